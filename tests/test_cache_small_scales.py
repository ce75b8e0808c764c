"""Binary16 pages whose value scales lie far below what commit makes of the type's values: they
are code times scale all the same, which is nothing beside the type's smallest number."""
import numpy as np
import pytest
import torch

from test_cache import Both, dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,value", [("e4m3", 1.75), ("int8", 1.984375)])
@pytest.mark.parametrize("counts", [[1, 3], [100, 70]])
@pytest.mark.parametrize("exponent", [-20, -30, -50, -62, -100, -118])
def test_value_scales_by_hand(dev, fmt, value, counts, exponent):  # noqa: F811
    """All pages, and every second one among ordinary pages; the values are the largest codes."""
    for every in (1, 2):
        b = Both(dev, 1, 2, 64, 2, 20, 9, 192, 64, fmt, "f16")

        def change(K, V, q):
            V[:] = value
        b.grow([512, 130], change)
        pages = b.model.table[b.model.table >= 0][::every]
        b.model.vs[:, pages] *= 2.0 ** exponent
        b.cache.v_scales[:, torch.from_numpy(pages).to(dev)] *= 2.0 ** exponent
        assert np.array_equal(b.cache.v_scales.double().cpu().numpy(), b.model.vs)

        def none(K, V, q):
            V[:] = 0
        q = b.draft(counts, none)
        b.attend(4, q)
        b.attend(4, q, longest=4000, sharp=4.0)
