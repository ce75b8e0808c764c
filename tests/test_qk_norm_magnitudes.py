"""Norms of queries and keys at any binary32 magnitude: the mean of squares may pass
either end of the range where the normed values do not.  References and bounds as in
``test_attention.py``'s norm tests: (4 + 6 + D / 2) 2^-24 of the rotation's terms;
results below the least normal number are off by 2^-149 of rounding at most."""
import numpy as np
import pytest
import torch

from test_attention import U, dev, norm64, rand, rotate64, table64  # noqa: F401

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,D,R,N", [(3, 64, 64, 1), (2, 64, 32, 33), (5, 80, 16, 130), (4, 128, 128, 257),
                                         (2, 33, 0, 40), (1, 256, 256, 600), (1, 2048, 64, 9)])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("sizes", [(1e25,), (1e37,), (1e-25,), (1e-37,), (3e-42,),
                                   (1.0, 1e30, 1e-30, 1e10, 1e19, 1e-19, 1e-12)])
def test_magnitudes(dev, heads, D, R, N, eps, sizes):  # noqa: F811
    print(f"[norm] {heads} x {D}, R {R}, N {N}, eps {eps}, {sizes}", flush=True)
    x = rand(D + N, 2 * heads * D, N).clamp(-3, 3)
    x = x * torch.tensor(sizes, dtype=torch.float32)[torch.arange(N) % len(sizes)]     # a size a token
    x[0, 0] = sizes[0]
    pos = torch.arange(N, dtype=torch.int32) % 50
    table = torch.from_numpy(table64(50, R).astype(np.float32)) if R else None
    t64 = np.zeros((2, 0, 1)) if table is None else table.double().numpy()
    w = 1 + 0.3 * rand(1, D)
    X = x.to(dev)
    q, k = X[: heads * D], X[heads * D:]
    got = nmg.qk_norm_rotary(q, k, heads, heads, w.to(dev), None, None if table is None else table.to(dev),
                             pos.to(dev), eps=eps)
    eps = float(np.float32(eps))
    for src, weight, y in ((q, w.double().numpy(), got[0]), (k, None, got[1])):
        ref, scale = rotate64(norm64(src.double().cpu().numpy(), heads, weight, eps), heads, t64,
                              pos.numpy(), "half")
        y = y.double().cpu().numpy()
        assert np.isfinite(y).all()
        assert (np.abs(y - ref) <= (4 + 6 + D / 2) * U * scale + 4 * 2.0 ** -149).all()
