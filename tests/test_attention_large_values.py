"""Binary32 attention with values near the end of their range: outputs are means of
values, so they are finite where the values are, whatever the order of the scores.
References and bounds as in ``test_attention.py``; a mean may pass its largest value
by the bound's relative (n + 32) 2^-24 + 4 e_s, so values stay below the largest
number by more than that."""
import math

import numpy as np
import pytest
import torch

from test_attention import attend64, check_attention, dev, rand  # noqa: F401

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu

# heads, kv_heads, D, queries, keys: few rows (the waves split the keys, one part and
# several), many rows, heads over 128, several parts of many rows
CASES = [(1, 1, 64, 1, 70), (2, 1, 64, 3, 5000), (4, 1, 128, 8, 900), (1, 1, 64, 300, 400),
         (2, 2, 128, 150, 700), (1, 1, 256, 2, 300), (3, 1, 256, 100, 200), (2, 2, 64, 128, 9000),
         (2, 1, 40, 130, 33)]


def go(dev, heads, kv_heads, q, k, v):  # noqa: F811
    n, keys = q.shape[1], k.shape[1]
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, n], [0], [keys])]
    got = nmg.attention(q.to(dev), k.to(dev), v.to(dev), heads, kv_heads, *ints)
    n64 = [t.double().numpy() for t in (q, k, v)]
    check_attention(got, attend64(*n64, heads, kv_heads, [0, n], [0], [keys]), n64[2], "f32")


@pytest.mark.parametrize("heads,kv_heads,D,n,keys", CASES)
@pytest.mark.parametrize("size", [1e31, 1e34, 3.3e38])
@pytest.mark.parametrize("scores", ["flat", "rising", "random"])
def test_values_of_one_sign(dev, heads, kv_heads, D, n, keys, size, scores):  # noqa: F811
    """Weights that grow by less than the running maximum's slack from tile to tile,
    equal ones over many keys, and ordinary ones."""
    print(f"[large] {heads}/{kv_heads} x {D}, {n} over {keys}, {size} {scores}", flush=True)
    q, k = rand(1, heads * D, n), rand(2, kv_heads * D, keys)
    if scores == "flat":
        q = q * 0
    elif scores == "rising":                  # by 11 after the first 32 keys
        q = torch.zeros_like(q)
        q[::D] = 1.0
        k = torch.zeros_like(k)
        k[::D, 32:] = 11.0 * math.sqrt(D)
    v = (1 - 0.01 * rand(3, kv_heads * D, keys).abs()) * size
    go(dev, heads, kv_heads, q, k, v)


@pytest.mark.parametrize("heads,kv_heads,D,n,keys", CASES)
def test_large_and_small_features(dev, heads, kv_heads, D, n, keys):  # noqa: F811
    """A head's features keep their own precision: some near the largest number, of
    either sign, some near the smallest."""
    print(f"[mixed] {heads}/{kv_heads} x {D}, {n} over {keys}", flush=True)
    q, k = rand(1, heads * D, n), rand(2, kv_heads * D, keys)
    size = torch.tensor([3e38, -3e38, 1e-34, 1.0, 1e20], dtype=torch.float32)
    v = (1 - 0.1 * rand(3, kv_heads * D, keys).abs().clamp(max=5)) * \
        size[torch.arange(kv_heads * D) % 5][:, None]
    go(dev, heads, kv_heads, q, k, v)


def test_largest_key_alone(dev):  # noqa: F811
    """Large values of which the softmax leaves almost nothing."""
    D, keys = 64, 500
    for n in (1, 200):
        q, k, v = rand(1, D, n).abs() + 0.5, rand(2, D, keys) * 0.1, rand(3, D, keys)
        k[:, 3] = -0.5                        # scores about -2 .. -6
        v[:, 3] = 3e38
        go(dev, 1, 1, q, k, v)
        k[:, 450] = 3.0
        v[:, 450] = -3e38
        go(dev, 1, 1, q, k, v)
