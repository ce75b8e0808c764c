"""Attention on matrices whose rows lie in unusual places: leading dimensions that are
odd, so that rows start between and on 4 bytes in turn, and heads that span more than
2^31 and 2^32 bytes with rows on 16 and on 4 bytes.  References and bounds as in
``test_attention.py``."""
import math

import numpy as np
import pytest
import torch

from test_attention import DT, attend64, check_attention, dev, offsets, rand  # noqa: F401

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu


def odd_rows(x, dtype, left, dev):  # noqa: F811
    """x on the GPU, `left` elements into an odd leading dimension; NaN around it."""
    rows, cols = x.shape
    ld = cols + left + 2
    ld += 1 - ld % 2
    assert ld % 2 == 1
    buf = torch.full((rows, ld), math.nan, dtype=DT[dtype], device=dev)
    buf[:, left:left + cols].copy_(x.to(DT[dtype]))
    return buf[:, left:left + cols]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv_heads,D,q_lens,kv_lens", [
    (2, 1, 64, [1, 1, 1], [64, 63, 65]), (4, 2, 64, [65, 1, 90], [130, 20, 257]), (3, 1, 32, [200], [333]),
    (8, 2, 128, [33, 7], [190, 65]), (2, 1, 128, [150], [1000]), (1, 1, 256, [40], [150]),
    (1, 1, 256, [100], [150]), (3, 3, 80, [9, 100], [77, 45]), (2, 1, 33, [17], [66]),
    (1, 1, 64, [2], [9000])])
def test_odd_leading_dimensions(dev, heads, kv_heads, D, q_lens, kv_lens, dtype):  # noqa: F811
    q_off, kv_off = offsets(q_lens), offsets(np.array(kv_lens) + 1)
    ke = kv_off[1:] - 1
    q = 1.5 * rand(1, heads * D, int(q_off[-1]))
    k, v = (rand(s, kv_heads * D, int(kv_off[-1])) for s in (2, 3))
    for t in (k, v):
        t[:, ke] = math.nan                   # between the sequences
    mask = np.ones(k.shape[1], np.uint8)
    mask[1::5] = 0
    ints = [torch.from_numpy(np.ascontiguousarray(t)).to(dev) for t in (q_off, kv_off[:-1], ke)]
    for left in (0, 1, 2, 3):
        print(f"[odd rows] {heads}/{kv_heads} x {D}, q {q_lens} kv {kv_lens} {dtype} {left}", flush=True)
        Q, K, V = (odd_rows(t, dtype, left, dev) for t in (q, k, v))
        n64 = [t.double().cpu().numpy() for t in (Q, K, V)]
        out = odd_rows(torch.zeros_like(q), dtype, left, dev)
        for m in (None, mask):
            ref = attend64(*n64, heads, kv_heads, q_off, kv_off[:-1], ke, m)
            given = None if m is None else torch.from_numpy(m).to(dev)
            got = nmg.attention(Q, K, V, heads, kv_heads, *ints, given, out=out)
            check_attention(got, ref, n64[2], dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("extra", [8, 2])
def test_heads_past_32_bit_offsets(dev, D, extra, dtype):  # noqa: F811
    """Rows on 16 bytes and on 4, two key heads, few query columns and many; a tree."""
    ld, n, left = (1 << 25) + (1 << 24) + extra, 400, 64
    if dtype == "f32":                        # (rows of less than 2^28 bytes)
        ld = (1 << 25) + extra
    cols = n + left + 7
    begin = ld - n - 7
    K, V = (torch.empty((2 * D, ld), dtype=DT[dtype], device=dev) for _ in range(2))
    for t, s in ((K, 2), (V, 3)):
        x = rand(s, 2 * D, cols)
        x[:, -7:] = math.nan                  # past the range
        t[:, ld - cols:].copy_(x.to(DT[dtype]))
    n64 = [t[:, begin:begin + n].double().cpu().numpy() for t in (K, V)]
    for q_len in (1, 70):
        print(f"[wide] D {D} ld +{extra} q {q_len} {dtype}", flush=True)
        Q = rand(1, 4 * D, q_len).to(DT[dtype]).to(dev)
        ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [begin], [begin + n])]
        got = nmg.attention(Q, K, V, 4, 2, *ints)
        q64 = Q.double().cpu().numpy()
        check_attention(got, attend64(q64, *n64, 4, 2, [0, q_len], [0], [n]), n64[1], dtype)
        tree = np.tril(np.ones((q_len, q_len), np.uint8))
        got = nmg.tree_attention(Q, K, V, 4, 2, *ints, torch.from_numpy(tree).to(dev))
        check_attention(got, attend64(q64, *n64, 4, 2, [0, q_len], [0], [n], None, tree), n64[1], dtype)
