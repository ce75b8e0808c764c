"""Attention for trees of drafted tokens when a branch is not finite: its keys and
values reach the tokens that attend to it and no others (``include/nmg.h``).
References and bounds as in ``test_attention.py``, where the reference is finite;
elsewhere NaN for NaN and the same infinity."""
import math

import numpy as np
import pytest
import torch

from test_attention import DT, attend64, check_attention, dev, offsets, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def branches(n):
    """(parents, tree) of n drafted tokens: four chains from the context, token i
    on chain i % 4."""
    parents = [i - 4 if i >= 4 else -1 for i in range(n)]
    tree = np.zeros((n, n), np.uint8)
    for i, up in enumerate(parents):
        if up >= 0:
            tree[i] = tree[up]
        tree[i, i] = 1
    return parents, tree


def check_all(got, ref, v, dtype):
    out = ref[0]
    finite = np.isfinite(out)
    assert finite.any() and not finite.all()
    g = got.double().cpu().numpy()
    assert (np.isnan(g) == np.isnan(out)).all(), "NaN in other places"
    assert (g[np.isinf(out)] == out[np.isinf(out)]).all(), "another infinity"
    check_attention(torch.from_numpy(np.where(finite, g, 0.0)),
                    [np.where(finite, r, 0.0) for r in ref], v, dtype)


# heads, kv_heads, D, drafted, context: few rows and many, one part of the keys and
# several, tiles that hold drafted and earlier keys, drafts over several tiles
CASES = [
    (2, 2, 64, [8], [50]),
    (2, 1, 64, [12], [3000]),
    (3, 1, 96, [70], [130]),
    (4, 1, 32, [6, 40], [0, 77]),
    (4, 2, 64, [66, 9], [300, 20]),
    (16, 2, 128, [63], [2000]),
    (8, 2, 128, [16], [63]),
    (1, 1, 256, [90], [40]),
    (2, 1, 256, [10], [500]),
    (2, 2, 80, [200], [17]),
]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv_heads,D,drafted,context", CASES)
def test_branches_not_finite(dev, heads, kv_heads, D, drafted, context, dtype):  # noqa: F811
    print(f"[branches] {heads}/{kv_heads} x {D} {drafted} {context} {dtype}", flush=True)
    q_off, kv_off = offsets(drafted), offsets(np.array(context) + np.array(drafted))
    N, S, T = int(q_off[-1]), int(kv_off[-1]), max(drafted)
    tree = np.zeros((N, T), np.uint8)
    for b, n in enumerate(drafted):
        tree[q_off[b]:q_off[b] + n, :n] = branches(n)[1]
    q, k, v = 1.2 * rand(1, heads * D, N), rand(2, kv_heads * D, S), rand(3, kv_heads * D, S)
    for b, n in enumerate(drafted):
        at = kv_off[b + 1] - n                # the draft's first column
        v[3, at] = math.inf                   # chain 0: one feature, one key head
        v[D - 1, at + 1] = -math.inf          # chain 1: an infinity, then its opposite
        if n > 5:
            v[D - 1, at + 5] = math.inf
        v[:, at + 2] = math.nan               # chain 2: everything, every key head
        k[:, at + 2] = math.nan
    K = torch.empty((kv_heads * D, S + S % 2 + 2), dtype=DT[dtype], device=dev)
    for odd in (0, 1):                        # rows that start on 4 bytes, and between
        V = torch.empty_like(K)
        Kv, Vv = (t[:, odd:odd + S] for t in (K, V))
        Kv.copy_(k.to(DT[dtype]))
        Vv.copy_(v.to(DT[dtype]))
        Q = q.to(DT[dtype]).to(dev)
        ints = [torch.from_numpy(np.ascontiguousarray(t)).to(dev) for t in (q_off, kv_off[:-1], kv_off[1:])]
        n64 = [t.double().cpu().numpy() for t in (Q, Kv, Vv)]
        with np.errstate(invalid="ignore"):
            ref = attend64(*n64, heads, kv_heads, q_off, kv_off[:-1], kv_off[1:], None, tree)
        t = torch.from_numpy(tree).to(dev)
        got = nmg_tree(Q, Kv, Vv, heads, kv_heads, ints, t)
        check_all(got, ref, n64[2], dtype)
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(nmg_tree(Q, Kv, Vv, heads, kv_heads,
                                                                           ints, t)))


def nmg_tree(Q, K, V, heads, kv_heads, ints, tree):
    from paper_2304_07613_amd import nmg

    return nmg.tree_attention(Q, K, V, heads, kv_heads, *ints, tree)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("share", [1, 40])
def test_kept_branch_keeps_its_values(dev, dtype, share):  # noqa: F811
    """What a sibling holds changes nothing, in binary16 to the last bit: two drafted
    tokens that do not see each other, the second one spoiled."""
    D, n = 64, 100
    Q = rand(1, share * D, 2).to(DT[dtype]).to(dev)
    K, V = (rand(s, D, n + 2).to(DT[dtype]).to(dev) for s in (2, 3))
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, 2], [0], [n + 2])]
    tree = torch.eye(2, dtype=torch.uint8, device=dev)
    clean = nmg_tree(Q, K, V, share, 1, ints, tree)
    # binary32 may sum in another order: twice (4 e_s + (n + 34) u) of the values, with
    # e_s = (D + 8) u times a score's absolute terms, here at most 6
    limit = 0.0 if dtype == "f16" else 2 * (4 * (D + 8) * 6 + n + 34) * 2.0 ** -24 * V.abs().max()
    for bad in (math.inf, -math.inf, math.nan):
        K2, V2 = K.clone(), V.clone()
        V2[::3, n + 1] = bad
        got = nmg_tree(Q, K, V2, share, 1, ints, tree)
        assert (got[:, 0].float() - clean[:, 0].float()).abs().max() <= limit
        spoiled = torch.arange(share * D, device=dev) % D % 3 == 0
        assert (~torch.isfinite(got[spoiled, 1])).all() and torch.isfinite(got[~spoiled, 1]).all()
        K2[5, n + 1] = bad
        got = nmg_tree(Q, K2, V2, share, 1, ints, tree)
        assert (got[:, 0].float() - clean[:, 0].float()).abs().max() <= limit
