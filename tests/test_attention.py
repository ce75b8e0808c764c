"""The attention operators between sparse projections: rotary positions, norms
of queries and keys with the rotation, attention over column ranges, attention
for trees of drafted tokens.

References are binary64 on the CPU, written from the formulas in
``include/nmg.h``.  Tolerances follow from the number of roundings:

  rotation   y = a c - b s: three roundings of terms and one of the sum in
             binary32, 4 u (|a c| + |b s|), u = 2^-24; behind a norm the factor
             x w / sqrt(mean + eps) carries the sum's D roundings halved by the
             square root and 6 more of its own
  attention  with e_s = (D + 8) u max_j scale sum_d |q_d k_dj| the error of a
             score and n keys, every weight is off by a factor 1 + 2 e_s at
             most, and the sums add n + 32 roundings: (4 e_s + (n + 32) u)
             sum_j p_j |v_j|; binary16 weights 2^-11 twice (numerator and
             denominator) and, where they are subnormal, 2^-30 n max |v|
  binary16   outputs add their rounding: 2^-11 |y| + 2^-24
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2304_07613_amd import build, nmg

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return nmg.lib()


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nmg.lib()
    return DEV


def rand(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32))


def placed(x, dtype, how, dev):
    """x on the GPU as a view: contiguous, rows padded, or starting at an odd
    element of an odd leading dimension.  What lies around it is NaN."""
    rows, cols = x.shape
    left, ld = {"dense": (0, cols), "padded": (8, (cols + 8) // 8 * 8 + 16),
                "odd": (3, cols + 4 + cols % 2)}[how]
    buf = torch.full((rows, ld), math.nan, dtype=dtype, device=dev)
    view = buf[:, left:left + cols]
    view.copy_(x.to(dtype))
    return view


# ---------------------------------------------------------------- references

def table64(length, dim, base=10000.0, scaling="none", factor=1.0, original=0.0, slow=1.0, fast=32.0,
            magnitude=1.0):
    i = np.arange(dim // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (dim / (dim - 2))
    f = base ** (-2 * i / dim)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        g = np.clip((original * f / (2 * np.pi) - slow) / (fast - slow), 0, 1)
        f = f * (g + (1 - g) / factor)
    a = f[:, None] * np.arange(length)[None, :]
    return np.stack((np.cos(a), np.sin(a))) * magnitude


def rotate64(x, heads, table, positions, pairs):
    """(result, error scale) of x (heads D x N, binary64)."""
    D, R = x.shape[0] // heads, 2 * table.shape[1]
    y, scale = x.copy(), np.abs(x)
    p = np.clip(positions, 0, table.shape[2] - 1)
    for h in range(heads):
        for i in range(R // 2):
            a, b = (2 * i, 2 * i + 1) if pairs == "interleaved" else (i, i + R // 2)
            a, b = h * D + a, h * D + b
            c, s = table[0, i, p], table[1, i, p]
            y[a], y[b] = x[a] * c - x[b] * s, x[a] * s + x[b] * c
            scale[a] = np.abs(x[a] * c) + np.abs(x[b] * s)
            scale[b] = np.abs(x[a] * s) + np.abs(x[b] * c)
    return y, scale


def norm64(x, heads, w, eps):
    D = x.shape[0] // heads
    y = x.reshape(heads, D, -1)
    y = y / np.sqrt((y * y).mean(axis=1, keepdims=True) + eps)
    return (y * (1 if w is None else w[None, :, None])).reshape(x.shape)


def attend64(q, k, v, heads, kv_heads, q_off, kb, ke, key_mask=None, tree=None, scale=None):
    """(result, sum of p |v|, e_s, keys) of every output, binary64."""
    D, share = q.shape[0] // heads, heads // kv_heads
    scale = D ** -0.5 if scale is None else scale
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    err, keys = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(kb)):
        n = q_off[b + 1] - q_off[b]
        cols = np.arange(kb[b], ke[b])
        for t in range(n):
            c = q_off[b] + t
            see = np.ones(len(cols), bool)
            if key_mask is not None:
                see &= key_mask[cols] != 0
            if tree is not None:
                i = cols - (ke[b] - n)
                own = i >= 0
                ok = i[own] < tree.shape[1]
                see[own] = ok & (tree[c, np.minimum(i[own], tree.shape[1] - 1)] != 0)
            mine = cols[see]
            if not len(mine):
                continue
            for h in range(heads):
                g = h // share
                rows = slice(h * D, (h + 1) * D)
                kk, vv = k[g * D:(g + 1) * D, mine], v[g * D:(g + 1) * D, mine]
                s = scale * (q[rows, c] @ kk)
                top = s.max()
                if top == -np.inf:
                    continue
                p = np.exp(s - top)
                p /= p.sum()
                out[rows, c] = vv @ p
                mag[rows, c] = np.abs(vv) @ p
                err[rows, c] = (D + 8) * U * scale * (np.abs(q[rows, c]) @ np.abs(kk)).max()
                keys[rows, c] = len(mine)
    return out, mag, err, keys


def check_attention(got, ref, v, dtype):
    out, mag, err, keys = ref
    tol = (4 * err + (keys + 32) * U) * mag
    if dtype == "f16":
        vmax = np.abs(v[np.isfinite(v)]).max(initial=0.0)
        tol = tol + 2 * 2.0 ** -11 * mag + 2.0 ** -30 * keys * vmax + 2.0 ** -11 * np.abs(out) + 2.0 ** -24
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), "not finite"
    worst = (np.abs(got - out) - tol).max(initial=-1.0)
    assert worst <= 0, f"off by {worst:.3g} more than the bound"


# ------------------------------------------------------------------- rotation

SCALINGS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
            dict(scaling="parts", factor=8.0, original=512.0, magnitude=1.2079),
            dict(scaling="parts", factor=8.0, original=8192.0, slow=1.0, fast=4.0, base=500000.0)]


@gpu
@pytest.mark.parametrize("kw", SCALINGS)
@pytest.mark.parametrize("dim,length", [(64, 1000), (2, 7), (128, 70001)])
def test_rotary_table(dev, kw, dim, length):
    if kw.get("scaling") == "ntk" and dim < 4:
        with pytest.raises(nmg.NmgError):
            nmg.rotary_table(length, dim, device=dev, **kw)
        return
    got = nmg.rotary_table(length, dim, device=dev, **kw).double().cpu().numpy()
    ref = table64(length, dim, **kw)
    assert got.shape == ref.shape
    # binary64 angles of up to 70000 carry 2^-53 * 70000 twice; one rounding to binary32
    assert np.abs(got - ref).max() <= U * np.abs(ref).max() + 1e-10


ROT = [  # heads, D, R, N
    (1, 2, 2, 1), (3, 64, 64, 1), (12, 64, 64, 8), (2, 64, 32, 33), (5, 80, 16, 130), (2, 7, 4, 65),
    (4, 128, 128, 257), (2, 96, 48, 1021), (1, 256, 256, 19), (3, 33, 0, 40), (2, 130, 128, 300),
    (7, 64, 64, 2047), (20, 32, 16, 515),
]


def rotary_inputs(seed, heads, D, R, N, length, dev):
    x = rand(seed, heads * D, N) * 3
    pos = torch.from_numpy(np.random.default_rng(seed + 1).integers(0, length, N).astype(np.int32))
    table = torch.from_numpy(table64(length, R).astype(np.float32)) if R else None
    return x, pos, table


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("heads,D,R,N", ROT)
def test_rotary(dev, heads, D, R, N, pairs, dtype):
    print(f"[rotary] {heads} x {D}, R {R}, N {N} {pairs} {dtype}", flush=True)
    x, pos, table = rotary_inputs(heads + D + N, heads, D, R, N, 700, dev)
    pos[0] = 699
    if N > 2:
        pos[1], pos[2] = -5, 100000          # outside: the nearest inside
    for how in ("dense", "padded", "odd"):
        X = placed(x, DT[dtype], how, dev)
        x64 = X.double().cpu().numpy()
        t64 = np.zeros((2, 0, 1)) if table is None else table.double().numpy()
        ref, scale = rotate64(x64, heads, t64, pos.numpy(), pairs)
        tol = 4 * U * scale + (2.0 ** -11 * np.abs(ref) + 2.0 ** -24 if dtype == "f16" else 0)
        tab = None if table is None else table.to(dev)
        Y = nmg.rotary(X, heads, tab, pos.to(dev), pairs)
        assert (np.abs(Y.double().cpu().numpy() - ref) <= tol).all(), how
        nmg.rotary(X, heads, tab, pos.to(dev), pairs, out=X)      # in place: the same bits
        assert torch.equal(X, Y)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("heads,D,R,N", ROT)
def test_qk_norm_rotary(dev, heads, D, R, N, pairs, dtype):
    print(f"[qk_norm] {heads} x {D}, R {R}, N {N} {pairs} {dtype}", flush=True)
    kv, eps = max(1, heads // 3), 1e-6
    x, pos, table = rotary_inputs(heads + D + N + 7, heads + 2 * kv, D, R, N, 700, dev)
    x[: D] = 0                                # a head of zeros: eps decides
    wq, wk = 1 + 0.3 * rand(1, D), 1 + 0.3 * rand(2, D)
    tab = None if table is None else table.to(dev)
    t64 = np.zeros((2, 0, 1)) if table is None else table.double().numpy()
    for how in ("dense", "odd"):
        X = placed(x, DT[dtype], how, dev)
        Q, K = X[: heads * D], X[heads * D:(heads + kv) * D]
        V = X[(heads + kv) * D:].clone()
        outs = nmg.qk_norm_rotary(Q, K, heads, kv, wq.to(dev), wk.to(dev), tab, pos.to(dev), pairs, eps)
        for src, h, w, got in ((Q, heads, wq, outs[0]), (K, kv, wk, outs[1])):
            y = norm64(src.double().cpu().numpy(), h, w.double().numpy(), eps)
            ref, scale = rotate64(y, h, t64, pos.numpy(), pairs)
            tol = (4 + 6 + D / 2) * U * scale
            tol = tol + (2.0 ** -11 * np.abs(ref) + 2.0 ** -24 if dtype == "f16" else 0)
            assert (np.abs(got.double().cpu().numpy() - ref) <= tol).all(), how
        nmg.qk_norm_rotary(Q, K, heads, kv, wq.to(dev), wk.to(dev), tab, pos.to(dev), pairs, eps, (Q, K))
        assert torch.equal(Q, outs[0]) and torch.equal(K, outs[1])
        assert torch.equal(X[(heads + kv) * D:], V)      # the values' rows are untouched


@gpu
def test_qk_norm_without_weights_or_table(dev):
    x = rand(3, 4 * 64, 50).to(dev)
    q, k = nmg.qk_norm_rotary(x[:192], x[192:], 3, 1, None, None)
    ref = norm64(x.double().cpu().numpy(), 4, None, 1e-6)
    assert np.abs(torch.cat((q, k)).double().cpu().numpy() - ref).max() <= (10 + 32) * U * 8


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_rotary_keeps_other_columns_out(dev, dtype):
    """NaN and infinity of one token stay in its column and, without a norm, in
    their pair."""
    x = rand(4, 2 * 64, 70)
    x[5, 3], x[64 + 40, 9] = math.nan, math.inf
    pos = torch.arange(70, dtype=torch.int32, device=dev)
    table = torch.from_numpy(table64(70, 32).astype(np.float32)).to(dev)
    y = nmg.rotary(x.to(DT[dtype]).to(dev), 2, table, pos).cpu()
    bad = ~torch.isfinite(y.float())
    assert bad.nonzero().tolist() == [[5, 3], [21, 3], [104, 9]]
    y, _ = nmg.qk_norm_rotary(x.to(DT[dtype]).to(dev), x.to(DT[dtype]).to(dev), 2, 2, None, None,
                              table, pos)
    bad = ~torch.isfinite(y.float().cpu())
    assert bad[:64, 3].all() and bad.sum() <= 64 + 64 and not bad[:, :3].any()


# ------------------------------------------------------------------ attention

def offsets(lens):
    return np.concatenate(([0], np.cumsum(lens))).astype(np.int32)


def run_attention(dev, dtype, heads, kv_heads, D, q_lens, kv_lens, how="dense", mask=None, seed=0,
                  scale=None, spread=1.5, gap=0):
    q_off, kv_off = offsets(q_lens), offsets(np.asarray(kv_lens) + gap)
    kb, ke = kv_off[:-1], kv_off[:-1] + np.asarray(kv_lens, dtype=np.int32)
    q = spread * rand(seed + 1, heads * D, int(q_off[-1]))
    k, v = rand(seed + 2, kv_heads * D, int(kv_off[-1])), rand(seed + 3, kv_heads * D, int(kv_off[-1]))
    for b in range(len(kb)):                  # gaps hold NaN: never read into a result
        k[:, ke[b]:kv_off[b + 1]] = math.nan
        v[:, ke[b]:kv_off[b + 1]] = math.nan
    if mask is not None:
        k[:, mask == 0] = math.inf
        v[:, mask == 0] = math.nan
    Q, K, V = (placed(t, DT[dtype], how, dev) for t in (q, k, v))
    ints = [torch.from_numpy(np.ascontiguousarray(t)).to(dev) for t in (q_off, kb, ke)]
    m = None if mask is None else torch.from_numpy(mask).to(dev)
    got = nmg.attention(Q, K, V, heads, kv_heads, *ints, m, scale)
    n64 = [t.double().cpu().numpy() for t in (Q, K, V)]
    ref = attend64(*n64, heads, kv_heads, q_off, kb, ke, mask, None, scale)
    check_attention(got, ref, n64[2], dtype)
    again = nmg.attention(Q, K, V, heads, kv_heads, *ints, m, scale)
    assert torch.equal(got, again)
    return got


ATTN = [  # heads, kv_heads, D, query lengths, key lengths
    (1, 1, 64, [1], [1]),
    (2, 1, 64, [1, 1, 1], [64, 63, 65]),
    (12, 12, 64, [1] * 8, [512, 1, 100, 37, 511, 0, 64, 3]),
    (4, 2, 64, [5, 0, 40, 1], [130, 20, 0, 257]),
    (2, 2, 64, [128, 129, 1], [128, 77, 300]),
    (3, 1, 64, [200], [333]),
    (8, 2, 128, [33, 7], [190, 65]),
    (2, 1, 128, [150], [1000]),
    (2, 2, 32, [70, 3], [40, 129]),
    (1, 1, 256, [40], [150]),
    (3, 3, 80, [9, 100], [77, 45]),
    (2, 2, 96, [31], [129]),
    (2, 1, 33, [17], [66]),
    (2, 2, 1, [5], [9]),
    (1, 1, 200, [3], [50]),
    (6, 1, 64, [1, 2], [2500, 1300]),
    (1, 1, 64, [2], [9000]),
]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv_heads,D,q_lens,kv_lens", ATTN)
def test_attention(dev, heads, kv_heads, D, q_lens, kv_lens, dtype):
    for how, gap in (("dense", 0), ("padded", 5), ("odd", 1)):
        print(f"[attention] {heads}/{kv_heads} x {D}, q {q_lens} kv {kv_lens} {dtype} {how}", flush=True)
        run_attention(dev, dtype, heads, kv_heads, D, q_lens, kv_lens, how, gap=gap, seed=D)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("q_lens", [[1, 1, 1], [100, 30, 7]])
def test_attention_key_mask(dev, D, q_lens, dtype):
    """Dropped keys, whole tiles of them, a sequence with none left; NaN and
    infinity behind the mask."""
    kv_lens = [300, 64, 129]
    mask = (np.random.default_rng(D).random(sum(kv_lens)) < 0.7).astype(np.uint8) * 3
    mask[40:240] = 0                          # tiles without a key
    mask[300:364] = 0                         # a sequence without a key
    for how in ("dense", "odd"):
        print(f"[mask] D {D} q {q_lens} {dtype} {how}", flush=True)
        got = run_attention(dev, dtype, 4, 2, D, q_lens, kv_lens, how, mask, seed=5)
        q0 = q_lens[0]
        assert (got[:, q0:q0 + q_lens[1]] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("q_len", [1, 130])
def test_attention_sharp_and_flat(dev, dtype, q_len):
    """Scores from hundreds apart to all equal, largest last: the running maximum
    moves in every tile; and a scale of the caller's."""
    D, n = 64, 400
    for what in ("sharp", "flat", "rising"):
        q, k, v = rand(1, D, q_len), rand(2, D, n), rand(3, D, n)
        if what == "sharp":
            q = q * 20
        elif what == "flat":
            q = q * 0
        else:
            q = q.abs() * 0.5
            k = k * 0.01 + torch.linspace(0, 12, n)[None, :]
        Q, K, V = (t.to(DT[dtype]).to(dev) for t in (q, k, v))
        ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [0], [n])]
        n64 = [t.double().cpu().numpy() for t in (Q, K, V)]
        for scale in (None, 0.3):
            got = nmg.attention(Q, K, V, 1, 1, *ints, scale=scale)
            ref = attend64(*n64, 1, 1, [0, q_len], [0], [n], scale=scale)
            check_attention(got, ref, n64[2], dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("q_len", [1, 70])
def test_attention_not_finite(dev, dtype, q_len):
    """Minus infinity as a score leaves its key out; a query whose scores are all
    minus infinity gives 0; NaN in a query or in a key that is seen reaches the
    rows that see it and no others; an infinity in V reaches its row of O."""
    D, n = 64, 200
    q, k, v = rand(1, 2 * D, q_len).abs() + 0.1, rand(2, D, n), rand(3, D, n)
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [0], [n])]

    def go(q, k, v):
        t = [x.to(DT[dtype]).to(dev) for x in (q, k, v)]
        return nmg.attention(*t, 2, 1, *ints).double().cpu().numpy()

    k1 = k.clone()
    k1[:, 10:150] = -math.inf
    kept = torch.cat((k[:, :10], k[:, 150:]), 1), torch.cat((v[:, :10], v[:, 150:]), 1)
    ref = attend64(*[x.to(DT[dtype]).double().numpy() for x in (q, *kept)], 2, 1, [0, q_len], [0], [60])
    check_attention(torch.from_numpy(go(q, k1, v)), ref, v.numpy(), dtype)
    assert (go(q, torch.full_like(k, -math.inf), v) == 0).all()
    q2 = q.clone()
    q2[D + 3, 0] = math.nan
    got = go(q2, k, v)
    assert np.isnan(got[D:, 0]).all() and np.isfinite(got[:D]).all() and np.isfinite(got[:, 1:]).all()
    v2 = v.clone()
    v2[7, 111] = math.inf
    got = go(q, k, v2)
    assert np.isinf(got[7]).all() and np.isinf(got[D + 7]).all() and np.isfinite(got[:7]).all()
    k2 = k.clone()
    k2[0, 5] = math.nan
    assert np.isnan(go(q, k2, v)).all()


TREE = [  # heads, kv_heads, D, drafted, context lengths
    (2, 2, 64, [1], [0]),
    (12, 12, 64, [8], [1000]),
    (4, 1, 64, [5, 16], [63, 64]),
    (8, 2, 128, [63, 63], [300, 17]),
    (2, 1, 80, [70], [130]),
    (6, 2, 64, [33, 2, 64], [0, 500, 1]),
    (4, 2, 32, [140], [50]),
]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv_heads,D,drafted,context", TREE)
def test_tree_attention(dev, heads, kv_heads, D, drafted, context, dtype):
    rng = np.random.default_rng(D + len(drafted))
    N, T = sum(drafted), max(drafted)
    q_off = offsets(drafted)
    room = max(c + d for c, d in zip(context, drafted)) + 3
    kb = np.array([b * room for b in range(len(drafted))], dtype=np.int32)
    ke = (kb + np.array(context) + np.array(drafted)).astype(np.int32)
    tree = np.zeros((N, T), np.uint8)
    for b, n in enumerate(drafted):
        for t in range(n):
            up = int(rng.integers(max(-1, t - 4), t)) if t else -1
            if up >= 0:
                tree[q_off[b] + t] = tree[q_off[b] + up]
            tree[q_off[b] + t, t] = 1
    q, k, v = 1.5 * rand(1, heads * D, N), rand(2, kv_heads * D, room * len(drafted)), \
        rand(3, kv_heads * D, room * len(drafted))
    for b in range(len(drafted)):             # past the end of a sequence's cache
        k[:, ke[b]:(b + 1) * room] = math.nan
        v[:, ke[b]:(b + 1) * room] = math.inf
    ints = [torch.from_numpy(t).to(dev) for t in (q_off, kb, ke)]
    for how in ("dense", "odd"):
        print(f"[tree] {heads}/{kv_heads} x {D} {drafted} {context} {dtype} {how}", flush=True)
        Q, K, V = (placed(t, DT[dtype], how, dev) for t in (q, k, v))
        n64 = [t.double().cpu().numpy() for t in (Q, K, V)]
        full = attend64(*n64, heads, kv_heads, q_off, kb, ke, None, tree)
        wide = torch.zeros((N, T + 5), dtype=torch.uint8, device=dev)     # a padded tree
        wide[:, :T] = torch.from_numpy(tree).to(dev)
        got = nmg.tree_attention(Q, K, V, heads, kv_heads, *ints, wide[:, :T])
        check_attention(got, full, n64[2], dtype)
    # a row that sees nothing of the draft, and behind an empty context nothing
    blind = torch.from_numpy(tree).to(dev)
    blind[N - 1] = 0
    got = nmg.tree_attention(Q, K, V, heads, kv_heads, *ints, blind)
    none = tree.copy()
    none[N - 1] = 0
    check_attention(got, attend64(*n64, heads, kv_heads, q_off, kb, ke, None, none), n64[2], dtype)
    # a tree narrower than a draft: the tokens beyond it are not attended to
    if T > 4:
        got = nmg.tree_attention(Q, K, V, heads, kv_heads, *ints, blind[:, :T - 3])
        ref = attend64(*n64, heads, kv_heads, q_off, kb, ke, None, none[:, :T - 3])
        check_attention(got, ref, n64[2], dtype)


@gpu
def test_tree_of_chains_equals_single_steps(dev):
    """A draft without branches gives what its tokens give one after another."""
    D, n, T = 64, 300, 6
    q, k, v = (rand(i, 2 * D, n + T).half().to(dev) for i in (1, 2, 3))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    chain = torch.tril(torch.ones((T, T), dtype=torch.bool, device=dev))
    got = nmg.tree_attention(q[:, n:], k, v, 2, 2, i32([0, T]), i32([0]), i32([n + T]), chain)
    for t in range(T):
        one = nmg.attention(q[:, n + t:n + t + 1], k, v, 2, 2, i32([0, 1]), i32([0]), i32([n + t + 1]))
        assert (got[:, t:t + 1].float() - one.float()).abs().max() <= 2 * 2.0 ** -11


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("q_len", [1, 40])
def test_attention_past_32_bit_offsets(dev, dtype, q_len):
    """Key and value rows further than 2^32 bytes and 2^31 elements apart."""
    D, ld, n = 64, (1 << 25) + (1 << 24) + 1, 700
    K = torch.empty((D, ld), dtype=DT[dtype], device=dev)
    V = torch.empty((D, ld), dtype=DT[dtype], device=dev)
    begin = ld - n - 1
    K[:, begin - 64:].copy_(rand(2, D, n + 65).to(DT[dtype]))
    V[:, begin - 64:].copy_(rand(3, D, n + 65).to(DT[dtype]))
    Q = rand(1, D, q_len).to(DT[dtype]).to(dev)
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [begin], [begin + n])]
    got = nmg.attention(Q, K, V, 1, 1, *ints)
    n64 = [t.double().cpu().numpy() for t in (Q, K[:, begin:begin + n], V[:, begin:begin + n])]
    check_attention(got, attend64(*n64, 1, 1, [0, q_len], [0], [n]), n64[2], dtype)


@gpu
def test_attention_ranges_cut_and_shared(dev):
    """Ranges past the matrices are cut; two sequences may read the same keys;
    a queryless tail column is left alone; no key columns at all give zeros."""
    D = 64
    q, k, v = (rand(i, D, 30).half().to(dev) for i in (1, 2, 3))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    out = torch.full((D, 30), 7.0, dtype=torch.float16, device=dev)
    nmg.attention(q, k, v, 1, 1, i32([0, 4, 20, 29]), i32([-3, -3, 25]), i32([10, 10, 99]), out=out)
    ref = attend64(*[t.double().cpu().numpy() for t in (q, k, v)], 1, 1, [0, 4, 20, 29], [0, 0, 25],
                   [10, 10, 30])
    assert (out[:, 29] == 7).all()
    check_attention(out[:, :29], [r[:, :29] for r in ref], v.double().cpu().numpy(), "f16")
    none = nmg.attention(q, k[:, :0], v[:, :0], 1, 1, i32([0, 30]), i32([0]), i32([0]))
    assert (none == 0).all()


@gpu
@pytest.mark.parametrize("q_len", [1, 40, 300])
def test_attention_with_and_without_workspace(dev, q_len):
    """Fewer splits for less workspace, and none without: each within the bound."""
    D, n = 64, 5000
    q, k, v = rand(1, D, q_len).half(), rand(2, D, n).half(), rand(3, D, n).half()
    Q, K, V = (t.to(dev) for t in (q, k, v))
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [0], [n])]
    L = nmg.lib()
    h = nmg._Heads(1, 1, D, nmg.F16)
    s = nmg._Sequences(1, *(t.data_ptr() for t in ints))
    full = L.nmg_attention_workspace_bytes(h, 1, q_len, n)
    ref = attend64(*[t.double().numpy() for t in (q, k, v)], 1, 1, [0, q_len], [0], [n])
    for nbytes in (0, 1000, full // 3, full):
        ws = torch.full((max(nbytes, 1),), 255, dtype=torch.uint8, device=dev)
        out = torch.empty_like(Q)
        st = L.nmg_attention(h, s, Q.data_ptr(), q_len, q_len, K.data_ptr(), n, V.data_ptr(), n, n, None,
                             0.125, out.data_ptr(), q_len, ws.data_ptr() if nbytes else None, nbytes,
                             torch.cuda.current_stream().cuda_stream)
        assert st == nmg.OK
        check_attention(out, ref, v.double().numpy(), "f16")


@gpu
def test_operators_in_a_graph_on_another_stream(dev):
    """Captured once, replayed while the cache grows in place."""
    D, H, cap = 64, 4, 900
    table = nmg.rotary_table(cap, D, device=dev)
    x, k, v = (rand(i, H * D, c).half().to(dev) for i, c in ((1, 2), (2, 2 * cap), (3, 2 * cap)))
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=dev)
    pos, q_off, kb, ke = i32([100, 200]), i32([0, 1, 2]), i32([0, cap]), i32([100, cap + 200])

    def step():
        q = nmg.rotary(x, H, table, pos)
        q, _ = nmg.qk_norm_rotary(q, q, H, H, None, None, table, pos)
        return nmg.attention(q, k, v, H, H, q_off, kb, ke)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for i in range(4):
        ke += 170
        pos += 31
        x.copy_(rand(20 + i, H * D, 2).half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, step())


@gpu
@pytest.mark.parametrize("q_len", [1, 70])
@pytest.mark.parametrize("scales", [(1, 1, 1e-30), (1, 1, 1e-33), (1, 1, 1e-36), (1, 1, 1e35), (1e20, 1e-20, 1),
                                    (1e-33, 1e33, 1), (1e30, 1e-30, 1e-34)])
def test_attention_magnitudes(dev, q_len, scales):
    """Binary32 keeps its precision at any magnitude of queries, keys and values."""
    D, n = 64, 200
    q, k, v = (rand(i, D, c) * np.float32(f) for i, c, f in zip((1, 2, 3), (q_len, n, n), scales))
    ints = [torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, q_len], [0], [n])]
    got = nmg.attention(q.to(dev), k.to(dev), v.to(dev), 1, 1, *ints)
    n64 = [t.double().numpy() for t in (q, k, v)]
    check_attention(got, attend64(*n64, 1, 1, [0, q_len], [0], [n]), n64[2], "f32")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("longest", [3, 60])
def test_attention_many_sequences(dev, dtype, longest):
    """More sequences than a wave has lanes, some without queries or keys."""
    rng = np.random.default_rng(longest)
    q_lens = rng.integers(0, longest + 1, 150).tolist()
    kv_lens = rng.integers(0, 90, 150).tolist()
    q_lens[64], q_lens[149], kv_lens[149] = longest, longest, 70
    run_attention(dev, dtype, 4, 2, 32, q_lens, kv_lens, "dense", seed=2)


@gpu
@pytest.mark.parametrize("dtype,D", [("f16", 64), ("f16", 128), ("f32", 64)])
def test_attention_repeats(dev, dtype, D):
    """Every pass over a full GPU gives the same bits, and those of its sequences
    alone: no result depends on when copies land."""
    H, n, B = 8, 640, 12
    q, k, v = (rand(i, H * D, B * n).to(DT[dtype]).to(dev) for i in (1, 2, 3))
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=dev)
    off = i32([n * b for b in range(B + 1)])
    first = nmg.attention(q, k, v, H, H, off, off[:-1].contiguous(), off[1:].contiguous())
    for _ in range(20):
        assert torch.equal(first, nmg.attention(q, k, v, H, H, off, off[:-1].contiguous(),
                                                off[1:].contiguous()))
    one = nmg.attention(q[:, :n].contiguous(), k, v, H, H, i32([0, n]), i32([0]), i32([n]))
    tol = 2.0 ** -9 if dtype == "f16" else 2.0 ** -17
    assert (one.float() - first[:, :n].float()).abs().max() <= tol * first.abs().max()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_many_rows(dev, dtype):
    """Rows that several waves share, where the tests above have few a sequence."""
    for heads, kv_heads, D, q_lens, kv_lens in [
            (4, 2, 64, [65, 1, 90], [130, 20, 257]), (1, 1, 256, [100], [150]), (3, 1, 80, [40, 33], [77, 45]),
            (2, 1, 96, [64], [129]), (4, 1, 33, [17], [66]), (2, 2, 1, [70], [9]), (12, 2, 64, [1] * 50, [70] * 50)]:
        for how, gap in (("dense", 0), ("odd", 1)):
            print(f"[rows] {heads}/{kv_heads} x {D}, q {q_lens} kv {kv_lens} {dtype} {how}", flush=True)
            run_attention(dev, dtype, heads, kv_heads, D, q_lens, kv_lens, how, gap=gap, seed=D)
    for D in (64, 80, 128):
        test_attention_key_mask(dev, D, [130, 70, 65], dtype)
    test_attention_past_32_bit_offsets(dev, dtype, 70)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("heads,kv_heads,D,drafted,context", [
    (6, 1, 64, [33, 2, 64], [0, 500, 1]), (8, 2, 80, [63, 17], [300, 5]), (1, 1, 256, [90], [40])])
def test_tree_attention_many_rows(dev, heads, kv_heads, D, drafted, context, dtype):
    test_tree_attention(dev, heads, kv_heads, D, drafted, context, dtype)


# ------------------------------------------------------------------- refusals

def test_rotary_refusals(lib):
    p, odd = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 2)
    ok = dict(dim=64, pairs=0, length=100, table=1 << 20, positions=1 << 20)

    def call(heads=2, D=64, X=p, ldx=32, N=32, Y=p, ldy=32, dtype=nmg.F32, **kw):
        return lib.nmg_rotary(dtype, heads, D, nmg._Rotary(**{**ok, **kw}), X, ldx, N, Y, ldy, None)

    assert call(dtype=9) == nmg.ERR_DTYPE
    assert lib.nmg_rotary(nmg.F32, 2, 64, None, p, 32, 32, p, 32, None) == nmg.ERR_NULL
    for kw in (dict(dim=63), dict(dim=66), dict(dim=-2), dict(pairs=2), dict(length=0), dict(heads=0),
               dict(ldx=31), dict(ldy=31), dict(N=0), dict(D=0, dim=0), dict(length=1 << 31),
               dict(ldy=40), dict(N=1 << 31, ldx=1 << 31, ldy=1 << 31)):
        assert call(**kw) == nmg.ERR_PARAM, kw
    for kw in (dict(X=None), dict(Y=None), dict(table=None), dict(positions=None)):
        assert call(**kw) == nmg.ERR_NULL, kw
    for kw in (dict(X=odd), dict(Y=odd), dict(table=(1 << 20) + 2), dict(positions=(1 << 20) + 1)):
        assert call(**kw) == nmg.ERR_ALIGN, kw

    def norm(qh=2, kh=1, eps=1e-6, K=p, YK=p, ldk=32, wq=p):
        return lib.nmg_qk_norm_rotary(nmg.F32, qh, kh, 64, nmg._Rotary(**ok), wq, None, eps, p, 32, K,
                                      ldk, 32, p, 32, YK, 32, None)

    assert norm(kh=-1) == norm(qh=0) == norm(eps=-1.0) == norm(eps=math.inf) == nmg.ERR_PARAM
    assert norm(eps=math.nan) == norm(ldk=31) == nmg.ERR_PARAM
    assert norm(K=None) == norm(YK=None) == nmg.ERR_NULL
    assert norm(wq=odd) == nmg.ERR_ALIGN

    def table(dim=64, length=10, base=1e4, scaling=0, factor=2.0, original=512.0, slow=1.0, fast=32.0,
              mag=1.0, out=p):
        return lib.nmg_rotary_table(dim, length, base, scaling, factor, original, slow, fast, mag, out, None)

    assert table(out=None) == nmg.ERR_NULL and table(out=odd) == nmg.ERR_ALIGN
    for kw in (dict(dim=0), dict(dim=7), dict(length=0), dict(base=0.0), dict(base=math.inf),
               dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=2, dim=2),
               dict(scaling=1, factor=math.nan), dict(scaling=3, original=0.0), dict(scaling=3, slow=32.0),
               dict(scaling=3, slow=-1.0), dict(mag=math.nan)):
        assert table(**kw) == nmg.ERR_PARAM, kw


def test_attention_refusals(lib):
    p, odd = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 1)

    def call(tree=False, heads=4, kv=2, D=64, dtype=nmg.F16, count=2, qo=1 << 20, kb=1 << 20, ke=1 << 20,
             Q=p, ldq=8, Nq=8, K=p, ldk=16, V=p, ldv=16, Nk=16, scale=0.125, O=p, ldo=8, ws=None, wb=0,
             tr=p, ldt=4, width=4):
        h, s = nmg._Heads(heads, kv, D, dtype), nmg._Sequences(count, qo, kb, ke)
        args = (h, s, Q, ldq, Nq, K, ldk, V, ldv, Nk)
        if tree:
            return lib.nmg_tree_attention(*args, tr, ldt, width, scale, O, ldo, ws, wb, None)
        return lib.nmg_attention(*args, None, scale, O, ldo, ws, wb, None)

    for tree in (False, True):
        assert call(tree, dtype=5) == nmg.ERR_DTYPE
        for kw in (dict(heads=3), dict(heads=0), dict(kv=0), dict(D=0), dict(count=0), dict(Nq=0),
                   dict(Nk=-1), dict(ldq=7), dict(ldo=7), dict(ldk=15), dict(ldv=15), dict(scale=0.0),
                   dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(wb=-1),
                   dict(Nq=1 << 31, ldq=1 << 31, ldo=1 << 31), dict(Nk=1 << 31, ldk=1 << 31, ldv=1 << 31),
                   dict(heads=1 << 24, kv=1 << 24, D=256)):
            assert call(tree, **kw) == nmg.ERR_PARAM, kw
        assert call(tree, D=257) == nmg.ERR_UNSUPPORTED
        for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(qo=None), dict(kb=None),
                   dict(ke=None)):
            assert call(tree, **kw) == nmg.ERR_NULL, kw
        for kw in (dict(Q=odd), dict(K=odd), dict(V=odd), dict(O=odd), dict(qo=(1 << 20) + 2),
                   dict(ws=ctypes.c_void_p(128), wb=64)):
            assert call(tree, **kw) == nmg.ERR_ALIGN, kw
    assert call(True, tr=None) == nmg.ERR_NULL
    assert call(True, ldt=3) == call(True, width=0) == nmg.ERR_PARAM
    assert lib.nmg_attention_workspace_bytes(nmg._Heads(3, 2, 64, 1), 1, 1, 1) == -1
    assert lib.nmg_attention_workspace_bytes(nmg._Heads(2, 2, 64, 1), 0, 1, 1) == -1


def test_bindings_refuse_cpu_tensors(lib):
    x, pos = torch.zeros(64, 4), torch.zeros(4, dtype=torch.int32)
    table, off = torch.zeros(2, 32, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        nmg.rotary(x, 1, table, pos)
    with pytest.raises(ValueError):
        nmg.qk_norm_rotary(x, x, 1, 1, None, None)
    with pytest.raises(ValueError):
        nmg.attention(x, x, x, 1, 1, off, off[:1], off[1:])
    with pytest.raises(ValueError):
        nmg.tree_attention(x, x, x, 1, 1, off, off[:1], off[1:], torch.zeros((4, 4), dtype=torch.uint8))
    with pytest.raises(TypeError):
        nmg.rotary(x.double(), 1, table, pos)


@gpu
def test_binding_refusals(dev):
    x = torch.zeros(128, 6, device=dev)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)
    table, pos = torch.zeros(2, 32, 8, device=dev), i32(6)
    for bad in (dict(heads=3), dict(table=table.double()), dict(table=table[:, :, ::2]),
                dict(positions=pos.long()), dict(positions=pos[:5]), dict(layout="other"),
                dict(out=torch.zeros(128, 5, device=dev)), dict(X=x.t()), dict(out=x.half())):
        kw = dict(X=x, heads=2, table=table, positions=pos)
        with pytest.raises(ValueError):
            nmg.rotary(**{**kw, **bad})
    w = torch.ones(64, device=dev)
    for bad in (dict(K=x[:64]), dict(q_weight=w[:32]), dict(q_weight=w.half()), dict(K=x[:, :5])):
        kw = dict(Q=x, K=x, heads=2, kv_heads=2, q_weight=w, k_weight=w, table=table, positions=pos)
        with pytest.raises(ValueError):
            nmg.qk_norm_rotary(**{**kw, **bad})
    with pytest.raises(TypeError):
        nmg.qk_norm_rotary(x, x.half(), 2, 2, w, w, table, pos)
    kw = dict(Q=x, K=x, V=x, heads=2, kv_heads=2, q_offsets=i32(2), kv_begin=i32(1), kv_end=i32(1))
    for bad in (dict(V=x[:64]), dict(kv_heads=1), dict(q_offsets=i32(3)), dict(kv_end=i32(2)),
                dict(kv_begin=torch.zeros(1, device=dev)), dict(key_mask=torch.ones(6, device=dev)),
                dict(key_mask=torch.ones(5, dtype=torch.bool, device=dev)), dict(Q=x.t())):
        with pytest.raises(ValueError):
            nmg.attention(**{**kw, **bad})
    with pytest.raises(TypeError):
        nmg.attention(**{**kw, "K": x.half()})
    with pytest.raises(nmg.NmgError):
        nmg.attention(**kw, scale=-1.0)
    for tree in (torch.ones((5, 6), dtype=torch.bool, device=dev), torch.ones((6, 6), device=dev)):
        with pytest.raises(ValueError):
            nmg.tree_attention(**kw, tree=tree)


def test_attention_size_limits(lib):
    """Rows of K or V of 2^28 bytes, and trees of 2^31, do not fit the kernels'
    offsets."""
    p = ctypes.c_void_p(1 << 20)

    def call(ldk, D=64, dtype=nmg.F16, ldt=None):
        h, s = nmg._Heads(1, 1, D, dtype), nmg._Sequences(1, 1 << 20, 1 << 20, 1 << 20)
        args = (h, s, p, 4, 4, p, ldk, p, 16, 16)
        if ldt is None:
            return lib.nmg_attention(*args, None, 0.125, p, 4, None, 0, None)
        return lib.nmg_tree_attention(*args, p, ldt, 4, 0.125, p, 4, None, 0, None)

    assert call(1 << 28) == call(1 << 27, dtype=nmg.F32) == nmg.ERR_UNSUPPORTED
    assert call(16, ldt=1 << 29) == nmg.ERR_UNSUPPORTED


@gpu
def test_binding_counts_arguments(dev):
    """The compiled marshalling refuses what is not a tensor or a number."""
    x, table = torch.zeros(64, 4, device=dev), torch.zeros(2, 32, 8, device=dev)
    pos = torch.zeros(4, dtype=torch.int32, device=dev)
    for bad in (dict(X=[1, 2]), dict(heads="a"), dict(table=3), dict(positions=None), dict(heads=1.5)):
        with pytest.raises(TypeError):
            nmg.rotary(**{**dict(X=x, heads=1, table=table, positions=pos), **bad})
    with pytest.raises(ValueError):
        nmg.rotary(x, 1, table, pos, layout=None)
    with pytest.raises(ValueError):
        nmg.rotary(x, 1 << 40, table, pos)
