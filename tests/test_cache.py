"""The 8-bit cache: drafted tokens in, kept ones to pages, attention over pages and
open tokens, pages handed out, shared, given back and moved.

References are numpy and binary64 on the CPU, written from ``include/nmg.h``.  What
is stored (codes, scales, open tokens, tables, counts) has to be equal.  Attention,
with u = 2^-24 and n keys:

  scores     e_s = (D + 8) u max_j scale sum_d |q_d k_dj|: D products and sums in
             binary32, the factor scale * log2 e (two roundings), its product, the difference
             from the maximum and the exponential.  Codes times scales are
             exact.
  weights    off by a factor 1 + 2 e_s; sums add n + 32 roundings:
             (4 e_s + (n + 32) u) sum_j p_j |v_j|
  binary16   weights are rounded once for the sums and not for the total: 2^-11
             sum_j p_j |v_j|, and 2^-34 n max |v| where they are subnormal (the
             largest is 2^9 to 2^15, a subnormal's half step 2^-25); outputs 2^-11 |y| + 2^-24
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2304_07613_amd import nmg

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16}
NP = {"f32": np.float32, "f16": np.float16}
CODES = {"e4m3": 448.0, "int8": 127.0}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nmg.lib()
    return DEV


def rand(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float32)


def i32(values, dev=DEV):
    return torch.tensor(list(values), dtype=torch.int32, device=dev)


def offsets(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


# ---------------------------------------------------------------- references

def codes64(x, fmt, largest):
    """(codes as values, scale) of one block, from the definition."""
    x = x.astype(np.float64)
    if not np.isfinite(x).all():
        return np.zeros(x.shape), math.nan
    most, top, e = CODES[fmt], np.abs(x).max(), -126
    while top > most * 2.0 ** e:
        e += 1
    y = x / 2.0 ** e
    if fmt == "int8":
        step = np.ones(y.shape)
    else:
        step = 2.0 ** (np.frexp(np.maximum(np.abs(y), 2.0 ** -6))[1] - 4)   # 4 significant bits
    c = np.rint(y / step) * step                                            # ties to even
    over = np.abs(c) * 2.0 ** e > largest
    below = np.abs(c) - (1.0 if fmt == "int8" else 16.0)                     # of 256, or 64
    return np.where(over, np.sign(c) * below, c), 2.0 ** e


class Model:
    """What a cache should hold, token by token."""

    def __init__(self, layers, heads, dim, sequences, pages, row, room, block, fmt, dtype):
        self.shape = (layers, heads, dim, sequences, pages, row, room, block)
        self.fmt, self.dtype, self.largest = fmt, dtype, float(np.finfo(NP[dtype]).max)
        wide = (dim + 15) // 16 * 16
        self.kp, self.vp = np.zeros((layers, pages, heads, block, wide)), np.zeros((layers, pages, heads, dim, block))
        self.ks, self.vs = np.zeros((layers, pages, heads)), np.zeros((layers, pages, heads))
        self.ko = np.zeros((layers, sequences, heads, room, wide))
        self.vo = np.zeros((layers, sequences, heads, dim, room))
        self.table, self.refs = np.full((sequences, row), -1), np.zeros(pages, int)
        self.n = np.zeros(sequences, int)

    def append(self, layer, K, V, q):
        L, H, D, B, P, row, room, block = self.shape
        for b in range(B):
            for i in range(q[b + 1] - q[b]):
                if self.n[b] % block + i >= room:
                    break
                at = (self.n[b] + i) % room
                self.ko[layer, b, :, at] = 0
                self.ko[layer, b, :, at, :D] = K[:, q[b] + i].reshape(H, D)
                self.vo[layer, b, :, :, at] = V[:, q[b] + i].reshape(H, D)

    def commit(self, kept):
        """kept: for every sequence the numbers of the drafted tokens that stay."""
        L, H, D, B, P, row, room, block = self.shape
        for b in range(B):
            n = self.n[b]
            full, picks = n // block * block, list(kept[b])[: max(0, room - n % block)]
            while True:                            # as far as there are pages
                whole = (n - full + len(picks)) // block
                held = [j for j in range(whole) if full // block + j < row and self.table[b, full // block + j] >= 0]
                if len(held) == whole:
                    break
                first = min(set(range(whole)) - set(held))
                picks = picks[: (first + 1) * block - 1 - (n - full)]
            slots = [p % room for p in range(full, n)] + [(n + p) % room for p in picks]
            k, v = self.ko[:, b][:, :, slots].copy(), self.vo[:, b][:, :, :, slots].copy()
            for j in range(whole):
                page = self.table[b, full // block + j]
                for layer in range(L):
                    for h in range(H):
                        s = slice(j * block, (j + 1) * block)
                        self.kp[layer, page, h], self.ks[layer, page, h] = codes64(k[layer, h, s], self.fmt, self.largest)
                        self.vp[layer, page, h], self.vs[layer, page, h] = codes64(v[layer, h, :, s], self.fmt, self.largest)
            for u in range(whole * block, len(slots)):
                self.ko[:, b, :, (full + u) % room] = k[:, :, u]
                self.vo[:, b, :, :, (full + u) % room] = v[:, :, :, u]
            self.n[b] = n + len(picks)

    def reserve(self, tokens):
        B, P, row, block = self.shape[3], self.shape[4], self.shape[5], self.shape[7]
        missing = 0
        for b in range(B):
            for j in range(self.n[b] // block, (self.n[b] + tokens[b]) // block):
                if j < row and self.table[b, j] >= 0:
                    continue
                free = np.flatnonzero(self.refs == 0)
                if j >= row or not len(free):
                    missing += 1
                    continue
                self.table[b, j] = free[0]
                self.refs[free[0]] = 1
        return missing

    def release(self, b):
        for p in self.table[b][self.table[b] >= 0]:
            self.refs[p] -= 1
        self.table[b], self.n[b] = -1, 0

    def fork(self, sources, targets):
        room, block = self.shape[6], self.shape[7]
        for a, b in zip(sources, targets):
            self.release(b)
            n = self.n[a]
            for j in range(n // block):
                self.table[b, j] = self.table[a, j]
                self.refs[self.table[a, j]] += 1
            slots = [p % room for p in range(n // block * block, n)]
            self.ko[:, b][:, :, slots] = self.ko[:, a][:, :, slots]
            self.vo[:, b][:, :, :, slots] = self.vo[:, a][:, :, :, slots]
            self.n[b] = n

    def compact(self):
        used = self.refs > 0
        live = int(used.sum())
        source, hole = np.flatnonzero(used[live:]) + live, np.flatnonzero(~used[:live])
        for x in (self.kp, self.vp, self.ks, self.vs):
            x[:, hole] = x[:, source]
        self.refs[hole] = self.refs[source]
        self.refs[source] = 0
        for a, b in zip(source, hole):
            self.table[self.table == a] = b
        return live

    def tokens(self, layer, b, drafts):
        """Keys and values (heads x tokens x dim) of what sequence b holds."""
        L, H, D, B, P, row, room, block = self.shape
        n = self.n[b]
        pages = self.table[b, : n // block]
        k = (self.kp[layer, pages] * self.ks[layer, pages][..., None, None])[..., :D]
        v = (self.vp[layer, pages] * self.vs[layer, pages][..., None, None])
        k = k.transpose(1, 0, 2, 3).reshape(H, -1, D)
        v = v.transpose(1, 0, 3, 2).reshape(H, -1, D)
        last = min(n + drafts, n // block * block + room)
        slots = [p % room for p in range(n // block * block, last)]
        return (np.concatenate((k, self.ko[layer, b][:, slots][..., :D]), 1),
                np.concatenate((v, self.vo[layer, b][:, :, slots].transpose(0, 2, 1)), 1))


def attend64(model, layer, Q, heads, q, tree=None, scale=None):
    """(result, error bound without the output's rounding) of every column."""
    L, H, D, B, P, row, room, block = model.shape
    scale, share = scale or D ** -0.5, heads // H
    out, bound = np.zeros(Q.shape), np.zeros(Q.shape)
    half = model.dtype == "f16"
    for b in range(B):
        T = q[b + 1] - q[b]
        k, v = model.tokens(layer, b, T)
        n, m = model.n[b], k.shape[1]
        for t in range(T):
            see = np.ones(m, bool)
            i = np.arange(m - n)
            see[n:] = i <= t if tree is None else (i < tree.shape[1]) & (
                tree[q[b] + t][np.minimum(i, tree.shape[1] - 1)] != 0)
            for h in range(heads):
                x = Q[h * D:(h + 1) * D, q[b] + t].astype(np.float64)
                kk, vv = k[h // share][see], v[h // share][see]
                if not len(kk):
                    continue
                s = scale * (kk @ x)
                at = slice(h * D, (h + 1) * D)
                if np.isnan(s).any() or s.max() == np.inf:
                    out[at, q[b] + t] = math.nan
                    continue
                if s.max() == -np.inf:
                    continue
                p = np.exp(s - s.max())
                p /= p.sum()
                e = (D + 8) * U * scale * (np.abs(np.where(np.isfinite(kk), kk, 0)) @ np.abs(x)).max()
                out[at, q[b] + t] = p @ vv
                w = np.where(np.isfinite(vv), np.abs(vv), 0)
                bound[at, q[b] + t] = (4 * e + (m + 32) * U + half * 2.0 ** -11) * (p @ w) + \
                    half * 2.0 ** -34 * m * w.max()
    return out, bound


def check(got, ref, dtype):
    ref, bound = ref
    bound = bound + (2.0 ** -11 * np.abs(ref) + 2.0 ** -24 if dtype == "f16" else 2 * U * np.abs(ref) + 2.0 ** -140)
    got = got.double().cpu().numpy()
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    worst = (np.abs(got - ref)[fine] / bound[fine]).max() if fine.any() else 0.0
    assert worst <= 1, f"error {worst:.2f} times its bound"
    return worst


class Both:
    """A cache on the GPU and its model, through the same calls."""

    def __init__(self, dev, layers=1, heads=2, dim=64, sequences=3, pages=40, row=12, room=128, block=64,
                 fmt="e4m3", dtype="f16"):
        self.model = Model(layers, heads, dim, sequences, pages, row, room, block, fmt, dtype)
        self.cache = nmg.Cache.empty(layers, heads, dim, sequences, pages, row, room, block, fmt, DT[dtype], dev)
        for t in (self.cache.k_open, self.cache.v_open):
            t.fill_(math.nan)                          # of what nobody wrote nothing may be seen
        self.lengths = i32([0] * sequences, dev)
        self.seed, self.dtype, self.dev = 1, dtype, dev
        self.rows = heads * dim

    def draft(self, counts, change=None):
        q = offsets(counts)
        N = max(1, int(q[-1]))
        for layer in range(self.model.shape[0]):
            self.seed += 2
            K, V = (rand(self.seed + i, self.rows, N).astype(NP[self.dtype]) for i in (0, 1))
            if change:
                change(K, V, q)
            self.model.append(layer, K, V, q)
            kv = torch.from_numpy(np.concatenate((K, V))).to(self.dev)
            nmg.cache_append(self.cache, layer, kv[: self.rows], kv[self.rows:], torch.from_numpy(q).to(self.dev),
                             self.lengths)
        return q

    def keep(self, kept, as_list=True):
        """The drafted tokens that stay; pages are there for them."""
        kept_offsets = torch.from_numpy(offsets([len(k) for k in kept])).to(self.dev)
        values = i32([i for k in kept for i in k], self.dev) if as_list else None
        self.model.commit(kept)
        self.lengths = nmg.cache_commit(self.cache, self.lengths, kept_offsets, values)

    def reserve(self, tokens):
        missing = nmg.cache_reserve(self.cache, self.lengths, i32(tokens, self.dev))
        assert missing.item() == self.model.reserve(tokens)

    def grow(self, counts, change=None):
        """Every sequence gets `counts` more tokens, a room at a time."""
        left, room = list(counts), self.model.shape[6] - self.model.shape[7] + 1
        while any(left):
            now = [min(n, room) for n in left]
            self.draft(now, change)
            self.reserve(now)
            self.keep([list(range(n)) for n in now], as_list=False)
            left = [a - b for a, b in zip(left, now)]

    def same(self):
        m, c = self.model, self.cache
        assert self.lengths.tolist() == m.n.tolist()
        assert np.array_equal(c.table.cpu().numpy(), m.table)
        assert np.array_equal(c.references.cpu().numpy(), m.refs)
        for name, ref in (("k_pages", m.kp), ("v_pages", m.vp), ("k_scales", m.ks), ("v_scales", m.vs)):
            got = getattr(c, name).float().cpu().numpy().astype(np.float64)
            assert np.array_equal(got, ref, equal_nan=True), name
        room, block = m.shape[6], m.shape[7]
        k, v = (t.cpu().numpy() for t in (c.k_open, c.v_open))
        for b in range(m.shape[3]):
            slots = [p % room for p in range(m.n[b] // block * block, m.n[b])]
            assert np.array_equal(k[:, b][:, :, slots].astype(np.float64), m.ko[:, b][:, :, slots], equal_nan=True)
            assert np.array_equal(v[:, b][..., slots].astype(np.float64), m.vo[:, b][..., slots], equal_nan=True)

    def attend(self, heads, q, tree=None, layer=0, longest=None, scale=None, sharp=1.5, Q=None, out=None):
        D = self.model.shape[2]
        if Q is None:
            self.seed += 1
            Q = (sharp * rand(self.seed, heads * D, max(1, int(q[-1])))).astype(NP[self.dtype])
        got = nmg.cache_attention(self.cache, layer, torch.from_numpy(Q).to(self.dev), heads,
                                  torch.from_numpy(q).to(self.dev), self.lengths,
                                  None if tree is None else torch.from_numpy(tree).to(self.dev), longest, scale, out)
        with np.errstate(all="ignore"):
            ref = attend64(self.model, layer, Q, heads, q, tree, scale)
        return check(got[:, : q[-1]], (ref[0][:, : q[-1]], ref[1][:, : q[-1]]), self.dtype)


def random_tree(seed, counts, width=None):
    rng, q = np.random.default_rng(seed), offsets(counts)
    width = width or max(1, max(counts))
    tree = np.zeros((max(1, int(q[-1])), width), np.uint8)
    for b, T in enumerate(counts):
        for i in range(T):
            up = int(rng.integers(-1, i)) if i else -1
            if up >= 0:
                tree[q[b] + i] = tree[q[b] + up]
            if i < width:
                tree[q[b] + i, i] = 1 + i % 200
    return tree


# ------------------------------------------------------------------ storage

@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,dim,block,room", [(2, 64, 64, 128), (1, 128, 128, 256), (3, 33, 64, 192),
                                                  (1, 1, 64, 64), (1, 256, 128, 128), (2, 80, 128, 384)])
def test_tokens_become_pages(dev, heads, dim, block, room, fmt, dtype):
    b = Both(dev, 2, heads, dim, 3, 30, 9, room, block, fmt, dtype)
    most = room - block + 1
    for counts in ([1, 0, most], [most, 1, 2], [0, 0, 0], [most, most // 2, 1], [1, 1, 1], [most, most, most]):
        print(counts, flush=True)
        b.draft(counts)
        b.reserve(counts)
        b.keep([list(range(n)) for n in counts], as_list=False)
        b.same()
    b.grow([block, 1, 2 * block])
    b.same()
    assert b.model.n.max() > 2 * block


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("block,room", [(64, 128), (128, 384), (64, 256)])
def test_paths_through_drafts(dev, block, room, dtype):
    rng = np.random.default_rng(block + room)
    b = Both(dev, 2, 2, 48, 4, 60, 20, room, block, "e4m3", dtype)
    for step in range(12):
        counts = [int(rng.integers(0, room - block + 2)) for _ in range(4)]
        b.draft(counts)
        kept = [sorted(rng.choice(n, rng.integers(0, n + 1), replace=False).tolist()) if n else [] for n in counts]
        if step % 3 == 0:
            kept = [list(range(n // 2, n)) for n in counts]       # the last ones, moved far
        if step % 5 == 0:
            kept[1] = []
        b.reserve([len(k) for k in kept])
        print(step, counts, [len(k) for k in kept], flush=True)
        b.keep(kept)
        b.same()


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_rounding_of_codes(dev, fmt, dtype):
    """Ties, largest and smallest values, blocks of zeros, scales at both ends, and
    values that are not finite."""
    rng = np.random.default_rng(5)
    top = float(np.finfo(NP[dtype]).max)
    tiny = float(np.finfo(NP[dtype]).smallest_subnormal)
    fills = [lambda x: rng.standard_normal(x.shape) * 10, lambda x: np.zeros(x.shape),
             lambda x: rng.integers(-2048, 2049, x.shape) / 8, lambda x: rng.integers(-3, 4, x.shape) * tiny,
             lambda x: rng.uniform(-top, top, x.shape), lambda x: np.where(rng.random(x.shape) < .5, top, -top),
             lambda x: np.full(x.shape, CODES[fmt]), lambda x: np.nextafter(np.full(x.shape, CODES[fmt], NP[dtype]), top),
             lambda x: np.exp2(rng.uniform(-14, 15, x.shape)), lambda x: rng.integers(0, 512, x.shape) - 255.5]
    B = len(fills)
    b = Both(dev, 1, 2, 64, B + 2, 40, 2, 64, 64, fmt, dtype)

    def fill(K, V, q):
        for i, f in enumerate(fills + [fills[0]] * 2):
            for x in (K, V):
                x[:, q[i]:q[i + 1]] = f(x[:, q[i]:q[i + 1]]).astype(NP[dtype])
        K[3, q[B] + 7], V[70, q[B + 1]] = math.nan, -math.inf

    b.draft([64] * (B + 2), fill)        # (room 64 takes as many while nothing is kept)
    b.reserve([64] * (B + 2))
    b.keep([list(range(64))] * (B + 2), as_list=False)
    b.same()
    scales = b.cache.k_scales[0][b.cache.table[:, 0].long()]
    assert torch.isnan(scales[B, 0]) and not torch.isnan(scales[B, 1]) and not torch.isnan(scales[:B]).any()
    codes = b.cache.k_pages.float() * b.cache.k_scales[..., None, None]
    assert codes[codes.isfinite()].abs().max() <= top and (~codes.isfinite()).sum() == 64 * 64


@gpu
def test_kept_only_as_far_as_pages_and_room(dev):
    b = Both(dev, 1, 1, 16, 3, 3, 2, 128, 64, "e4m3", "f16")
    b.draft([65, 65, 65])
    b.reserve([65, 65, 65])
    b.keep([list(range(65))] * 3, as_list=False)
    b.same()
    b.draft([65, 64, 3])
    b.reserve([65, 64, 3])                 # no page is free any more
    b.keep([list(range(65)), list(range(0, 64)), [0, 2]])
    b.same()
    assert b.model.n.tolist() == [127, 127, 67]
    nmg.cache_free(b.cache, b.lengths, [2])
    b.model.release(2)
    b.reserve([1, 0, 0])
    b.draft([65, 0, 200])                  # past the room of sequence 2
    b.keep([[5, 64], [], list(range(200))])
    b.same()


@gpu
def test_an_empty_list_keeps_nothing(dev):
    b = Both(dev)
    b.grow([70, 3, 0])
    b.draft([5, 5, 5])
    b.keep([[], [], []])
    b.same()
    assert b.lengths.tolist() == [70, 3, 0]


@gpu
def test_rows_and_slots_of_others_stay(dev):
    """A call touches the sequences it names: what lies around their tokens, in
    rings and pages, keeps its bits."""
    b = Both(dev, 2, 2, 40, 4, 20, 6, 128, 64)
    b.grow([70, 10, 130, 0])
    before = {k: t.view(torch.uint8).clone() for k, t in b.cache.buffers.items()}
    b.draft([0, 20, 0, 0])
    for name in ("k_open", "v_open"):
        now, old = getattr(b.cache, name).view(torch.uint8), before[name]
        for s in (0, 2, 3):
            assert torch.equal(now[:, s], old[:, s])
    assert (b.cache.k_open[:, 1, :, 30:].isnan()).all()      # slots behind the draft
    for name in ("k_pages", "v_pages", "table", "references"):
        assert torch.equal(getattr(b.cache, name).view(torch.uint8), before[name])
    before = {k: t.view(torch.uint8).clone() for k, t in b.cache.buffers.items()}
    nmg.cache_fork(b.cache, b.lengths, [1], [3])
    b.model.fork([1], [3])
    b.same()
    for name in ("k_open", "v_open"):
        now, old = getattr(b.cache, name).view(torch.uint8), before[name]
        assert torch.equal(now[:, :3], old[:, :3])
    assert (b.cache.k_open[:, 3, :, 10:].isnan()).all() and (b.cache.v_open[:, 3, :, :, 10:].isnan()).all()


# ---------------------------------------------------------------------- pages

@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_requests_come_and_go(dev, dtype):
    rng = np.random.default_rng(11)
    b = Both(dev, 2, 2, 32, 6, 50, 8, 128, 64, "int8", dtype)
    for step in range(20):
        counts = [int(rng.integers(0, 66)) if rng.random() < .7 else 0 for _ in range(6)]
        b.draft(counts)
        b.reserve(counts)
        b.keep([list(range(n)) for n in counts], as_list=step % 2 == 0)
        if step % 3 == 1:
            order = rng.permutation(6).tolist()
            pairs = int(rng.integers(1, 4))
            nmg.cache_fork(b.cache, b.lengths, order[3:3 + pairs], order[:pairs])
            b.model.fork(order[3:3 + pairs], order[:pairs])
        if step % 4 == 2:
            gone = rng.permutation(6)[: rng.integers(1, 3)].tolist()
            nmg.cache_free(b.cache, b.lengths, gone)
            for s in gone:
                b.model.release(s)
        if step % 5 == 3:
            assert nmg.cache_compact(b.cache).item() == b.model.compact()
        print(step, counts, b.model.n.tolist(), flush=True)
        b.same()
    b.attend(4, b.draft([3, 1, 2, 0, 5, 1]))


@gpu
def test_compaction_into_other_tables(dev):
    b = Both(dev, 1, 1, 16, 4, 30, 6, 128, 64)
    b.grow([200, 130, 70, 300])
    nmg.cache_fork(b.cache, b.lengths, [3], [1])
    b.model.fork([3], [1])
    nmg.cache_free(b.cache, b.lengths, [0])
    b.model.release(0)
    table, references = b.cache.table.clone(), b.cache.references.clone()
    old = b.cache.table.clone(), b.cache.references.clone()
    for _ in range(2):       # sources stay as they are, so a second call does the same
        live = nmg.cache_compact(b.cache, table, references)
        assert torch.equal(b.cache.table, old[0]) and torch.equal(b.cache.references, old[1])
    assert live.item() == b.model.compact()
    b.cache.table.copy_(table)
    b.cache.references.copy_(references)
    b.same()
    assert nmg.cache_compact(b.cache).item() == live.item()      # nothing left to move
    b.same()


@gpu
@pytest.mark.parametrize("pages,row,sequences", [(1, 1, 1), (3000, 2, 1100), (5000, 40, 2100)])
def test_many_pages_and_sequences(dev, pages, row, sequences):
    rng = np.random.default_rng(pages)
    cache = nmg.Cache.empty(1, 1, 1, sequences, pages, row, 64, 64, device=dev)
    model = Model(1, 1, 1, sequences, pages, row, 64, 64, "e4m3", "f16")
    tokens = rng.integers(0, 64 * row, sequences)
    lengths = i32([0] * sequences)
    for _ in range(2):
        assert nmg.cache_reserve(cache, lengths, i32(tokens)).item() == model.reserve(tokens)
        assert np.array_equal(cache.table.cpu().numpy(), model.table)
        assert np.array_equal(cache.references.cpu().numpy(), model.refs)
        gone = np.flatnonzero(rng.random(sequences) < .5).tolist()
        nmg.cache_free(cache, lengths, gone)
        for b in gone:
            model.release(b)
        assert nmg.cache_compact(cache).item() == model.compact()
        assert np.array_equal(cache.table.cpu().numpy(), model.table)
        assert np.array_equal(cache.references.cpu().numpy(), model.refs)


@gpu
def test_compaction_moves_whole_pages(dev):
    """Pages of many chunks, random bytes."""
    cache = nmg.Cache.empty(3, 5, 96, 2, 37, 20, 128, 128, "int8", device=dev)
    gen = torch.Generator(device=dev).manual_seed(1)
    for t in (cache.k_pages, cache.v_pages):
        t.copy_(torch.randint(-128, 128, t.shape, generator=gen, device=dev, dtype=torch.int8))
    for t in (cache.k_scales, cache.v_scales):
        t.copy_(torch.rand(t.shape, generator=gen, device=dev))
    used = torch.randperm(37, generator=gen, device=dev)[:17]
    cache.references[used] = 1
    cache.table[0, :17] = used.int()
    old = {k: getattr(cache, k).clone() for k in ("k_pages", "v_pages", "k_scales", "v_scales")}
    assert nmg.cache_compact(cache).item() == 17
    now = cache.table[0, :17].long()
    assert now.max() == 16 and cache.references.tolist() == [1] * 17 + [0] * 20
    for name, t in old.items():
        assert torch.equal(getattr(cache, name)[:, now], t[:, used])


# ------------------------------------------------------------------ attention

SHAPES = [(2, 2, 64), (4, 2, 64), (8, 1, 32), (4, 1, 128), (3, 3, 80), (2, 1, 96), (6, 2, 33), (2, 2, 1),
          (2, 1, 256), (1, 1, 200), (5, 1, 17)]


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
def test_attention_of_single_tokens_and_trees(dev, heads, kv_heads, dim, dtype):
    for block, fmt in ((64, "e4m3"), (128, "int8")):
        b = Both(dev, 2, kv_heads, dim, 4, 30, 8, 2 * block, block, fmt, dtype)
        for kept in ([0, 1, block - 1, block], [1, 70, 66, 3], [130, 0, 200, 1]):
            b.grow(kept)
            for counts in ([1, 1, 1, 1], [3, 0, 17, 1], [block + 1, 2, 5, 33]):
                print(f"{heads}/{kv_heads} x {dim} {dtype} {fmt} kept {b.model.n.tolist()} drafts {counts}", flush=True)
                q = b.draft(counts)
                b.attend(heads, q, layer=1)
                b.attend(heads, q, random_tree(dim, counts))


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attention_over_long_caches(dev, fmt, dtype):
    """Keys split into parts, with and without scratch memory."""
    b = Both(dev, 1, 1, 64, 2, 200, 120, 512, 64, fmt, dtype)
    b.grow([5000, 37])
    for counts in ([1, 1], [40, 3]):
        q = b.draft(counts)
        for longest in (None, 5000, 64, 1):
            print(fmt, dtype, counts, longest, flush=True)
            b.attend(4, q, longest=longest)
            b.attend(4, q, random_tree(3, counts), longest=longest)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("sequences", [64, 65, 200, 4500])
def test_many_sequences(dev, sequences, dtype):
    """Few with a draft among many, some of them long; the splits aim at more workgroups than
    there are row tiles, or not."""
    rng = np.random.default_rng(sequences)
    b = Both(dev, 1, 1, 16, sequences, 60 + sequences // 64, 40, 256, 64, "int8", dtype)
    grown = [0] * sequences
    for s in rng.permutation(sequences)[:20]:
        grown[s] = int(rng.integers(1, 100))
    grown[3] = 1500
    b.grow(grown)
    for most in (1, 100):
        counts = [0] * sequences
        for s in rng.permutation(sequences)[:12]:
            counts[s] = int(rng.integers(1, most + 1))
        counts[3] = most
        print(sequences, dtype, counts[:20], flush=True)
        q = b.draft(counts)
        b.attend(2, q)
        b.attend(2, q, random_tree(1, counts), longest=1500)
        kept = [list(range(0, n, 2)) for n in counts]
        b.reserve([len(k) for k in kept])
        b.keep(kept)
        b.same()


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_prompt_in_pieces(dev, dtype):
    """A prompt's pieces attend to what came before and causally to themselves."""
    b = Both(dev, 1, 2, 64, 2, 60, 16, 512, 64, "e4m3", dtype)
    for counts in ([300, 449], [1, 200], [130, 7]):
        print(counts, flush=True)
        q = b.draft(counts)
        b.attend(4, q)
        b.reserve(counts)
        b.keep([list(range(n)) for n in counts], as_list=False)
    b.same()


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_values_that_are_not_finite_reach_those_who_see_them(dev, dtype):
    for bad in (math.nan, math.inf, -math.inf):
        b = Both(dev, 1, 2, 48, 3, 20, 6, 192, 64, "e4m3", dtype)
        b.grow([70, 5, 100])
        counts = [9, 70, 1]
        tree = random_tree(4, counts)

        def change(K, V, q):
            V[3, q[0] + 4], V[60, q[1] + 66], K[10, q[1] + 2] = bad, bad, bad

        print(bad, dtype, flush=True)
        q = b.draft(counts, change)
        b.attend(4, q, tree)
        b.attend(2, q)
        rng = np.random.default_rng(3)
        Q = rng.standard_normal((96, q[-1])).astype(NP[dtype])
        Q[5, 2], Q[50, 30] = bad, bad
        b.draft(counts)
        b.attend(2, q, tree, Q=Q)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_pages_that_are_not_finite(dev, fmt, dtype):
    b = Both(dev, 1, 2, 32, 3, 20, 6, 128, 64, fmt, dtype)

    def change(K, V, q):
        K[3, q[0] + 4], V[40, q[1] + 3] = math.nan, math.inf

    b.grow([64, 64, 64], change)
    b.grow([70, 3, 1])
    b.attend(4, b.draft([2, 1, 20]))
    nmg.cache_free(b.cache, b.lengths, [0, 1])
    for s in (0, 1):
        b.model.release(s)
    b.grow([130, 130, 10])           # the same pages again, finite now
    worst = b.attend(4, b.draft([2, 1, 20]))
    assert worst <= 1


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rows_that_see_nothing(dev, dtype):
    b = Both(dev, 1, 1, 64, 3, 20, 6, 128, 64, "e4m3", dtype)
    b.grow([0, 0, 66])
    counts = [5, 20, 3]
    q = b.draft(counts)
    tree = random_tree(1, counts)
    tree[2], tree[7], tree[-1] = 0, 0, 0
    b.attend(2, q, tree)
    b.attend(2, q, tree[:, :3].copy())            # narrower than the drafts
    b.attend(2, q, np.concatenate((tree, np.ones_like(tree)), 1))      # wider


@gpu
def test_scores_of_minus_infinity(dev):
    b = Both(dev, 1, 1, 16, 2, 4, 2, 128, 64, "e4m3", "f32")
    b.draft([2, 3], lambda K, V, q: K.__setitem__((0, slice(None)), -math.inf))
    q = offsets([2, 3])
    Q = np.zeros((16, 5), np.float32)
    Q[0] = 1.0
    got = nmg.cache_attention(b.cache, 0, torch.from_numpy(Q).to(dev), 1, torch.from_numpy(q).to(dev), b.lengths)
    # 0 * finite + 1 * -inf: every score is minus infinity
    assert (got == 0).all()


@gpu
@pytest.mark.parametrize("k_size,v_size,q_size", [(1e30, 1e30, 1e-30), (1e-30, 1e-30, 1e30), (1e18, 3e38, 1e-18),
                                                  (1.0, 1e-37, 1.0), (3e38, 1.0, 1e-38)])
def test_values_of_any_size_in_binary32(dev, k_size, v_size, q_size):
    b = Both(dev, 1, 1, 64, 2, 20, 6, 128, 64, "e4m3", "f32")

    def change(K, V, q):
        K *= np.float32(k_size) / 5
        V *= np.float32(v_size) / 5

    b.grow([130, 10], change)
    q = b.draft([5, 20], change)
    Q = (rand(3, 128, 25) * np.float32(q_size)).astype(np.float32)
    b.attend(2, q, Q=Q)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 64), (3, 1, 80), (6, 1, 96), (4, 1, 128), (2, 1, 200),
                                                (2, 2, 256), (8, 1, 16)])
def test_many_rows(dev, heads, kv_heads, dim, dtype):
    """Drafts long enough for every kernel: sequences of unequal length, a wave or a
    workgroup without rows, the last key tile partly filled, values that are not finite."""
    for block, fmt in ((64, "int8"), (128, "e4m3")):
        b = Both(dev, 1, kv_heads, dim, 4, 40, 8, 384, block, fmt, dtype)
        b.grow([200, 0, 129, 64])
        for counts in ([130, 255, 1, 70], [64, 64, 64, 64], [0, 257, 0, 0]):
            print(f"{heads}/{kv_heads} x {dim} {dtype} {fmt} {counts}", flush=True)
            tree = random_tree(dim, counts)
            q = b.draft(counts)
            b.attend(heads, q)
            b.attend(heads, q, tree)
            b.attend(heads, q, tree, longest=4000)
            q = b.draft(counts, lambda K, V, q: V.__setitem__((dim // 2, slice(None, None, 50)), math.nan))
            b.attend(heads, q, tree)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_many_rows_over_parts(dev, dtype):
    for dim, fmt in ((64, "e4m3"), (128, "int8"), (256, "e4m3")):
        b = Both(dev, 1, 1, dim, 2, 60, 50, 512, 64, fmt, dtype)
        b.grow([2000, 300])
        q = b.draft([100, 37])
        for longest in (None, 2000, 100):
            print(dim, fmt, dtype, longest, flush=True)
            b.attend(3, q, random_tree(dim, [100, 37]), longest=longest)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_pages_of_very_different_sizes(dev, dtype):
    """Attention that looks at one page whose values are tiny beside the others'."""
    b = Both(dev, 1, 1, 64, 1, 20, 8, 128, 64, "e4m3", dtype)
    sizes = iter((1.0, 1e-4, 0.0, 300.0, 1e-6))

    def change(K, V, q):
        V *= NP[dtype](next(sizes))

    for _ in range(5):
        b.draft([64], change)
        b.reserve([64])
        b.keep([list(range(64))], as_list=False)
    q = b.draft([4], lambda K, V, q: V.__imul__(NP[dtype](1e-3)))
    for at in range(5):
        k = b.model.kp[0, b.model.table[0, at], 0, 5] * b.model.ks[0, b.model.table[0, at], 0]
        Q = np.repeat((8 * k[:, None]).astype(NP[dtype]), 4, 1)
        b.attend(1, q, Q=Q)


@gpu
def test_offsets_past_32_bits(dev):
    """Pools and rings of more than 2^32 bytes: the last pages, layer and sequence."""
    pages = 70000
    cache = nmg.Cache.empty(2, 2, 256, 2, pages, 8, 128, 64, device=dev)
    assert cache.k_pages[0].numel() > 1 << 31 and cache.k_pages.numel() > 1 << 32
    b = Both(dev, 2, 2, 256, 2, 8, 8, 128, 64)
    b.grow([200, 150])
    q = b.draft([3, 1])
    shift = pages - 8
    for name in ("k_pages", "v_pages"):
        for layer in (0, 1):
            getattr(cache, name)[layer, shift:].view(torch.uint8).copy_(getattr(b.cache, name)[layer].view(torch.uint8))
    for name in ("k_scales", "v_scales"):
        getattr(cache, name)[:, shift:] = getattr(b.cache, name)
    for name in ("k_open", "v_open"):
        getattr(cache, name).copy_(getattr(b.cache, name))
    cache.table.copy_(torch.where(b.cache.table >= 0, b.cache.table + shift, b.cache.table))
    b.cache = cache
    for layer in (0, 1):
        b.attend(4, q, layer=layer)
    cache.references[cache.table[cache.table >= 0].long()] = 1
    assert nmg.cache_compact(cache).item() == 5
    order = {p: i for i, p in enumerate(sorted(set(b.model.table[b.model.table >= 0].tolist())))}
    assert cache.table.cpu().tolist() == [[order.get(p, -1) for p in r] for r in b.model.table.tolist()]
    b.attend(4, q, layer=1)


@gpu
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_matrices_in_unusual_places(dev, dtype):
    """Odd leading dimensions and starts for Q, K, V and O; a strided tree; columns of
    no sequence are not written."""
    b = Both(dev, 1, 2, 40, 3, 20, 6, 128, 64, "int8", dtype)
    b.grow([70, 5, 0])
    counts, skip = [3, 9, 1], 4
    q = offsets(counts) + skip
    N = int(q[-1]) + 3

    def odd(rows):
        buf = torch.full((rows, N + 8), 7.0, dtype=DT[dtype], device=dev)
        return buf[:, 5:5 + N]

    K, V, Q = (rand(s, r, N).astype(NP[dtype]) for s, r in ((1, 80), (2, 80), (3, 160)))
    b.model.append(0, K, V, q)
    views = [odd(x.shape[0]) for x in (K, V, Q)]
    for view, x in zip(views, (K, V, Q)):
        view.copy_(torch.from_numpy(x))
    offs = torch.from_numpy(q).to(dev)
    nmg.cache_append(b.cache, 0, views[0], views[1], offs, b.lengths)
    tree = np.zeros((N, 12), np.uint8)
    tree[skip:skip + 13, :9] = random_tree(2, counts, 9)
    wide = torch.zeros((N, 31), dtype=torch.uint8, device=dev)
    wide[:, 3:15] = torch.from_numpy(tree).to(dev)
    out = odd(160)
    got = nmg.cache_attention(b.cache, 0, views[2], 4, offs, b.lengths, wide[:, 3:15].bool()
                              if dtype == "f16" else wide[:, 3:15], out=out)
    assert got.data_ptr() == out.data_ptr()
    ref = attend64(b.model, 0, Q, 4, q, tree)
    inside = slice(skip, int(q[-1]))
    check(out[:, inside], (ref[0][:, inside], ref[1][:, inside]), dtype)
    whole = out._base
    assert (whole[:, :5 + skip] == 7).all() and (whole[:, 5 + int(q[-1]):] == 7).all()


@gpu
def test_drafts_past_the_room_are_seen_by_none(dev):
    b = Both(dev, 1, 1, 32, 2, 8, 4, 128, 64)
    b.grow([60, 64])
    q = b.draft([100, 3])
    b.attend(1, q)
    b.attend(1, q, random_tree(1, [100, 3]))


@gpu
def test_parts_do_not_depend_on_what_lies_in_scratch_memory(dev):
    b = Both(dev, 1, 2, 64, 2, 100, 80, 128, 64)
    b.grow([4000, 900])
    q = b.draft([1, 2])
    Q = torch.randn(256, 3, device=dev).half()
    args = b.cache.c, 0, 4, i32(q).data_ptr(), b.lengths.data_ptr(), Q.data_ptr(), 3, 3, None, 0, 0, 4000, 0.125
    L, outs = nmg.lib(), []
    qo = i32(q)
    args = (b.cache.c, 0, 4, qo.data_ptr(), *args[4:])
    need = L.nmg_cache_attention_workspace_bytes(b.cache.c, 4, 3, 4000)
    assert need > 0
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=dev)
        O = torch.empty_like(Q)
        assert L.nmg_cache_attention(*args, O.data_ptr(), 3, ws.data_ptr(), need, None) == 0
        outs.append(O)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    for room in (0, 256, need // 2, need - 1):       # less of it: fewer parts, the same within rounding
        ws = torch.full((max(room, 1),), 255, dtype=torch.uint8, device=dev)
        O = torch.empty_like(Q)
        assert L.nmg_cache_attention(*args, O.data_ptr(), 3, ws.data_ptr(), room, None) == 0
        ref = attend64(b.model, 0, Q.cpu().numpy(), 4, q)
        check(O, ref, "f16")


# ----------------------------------------------- streams, graphs, bad contents

@gpu
def test_captured_steps_follow_lengths_and_tables(dev):
    """append, attention, reserve and commit captured once, replayed with the program's own
    work between the replays: each replay is one step of the eager cache."""
    a, b = Both(dev, 2, 2, 64, 3, 30, 8, 128, 64), Both(dev, 2, 2, 64, 3, 30, 8, 128, 64)
    for x in (a, b):
        x.grow([60, 3, 130])
    q = i32([0, 1, 2, 3])
    kv, Q, ones = torch.zeros(256, 3, device=dev).half(), torch.zeros(256, 3, device=dev).half(), i32([1, 1, 1])
    lengths, new = a.lengths.clone(), torch.empty_like(a.lengths)

    def step(cache, lengths, new):
        outs = []
        for layer in (0, 1):
            nmg.cache_append(cache, layer, kv[:128], kv[128:], q, lengths)
            outs.append(nmg.cache_attention(cache, layer, Q, 4, q, lengths, longest=200))
        nmg.cache_reserve(cache, lengths, ones)
        nmg.cache_commit(cache, lengths, q, out=new)
        lengths.copy_(new)
        return outs

    side = torch.cuda.Stream()
    saved = {k: t.clone() for k, t in a.cache.buffers.items()}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a.cache, lengths, new)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(a.cache, lengths, new)
    for k, t in a.cache.buffers.items():
        t.view(torch.uint8).copy_(saved[k].view(torch.uint8))
    lengths.copy_(a.lengths)
    eager_lengths, eager_new = b.lengths.clone(), torch.empty_like(b.lengths)
    for i in range(8):
        kv.copy_(torch.from_numpy(rand(i, 256, 3)))
        Q.copy_(torch.from_numpy(rand(90 + i, 256, 3)))
        graph.replay()
        want = step(b.cache, eager_lengths, eager_new)
        torch.cuda.synchronize()
        assert torch.equal(lengths, eager_lengths)
        for x, y in zip(outs, want):
            assert torch.equal(x, y)
        for k, t in a.cache.buffers.items():
            u, w = t.view(torch.uint8), getattr(b.cache, k).view(torch.uint8)
            assert torch.equal(u, w), k
    assert lengths.tolist() == [68, 11, 138]


@gpu
def test_calls_run_on_the_current_stream(dev):
    b = Both(dev, 1, 2, 64, 2, 20, 8, 128, 64)
    b.grow([100, 5])
    q = b.draft([1, 2])
    Q = torch.randn(256, 3, device=dev).half()
    want = nmg.cache_attention(b.cache, 0, Q, 4, i32(q), b.lengths)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = torch.zeros_like(Q)
        for _ in range(20):
            late = late + 0.05 * Q.float().mean() * 0      # work that the call has to wait for
        got = nmg.cache_attention(b.cache, 0, Q + late.half(), 4, i32(q), b.lengths)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@gpu
def test_bad_lengths_tables_and_lists_stay_inside(dev):
    """Contents that are not as described: every call ends, and nothing outside the
    cache's buffers is touched (they lie between guards)."""
    guard, parts = 4096, {}
    shapes = nmg.Cache.empty(1, 2, 32, 3, 4, 3, 128, 64, device=dev).buffers
    for name, t in shapes.items():
        buf = torch.full((t.numel() * t.element_size() + 2 * guard,), 0x5A, dtype=torch.uint8, device=dev)
        inner = buf[guard:-guard]
        inner.copy_(t.reshape(-1).view(torch.uint8))
        parts[name] = buf, inner.view(t.dtype).view(t.shape)
    cache = nmg.Cache(*(v for _, v in parts.values()))
    K = torch.ones(64, 9, device=dev).half()
    Q = torch.ones(128, 9, device=dev).half()
    for lengths in ([-5, 1 << 30, 2147483647], [-2147483648, 255, 256], [64, 191, 192]):
        for table in (-1, 1 << 30, -2147483648, 4, 3):
            for q in ([0, 3, 6, 9], [0, 9, 3, 9], [5, 4, 2, 1], [-7, 100, -3, 1 << 30], [9, 9, 9, 9]):
                cache.table.fill_(table)
                n, qo = i32(lengths), i32(q)
                nmg.cache_append(cache, 0, K, K, qo, n)
                nmg.cache_attention(cache, 0, Q, 4, qo, n)
                nmg.cache_attention(cache, 0, Q, 4, qo, n, torch.ones(9, 5, dtype=torch.uint8, device=dev))
                nmg.cache_commit(cache, n, qo)
                nmg.cache_commit(cache, n, qo, i32([7, -5, 1 << 30, 0, 2, 2]))
                nmg.cache_reserve(cache, n, i32([1 << 30, -4, 64]))
                nmg.cache_fork(cache, n, [0], [2])
                nmg.cache_compact(cache)
                nmg.cache_free(cache, n, [1, 0])
                torch.cuda.synchronize()
                for name, (buf, _) in parts.items():
                    assert (buf[:guard] == 0x5A).all() and (buf[-guard:] == 0x5A).all(), name


# ------------------------------------------------------------------- refusals

def struct(**change):
    """A cache whose pointers are never followed: every call below is refused first."""
    c = nmg._Cache(1, 2, 64, nmg.F16, 0, 64, 8, 3, 4, 128, *[4096] * 8)
    for k, v in change.items():
        setattr(c, k, v)
    return c


SIZES = [dict(layers=0), dict(kv_heads=0), dict(head_dim=0), dict(pages=0), dict(sequences=0), dict(row=0),
         dict(room=0), dict(room=96), dict(format=2), dict(format=-1)]
UNSUPPORTED = [dict(head_dim=257), dict(block=32), dict(block=0), dict(block=-64), dict(row=1 << 25),
               dict(layers=40000), dict(kv_heads=32767, head_dim=256), dict(sequences=1 << 24),
               dict(sequences=1 << 20, row=1 << 12)]


def calls(c):
    L, p, lists = nmg.lib(), 4096, (ctypes.c_int32 * 2)(0, 1)
    return {"append": lambda: L.nmg_cache_append(c, 0, p, p, p, 9, p, 9, 9, None),
            "attention": lambda: L.nmg_cache_attention(c, 0, 4, p, p, p, 9, 9, None, 0, 0, 0, 1.0, p, 9, None, 0, None),
            "commit": lambda: L.nmg_cache_commit(c, p, p, None, 0, p + 64, None),
            "reserve": lambda: L.nmg_cache_reserve(c, p, p, p, None),
            "fork": lambda: L.nmg_cache_fork(c, p, 1, lists, ctypes.cast(ctypes.addressof(lists) + 4,
                                                                         ctypes.POINTER(ctypes.c_int32)), None),
            "free": lambda: L.nmg_cache_free(c, p, 1, lists, None),
            "compact": lambda: L.nmg_cache_compact(c, p, p, p, p, 1 << 20, None)}


def test_caches_of_wrong_sizes_are_refused():
    for change, status in [(c, nmg.ERR_PARAM) for c in SIZES] + [(c, nmg.ERR_UNSUPPORTED) for c in UNSUPPORTED] + \
            [(dict(dtype=7), nmg.ERR_DTYPE)]:
        c = struct(**change)
        for name, call in calls(c).items():
            assert call() == status, (change, name)
        assert nmg.lib().nmg_cache_compact_workspace_bytes(c) == -1
        assert nmg.lib().nmg_cache_attention_workspace_bytes(c, 4, 9, 0) == -1
    for field in ("k_pages", "v_pages", "k_scales", "v_scales", "k_open", "v_open", "table", "references"):
        wide = field in ("k_pages", "v_pages", "k_open", "v_open")
        for value, status in ((None, nmg.ERR_NULL), (4096 + (8 if wide else 2), nmg.ERR_ALIGN)):
            for name, call in calls(struct(**{field: value})).items():
                assert call() == status, (field, name)
    for name, call in calls(None).items():
        assert call() == nmg.ERR_NULL, name


def test_wrong_arguments_are_refused():
    L, c, p = nmg.lib(), struct(), 4096
    N, P, A, U_ = nmg.ERR_NULL, nmg.ERR_PARAM, nmg.ERR_ALIGN, nmg.ERR_UNSUPPORTED

    def append(layer=0, q=p, n=p, K=p, ldk=9, V=p, ldv=9, cols=9):
        return L.nmg_cache_append(c, layer, q, n, K, ldk, V, ldv, cols, None)
    for kw, status in ((dict(layer=1), P), (dict(layer=-1), P), (dict(q=None), N), (dict(n=None), N), (dict(K=None), N),
                       (dict(V=None), N), (dict(ldk=8), P), (dict(ldv=8), P), (dict(cols=0), P), (dict(cols=1 << 31), P),
                       (dict(K=p + 1), A), (dict(V=p + 1), A), (dict(q=p + 2), A), (dict(n=p + 1), A)):
        assert append(**kw) == status, kw

    def attention(layer=0, heads=4, q=p, n=p, Q=p, ldq=9, cols=9, tree=None, ldtree=0, width=0, longest=0, scale=1.0,
                  O=p, ldo=9, ws=None, room=0):
        return L.nmg_cache_attention(c, layer, heads, q, n, Q, ldq, cols, tree, ldtree, width, longest, scale, O, ldo,
                                     ws, room, None)
    for kw, status in ((dict(layer=1), P), (dict(heads=0), P), (dict(heads=3), P), (dict(heads=-2), P), (dict(q=None), N),
                       (dict(n=None), N), (dict(Q=None), N), (dict(O=None), N), (dict(ldq=8), P), (dict(ldo=8), P),
                       (dict(cols=0), P), (dict(cols=1 << 31, ldq=1 << 31, ldo=1 << 31), P), (dict(longest=-1), P),
                       (dict(scale=0.0), P), (dict(scale=-1.0), P), (dict(scale=math.nan), P), (dict(scale=math.inf), P),
                       (dict(tree=p, width=0, ldtree=4), P), (dict(tree=p, width=5, ldtree=4), P),
                       (dict(tree=p, width=1 << 31, ldtree=1 << 31), P), (dict(ws=p + 64, room=64), A),
                       (dict(ws=p, room=-1), P), (dict(Q=p + 1), A), (dict(O=p + 1), A), (dict(q=p + 1), A),
                       (dict(heads=1 << 20, cols=1 << 20, ldq=1 << 20, ldo=1 << 20), U_)):
        assert attention(**kw) == status, kw

    def commit(n=p, ko=p, kept=None, count=0, new=p + 64):
        return L.nmg_cache_commit(c, n, ko, kept, count, new, None)
    for kw, status in ((dict(n=None), N), (dict(ko=None), N), (dict(new=None), N), (dict(new=p), P),
                       (dict(kept=p + 2), A), (dict(kept=p, count=-1), P), (dict(kept=p, count=1 << 31), P),
                       (dict(new=p + 2), A)):
        assert commit(**kw) == status, kw
    for args, status in (((None, p, p), N), ((p, None, p), N), ((p, p, None), N), ((p, p, p + 1), A)):
        assert L.nmg_cache_reserve(c, *args, None) == status
    need = L.nmg_cache_compact_workspace_bytes(c)
    assert need > 0
    for args, status in (((None, p, p, p, need), N), ((p, None, p, p, need), N), ((p, p, None, p, need), N),
                         ((p, p, p, None, need), N), ((p, p, p, p + 64, need), A),
                         ((p, p, p, p, need - 1), nmg.ERR_CAPACITY)):
        assert L.nmg_cache_compact(c, *args, None) == status


def test_lists_of_sequences_are_refused():
    L, c, p = nmg.lib(), struct(), 4096
    ints = lambda *v: (ctypes.c_int32 * len(v))(*v)   # noqa: E731
    for a, b in (((0,), (0,)), ((0, 1), (2, 2)), ((0, 1), (1, 2)), ((3,), (0,)), ((0,), (3,)), ((-1,), (0,)), ((0,), (-1,)),
                 ((0, 0, 0, 0), (1, 2, 1, 2))):
        assert L.nmg_cache_fork(c, p, len(a), ints(*a), ints(*b), None) == nmg.ERR_PARAM, (a, b)
    assert L.nmg_cache_fork(c, p, -1, ints(0), ints(1), None) == nmg.ERR_PARAM
    assert L.nmg_cache_fork(c, p, 1, None, ints(1), None) == nmg.ERR_NULL
    assert L.nmg_cache_fork(c, None, 1, ints(0), ints(1), None) == nmg.ERR_NULL
    assert L.nmg_cache_fork(c, p, 0, None, None, None) == nmg.OK
    for v in ((0, 0), (3,), (-1,), (0, 1, 2, 0)):
        assert L.nmg_cache_free(c, p, len(v), ints(*v), None) == nmg.ERR_PARAM
    assert L.nmg_cache_free(c, p, 1, None, None) == nmg.ERR_NULL
    assert L.nmg_cache_free(c, p, 0, None, None) == nmg.OK


@gpu
def test_the_binding_refuses(dev):
    b = Both(dev)
    c, n, q = b.cache, b.lengths, i32([0, 1, 2, 3])
    K = torch.zeros(128, 3, device=dev).half()
    for bad in ((K.float(), K), (K, K.float())):
        with pytest.raises(TypeError):
            nmg.cache_append(c, 0, *bad, q, n)
    for K2, V2, q2, n2 in ((K[:64], K[:64], q, n), (K, K[:, :2], q, n), (K.t(), K.t(), q, n), (K, K, q[:3], n),
                           (K, K, q.long(), n), (K, K, q, n[:2]), (K, K, q, n.float()), (K.cpu(), K, q, n)):
        with pytest.raises(ValueError):
            nmg.cache_append(c, 0, K2, V2, q2, n2)
    with pytest.raises(nmg.NmgError):
        nmg.cache_append(c, 1, K, K, q, n)
    Q = torch.zeros(256, 3, device=dev).half()
    for kw in (dict(heads=3), dict(heads=0), dict(Q=Q.float()), dict(tree=torch.ones(2, 3, device=dev, dtype=torch.uint8)),
               dict(tree=torch.ones(3, 3, device=dev)), dict(out=Q.float()), dict(out=Q[:, :2]), dict(heads=8),
               dict(longest=-1), dict(scale=0.0), dict(longest=1 << 40), dict(q=q[1:]), dict(n=q)):
        args = dict(Q=Q, heads=4, q=q, n=n) | kw
        with pytest.raises((ValueError, TypeError, nmg.NmgError)):
            nmg.cache_attention(c, 0, args["Q"], args["heads"], args["q"], args["n"], args.get("tree"),
                                args.get("longest"), args.get("scale"), args.get("out"))
    for args in ((q, q), (n, n), (n.long(), q), (n, q, q.float()), (n, q, None, n), (n, q, None, q)):
        with pytest.raises((ValueError, nmg.NmgError)):
            nmg.cache_commit(c, *args)
    for a, t in (([0], [0]), ([0, 1], [2]), ([0], [7]), ([-1], [0]), ([1 << 40], [0]), ([0, 0], [1, 1])):
        with pytest.raises((ValueError, nmg.NmgError)):
            nmg.cache_fork(c, n, a, t)
    for which in ([0, 0], [3], [-1]):
        with pytest.raises(nmg.NmgError):
            nmg.cache_free(c, n, which)
    with pytest.raises(ValueError):
        nmg.cache_compact(c, c.table[:1])
    with pytest.raises(ValueError):
        nmg.cache_reserve(c, n, n.long())
    buffers = dict(c.buffers)
    for name, t in c.buffers.items():
        for wrong in (t.cpu(), t[:, :1] if t.dim() > 1 else t[:1], t.to(torch.float64)):
            with pytest.raises((ValueError, TypeError)):
                nmg.Cache(*(buffers | {name: wrong}).values())
    with pytest.raises(nmg.NmgError):
        nmg.Cache.empty(1, 1, 64, 1, 4, 4, 128, 32, device=dev)
    with pytest.raises(ValueError):
        nmg.Cache.empty(1, 1, 64, 1, 4, 4, 128, 64, "e5m2", device=dev)
