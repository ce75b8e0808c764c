"""Values that are not finite at scores far below the maximum: a weight of e^-300 is no
zero, so an infinity or NaN reaches the output that has it, whichever wave or part of the
keys holds the token, whatever `longest` and the scratch memory.  References and bounds as in
``test_cache.py``, whose binary64 weights are positive down to e^-745."""
import math

import numpy as np
import pytest
import torch

from test_cache import Both, attend64, check, dev, i32, offsets, random_tree  # noqa: F401

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu
FAR = 30.0          # of the queries' first feature; the key of the maximum has 10 there


def sharp(b, heads, q, size=FAR, seed=5):
    Q = np.random.default_rng(seed).standard_normal((heads * b.model.shape[2], max(1, int(q[-1]))))
    Q[::b.model.shape[2]] = size
    return Q.astype(np.float16 if b.dtype == "f16" else np.float32)


def places(b, top, bad=()):
    """change() for draft and grow: the key at position `top` of every sequence has the largest
    score; (position, feature, value) of `bad` go into the values."""
    D = b.model.shape[2]

    def change(K, V, q):
        K *= 0.3
        K[::D] = 0
        for s, n in enumerate(b.model.n):
            at = lambda p: q[s] + p - n if n <= p < n + q[s + 1] - q[s] else None   # noqa: E731
            if at(top) is not None:
                K[::D, at(top)] = 10
            for p, d, value in bad:
                if at(p) is not None:
                    V[d::D, at(p)] = value
    return change


# kept tokens, drafted ones: one wave's tiles and the others'; parts; many rows and their parts
SIZES = [(200, 1), (700, 3), (2500, 1), (700, 70), (2500, 140)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kept,drafted", SIZES)
@pytest.mark.parametrize("size", [6.0, FAR])
def test_a_page_without_a_finite_value(dev, kept, drafted, size, dtype):  # noqa: F811
    for page in (0, kept // 128, kept // 64 - 1):
        for top in (page * 64 + 5, (page * 64 + kept // 2) % kept, kept - 1, kept):
            b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, "e4m3", dtype)
            change = places(b, top, [(page * 64 + 9, 3, math.inf)])
            b.grow([kept], change)
            q = b.draft([drafted], change)
            print(kept, drafted, page, top, dtype, flush=True)
            for longest in (None, kept, 64):
                b.attend(2, q, longest=longest, scale=1.0, Q=sharp(b, 2, q, size))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kept,drafted", SIZES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_open_values(dev, kept, drafted, bad, dtype):  # noqa: F811
    for where in (kept, kept + drafted - 1, kept - 1):         # an open token, kept or drafted
        for top in (3, kept // 2, kept):
            b = Both(dev, 1, 2, 48, 1, 60, 50, 256, 64, "int8", dtype)
            change = places(b, top, [(where, 7, bad), (kept, 40, 5.0)])
            b.grow([kept], change)
            q = b.draft([drafted], change)
            print(kept, drafted, where, top, bad, dtype, flush=True)
            for size in (6.0, FAR):
                for longest in (None, kept, 64):
                    b.attend(4, q, longest=longest, scale=1.0, Q=sharp(b, 4, q, size))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kept,drafted", SIZES)
def test_infinities_of_both_signs(dev, kept, drafted, dtype):  # noqa: F811
    """One far below the maximum, one with it, and both: their sum is NaN."""
    for top in (3, kept):
        b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, "e4m3", dtype)
        last = kept + drafted - 1
        change = places(b, top, [(last, 1, math.inf), (kept, 2, -math.inf), (last, 5, -math.inf), (kept - 1, 5, math.inf)])
        b.grow([kept - kept % 64], change)
        b.grow([kept % 64], change)
        q = b.draft([drafted], change)
        for longest in (None, 64):
            b.attend(2, q, longest=longest, scale=1.0, Q=sharp(b, 2, q))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kept,drafted", SIZES)
def test_a_weight_that_is_zero(dev, kept, drafted, dtype):  # noqa: F811
    """A score of minus infinity has the weight 0, and 0 times infinity is NaN."""
    for top in (3, kept):
        b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, "e4m3", dtype)
        far = places(b, top, [(kept, 9, math.inf), (kept, 11, 1.0)])

        def change(K, V, q):
            far(K, V, q)
            K[1, q[0]] = -math.inf if b.model.n[0] == kept else 0.0

        b.grow([kept], far)
        q = b.draft([drafted], change)
        Q = sharp(b, 2, q)
        Q[1::64] = 0.5
        for longest in (None, 64):
            b.attend(2, q, longest=longest, scale=1.0, Q=Q)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("counts", [[2, 3], [90, 100]])
def test_no_weight_at_all(dev, counts, dtype):  # noqa: F811
    """Scores of minus infinity alone give 0, whatever the values are."""
    b = Both(dev, 1, 1, 32, 2, 4, 2, 128, 64, "e4m3", dtype)

    def change(K, V, q):
        K[0] = -math.inf
        V[3], V[9, 0] = math.inf, math.nan

    q = b.draft(counts, change)
    Q = np.zeros((32, q[-1]), np.float16 if dtype == "f16" else np.float32)
    Q[0] = 1.0
    b.attend(1, q, Q=Q)
    b.attend(1, q, random_tree(1, counts), Q=Q)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_scratch_memory_and_splits_change_nothing(dev, dtype):  # noqa: F811
    """NaN or a number does not depend on the number of parts."""
    b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, "e4m3", dtype)
    change = places(b, 1900, [(70, 3, math.nan), (2500, 4, math.inf)])
    b.grow([2500], change)
    q = b.draft([1], change)
    Q = torch.from_numpy(sharp(b, 1, q)).to(dev)
    with np.errstate(all="ignore"):
        ref = attend64(b.model, 0, Q.cpu().numpy(), 1, q, None, 1.0)
    L, qo = nmg.lib(), torch.from_numpy(q).to(dev)
    most = L.nmg_cache_attention_workspace_bytes(b.cache.c, 1, 1, 2500)
    assert most > 0
    for nbytes in (0, most // 3 // 256 * 256, most):
        space = torch.full((max(nbytes, 256),), 255, dtype=torch.uint8, device=dev)
        out = torch.zeros_like(Q)
        st = L.nmg_cache_attention(b.cache.c, 0, 1, qo.data_ptr(), b.lengths.data_ptr(), Q.data_ptr(), 1, 1, None, 0, 0,
                                   2500, 1.0, out.data_ptr(), 1, space.data_ptr(), nbytes,
                                   torch.cuda.current_stream().cuda_stream)
        assert st == 0
        check(out, ref, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("heads,dim", [(2, 64), (3, 80), (1, 200), (4, 128)])
def test_many_values_that_are_not_finite(dev, heads, dim, dtype):  # noqa: F811
    """Features with infinities of one sign, of both, NaN, and none, keys whose score is minus
    infinity among them, seen by some."""
    rng = np.random.default_rng(11)
    for counts in ([7, 1, 40], [130, 255, 70]):
        b = Both(dev, 1, 1, dim, 3, 30, 6, 384, 64, "e4m3", dtype)
        b.grow([100, 0, 70])

        def change(K, V, q):
            some = rng.random(V.shape) < 0.05
            kinds = np.array([math.inf, -math.inf, math.nan, 1.0, math.inf])[np.arange(dim) % 5]
            signs = np.where(rng.random(V.shape) < 0.5, -1, 1)
            V[:] = np.where(some, np.where((np.arange(dim) % 5 == 4)[:, None], signs, 1) * kinds[:, None], V)
            K[0, rng.random(V.shape[1]) < 0.1] = -math.inf
        q = b.draft(counts, change)
        Q = np.random.default_rng(5).standard_normal((heads * dim, int(q[-1])))
        Q[::dim] = 0.5
        Q = Q.astype(np.float16 if dtype == "f16" else np.float32)
        print(heads, dim, counts, dtype, flush=True)
        b.attend(heads, q, random_tree(3, counts), Q=Q)
        b.attend(heads, q, Q=Q)
        b.attend(heads, q, random_tree(4, counts), Q=Q, longest=4000)
