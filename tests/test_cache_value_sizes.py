"""Binary32 values of very different sizes in one cache: what a row does not see, or hardly weighs,
costs no precision of what it sees.  References and bounds as in ``test_cache.py``: relative to
sum_j p_j |v_j| of the row and feature."""
import numpy as np
import pytest

from test_cache import Both, dev, random_tree  # noqa: F401
from test_cache_far_values import SIZES, places, sharp

pytestmark = pytest.mark.gpu


def small(V, size=1e-5):
    """Values of `size`, none much smaller."""
    V[:] = np.where(V < 0, -1, 1) * (0.5 + np.abs(V) / 8) * np.float32(size)


@pytest.mark.parametrize("size", [1e-5, 1.0, 1e-25])
@pytest.mark.parametrize("heads,dim", [(2, 64), (1, 128), (8, 80), (2, 200)])
def test_drafts_that_a_row_does_not_see(dev, heads, dim, size):  # noqa: F811
    counts = [5, 1, 70, 30]
    b = Both(dev, 1, 1, dim, 4, 60, 12, 192, 64, "e4m3", "f32")
    b.grow([130, 0, 64, 200], lambda K, V, q: small(V, size))
    tree = random_tree(3, counts)
    for huge in (3e38, -1e30, 1e20, 1e12):
        def change(K, V, q):
            small(V, size)
            for s, T in enumerate(counts):
                V[1::3, q[s] + T // 2] = huge
                V[2::5, q[s] + T - 1] = huge
        print(heads, dim, huge, flush=True)
        q = b.draft(counts, change)
        b.attend(heads, q)
        b.attend(heads, q, tree)
        b.attend(heads, q, tree, longest=3000)


@pytest.mark.parametrize("kept,drafted", SIZES)
@pytest.mark.parametrize("gap", [60.0, 90.0, 110.0])
def test_tokens_of_almost_no_weight(dev, kept, drafted, gap):  # noqa: F811
    """A page, a kept and a drafted token near the largest number, e^-gap below the rest."""
    for fmt in ("e4m3", "int8"):
        for huge in (3e38, 1e30, 1e19):
            b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, fmt, "f32")

            def change(K, V, q):
                K *= 0.1
                K[0] = 10
                small(V)
                n = b.model.n[0]
                for p in (5, kept - 1, kept + drafted // 2):
                    if n <= p < n + q[1] and (p < 64 or kept - kept % 64 <= p):
                        K[0, q[0] + p - n], V[3:50, q[0] + p - n] = 0, huge
            b.grow([kept], change)
            q = b.draft([drafted], change)
            print(kept, drafted, gap, huge, fmt, flush=True)
            for longest in (None, 64):
                b.attend(2, q, longest=longest, scale=1.0, Q=sharp(b, 2, q, gap / 10))


@pytest.mark.parametrize("kept,drafted", SIZES)
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_blocks_of_all_sizes(dev, kept, drafted, fmt):  # noqa: F811
    """Every block and open token of a size of its own, 1e-30 to 1e30, weighed as scores happen."""
    for sharpness in (1.5, 20.0):
        b = Both(dev, 1, 2, 64, 1, 60, 50, 256, 64, fmt, "f32")
        sizes = 10.0 ** np.random.default_rng(1).uniform(-30, 30, 4000)

        def change(K, V, q):
            n = b.model.n[0]
            for i in range(q[1]):
                p = n + i
                V[:, i] *= np.float32(sizes[p // 64 if p < kept // 64 * 64 else p])
        b.grow([kept], change)
        q = b.draft([drafted], change)
        print(kept, drafted, fmt, sharpness, flush=True)
        for longest in (None, 64):
            b.attend(4, q, longest=longest, sharp=sharpness)


@pytest.mark.parametrize("kept,drafted", SIZES)
@pytest.mark.parametrize("size", [1e31, 3.2e38])
def test_values_near_the_largest(dev, kept, drafted, size):  # noqa: F811
    """Of one sign: means, finite whatever the order of the scores."""
    for scores in ("flat", "rising", "random"):
        b = Both(dev, 1, 1, 64, 1, 60, 50, 256, 64, "int8", "f32")

        def change(K, V, q):
            small(V, 1)
            V[:] = np.float32(size) * (1 - 0.02 * np.abs(V))
            n = b.model.n[0]
            if scores == "rising":                 # by less than what moves the reference
                K[:] = 0
                K[0] = [4.0 * (n + i) / (kept + drafted) for i in range(q[1])]
        b.grow([kept], change)
        q = b.draft([drafted], change)
        Q = np.zeros((128, q[-1]), np.float32) if scores == "flat" else sharp(b, 2, q, 1.0) / 4
        print(kept, drafted, size, scores, flush=True)
        for longest in (None, 64):
            b.attend(2, q, longest=longest, scale=1.0, Q=Q)


@pytest.mark.parametrize("kept,drafted", [(130, 3), (1000, 1), (64, 70), (2500, 33)])
def test_large_and_small_features(dev, kept, drafted):  # noqa: F811
    """A token's features keep their own precision (open tokens; a block has one scale)."""
    sizes = np.array([3e38, -3e38, 1e-34, 1.0, 1e20], np.float32)
    for heads, dim in ((2, 64), (1, 200)):
        b = Both(dev, 1, 1, dim, 1, 60, 50, 256, 64, "e4m3", "f32")

        def change(K, V, q):
            small(V, 1)
            n = b.model.n[0]
            V *= (0 if n < kept // 64 * 64 else 0.9 * sizes[np.arange(dim) % 5][:, None])
        b.grow([kept // 64 * 64], change)
        b.grow([kept % 64], change)
        q = b.draft([drafted], change)
        b.attend(heads, q)
        b.attend(heads, q, random_tree(1, [drafted]), longest=200)


def test_hidden_infinities_beside_large_values(dev):  # noqa: F811
    counts = [6, 40]
    b = Both(dev, 1, 2, 64, 2, 60, 12, 192, 64, "e4m3", "f32")
    b.grow([100, 70], lambda K, V, q: small(V))
    tree = random_tree(3, counts)

    def change(K, V, q):
        small(V)
        V[1, q[0] + 3], V[2, q[1] + 20], V[2, q[1] + 21] = np.inf, 3e38, -np.inf
        V[3, q[1] + 39], V[4, q[0]] = np.nan, 1e25
    q = b.draft(counts, change)
    b.attend(4, q)
    b.attend(4, q, tree)
