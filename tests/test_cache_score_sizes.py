"""Binary32 queries and keys of very different sizes: scores of open tokens and pages to the
bounds of ``test_cache.py``, relative to scale sum_d |q_d k_d| of the row."""
import numpy as np
import pytest

from test_cache import Both, dev, random_tree  # noqa: F401

pytestmark = pytest.mark.gpu


def go(dev, heads, dim, sizes_k, sizes_q, counts=(5, 33), kept=(130, 10), scale=None):  # noqa: F811
    """sizes_k(open, N): sizes of N tokens' keys, by feature or not."""
    b = Both(dev, 1, 1, dim, 2, 20, 6, 192, 64, "e4m3", "f32")

    def change(K, V, q):
        K *= np.asarray(sizes_k(K.shape[1]), np.float64).astype(np.float32)
        V *= 0.1
    b.grow(list(kept), change)
    q = b.draft(list(counts), change)
    Q = np.random.default_rng(7).standard_normal((heads, dim, q[-1]))
    with np.errstate(over="ignore"):      # (an infinite query or two)
        Q = (Q * np.broadcast_to(np.asarray(sizes_q(q[-1]), np.float64).reshape(-1, 1), (dim, q[-1]))).astype(np.float32)
    Q = Q.reshape(heads * dim, -1)
    print(heads, dim, flush=True)
    b.attend(heads, q, Q=Q, scale=scale)
    b.attend(heads, q, random_tree(2, counts), Q=Q, scale=scale)


@pytest.mark.parametrize("heads,dim", [(2, 64), (5, 80), (1, 200), (4, 128)])
@pytest.mark.parametrize("k,q", [(1e-37, 1e37), (4e-39, 1e38), (1e-36, 3e36), (1e37, 1e-37), (3e37, 4e-39)])
def test_keys_and_queries_of_one_size(dev, heads, dim, k, q):  # noqa: F811
    go(dev, heads, dim, lambda N: k, lambda N: q)


@pytest.mark.parametrize("heads,dim", [(2, 64), (1, 200)])
@pytest.mark.parametrize("large", [2.0 ** 30, 2.0 ** 60, 2.0 ** 90])
def test_features_of_several_sizes(dev, heads, dim, large):  # noqa: F811
    """Large in one, small in the other: every product counts the same."""
    by = np.where(np.arange(dim) % 2, large, 1 / large)
    go(dev, heads, dim, lambda N: by[:, None], lambda N: 1 / by, kept=(10, 3))


@pytest.mark.parametrize("heads,dim", [(2, 64), (3, 80)])
def test_tokens_of_several_sizes(dev, heads, dim):  # noqa: F811
    """A key near the largest number beside others of 1e-5 that count: its score is
    far below theirs, or it is nothing in the feature that is large."""
    def sizes(N):
        s = np.full((dim, N), 1e-5)
        s[1::2, N // 2] = 1e37                     # met by queries of 0
        return s
    by = np.where(np.arange(dim) % 2, 0.0, 1e5)
    go(dev, heads, dim, sizes, lambda N: by, kept=(10, 3))


@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** -100])
def test_products_past_the_range_with_scores_inside(dev, scale):  # noqa: F811
    """scale q k where the sum of products is past 2^128."""
    go(dev, 2, 64, lambda N: 1e25, lambda N: 5e13 * 2.0 ** -40 / scale, kept=(10, 3), scale=scale)
