"""The norm of a sum that is past binary16, or far below it: scale, weights and biases are binary32, and
the second norm is of the sum in binary32.  References and bounds as in ``test_residual_norm.py``."""
import numpy as np
import pytest
import torch

from test_residual_norm import DT, NP, U, dev, rand, reference  # noqa: F401

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu
LARGEST = {"f16": 65504.0, "f32": float(np.finfo(np.float32).max)}


def check(got, ref, dtype):
    """Values past the type round to infinity; one within the bound of that border may do either."""
    y, e = ref
    e = np.where(np.isfinite(e) & np.isfinite(y), e, 0)
    half = 2.0 ** -11 if dtype == "f16" else U
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(y))
    border = LARGEST[dtype] * (1 + half)
    inf = np.abs(y) > border + e
    assert np.array_equal(got[inf], np.sign(y[inf]) * np.inf)
    fine = np.abs(y) < border - e
    assert np.isfinite(got[fine]).all()
    e = e + half * np.abs(y) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -149)
    assert (np.abs(got - y)[fine] <= e[fine]).all(), (np.abs(got - y)[fine] / e[fine]).max()


def run(dev, M, N, dtype, after, before, scale, gate, residual, weight=1.0, bias=0.0, eps=0.0, A=None, R=None):  # noqa: F811
    A = (rand(1, M, N) if A is None else A).astype(NP[dtype])
    R = (rand(3, M, N) if R is None else R).astype(NP[dtype]) if residual else None
    G = (1 + rand(4, M, N) / 8).astype(NP[dtype]) if gate else None
    w = ((1 + rand(5, M) / 8) * np.float32(weight)).astype(np.float32)
    b = (rand(6, M) * np.float32(bias)).astype(np.float32)
    w2 = (1 + rand(7, M) / 8).astype(np.float32)
    up = lambda t: None if t is None else torch.from_numpy(t).to(dev)   # noqa: E731
    with np.errstate(all="ignore"):
        ref = reference(A, R, G, np.float64(np.float32(scale)), (after, w, b, eps), (before, w2, None, eps))
    got = nmg.residual_norm(up(A), up(R), up(G), scale, nmg.Norm(after, up(w), up(b), eps),
                            nmg.Norm(before, up(w2), None, eps))
    for g, r in zip(got, ref):
        check(g, r, dtype)


# one token to a workgroup's most; few rows and more than vector loads are for
SIZES = [(96, 10), (768, 1), (768, 300), (4097, 9), (9000, 3)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("before", ["rms", "layer"])
@pytest.mark.parametrize("after", ["none", "rms", "layer"])
@pytest.mark.parametrize("scale", [1e20, -1e30, 1e10, 1e-25, 1e-12])
def test_scales_of_any_size(dev, M, N, after, before, scale, dtype):  # noqa: F811
    for eps in (0.0, 1e-6):
        run(dev, M, N, dtype, after, before, scale, False, False, eps=eps)
        run(dev, M, N, dtype, after, before, scale, True, abs(scale) > 1, eps=eps)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("before", ["rms", "layer"])
@pytest.mark.parametrize("weight,bias", [(1e25, 0.0), (1e-30, 0.0), (1.0, 1e22), (1e-28, 1e-28)])
def test_weights_and_biases_of_any_size(dev, before, weight, bias, dtype):  # noqa: F811
    for M, N in SIZES:
        run(dev, M, N, dtype, "rms", before, 0.5, True, False, weight, bias)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_tokens_of_different_sizes(dev, dtype):  # noqa: F811
    """Beside a token whose sum is large or small others keep what they had."""
    M, N = 512, 40
    G = np.ones((M, N))
    for scale in (1e24, 1e-20):
        A = rand(1, M, N)
        A[:, ::3] = 0
        A[0, ::3] = 2.0 ** -20
        run(dev, M, N, dtype, "none", "rms", scale, False, True, A=A, R=rand(2, M, N) * (G if scale > 1 else 0 * G))
