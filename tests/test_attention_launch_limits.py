"""Calls of more workgroups than a launch holds (2^32 threads) are refused before
anything is enqueued, and say so (``include/nmg.h``)."""
import ctypes

import pytest

from paper_2304_07613_amd import nmg

P = ctypes.c_void_p(1 << 20)


def attention(dtype, heads, kv, D, sequences, Nq, Nk, tree):
    h = nmg._Heads(heads, kv, D, dtype)
    s = nmg._Sequences(sequences, 1 << 20, 1 << 20, 1 << 20)
    args = (h, s, P, Nq, Nq, P, Nk, P, Nk, Nk)
    if tree:
        return nmg.lib().nmg_tree_attention(*args, P, 1, 1, 0.125, P, Nq, None, 0, None)
    return nmg.lib().nmg_attention(*args, None, 0.125, P, Nq, None, 0, None)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype,heads,kv,D,sequences,Nq,Nk", [
    (nmg.F16, 12, 12, 8, 1 << 21, 1 << 21, 1 << 21),   # 256 threads a workgroup
    (nmg.F32, 16, 16, 8, 1 << 20, 1 << 20, 1 << 20),   # exactly 2^32 threads
    (nmg.F32, 16, 16, 64, 1 << 19, 1 << 19, (1 << 26) - 4),   # 512 threads a workgroup: 2^32
    (nmg.F16, 1 << 12, 1 << 12, 1, 1, 1 << 20, 64),    # one sequence
])
def test_attention_past_a_launch(dtype, heads, kv, D, sequences, Nq, Nk, tree):
    assert attention(dtype, heads, kv, D, sequences, Nq, Nk, tree) == nmg.ERR_UNSUPPORTED


@pytest.mark.parametrize("heads,D,N", [(1 << 28, 2, 3), (1 << 13, 64, 1 << 21)])
def test_rotary_past_a_launch(heads, D, N):
    r = nmg._Rotary(2, 0, 8, 1 << 20, 1 << 20)
    assert nmg.lib().nmg_rotary(nmg.F16, heads, D, r, P, N, N, P, N, None) == nmg.ERR_UNSUPPORTED
    assert nmg.lib().nmg_qk_norm_rotary(nmg.F16, heads, 1, D, r, None, None, 1e-6, P, N, P, N, N, P, N, P,
                                        N, None) == nmg.ERR_UNSUPPORTED


def test_workspace_of_such_calls():
    """The query stays pure host code and gives a size, or none."""
    h = nmg._Heads(12, 12, 8, nmg.F16)
    assert nmg.lib().nmg_attention_workspace_bytes(h, 1 << 21, 1 << 21, 1 << 21) >= 0
