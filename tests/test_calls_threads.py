"""The compiled calls run the library without the interpreter lock: threads with
streams of their own do not wait for each other's launches."""
import ctypes

import pytest
import torch

from paper_2304_07613_amd import nmg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture
def lock_seen():
    """The binding with every function of the library replaced by the question
    whether the caller holds the interpreter lock: 0 (no error) if not, else an
    error status."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    module = nmg._load_calls()
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    names = ("nmg_rotary", "nmg_qk_norm_rotary", "nmg_attention", "nmg_tree_attention",
             "nmg_attention_workspace_bytes")
    module.bind({n: held for n in names}, nmg._check, torch._C._cuda_getDevice,
                torch._C._cuda_getCurrentRawStream)
    yield
    nmg._load_calls()


def test_calls_release_the_lock(lock_seen):
    x = torch.zeros(64, 4, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    table, out = torch.zeros(2, 32, 8, device=DEV), torch.empty_like(x)
    ranges = i32(0, 4), i32(0), i32(4)
    for o in (None, out):
        nmg.rotary(x, 1, table, i32(0, 1, 2, 3), out=o)
        nmg.qk_norm_rotary(x, x, 1, 1, None, None, table, i32(0, 1, 2, 3), out=o if o is None else (o, o))
        nmg.attention(x, x, x, 1, 1, *ranges, out=o)
        nmg.tree_attention(x, x, x, 1, 1, *ranges, torch.ones(4, 4, dtype=torch.bool, device=DEV), out=o)


def test_refusals_come_back_with_the_lock():
    x = torch.zeros(64, 4, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    with pytest.raises(nmg.NmgError):
        nmg.attention(x, x, x, 1, 1, i32(0, 4), i32(0), i32(4), scale=-1.0)
    with pytest.raises(nmg.NmgError):
        nmg.rotary(x[:, :0], 1, None, None)
    for call in (lambda o: nmg.rotary(x, 1, None, None, out=o),
                 lambda o: nmg.attention(x, x, x, 1, 1, i32(0, 4), i32(0), i32(4), out=o)):
        for bad in (x.half(), x[:, :3], x.t().contiguous().t()):
            with pytest.raises(ValueError):
                call(bad)
        y = torch.empty(64, 9, device=DEV)[:, 2:6]
        assert call(y).data_ptr() == y.data_ptr()
