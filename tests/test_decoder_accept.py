"""What ``SparseDecoder.accept`` refuses: anything but one path from the kept tokens
through the last draft of each sequence."""
import pytest
import torch

from paper_2304_07613_amd import nmg
from paper_2304_07613_amd.decoder import DecoderShape, SparseDecoder

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nmg.lib()


def decoder(capacity=8):
    shape = DecoderShape(hidden=64, ffn=64, heads=2, kv_heads=1, head_dim=32, g=8, m=4)
    return SparseDecoder.random(shape, 1, sequences=2, capacity=capacity)


def draft(dec, parents):
    n = sum(len(p) for p in parents)
    return dec.step(torch.randn(64, n, generator=torch.Generator().manual_seed(n)).half().to(DEV), parents)


PARENTS = [[-1, 0, 0, 2, -1], [-1, 0]]


@pytest.mark.parametrize("kept", [
    [[5], []],              # past the draft of its sequence
    [[], [2]],
    [[-1], []],             # before it
    [[0, 0], []],           # a token twice
    [[1], []],              # a path starts behind the kept tokens
    [[0, 3], []],           # ... and leaves out no node
    [[0, 1, 2], []],        # siblings
    [[2, 0], []],           # from the end
    [[0, 4], []],           # two paths
    [[0], [1]],             # the second sequence's
    [[0, 2, 3, 5, 6, 7, 8, 9], []],
    [[0]],
])
def test_accept_refuses(kept):
    dec = decoder()
    draft(dec, PARENTS)
    keys = dec.layers[0].keys.clone()
    with pytest.raises(ValueError):
        dec.accept(kept)
    assert dec.lengths.tolist() == [0, 0] and torch.equal(dec.layers[0].keys, keys)
    dec.accept([[0, 2, 3], [0, 1]])           # the draft is still there to accept from
    assert dec.lengths.tolist() == [3, 2]


def test_a_draft_is_accepted_once():
    dec = decoder()
    with pytest.raises(ValueError):
        dec.accept([[0], []])                 # nothing was drafted
    dec.accept([[], []])
    draft(dec, PARENTS)
    dec.accept([[4], []])
    for again in ([[4], []], [[0], []], [[], [0]]):
        with pytest.raises(ValueError):
            dec.accept(again)
    dec.accept([[], []])
    assert dec.lengths.tolist() == [1, 0]


def test_lengths_stay_within_the_capacity():
    dec = decoder(capacity=3)
    for _ in range(3):
        draft(dec, [[-1], [-1]])
        dec.accept([[0], [0]])
    with pytest.raises(ValueError):
        draft(dec, [[-1], []])
    with pytest.raises(ValueError):           # the refused draft is none
        dec.accept([[0], []])
    assert dec.lengths.tolist() == [3, 3]
