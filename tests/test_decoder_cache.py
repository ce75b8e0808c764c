"""The sparse decoder over an 8-bit cache and with norms around its blocks.

Cache: against the decoder over a cache in the activations' type that is given what the
pages stand for, so that both see the same keys and values.  The two round their
activations alike and differ in the attention's roundings: with about 10 roundings
of an activation on the way through a layer, 40 x 2^-11 (binary16) or 1e-4 (binary32)
of the outputs' scale for two layers.

Norms: against the layers in binary64 from the densified weights, same bound."""
import math

import pytest
import torch

from paper_2304_07613_amd import nmg
from paper_2304_07613_amd.decoder import BLOCKS, DecoderShape, SparseDecoder

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nmg.lib()


def shape_of(dtype):
    return DecoderShape(hidden=128, ffn=192, heads=4, kv_heads=2, head_dim=32, encoder_hidden=64,
                        n=2, m=4, g=8, dtype=dtype)


def chains(counts):
    return [list(range(-1, n - 1)) for n in counts]


def give_pages(paged, plain):
    """The plain cache's columns of whole blocks become what the pages stand for."""
    c, rows = paged.cache, paged.shape.kv_heads * paged.shape.head_dim
    for b, n in enumerate(paged.kept):
        for j in range(n // c.block):
            page = int(c.table[b, j])
            at = b * plain.capacity + j * c.block
            for i, layer in enumerate(plain.layers):
                k = c.k_pages[i, page].float()[..., : c.head_dim] * c.k_scales[i, page][:, None, None]
                v = c.v_pages[i, page].float() * c.v_scales[i, page][:, None, None]
                layer.keys[:, at:at + c.block] = k.transpose(1, 2).reshape(rows, -1).to(layer.keys.dtype)
                layer.values[:, at:at + c.block] = v.reshape(rows, -1).to(layer.values.dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("fmt,block", [("e4m3", 64), ("int8", 128)])
@pytest.mark.parametrize("block_norms", [None, "rms"])
def test_drafts_over_pages(fmt, block, block_norms, dtype):
    kw = dict(sequences=3, capacity=300, seed=3, block_norms=block_norms)
    paged = SparseDecoder.random(shape_of(dtype), 2, cache=fmt, block=block, max_draft=140, pages=7, **kw)
    plain = SparseDecoder.random(shape_of(dtype), 2, **kw)
    limit = 40 * 2.0 ** -11 if dtype == torch.float16 else 1e-4
    g = torch.Generator().manual_seed(5)
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32, device=DEV)   # noqa: E731
    states = torch.randn(64, 50, generator=g).to(dtype).to(DEV)
    for dec in (paged, plain):
        dec.set_encoder(states, i32(0, 30, 0), i32(30, 50, 10))

    def step(parents, keep):
        x = torch.randn(128, sum(len(p) for p in parents), generator=g).to(dtype).to(DEV)
        y, z = (dec.step(x, parents).double() for dec in (paged, plain))
        err = (y - z).abs().max() / z.abs().max()
        print(fmt, dtype, paged.kept, float(err), flush=True)
        assert err <= limit
        for dec in (paged, plain):
            dec.accept(keep)
        assert paged.lengths.tolist() == plain.lengths.tolist() == paged.kept == plain.kept
        give_pages(paged, plain)

    step(chains([140, 50, 1]), [list(range(140)), list(range(50)), [0]])
    step([[-1, 0, 1, 1, 0], [-1, -1], [-1]], [[0, 1, 3], [1], [0]])
    step(chains([1, 100, 70]), [[0], list(range(100)), []])
    step(chains([1, 1, 1]), [[0], [0], [0]])
    # sequence 2 goes on from sequence 0, which goes
    paged.fork([0], [2])
    for layer in plain.layers:
        for cache in (layer.keys, layer.values):
            cache[:, 2 * 300:3 * 300] = cache[:, :300]
    plain.lengths[2], plain.kept[2] = plain.lengths[0], plain.kept[0]
    plain.encoder_begin, plain.encoder_end = i32(0, 30, 0), i32(30, 50, 30)     # and its encoder's columns
    step(chains([2, 2, 2]), [[0], [0, 1], [0, 1]])
    paged.free([0])
    plain.lengths[0], plain.kept[0] = 0, 0
    used = int((paged.cache.references > 0).sum())
    assert paged.compact() == used and (paged.cache.references[used:] == 0).all()
    step(chains([3, 3, 3]), [[0, 1, 2], [0], [0]])


def test_a_pool_that_runs_out():
    dec = SparseDecoder.random(shape_of(torch.float16), 1, sequences=2, capacity=200, cache="e4m3", pages=1)
    x = lambda n: torch.randn(128, n, generator=torch.Generator().manual_seed(n)).half().to(DEV)   # noqa: E731
    dec.step(x(120), chains([60, 60]))
    dec.accept([list(range(60))] * 2)
    dec.step(x(20), chains([10, 10]))
    with pytest.raises(RuntimeError):
        dec.accept([list(range(10))] * 2)
    assert dec.lengths.tolist() == [60, 60]
    dec.accept([[0], [0]])
    assert dec.kept == [61, 61]
    dec.free([1])
    dec.step(x(10), chains([10, 0]))
    dec.accept([list(range(10)), []])
    assert dec.kept == [71, 0] and dec.lengths.tolist() == [71, 0]


def test_fork_and_free_leave_other_drafts():
    """What an exhausted pool's error asks for: free a sequence, accept the draft again."""
    make = lambda pages: SparseDecoder.random(shape_of(torch.float16), 1, sequences=3, capacity=200,  # noqa: E731
                                              cache="e4m3", pages=pages)
    few, many = make(1), make(9)
    g = torch.Generator().manual_seed(8)
    xs = [torch.randn(128, n, generator=g).half().to(DEV) for n in (150, 30, 2)]
    for dec in (few, many):
        dec.step(xs[0], chains([60, 60, 30]))
        dec.accept([list(range(60)), list(range(60)), list(range(30))])
        dec.step(xs[1], chains([10, 10, 10]))
    with pytest.raises(RuntimeError):
        few.accept([list(range(10))] * 2 + [[0]])
    for dec in (few, many):
        dec.free([0])
        dec.fork([1], [2])
        for path in ([[0], [], []], [[], [], [0]]):     # the drafts of a freed sequence and of a target are gone
            with pytest.raises(ValueError):
                dec.accept(path)
        dec.accept([[], list(range(10)), []])
        assert dec.kept == dec.lengths.tolist() == [0, 70, 60]
    a, b = (dec.step(xs[2], chains([0, 1, 1])) for dec in (few, many))
    assert torch.equal(a, b)


def test_refusals():
    dec = SparseDecoder.random(shape_of(torch.float16), 1, sequences=2, capacity=200)
    for call in (lambda: dec.fork([0], [1]), lambda: dec.free([0]), dec.compact):
        with pytest.raises(ValueError):
            call()
    dec = SparseDecoder.random(shape_of(torch.float16), 1, sequences=2, capacity=200, cache="int8", max_draft=5)
    with pytest.raises(ValueError):
        dec.step(torch.zeros(128, 6, dtype=torch.float16, device=DEV), chains([6, 0]))
    for a, b in (([0], [0]), ([0], [2]), ([0, 1], [1, 0])):
        with pytest.raises(nmg.NmgError):
            dec.fork(a, b)
    with pytest.raises(nmg.NmgError):
        dec.free([1, 1])
    dec.layers.append(SparseDecoder.random(shape_of(torch.float16), 1, 2, 200, block_norms="rms").layers[0])
    with pytest.raises(ValueError):
        SparseDecoder(dec.shape, dec.layers, 2, 200)
    for name in BLOCKS:                                                      # some blocks without
        layers = SparseDecoder.random(shape_of(torch.float16), 1, 2, 200, block_norms="rms").layers
        del layers[0].before[name]
        with pytest.raises(ValueError):
            SparseDecoder(dec.shape, layers, 2, 200)
    layers[0].before.clear()                                                 # norms after alone
    with pytest.raises(ValueError):
        SparseDecoder(dec.shape, layers, 2, 200)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norms_around_blocks(kind, dtype):
    """One token a sequence, so that attention over oneself is the value itself."""
    s = shape_of(dtype)
    dec = SparseDecoder.random(s, 2, sequences=3, capacity=8, seed=4, norms=False, block_norms=kind, branch_scale=0.6)
    dense = [{n: nmg.densify(*p).double().cpu() for n, p in layer.packed.items()} for layer in dec.layers]

    def norm(x, n):
        if kind == "layer":
            x = x - x.mean(0)
        x = x / (x.square().mean(0) + n.eps).sqrt() * n.weight.double().cpu()[:, None]
        return x if n.bias is None else x + n.bias.double().cpu()[:, None]

    x0 = torch.randn(128, 3, generator=torch.Generator().manual_seed(1)).to(dtype)
    x = x0.double()
    for layer, W in zip(dec.layers, dense):
        v = (W["qkv"] @ norm(x, layer.before["attention"]))[6 * 32:].view(2, 32, 3)
        a = W["ao"] @ v.repeat_interleave(2, 0).reshape(128, 3)
        x = x + 0.6 * norm(a, layer.after["attention"])
        u = W["up"] @ norm(x, layer.before["ffn"])
        x = x + 0.6 * norm(W["down"] @ (0.5 * u * (1 + torch.erf(u / math.sqrt(2)))), layer.after["ffn"])
    y = dec.step(x0.to(DEV), chains([1, 1, 1])).double().cpu()
    assert set(dec.layers[0].before) == set(BLOCKS)
    assert (y - x).abs().max() / x.abs().max() <= (40 * 2.0 ** -11 if dtype == torch.float16 else 1e-4)
