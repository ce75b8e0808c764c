"""The sparse decoder (``decoder.py``): drafts, kept tokens and an encoder's
states, against the same layers in binary64 from the densified weights, token
after token.

Tolerance: a layer rounds about 10 activations on the way to its output; in
binary16 (2^-11 each) two layers stay within 40 x 2^-11 of the outputs' scale,
in binary32 the sums' roundings stay within 1e-4 of it."""
import math

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


def reference(dec, dense, norms, states, path):
    """Outputs (binary64) of the tokens of `path` (hidden x tokens), each attending
    to itself and those before it and to `states`."""
    s, D = dec.shape, dec.shape.head_dim
    table = dec.table.double().cpu()
    c, n = (t[:, : path.shape[1]] for t in table)
    share, N = s.heads // s.kv_heads, path.shape[1]

    def rotate(x):                               # heads x D x N
        a, b = x[:, : D // 2], x[:, D // 2:]
        return torch.cat((a * c - b * n, a * n + b * c), 1)

    def norm(x, w):
        return x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * w[:, None]

    def attend(q, k, v, mask):
        out = torch.empty_like(q)
        for h in range(s.heads):
            score = q[h].t() @ k[h // share] / math.sqrt(D)
            out[h] = v[h // share] @ torch.softmax(score.masked_fill(~mask, -math.inf), 1).t()
        return out.reshape(s.heads * D, -1)

    x = path
    for W, (qn, kn) in zip(dense, norms):
        qkv = (W["qkv"] @ x).view(-1, D, N)
        q, k, v = qkv[: s.heads], qkv[s.heads:s.heads + s.kv_heads], qkv[s.heads + s.kv_heads:]
        if qn is not None:
            q, k = norm(q, qn), norm(k, kn)
        h = x + W["ao"] @ attend(rotate(q), rotate(k), v, torch.ones(N, N).tril().bool())
        kv = (W["cross_kv"] @ states).view(2, s.kv_heads, D, -1)
        a = attend((W["cross_q"] @ h).view(s.heads, D, N), kv[0], kv[1],
                   torch.ones(N, states.shape[1]).bool())
        h = h + W["cross_o"] @ a
        u = W["up"] @ h
        x = h + W["down"] @ (0.5 * u * (1 + torch.erf(u / math.sqrt(2))))
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("norms", [True, False])
def test_drafts_and_kept_tokens(dtype, norms):
    shape = DecoderShape(hidden=128, ffn=192, heads=4, kv_heads=2, head_dim=32, encoder_hidden=64,
                         n=2, m=4, g=8, dtype=dtype)
    dec = SparseDecoder.random(shape, 2, sequences=2, capacity=40, seed=3, norms=norms)
    dense = [{n: nmg.densify(*p).double().cpu() for n, p in layer.packed.items()} for layer in dec.layers]
    scales = [(None, None) if layer.q_norm is None else
              (layer.q_norm.double().cpu(), layer.k_norm.double().cpu()) for layer in dec.layers]
    g = torch.Generator().manual_seed(5)
    states = torch.randn(64, 50, generator=g).to(dtype)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)
    spans = ([0, 30], [30, 47])                  # the second sequence's states are shorter
    dec.set_encoder(states.to(DEV), i32(spans[0]), i32(spans[1]))
    limit = 40 * 2.0 ** -11 if dtype == torch.float16 else 1e-4

    kept = [torch.zeros(128, 0, dtype=torch.float64)] * 2
    drafts = [([[-1, 0, 1, 1, 0], [-1, -1]], [[0, 1, 3], [1]]),
              ([[-1], [-1, 0, 0, 2, 3, -1, 5, 6]], [[0], [0, 2, 3]]),
              ([[-1, 0], [-1]], [[], [0]]),
              ([[-1], [-1]], [[0], [0]])]
    for parents, keep in drafts:
        total = sum(len(p) for p in parents)
        x = torch.randn(128, total, generator=g).to(dtype)
        y = dec.step(x.to(DEV), parents).double().cpu()
        at = 0
        for b, p in enumerate(parents):
            for i in range(len(p)):
                line, up = [], i
                while up >= 0:
                    line.insert(0, at + up)
                    up = p[up]
                path = torch.cat((kept[b], x[:, line].double()), 1)
                ref = reference(dec, dense, scales, states[:, spans[0][b]:spans[1][b]].double(), path)
                err = (y[:, at + i] - ref[:, -1]).abs().max() / ref[:, -1].abs().max()
                assert err <= limit, (b, i, float(err))
            kept[b] = torch.cat((kept[b], x[:, [at + i for i in keep[b]]].double()), 1)
            at += len(p)
        dec.accept(keep)
        assert dec.lengths.tolist() == [k.shape[1] for k in kept]


def test_step_refusals():
    dec = SparseDecoder.random(DecoderShape(hidden=64, ffn=64, heads=2, kv_heads=1, head_dim=32, g=8, m=4),
                               1, sequences=1, capacity=4)
    x = torch.zeros(64, 2, dtype=torch.float16, device=DEV)
    for bad in ([[-1]], [[-1, 1]], [[-1, 0], [-1]], [[-2, 0]]):
        with pytest.raises(ValueError):
            dec.step(x, bad)
    with pytest.raises(ValueError):
        dec.step(torch.zeros(64, 5, dtype=torch.float16, device=DEV), [[-1, 0, 1, 2, 3]])
    with pytest.raises(ValueError):
        dec.accept([[0], [0]])
