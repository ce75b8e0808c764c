"""A decoder on n:m:g weights: drafted tokens over a cache, an encoder's states.

Every projection of a layer is a sparse weight packed by ``nmg.compress``; what
stands between them are the attention operators.  Activations are features x
tokens.  A layer (residual sums as in ``stack.py``, no LayerNorm):

    q, k, v = rows of QKV x
    q, k    = norms of every head and the rotation (or the rotation alone)
    h       = x + AO(attention of the drafted tokens to cache and ancestors)
    h       = h + CO(attention of CQ h to the encoder's keys and values)
    y       = h + Down(GELU(Up(h)))

Several tokens are drafted at once as a tree (``step``); those that turn out
right are kept (``accept``), the others' columns of the cache are overwritten by
the next draft.  One token a sequence is a tree of one node.

The cache of a layer holds keys and values of `capacity` columns for every
sequence side by side; ``torch`` holds the buffers and moves cache columns.
"""
from __future__ import annotations

from dataclasses import dataclass, field

import torch

from . import nmg, synth

NAMES = ("qkv", "ao", "cross_q", "cross_kv", "cross_o", "up", "down")


@dataclass(frozen=True)
class DecoderShape:
    hidden: int = synth.BERT_HIDDEN
    ffn: int = synth.BERT_FFN
    heads: int = 12
    kv_heads: int = 12
    head_dim: int = 64
    encoder_hidden: int = synth.BERT_HIDDEN
    n: int = 2
    m: int = 8
    g: int = 8
    dtype: torch.dtype = torch.float16

    def weights(self) -> dict:
        """Rows and columns of every projection."""
        q, kv = self.heads * self.head_dim, self.kv_heads * self.head_dim
        return {"qkv": (q + 2 * kv, self.hidden), "ao": (self.hidden, q),
                "cross_q": (q, self.hidden), "cross_kv": (2 * kv, self.encoder_hidden),
                "cross_o": (self.hidden, q), "up": (self.ffn, self.hidden),
                "down": (self.hidden, self.ffn)}


@dataclass
class DecoderLayer:
    packed: dict                                 # name -> (values, indices, layout)
    q_norm: torch.Tensor | None = None           # float32, head_dim; None: rotation alone
    k_norm: torch.Tensor | None = None
    keys: torch.Tensor | None = None             # the cache: kv_heads * head_dim x columns
    values: torch.Tensor | None = None
    cross: tuple = field(default_factory=tuple)  # the encoder's keys and values

    def linear(self, name, x):
        v, idx, layout = self.packed[name]
        return nmg.spmm(v, idx, x, layout)

    def fused(self, name, x, epilogue, r=None):
        v, idx, layout = self.packed[name]
        return nmg.spmm_epilogue(v, idx, x, layout, epilogue, r)


class SparseDecoder:
    def __init__(self, shape: DecoderShape, layers, sequences: int, capacity: int,
                 base: float = 10000.0, pairs: str = "half", **scaling):
        self.shape, self.layers, self.capacity, self.pairs = shape, layers, capacity, pairs
        device = layers[0].packed["qkv"][0].device
        self.table = nmg.rotary_table(capacity, shape.head_dim, base, device=device, **scaling)
        rows = shape.kv_heads * shape.head_dim
        for layer in layers:
            layer.keys = torch.zeros((rows, sequences * capacity), dtype=shape.dtype, device=device)
            layer.values = torch.zeros_like(layer.keys)
        self.begin = torch.arange(sequences, dtype=torch.int32, device=device) * capacity
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)   # kept tokens
        self.encoder_begin = self.encoder_end = None
        self.draft = [[] for _ in range(sequences)]     # the parents of the last step

    @classmethod
    def random(cls, shape: DecoderShape, n_layers: int, sequences: int, capacity: int, seed: int = 0,
               norms: bool = True, device="cuda:0", **kw):
        """A decoder of seeded normal weights."""
        layers = []
        for i in range(n_layers):
            packed = {}
            for j, (name, (M, K)) in enumerate(shape.weights().items()):
                W = synth.normal((M, K), 1000 * seed + 10 * i + j, synth.W_STD, shape.dtype).to(device)
                packed[name] = nmg.compress(W, shape.n, shape.m, shape.g)
            layer = DecoderLayer(packed)
            if norms:
                layer.q_norm = (1 + 0.1 * synth.normal((shape.head_dim,), 7 + i)).to(device)
                layer.k_norm = (1 + 0.1 * synth.normal((shape.head_dim,), 57 + i)).to(device)
            layers.append(layer)
        return cls(shape, layers, sequences, capacity, **kw)

    def set_encoder(self, states: torch.Tensor, begin: torch.Tensor, end: torch.Tensor):
        """The encoder's states (encoder_hidden x columns) that sequence b attends
        to: columns begin[b] .. end[b] - 1 (int32).  Their keys and values are made
        once."""
        rows = self.shape.kv_heads * self.shape.head_dim
        self.encoder_begin, self.encoder_end = begin, end
        for layer in self.layers:
            kv = layer.linear("cross_kv", states)
            layer.cross = (kv[:rows], kv[rows:])

    def step(self, x: torch.Tensor, parents: list) -> torch.Tensor:
        """One pass over drafted tokens: x (hidden x tokens) holds every sequence's
        draft in turn; parents[b][i] is the draft's index of token i's parent, -1
        for one that follows the kept tokens.  Returns their outputs."""
        counts = [len(p) for p in parents]
        if len(counts) != len(self.begin) or sum(counts) != x.shape[1] or not sum(counts):
            raise ValueError("x must hold one column for every drafted token of every sequence")
        tree = torch.zeros((sum(counts), max(counts)), dtype=torch.uint8)
        depth, row = [], 0
        for p in parents:
            for i, up in enumerate(p):
                if not -1 <= up < i:
                    raise ValueError("a parent comes before its token")
                if up >= 0:
                    tree[row + i] = tree[row + up]
                tree[row + i, i] = 1
                depth.append(int(tree[row + i].sum()) - 1)
            row += len(p)
        dev = x.device
        tree, depth = tree.to(dev), torch.tensor(depth, dtype=torch.int32, device=dev)
        counts = torch.tensor(counts, dtype=torch.int32, device=dev)
        if int((self.lengths + counts).max()) > self.capacity:
            raise ValueError("the cache is full")
        offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).int()
        which = torch.repeat_interleave(torch.arange(len(counts), device=dev), counts)
        ends = self.begin + self.lengths + counts
        # drafted token i of a sequence goes behind its kept tokens
        columns = (self.begin + self.lengths - offsets[:-1])[which] + \
            torch.arange(x.shape[1], device=dev)
        positions = (self.lengths[which] + depth).int()
        self.draft = [[] for _ in parents]
        s = self.shape
        q_rows, kv_rows = s.heads * s.head_dim, s.kv_heads * s.head_dim
        for layer in self.layers:
            qkv = layer.linear("qkv", x)
            q, k, v = qkv[:q_rows], qkv[q_rows:q_rows + kv_rows], qkv[q_rows + kv_rows:]
            if layer.q_norm is not None:
                nmg.qk_norm_rotary(q, k, s.heads, s.kv_heads, layer.q_norm, layer.k_norm, self.table,
                                   positions, self.pairs, out=(q, k))
            else:   # queries and keys are rows of one matrix: heads of one call
                qk = qkv[:q_rows + kv_rows]
                nmg.rotary(qk, s.heads + s.kv_heads, self.table, positions, self.pairs, out=qk)
            layer.keys.index_copy_(1, columns, k)
            layer.values.index_copy_(1, columns, v)
            a = nmg.tree_attention(q, layer.keys, layer.values, s.heads, s.kv_heads, offsets,
                                   self.begin, ends, tree)
            h = layer.fused("ao", a, "add", x)
            if layer.cross:
                a = nmg.attention(layer.linear("cross_q", h), *layer.cross, s.heads, s.kv_heads,
                                  offsets, self.encoder_begin, self.encoder_end)
                h = layer.fused("cross_o", a, "add", h)
            x = layer.fused("down", layer.fused("up", h, "gelu"), "add", h)
        self.draft = [list(p) for p in parents]
        return x

    def accept(self, kept: list):
        """Keep drafted tokens of the last step: kept[b] are indices of sequence b's
        draft along one path, the first one's parent -1; their columns move behind
        the kept tokens.  A draft is accepted from once."""
        if len(kept) != len(self.begin):
            raise ValueError("one list of kept tokens for every sequence")
        for path, parents in zip(kept, self.draft):
            last = -1
            for i in path:
                if not 0 <= i < len(parents) or parents[i] != last:
                    raise ValueError("kept tokens are one path through their sequence's last draft")
                last = i
        start = (self.begin + self.lengths).tolist()
        source = [start[b] + i for b, path in enumerate(kept) for i in path]
        target = [start[b] + i for b, path in enumerate(kept) for i in range(len(path))]
        if source:
            dev = self.begin.device
            source, target = (torch.tensor(t, device=dev) for t in (source, target))
            for layer in self.layers:
                for cache in (layer.keys, layer.values):
                    cache.index_copy_(1, target, cache.index_select(1, source))
        self.lengths += torch.tensor([len(path) for path in kept], dtype=torch.int32,
                                     device=self.begin.device)
        self.draft = [[] for _ in kept]
