"""The attention operators between sparse projections, as their users call them.

Activations are features x tokens, as everywhere in this library: a head's
rows, tokens contiguous.  Sequences are ranges of columns.

Every case is a plain dict; ``listed()`` holds the standing ones, ``draw(rng)``
one more of the same ranges.  ``prepare(case, seed)`` gives what a program has
in hand before the call, ``run(state)`` makes one pass: through the library's
entry points where ``own`` is true, else by elementary torch operations in
binary32.  ``work(case)`` is what a pass cannot do without, ``exact(case,
seed)`` its result in 64 bits.

Kinds:

    rotary    position rotation of the rows of ``heads`` heads (keys, or the
              queries of a layer without norms)
    qk_norm   RMS norm of every query and key head and the rotation, one pass
    cross     attention of each sequence's queries to a range of key columns
              (an encoder's states, packed; or the sequence itself)
    tree      attention of a tree of drafted tokens to a cache and to each
              other's ancestors
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16}
EPS = 1e-6
ROPE_BASE = 10000.0


def listed():
    return [
        # a decode step of a served batch of 8: one token each, where the launch counts
        dict(name="rotary_decode_f16", kind="rotary", dtype="f16", heads=12, dim=64, rot=64,
             inter=False, batch=8, tokens=8, context=512, scaling="none"),
        # a packed, unpadded batch; a quarter of the head rotated, pairs side by side
        dict(name="rotary_ragged_f16", kind="rotary", dtype="f16", heads=16, dim=64, rot=16,
             inter=True, batch=5, tokens=2047, context=1024, scaling="linear"),
        # one long prompt in binary32, frequencies scaled by parts for 8 times the context
        dict(name="rotary_long_f32", kind="rotary", dtype="f32", heads=16, dim=128, rot=128,
             inter=False, batch=1, tokens=16384, context=32768, scaling="parts"),
        # the same decode step for a model that norms its queries and keys
        dict(name="qk_norm_decode_f16", kind="qk_norm", dtype="f16", heads=12, kv_heads=12, dim=64,
             rot=64, inter=False, batch=8, tokens=8, context=512, scaling="none"),
        # the BERT-base-shaped encoder batch, 8 x 512 tokens, 12 heads
        dict(name="qk_norm_batch_f16", kind="qk_norm", dtype="f16", heads=12, kv_heads=12, dim=64,
             rot=64, inter=False, batch=8, tokens=4096, context=512, scaling="none"),
        # shared key heads, an odd number of packed tokens, binary32
        dict(name="qk_norm_ragged_f32", kind="qk_norm", dtype="f32", heads=16, kv_heads=4, dim=128,
             rot=64, inter=True, batch=7, tokens=8191, context=4096, scaling="ntk"),
        # a decoder's step: one query a sequence against the encoder's 512 states
        dict(name="cross_decode_f16", kind="cross", dtype="f16", heads=12, kv_heads=12, dim=64,
             batch=8, q_len=1, kv_len=512, ragged=False, masked=False),
        # the encoder batch attending to itself, 8 x 512
        dict(name="cross_batch_f16", kind="cross", dtype="f16", heads=12, kv_heads=12, dim=64,
             batch=8, q_len=512, kv_len=512, ragged=False, masked=False),
        # unpadded batch in binary32, padding and dropped states masked, one source empty
        dict(name="cross_ragged_f32", kind="cross", dtype="f32", heads=12, kv_heads=12, dim=64,
             batch=8, q_len=250, kv_len=701, ragged=True, masked=True),
        # a long target over a long source, shared key heads
        dict(name="cross_long_f16", kind="cross", dtype="f16", heads=16, kv_heads=4, dim=128,
             batch=1, q_len=4096, kv_len=16384, ragged=False, masked=False),
        # a short draft of a small model for one user
        dict(name="tree_short_f16", kind="tree", dtype="f16", heads=12, kv_heads=12, dim=64,
             batch=1, draft=8, kv_len=1000, ragged=False),
        # a wide draft over long caches, shared key heads
        dict(name="tree_long_f16", kind="tree", dtype="f16", heads=32, kv_heads=8, dim=128,
             batch=4, draft=63, kv_len=32768, ragged=True),
    ]


# The costliest listed cases: bytes moved, and scores (query heads x queries x
# keys), which the plain form holds in memory
_MOST_BYTES = 2 * 16 * 128 * 16384 * 4
_MOST_SCORES = 16 * 4096 * 16384


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("rotary", "qk_norm", "cross", "tree"))
    heads, kv_heads = rng.choice(((12, 12), (16, 16), (16, 4), (8, 1), (32, 8), (6, 2), (5, 5)))
    case = dict(kind=kind, dtype=rng.choice(("f32", "f16", "f16")), heads=heads,
                dim=rng.choice((64, 64, 128, 128, 32, 80, 96)))
    if kind in ("rotary", "qk_norm"):
        if kind == "qk_norm":
            case["kv_heads"] = kv_heads
        tokens = _log_int(rng, 1, 16384)
        case.update(rot=rng.choice((case["dim"], case["dim"] // 2, 16)), inter=rng.random() < 0.5,
                    batch=min(tokens, rng.randint(1, 9)), tokens=tokens,
                    context=_log_int(rng, 512, 32768),
                    scaling=rng.choice(("none", "linear", "ntk", "parts")))
        return case
    case.update(kv_heads=kv_heads, batch=_log_int(rng, 1, 16))
    if kind == "cross":
        case.update(q_len=_log_int(rng, 1, 4096), kv_len=_log_int(rng, 1, 16384),
                    ragged=rng.random() < 0.6, masked=rng.random() < 0.4)
    else:
        case.update(draft=_log_int(rng, 1, 64), kv_len=_log_int(rng, 16, 32768),
                    ragged=rng.random() < 0.6)
    return case


def draw(rng):
    while True:
        case = _draw_once(rng)
        w = work(case)
        if w["bytes"] > _MOST_BYTES:
            continue
        if case["kind"] in ("cross", "tree"):
            q, kv = _lengths(case)
            # half of the listed maximum: ragged cases are padded by the plain form,
            # and binary32 arithmetic costs more
            if 2 * case["heads"] * case["batch"] * max(q) * max(kv) > _MOST_SCORES:
                continue
        return case


# ------------------------------------------------------------------- lengths

def _spread(total, parts):
    """`parts` positive lengths of sum `total`, uneven where that is possible."""
    base = [total // parts + (1 if i < total % parts else 0) for i in range(parts)]
    for i in range(0, parts - 1, 2):
        d = base[i] // 3
        base[i], base[i + 1] = base[i] - d, base[i + 1] + d
    return base


def _lengths(case):
    """Queries and keys of every sequence (a function of the case alone)."""
    B = case["batch"]
    q_len = case["draft"] if case["kind"] == "tree" else case["q_len"]
    kv_len = case["kv_len"] + (case["draft"] if case["kind"] == "tree" else 0)
    if not case["ragged"]:
        return [q_len] * B, [kv_len] * B
    q = [q_len] * B if case["kind"] == "tree" else [max(1, q_len - (i * 37) % (q_len // 2 + 1))
                                                    for i in range(B)]
    kv = [max(q_len if case["kind"] == "tree" else 1, kv_len - (i * 971) % (kv_len // 2 + 1))
          for i in range(B)]
    return q, kv


def _kept(case, kv):
    """Per sequence, the keys a masked case keeps: about 7 of 8, the last of
    several sequences none."""
    if not case.get("masked"):
        return kv
    return [0 if i == len(kv) - 1 and i > 0 else k - k // 8 for i, k in enumerate(kv)]


# -------------------------------------------------------------------- inputs

def _frequencies(case):
    """Rotation frequencies in binary64, and the factor on cos and sin."""
    R, factor, scaling = case["rot"], 8.0, case["scaling"]
    base = ROPE_BASE * factor ** (R / (R - 2)) if scaling == "ntk" else ROPE_BASE
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        turns = (case["context"] / factor) * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        return f * (keep + (1 - keep) / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _token_tensors(case, seed):
    gen, dt = _gen(seed), DTYPES[case["dtype"]]
    D, N, L = case["dim"], case["tokens"], case["context"]
    kv = case.get("kv_heads", 0)
    # rows of a fused projection's output: queries, then keys, then values; a
    # feature's own scale beside N(0, 1)
    rows = (case["heads"] + 2 * kv) * D
    x = _randn(gen, (rows, N)) * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda"))
    s = dict(kind=case["kind"], dtype=dt, heads=case["heads"], kv_heads=kv, dim=D, rot=case["rot"],
             layout="interleaved" if case["inter"] else "half", x=x.to(dt))
    # each sequence's tokens follow one another from where its context ends
    lens = _spread(N, case["batch"])
    room = torch.tensor([max(1, L - n + 1) for n in lens], device="cuda")
    start = (torch.rand(len(lens), generator=gen, device="cuda", dtype=torch.float64) * room).long()
    ahead = torch.cat([torch.arange(n, device="cuda") for n in lens])
    s["positions"] = ((torch.repeat_interleave(start, torch.tensor(lens, device="cuda")) + ahead) % L).int()
    f, mag = _frequencies(case)
    angle = f.cuda()[:, None] * torch.arange(L, device="cuda", dtype=torch.float64)
    s["table"] = (torch.stack((angle.cos(), angle.sin())) * mag).float()
    if kv:
        s["wq"] = 1 + 0.1 * _randn(gen, (D,))
        s["wk"] = 1 + 0.1 * _randn(gen, (D,))
    return s


def _attention_tensors(case, seed):
    gen, dt = _gen(seed), DTYPES[case["dtype"]]
    H, G, D, B = case["heads"], case["kv_heads"], case["dim"], case["batch"]
    q, kv = _lengths(case)
    s = dict(kind=case["kind"], heads=H, kv_heads=G, dim=D, max_q=max(q), max_kv=max(kv),
             scale=1 / math.sqrt(D), q_offsets=_i32(_offsets(q)))
    # queries a little sharper than N(0, 1): attention that looks somewhere
    s["q"] = (1.5 * _randn(gen, (H * D, sum(q)))).to(dt)
    if case["kind"] == "tree":
        # caches of one capacity side by side; columns past a sequence's end
        # hold what earlier requests left there
        room = -(-(max(kv) + 1) // 64) * 64
        begin = [i * room for i in range(B)]
        cols = B * room
    else:
        begin = _offsets(kv)[:-1]
        cols = sum(kv)
    s["kv"] = _randn(gen, (2 * G * D, cols)).to(dt)
    s["kv_begin"] = _i32(begin)
    s["kv_end"] = _i32([b + n for b, n in zip(begin, kv)])
    if case["kind"] == "tree":
        T = case["draft"]
        # a random tree for every sequence: the parent of node i is the context
        # (-1) or an earlier node, near ones more often
        parent = torch.arange(T, device="cuda") - 1 - (
            torch.rand((B, T), generator=gen, device="cuda").square() * 4).long()
        see = torch.zeros((B, T, T), dtype=torch.bool, device="cuda")
        see[:, range(T), range(T)] = True
        for i in range(T):
            up = parent[:, i]
            rows = see[torch.arange(B, device="cuda"), up.clamp(min=0)] & (up >= 0)[:, None]
            see[:, i] |= rows
        s["tree"] = see.reshape(B * T, T).to(torch.uint8).contiguous()
    elif case["masked"]:
        # dropped states, and a last sequence whose states are all padding
        keep = torch.ones(cols, dtype=torch.uint8, device="cuda")
        at = 0
        for i, n in enumerate(kv):
            left = _kept(case, kv)[i]
            drop = torch.randperm(n, generator=gen, device="cuda")[: n - left]
            keep[at + drop] = 0
            at += n
        s["key_mask"] = keep
    return s


def prepare(case, seed):
    if case["kind"] in ("rotary", "qk_norm"):
        return _token_tensors(case, seed)
    return _attention_tensors(case, seed)


# ------------------------------------------------------------------ one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2304_07613_amd import nmg

    kind = s["kind"]
    if kind == "rotary":
        return nmg.rotary(s["x"], s["heads"], s["table"], s["positions"], s["layout"])
    if kind == "qk_norm":
        at, end = s["heads"] * s["dim"], (s["heads"] + s["kv_heads"]) * s["dim"]
        return nmg.qk_norm_rotary(s["x"][:at], s["x"][at:end], s["heads"], s["kv_heads"], s["wq"],
                                  s["wk"], s["table"], s["positions"], s["layout"], EPS)
    half = s["kv"].shape[0] // 2
    k, v = s["kv"][:half], s["kv"][half:]
    if kind == "cross":
        return nmg.attention(s["q"], k, v, s["heads"], s["kv_heads"], s["q_offsets"], s["kv_begin"],
                             s["kv_end"], s.get("key_mask"), s["scale"])
    return nmg.tree_attention(s["q"], k, v, s["heads"], s["kv_heads"], s["q_offsets"], s["kv_begin"],
                              s["kv_end"], s["tree"], s["scale"])


def _rotate(x, s):
    """x: heads x D x N in binary32."""
    R, at = s["rot"], s["positions"].long()
    c, n = s["table"][0][:, at], s["table"][1][:, at]
    if s["layout"] == "half":
        a, b = x[:, : R // 2], x[:, R // 2:R]
        turned = torch.cat((a * c - b * n, a * n + b * c), dim=1)
    else:
        a, b = x[:, 0:R:2], x[:, 1:R:2]
        turned = torch.stack((a * c - b * n, a * n + b * c), dim=2).flatten(1, 2)
    return torch.cat((turned, x[:, R:]), dim=1)


def _normed(x, w):
    return x * (1 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)) * w[:, None]


def _run_plain(s):
    kind, H, D = s["kind"], s["heads"], s["dim"]
    if kind == "rotary":
        x = s["x"].float().view(H, D, -1)
        return _rotate(x, s).reshape(H * D, -1).to(s["dtype"])
    if kind == "qk_norm":
        at, end = H * D, (H + s["kv_heads"]) * D
        q = _normed(s["x"][:at].float().view(H, D, -1), s["wq"])
        k = _normed(s["x"][at:end].float().view(s["kv_heads"], D, -1), s["wk"])
        return (_rotate(q, s).reshape(at, -1).to(s["dtype"]),
                _rotate(k, s).reshape(end - at, -1).to(s["dtype"]))
    return _attend_plain(s)


def _attend_plain(s):
    H, G, D, T, S = s["heads"], s["kv_heads"], s["dim"], s["max_q"], s["max_kv"]
    dev, q, kv = s["q"].device, s["q"], s["kv"]
    offsets, begin, end = s["q_offsets"].long(), s["kv_begin"].long(), s["kv_end"].long()
    B = begin.shape[0]
    step_q, step_k = torch.arange(T, device=dev), torch.arange(S, device=dev)
    # every sequence padded to the longest one's queries and keys
    q_at = (offsets[:-1, None] + step_q).clamp(max=q.shape[1] - 1)
    k_at = (begin[:, None] + step_k).clamp(max=kv.shape[1] - 1)
    allowed = ((begin[:, None] + step_k) < end[:, None])[:, None, :]              # B x 1 x S
    if "key_mask" in s:
        allowed = allowed & (s["key_mask"][k_at] != 0)[:, None, :]
    if "tree" in s:
        drafted = step_k - (end - begin - T)[:, None]                             # B x S
        seen = s["tree"].view(B, T, T).gather(2, drafted.clamp(0, T - 1)[:, None, :].expand(B, T, S))
        allowed = allowed & ((drafted < 0)[:, None, :] | (seen != 0))             # B x T x S
    qp = q[:, q_at].float().view(G, H // G, D, B, T).permute(3, 0, 1, 4, 2).reshape(B, G, -1, D)
    kp = kv[: G * D][:, k_at].float().view(G, D, B, S).permute(2, 0, 1, 3).contiguous()
    vp = kv[G * D:][:, k_at].float().view(G, D, B, S).permute(2, 0, 3, 1).contiguous()
    score = torch.matmul(qp, kp).mul_(s["scale"]).view(B, G, H // G, T, S)
    score = score.masked_fill_(~allowed[:, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True).clamp_(min=-3.0e38)       # a row with nothing left: 0
    weight = score.sub_(top).exp_()
    total = weight.sum(dim=-1, keepdim=True)
    weight = weight.div_(torch.where(total == 0, torch.ones_like(total), total))
    out = torch.matmul(weight.view(B, G, -1, S), vp).view(B, H, T, D)
    # back to packed columns
    column = torch.arange(q.shape[1], device=dev)
    which = torch.searchsorted(offsets, column, right=True) - 1
    return out[which, :, column - offsets[which]].permute(1, 2, 0).reshape(H * D, -1).to(q.dtype)


# ---------------------------------------------------------------------- work

def work(case):
    es, D, H = (4 if case["dtype"] == "f32" else 2), case["dim"], case["heads"]
    if case["kind"] in ("rotary", "qk_norm"):
        N, R = case["tokens"], case["rot"]
        heads = H + case.get("kv_heads", 0)
        positions = min(max(_spread(N, case["batch"])), case["context"])
        norm = 4 * D if case["kind"] == "qk_norm" else 0
        return dict(bytes=2 * heads * D * N * es + 4 * N + 4 * R * positions,
                    flops=heads * N * (3 * R + norm))
    q, kv = _lengths(case)
    kept = _kept(case, kv)
    flops = 4 * D * H * sum(a * b for a, b in zip(q, kept))
    extra = 4 * (3 * len(q) + 1)
    if case["kind"] == "tree":
        T = case["draft"]
        # a drafted token sees at least itself of the draft
        flops = 4 * D * H * sum(a * (b - T + 1) for a, b in zip(q, kv))
        extra += len(q) * T * T
    elif case["masked"]:
        extra += sum(kv)
    return dict(bytes=2 * H * D * sum(q) * es + 2 * case["kv_heads"] * D * sum(kept) * es + extra,
                flops=flops)


# ------------------------------------------------------------- 64-bit results

def _turn64(x, case, positions):
    """The rotation of x (rows of one head x N, binary64) as complex numbers."""
    f, mag = _frequencies(case)
    R = case["rot"]
    # the angles' cosines and sines are binary32 inputs
    a = f.cuda()[:, None] * positions.double()[None, :]
    e = torch.complex((a.cos() * mag).float().double(), (a.sin() * mag).float().double())
    y = x.clone()
    first = slice(0, R, 2) if case["inter"] else slice(0, R // 2)
    second = slice(1, R, 2) if case["inter"] else slice(R // 2, R)
    z = torch.complex(x[first].contiguous(), x[second].contiguous()) * e
    y[first], y[second] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    H, D = case["heads"], case["dim"]
    if case["kind"] in ("rotary", "qk_norm"):
        groups = [(s["x"][: H * D], s.get("wq"))]
        if case["kind"] == "qk_norm":
            groups.append((s["x"][H * D:(H + case["kv_heads"]) * D], s["wk"]))
        outs = []
        for x, w in groups:
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[0] // D):
                r = x[h * D:(h + 1) * D].double()
                if w is not None:
                    r = r / ((r * r).sum(dim=0) / D + EPS).sqrt() * w.double()[:, None]
                y[h * D:(h + 1) * D] = _turn64(r, case, s["positions"])
            outs.append(y)
        return outs[0] if len(outs) == 1 else tuple(outs)
    q_len, kv_len = _lengths(case)
    starts, begins = _offsets(q_len), s["kv_begin"].tolist()
    share = H // case["kv_heads"]
    half = s["kv"].shape[0] // 2
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        cols = torch.arange(begins[b], begins[b] + kv_len[b], device="cuda")
        if "key_mask" in s:
            cols = cols[s["key_mask"][cols] != 0]
        if cols.numel() == 0:
            continue
        at = slice(starts[b], starts[b + 1])
        hidden = None
        if "tree" in s:
            hidden = torch.zeros((q_len[b], kv_len[b]), dtype=torch.bool, device="cuda")
            hidden[:, kv_len[b] - q_len[b]:] = s["tree"][at][:, : q_len[b]] == 0
        for h in range(H):
            g = h // share
            k = s["kv"][g * D:(g + 1) * D, cols].double()
            v = s["kv"][half + g * D:half + (g + 1) * D, cols].double()
            logit = (s["q"][h * D:(h + 1) * D, at].double().t().contiguous() @ k) * s["scale"]
            if hidden is not None:
                logit[hidden] = -math.inf
            out[h * D:(h + 1) * D, at] = (torch.softmax(logit, dim=1) @ v.t().contiguous()).t()
    return out
