"""More operators of a decoder layer, as the executor of a placement runs them: the norms around a block with its gate
and residual scale, and a paged cache held in 8 bits, with keys rotated into it on the way and the attention that reads it.

Cases, states and outputs are those of operators.py: ``run`` makes one pass through one operator, in its plain form
(elementary torch operations in 32 bits, rounded once at the end) or, where ``own`` is true, through ``gmgop``.

A cache in 8 bits: a page holds codes [layers, 2 (K, V), kv_heads, page tokens, dim] in e4m3, then, in fp32, a scale
[layers, 2, kv_heads, page tokens / 16] for each block of 16 tokens and head; a value is its code times its scale.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
DEV = "cuda"
BLOCK = 16                       # tokens that share a scale
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _norm(name, rows, n, kind="rms", dtype="bf16", stream="same", block=True, after=False, bias=False, gate="none",
          scale=1.0):
    return dict(name=name, op="norm", rows=rows, n=n, kind=kind, dtype=dtype, stream=stream, block=block, after=after,
                bias=bias, gate=gate, scale=scale)


def _append(name, tokens, seqs, heads, kv_heads, dim, rotary, top, dtype="bf16", interleaved=False, page=16):
    return dict(name=name, op="append", tokens=tokens, seqs=seqs, heads=heads, kv_heads=kv_heads, dim=dim,
                rotary=rotary, top=top, dtype=dtype, interleaved=interleaved, page=page)


def _attend(name, groups, members, prefix, suffix, q_max, heads, kv_heads, dim, page=16, dtype="bf16", lens=1):
    return dict(name=name, op="attend", groups=groups, members=members, prefix=prefix, suffix=suffix, q_max=q_max,
                heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, lens=lens)


def listed():
    return [
        # one token of one request: the projection's result added to the residual stream and the next block's input
        # normalised, where the launch is all that counts
        _norm("norm_token", 1, 4096),
        # a ragged batch of odd width, with means, biases and a gate for each token
        _norm("norm_ragged", 333, 5003, kind="layer", dtype="fp16", bias=True, gate="row", scale=0.25),
        # prompts with the residual stream in 32 bits, norms on both sides of the block and a gate for each channel
        _norm("norm_prompt", 16384, 4096, stream="fp32", after=True, gate="column", scale=0.5),
        # a decode step of 16 requests: rotate one token each into blocks that are partly filled
        _append("append_step", 16, 16, 32, 8, 128, 128, 8000),
        # drafted and resumed tokens of several requests at odd positions, a partly rotated and interleaved head
        _append("append_chunk", 777, 9, 20, 4, 80, 32, 6000, dtype="fp16", interleaved=True, page=64),
        # the prompts of a long context
        _append("append_prompt", 32768, 3, 32, 8, 128, 128, 200000),
        # a small decode step over a short shared prompt
        _attend("attend8_step", 1, 8, 500, 60, 1, 32, 8, 128),
        # a decode step of many requests with histories of their own: reading the cache is all that counts
        _attend("attend8_decode", 64, 1, 9000, 300, 1, 32, 8, 128, lens=2),
        # drafted tokens of a single long request, spread over the whole GPU
        _attend("attend8_long", 1, 1, 131072, 40, 4, 40, 8, 128, page=64, dtype="fp16", lens=3),
        # a large decode step over a long shared document
        _attend("attend8_shared", 1, 96, 32768, 700, 1, 32, 8, 128, lens=4),
        # chunks of new prompt tokens behind the prompts of several tenants
        _attend("attend8_chunk", 4, 6, 4000, 900, 700, 24, 8, 64, page=32, lens=5),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("norm", "append", "attend", "attend"))
    if op == "norm":
        n = _log(rng, 64, 16384)
        if rng.random() < 0.7:
            n = -(-n // 64) * 64
        c = _norm("", _log(rng, 1, min(16384, 16384 * 4096 // n)), n, kind=rng.choice(("rms", "layer")),
                  dtype=rng.choice(("bf16", "fp16")), stream=rng.choice(("same", "fp32")), block=rng.random() < 0.8,
                  after=rng.random() < 0.4, bias=rng.random() < 0.4, gate=rng.choice(("none", "row", "column", "full")),
                  scale=rng.choice((1.0, 0.5, 0.22)))
        if not c["block"]:
            c.update(after=False, gate="none", scale=1.0)
    elif op == "append":
        dim, kv = rng.choice((64, 80, 96, 128)), rng.choice((1, 2, 4, 8))
        tokens = _log(rng, 1, 32768)
        seqs = min(tokens, _log(rng, 1, 64))
        c = _append("", tokens, seqs, kv * rng.choice((1, 4, 5)), kv, dim, rng.choice((dim, dim // 2, 32)),
                    max(rng.choice((6000, 40000, 200000)), 2 * (-(-tokens // seqs))), dtype=rng.choice(("bf16", "fp16")),
                    interleaved=rng.random() < 0.5, page=rng.choice((16, 32, 64)))
    else:
        while True:
            groups, members = _log(rng, 1, 64), 1 if rng.random() < 0.4 else _log(rng, 2, 96)
            prefix, suffix = _log(rng, 16, 131072), _log(rng, 4, 1000)
            q_max = 1 if rng.random() < 0.6 else _log(rng, 2, 700)
            tokens = groups * members * q_max
            if groups * members <= 128 and tokens * (prefix + suffix) <= 50_000_000 and groups * prefix <= 500_000:
                break
        kv = rng.choice((1, 2, 8))
        c = _attend("", groups, members, prefix, suffix, q_max, kv * rng.choice((1, 4, 5, 8)), kv,
                    rng.choice((64, 80, 128)), page=rng.choice((16, 32, 64)), dtype=rng.choice(("bf16", "fp16")),
                    lens=rng.randrange(1 << 30))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Lengths, tables and pages of a case
# ---------------------------------------------------------------------------

def _attend_lens(c):
    """(prefix of each group, group of each request, new tokens of each request, cached tokens of each request)."""
    r = random.Random(c["lens"])
    prefix = [r.randint((3 * c["prefix"] + 3) // 4, c["prefix"]) for _ in range(c["groups"])]
    group, q, kv = [], [], []
    for g in range(c["groups"]):
        for _ in range(c["members"]):
            n = 1 if c["q_max"] == 1 else r.randint(max(1, c["q_max"] // 7), c["q_max"])
            group.append(g)
            q.append(n)
            kv.append(prefix[g] + n + r.randint(0, max(0, c["suffix"] - n)))
    return prefix, group, q, kv


def _freqs(c):
    """The angle of one position for each pair, in 64 bits."""
    return 10000.0 ** (-2.0 * np.arange(c["rotary"] // 2) / c["rotary"])


def _pool(g, n_pages, kv_heads, page, dim):
    """Pages in 8 bits with random contents: (pool, its codes, its scales); the scales are powers of two, as values of
    blocks of different size leave them."""
    n = 2 * kv_heads * page * dim
    more = 2 * kv_heads * (page // BLOCK) * 4
    pool = torch.zeros(n_pages, -(-(n + more) // 128) * 128, dtype=torch.uint8, device=DEV)
    codes = pool[:, :n].unflatten(1, (1, 2, kv_heads, page, dim))
    for a in range(0, n_pages, 4096):
        part = codes[a:a + 4096]
        part.copy_((torch.randn(part.shape, generator=g, device=DEV) * 80).clamp(-448, 448).to(F8).view(torch.uint8))
    scales = pool[:, n:n + more].view(torch.float32).unflatten(1, (1, 2, kv_heads, page // BLOCK))
    scales.copy_(torch.exp2(torch.randint(-7, -4, scales.shape, generator=g, device=DEV).float()))
    return pool, codes, scales


def _powers(least, most, dtype):
    """2 ^ least .. 2 ^ most, exactly."""
    return torch.tensor([2.0 ** i for i in range(least, most + 1)], dtype=dtype, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2 + 1)
    return g


# ---------------------------------------------------------------------------
# What a program has in hand before the call
# ---------------------------------------------------------------------------

def prepare(case, seed):
    s = dict(case=case)
    g = _gen(seed)
    c, dt = case, DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    if c["op"] == "norm":
        m, n = c["rows"], c["n"]
        # a residual stream grows over the layers, and some channels are far larger than the others
        size = torch.exp(torch.randn(n, generator=g, device=DEV))
        s.update(x=((torch.randn(m, n, generator=g, device=DEV) + 0.1) * size).to(dt if c["stream"] == "same" else torch.float32),
                 w=1 + normal(n, scale=0.2), bias=normal(n, scale=0.1) if c["bias"] else None,
                 y=normal(m, n) + 0.25 if c["block"] else None, y_w=1 + normal(n, scale=0.2) if c["after"] else None,
                 y_bias=normal(n, scale=0.1) if c["after"] and c["bias"] else None,
                 gate={"none": lambda: None, "row": lambda: normal(m, 1), "column": lambda: normal(n),
                       "full": lambda: normal(m, n)}[c["gate"]]())
        return s
    if c["op"] == "append":
        T, H, Hk, D, page = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["page"]
        # tokens of each request follow one another; the heads lie in one row, as the product before leaves them
        per = -(-T // c["seqs"])
        seq = np.arange(T) // per
        first = np.random.default_rng(seed).integers(0, c["top"] - per, c["seqs"])
        pos = first[seq] + np.arange(T) % per
        cols = -(-c["top"] // page) + 1
        table = np.full((c["seqs"], cols), -1, np.int32)
        used = [np.unique(pos[seq == b] // page) for b in range(c["seqs"])]
        n = c["seqs"] * (-(-per // page) + 1) + 3                # as many pages as any first positions take
        ids = np.random.default_rng(seed + 1).permutation(n).astype(np.int32)
        at = 0
        for b, u in enumerate(used):
            table[b, u] = ids[at:at + len(u)]
            at += len(u)
        s.update(row=normal(T, (H + 2 * Hk) * D, scale=1.4), pos=torch.from_numpy(pos.astype(np.int32)).to(DEV),
                 seq=torch.from_numpy(seq.astype(np.int32)).to(DEV), table=torch.from_numpy(table).to(DEV), freqs=_freqs(c))
        s["pool"], s["codes"], s["scales"] = _pool(g, n, Hk, page, D)
        if own:
            from paper_2608_15762_gb300 import gmgop
            s["rope"] = gmgop.Rope(c["rotary"], freqs=s["freqs"], interleaved=c["interleaved"], device=DEV)
            s["cache"] = gmgop.PageCache8(s["pool"], 1, Hk, page, D, table=s["table"])
        else:
            # a program without the operator keeps the angles' cosines and sines
            a = torch.arange(c["top"], device=DEV, dtype=torch.float64)[:, None] * torch.from_numpy(s["freqs"]).to(DEV)
            s["cos"], s["sin"] = torch.cos(a).float(), torch.sin(a).float()
        return s
    prefix, group, q, kv = _attend_lens(c)
    B, page, Hk, D = len(q), c["page"], c["kv_heads"], c["dim"]
    cols = max(-(-n // page) for n in kv)
    table, at = np.full((B, cols), -1, np.int32), 0
    total = sum(p // page for p in prefix) + sum(-(-kv[b] // page) - prefix[group[b]] // page for b in range(B))
    ids = np.random.default_rng(seed).permutation(total + 2).astype(np.int32)
    for b in range(B):
        full, need = prefix[group[b]] // page, -(-kv[b] // page)
        full_from = full if b % c["members"] else 0
        table[b, :full_from] = table[b - b % c["members"], :full_from]
        table[b, full_from:need] = ids[at:at + need - full_from]
        at += need - full_from
    pool, codes, scales = _pool(g, total + 2, Hk, page, D)
    # a page that the prefix ends in was copied, scales and all, when the requests were forked; what a request wrote
    # behind it came with scales of its own, but for the block that the prefix ends in
    for b in range(B):
        lead, tail = b - b % c["members"], prefix[group[b]] % page
        if tail and b != lead:
            k = prefix[group[b]] // page
            to, frm = int(table[b, k]), int(table[lead, k])
            codes[to, :, :, :, :tail] = codes[frm, :, :, :, :tail]
            scales[to, :, :, :, :-(-tail // BLOCK)] = scales[frm, :, :, :, :-(-tail // BLOCK)]
    s.update(q=normal(sum(q), c["heads"], D), pool=pool, codes=codes, scales=scales, table=torch.from_numpy(table).to(DEV),
             scale=D ** -0.5, lens=(prefix, group, q, kv))
    if own:
        from paper_2608_15762_gb300 import gmgop
        s["cache"] = gmgop.PageCache8(pool, 1, Hk, page, D, table=s["table"])
        shared = {} if c["members"] == 1 else dict(group_off=[i * c["members"] for i in range(c["groups"] + 1)],
                                                   prefix=prefix)
        s["plan"] = gmgop.AttendPlan8(q, kv, c["heads"], Hk, D, page, device=DEV, **shared)
    else:
        first = np.cumsum([0] + q)[:-1]
        b_of = np.repeat(np.arange(B), q)
        qi = np.arange(sum(q)) - first[b_of]
        g_of = np.asarray(group)[b_of]
        g_first = np.asarray([first[i * c["members"]] for i in range(c["groups"])])
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).to(DEV)  # noqa: E731
        s.update(b_of=up(b_of), qi=up(qi), g_of=up(g_of), gi=up(np.arange(sum(q)) - g_first[g_of]),
                 kv=up(np.asarray(kv)), n_q=up(np.asarray(q)), pre=up(np.asarray(prefix)), grp=up(np.asarray(group)),
                 lead=up(np.arange(c["groups"]) * c["members"]))
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

EPS = 1e-6


def _normed(v, w, bias, kind):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w.float()
    return v if bias is None else v + bias.float()


def _plain_norm(s):
    c, r = s["case"], s["x"].float()
    dt = s["w"].dtype
    if s["y"] is None:
        return _normed(r, s["w"], s["bias"], c["kind"]).to(dt)
    z = s["y"].float()
    if s["y_w"] is not None:
        z = _normed(z, s["y_w"], s["y_bias"], c["kind"])
    if s["gate"] is not None:
        z = z * s["gate"].float()
    r = r + z * c["scale"]
    return _normed(r, s["w"], s["bias"], c["kind"]).to(dt), r.to(s["x"].dtype)


def _heads(s):
    c = s["case"]
    T, H, Hk, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
    row = s["row"]
    return (row[:, :H * D].view(T, H, D), row[:, H * D:(H + Hk) * D].view(T, Hk, D),
            row[:, (H + Hk) * D:].view(T, Hk, D))


def _turn(s, x):
    """The rotated heads of x [T, heads, dim], in 32 bits."""
    c, R = s["case"], s["case"]["rotary"]
    pos = s["pos"].long()
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    x = x.float()
    if c["interleaved"]:
        u, v = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((u * cos - v * sin, u * sin + v * cos), -1).flatten(-2)
    else:
        u, v = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _needed(top):
    """The least power of two that brings `top` to at most 448."""
    m, e = torch.frexp(top)
    e = torch.where(top == 0, -60, e - 9 + (m > 0.875))
    return _powers(-60, 60, top.dtype)[e.clamp(-60, 60).long() + 60]


def _put(s, which, x):
    """x [T, kv_heads, dim] into the keys (0) or values (1) of the cache: the blocks that it touches get the scale that
    they need, and what they held before its first token is rounded again where that one is larger."""
    c, page = s["case"], s["case"]["page"]
    pos, seq = s["pos"].long(), s["seq"].long()
    codes, scales = s["codes"][:, 0, which], s["scales"][:, 0, which]
    at = s["table"][seq, pos // page].long()
    place = at * (page // BLOCK) + pos % page // BLOCK
    _, group = torch.unique_consecutive(place, return_inverse=True)
    head = torch.ones_like(group, dtype=torch.bool)
    head[1:] = group[1:] != group[:-1]
    lead = head.nonzero()[:, 0]
    p, b, first = at[lead], pos[lead] % page // BLOCK, pos[lead] % BLOCK
    tops = x.abs().amax(-1)
    need = _needed(torch.zeros(len(lead), x.shape[1], device=x.device, dtype=x.dtype).scatter_reduce_(
        0, group[:, None].expand_as(tops), tops, "amax"))
    old = scales[p, :, b].to(x.dtype)
    new = torch.where(first[:, None] > 0, torch.maximum(old, need), need)
    slots = torch.arange(BLOCK, device=x.device)
    where = b[:, None] * BLOCK + slots
    held = codes[p[:, None], :, where].view(F8).to(x.dtype) * (old / new)[:, None, :, None]
    kept = (slots < first[:, None])[..., None, None]
    codes[p[:, None], :, where] = torch.where(kept, held.to(F8).view(torch.uint8), codes[p[:, None], :, where])
    codes[at, :, pos % page] = (x / new[group][..., None]).to(F8).view(torch.uint8)
    scales[p, :, b] = new.float()


def _plain_append(s):
    q, k, v = _heads(s)
    _put(s, 0, _turn(s, k))
    _put(s, 1, v.float())
    return _turn(s, q).to(q.dtype), s["codes"].view(F8), s["scales"]


def _values(s, which, pages, slot=None):
    """The values of keys (0) or values (1) of whole pages, or of one slot of each, in 32 bits."""
    codes, scales = s["codes"][:, 0, which], s["scales"][:, 0, which]
    if slot is None:
        return codes[pages].view(F8).float() * scales[pages].repeat_interleave(BLOCK, -1)[..., None]
    return codes[pages, :, slot].view(F8).float() * scales[pages, :, slot // BLOCK][..., None]


def _plain_attend(s):
    c = s["case"]
    H, Hk, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    G, q = H // Hk, s["q"]
    prefix, _, n_q, kv = s["lens"]
    ng, B, T = c["groups"], len(n_q), sum(n_q)
    # the prefix: all queries of a group against its keys
    np_ = -(-max(prefix) // page)
    rows = s["table"][s["lead"]][:, :np_].long().clamp(min=0)
    kp, vp = (_values(s, i, rows).transpose(1, 2).reshape(ng, Hk, np_ * page, D) for i in (0, 1))
    most = int(max(sum(n_q[b] for b in range(g * c["members"], (g + 1) * c["members"])) for g in range(ng)))
    qf = q.float() * s["scale"]
    qg = qf.new_zeros(ng, most, H, D)
    qg[s["g_of"], s["gi"]] = qf
    sp = qg.view(ng, most, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(ng, Hk, most * G, D) @ kp.transpose(-1, -2)
    sp.masked_fill_((torch.arange(np_ * page, device=DEV) >= s["pre"][:, None])[:, None, None], -math.inf)
    # what follows it: each request's own queries against its own keys
    Sm = max(kv[b] - prefix[b // c["members"]] for b in range(B))
    Qm = max(n_q)
    at = s["pre"][s["grp"]][:, None] + torch.arange(Sm, device=DEV)
    here = at < s["kv"][:, None]
    col = (at // page).clamp(max=s["table"].shape[1] - 1)
    pages = s["table"].gather(1, col).long().clamp(min=0)
    ks, vs = (_values(s, i, pages, at % page).masked_fill_(~here[..., None, None], 0).transpose(1, 2) for i in (0, 1))
    qs = qf.new_zeros(B, Qm, H, D)
    qs[s["b_of"], s["qi"]] = qf
    ss = qs.view(B, Qm, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, Qm * G, D) @ ks.transpose(-1, -2)
    where = (s["kv"] - s["n_q"])[:, None] + torch.arange(Qm, device=DEV)
    hide = (at[:, None] > where[:, :, None]).repeat_interleave(G, 1)[:, None]
    ss.masked_fill_(hide, -math.inf)

    def to_tokens(x, first, second, n, m):
        """[n, Hk, m * G, ...] by request or group to [T, H, ...]."""
        x = x.view(n, Hk, m, G, *x.shape[3:])
        return x[first, :, second].reshape(T, H, *x.shape[4:])

    mp = to_tokens(sp.amax(-1), s["g_of"], s["gi"], ng, most)
    ms = to_tokens(ss.amax(-1), s["b_of"], s["qi"], B, Qm)
    m = torch.maximum(mp, ms)
    mg, mb = m.new_zeros(ng, most, H), m.new_zeros(B, Qm, H)
    mg[s["g_of"], s["gi"]], mb[s["b_of"], s["qi"]] = m, m
    sp = torch.exp_(sp.sub_(mg.view(ng, most, Hk, G).transpose(1, 2).reshape(ng, Hk, most * G, 1)))
    ss = torch.exp_(ss.sub_(mb.view(B, Qm, Hk, G).transpose(1, 2).reshape(B, Hk, Qm * G, 1)))
    total = (to_tokens(sp.sum(-1), s["g_of"], s["gi"], ng, most) + to_tokens(ss.sum(-1), s["b_of"], s["qi"], B, Qm))
    o = to_tokens(sp @ vp, s["g_of"], s["gi"], ng, most) + to_tokens(ss @ vs, s["b_of"], s["qi"], B, Qm)
    return (o / total[..., None]).to(q.dtype), m + torch.log(total)


def run(state):
    s, c = state, state["case"]
    if c["op"] == "norm":
        if not own:
            return _plain_norm(s)
        from paper_2608_15762_gb300 import gmgop
        return gmgop.norm(s["x"], s["w"], s["bias"], kind=c["kind"], eps=EPS, y=s["y"], after=c["after"], y_w=s["y_w"],
                          y_bias=s["y_bias"], gate=s["gate"], scale=c["scale"])
    if c["op"] == "append":
        if not own:
            return _plain_append(s)
        from paper_2608_15762_gb300 import gmgop
        q, k, v = _heads(s)
        return gmgop.rope_append8(s["rope"], q, k, v, s["pos"], s["seq"], s["cache"], 0), s["cache"].codes, s["cache"].scales
    if not own:
        return _plain_attend(s)
    from paper_2608_15762_gb300 import gmgop
    return gmgop.attend8(s["plan"], s["q"], s["cache"], 0, scale=s["scale"], lse=True)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "norm":
        m, n, x = c["rows"], c["n"], 4 if c["stream"] == "fp32" else 2
        gate = {"none": 0, "row": m, "column": n, "full": m * n}[c["gate"]]
        vectors = (1 + c["bias"]) * (1 + c["after"]) * n
        each = (x + 2) + ((2 + x) if c["block"] else 0)     # x, h; y, the new x
        return {"bytes": m * n * each + 2 * (gate + vectors), "flops": m * n * (4 + (2 if c["block"] else 0) + (4 if c["after"] else 0))}
    if c["op"] == "append":
        T, H, Hk, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        return {"bytes": T * (4 * H * D + 3 * 2 * Hk * D + 8) + T // BLOCK * 2 * Hk * 4, "flops": 3 * T * (H + Hk) * c["rotary"]}
    prefix, group, q, kv = _attend_lens(c)
    own_keys = sum(kv[b] - prefix[group[b]] for b in range(len(q)))
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(q, kv))
    return {"bytes": 2 * (sum(prefix) + own_keys) * c["kv_heads"] * (c["dim"] + 4 / BLOCK)
            + 2 * 2 * sum(q) * c["heads"] * c["dim"] + 4 * sum(q) * c["heads"],
            "flops": 4 * pairs * c["heads"] * c["dim"]}


# ---------------------------------------------------------------------------
# The definition, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        def standard(v, w, b):
            if c["kind"] == "layer":
                spread, mean = torch.var_mean(v, -1, correction=0, keepdim=True)
                v = v - mean
            else:
                spread = torch.linalg.vector_norm(v, dim=-1, keepdim=True) ** 2 / v.shape[-1]
            v = v / torch.sqrt(spread + EPS) * w.double()[None]
            return v if b is None else v + b.double()[None]

        r = s["x"].double()
        if s["y"] is None:
            return standard(r, s["w"], s["bias"])
        z = s["y"].double()
        z = z if s["y_w"] is None else standard(z, s["y_w"], s["y_bias"])
        r = torch.addcmul(r, z, torch.ones((), dtype=torch.float64, device=DEV) if s["gate"] is None else s["gate"].double(),
                          value=c["scale"])
        return standard(r, s["w"], s["bias"]), r
    if c["op"] == "append":
        R, f, page = c["rotary"], torch.from_numpy(s["freqs"]).to(DEV), c["page"]
        turn = torch.polar(torch.ones(c["tokens"], R // 2, dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * f)[:, None]

        def turned(x):
            x = x.double().clone()
            if c["interleaved"]:
                z = torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) * turn
                x[..., :R] = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * turn
                x[..., :R // 2], x[..., R // 2:R] = z.real, z.imag
            return x

        def rounded(x):
            """To the nearest number of 4 significant bits, or multiple of 2^-9: the same in 64 bits."""
            powers = _powers(-6, 9, torch.float64)
            step = powers[torch.searchsorted(powers, x.abs().clamp(min=2.0 ** -6), right=True) - 1] / 8
            return torch.round(x / step) * step

        q, k, v = _heads(s)
        codes, scales = s["codes"].view(F8).double(), s["scales"].double()
        pos, seq = s["pos"].cpu().numpy(), s["seq"].cpu().numpy()
        table = s["table"].cpu().numpy()
        # by block: (page, block in it, first slot, the tokens of the call), as padded lists
        key = table[seq, pos // page].astype(np.int64) * (page // BLOCK) + pos % page // BLOCK
        place, start, count = np.unique(key, return_index=True, return_counts=True)
        where = torch.from_numpy(place).to(DEV)
        which = torch.from_numpy(start[:, None] + np.minimum(np.arange(BLOCK), count[:, None] - 1)).to(DEV)   # the last one again
        first = torch.from_numpy(pos[start] % BLOCK).to(DEV).long()
        for i, x in ((0, turned(k)), (1, v.double())):
            c8 = codes[:, 0, i].unflatten(2, (-1, BLOCK)).transpose(1, 2).flatten(0, 1)      # [blocks, heads, 16, dim]
            s8 = scales[:, 0, i].transpose(1, 2).flatten(0, 1)
            held = x[which].transpose(1, 2)                                                    # [n, heads, 16, dim]
            powers = _powers(-60, 60, torch.float64)
            need = powers[torch.searchsorted(powers * 448, held.abs().amax((2, 3))).clamp(max=120)]
            new = torch.where(first[:, None] == 0, need, torch.maximum(s8[where], need))
            slot = torch.arange(BLOCK, device=DEV)
            keep = rounded(c8[where] * (s8[where] / new)[..., None, None])
            block = torch.where((slot < first[:, None])[:, None, :, None], keep, c8[where])
            to = torch.from_numpy(pos).to(DEV).long()[which] % BLOCK
            block.scatter_(2, to[:, None, :, None].expand_as(held), rounded(held / new[..., None, None]))
            c8[where], s8[where] = block, new
            codes[:, 0, i] = c8.unflatten(0, (-1, page // BLOCK)).transpose(1, 2).flatten(2, 3)
            scales[:, 0, i] = s8.unflatten(0, (-1, page // BLOCK)).transpose(1, 2)
        return turned(q), codes, scales
    # attention: request by request, over all its cached tokens
    _, _, n_q, kv = s["lens"]
    H, Hk, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    if 4 * H * D * sum(n * t for n, t in zip(n_q, kv)) > 6e12:
        return None
    o = torch.empty(sum(n_q), H, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(sum(n_q), H, dtype=torch.float64, device=DEV)
    at = 0
    for b, n in enumerate(n_q):
        t = kv[b]
        pages = s["table"][b, :-(-t // page)].long()
        k, v = ((s["codes"][pages, 0, i].view(F8).double().unflatten(2, (-1, BLOCK))
                 * s["scales"][pages, 0, i].double()[..., None, None]).flatten(2, 3).permute(1, 0, 2, 3).flatten(1, 2)[:, :t]
                for i in (0, 1))
        x = s["q"][at:at + n].double()
        sees = torch.arange(t, device=DEV)[None] <= torch.arange(t - n, t, device=DEV)[:, None]
        for h in range(H):
            z = (x[:, h] @ k[h * Hk // H].t() * s["scale"]).masked_fill(~sees, -math.inf)
            lse[at:at + n, h] = torch.logsumexp(z, -1)
            o[at:at + n, h] = torch.softmax(z, -1) @ v[h * Hk // H]
        at += n
    return o, lse
