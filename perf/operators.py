"""The operators of a decoder layer on a paged cache, as the executor of a placement runs them: matrix products with
their epilogue, rotary positions written into the cache, attention of requests that share a retained prefix, and the
pages of the cache themselves.

A case is a dict of plain values.  ``run`` makes one pass through one operator: in its plain form (elementary torch
operations in 32 bits, rounded once at the end) or, where ``own`` is true, through ``gmgop``.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
DEV = "cuda"


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _linear(name, tokens, k, n, act="none", gated=False, bias=False, residual=False, dtype="bf16"):
    return dict(name=name, op="linear", tokens=tokens, k=k, n=n, act=act, gated=gated, bias=bias, residual=residual,
                dtype=dtype)


def _rope(name, tokens, seqs, heads, kv_heads, dim, rotary, top, dtype="bf16", interleaved=False, scaling="none",
          append=True, page=16):
    return dict(name=name, op="rope", tokens=tokens, seqs=seqs, heads=heads, kv_heads=kv_heads, dim=dim, rotary=rotary,
                top=top, dtype=dtype, interleaved=interleaved, scaling=scaling, append=append, page=page)


def _attend(name, groups, members, prefix, suffix, q_max, heads, kv_heads, dim, page=16, dtype="bf16", lens=1):
    return dict(name=name, op="attend", groups=groups, members=members, prefix=prefix, suffix=suffix, q_max=q_max,
                heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, lens=lens)


def _pages(name, action, n_pages, seqs, length, moved, layers, kv_heads, dim, page=16, lens=1):
    return dict(name=name, op="pages", action=action, n_pages=n_pages, seqs=seqs, length=length, moved=moved,
                layers=layers, kv_heads=kv_heads, dim=dim, page=page, lens=lens)


def listed():
    return [
        # one token of one request: the output projection added to the residual stream, where reading the weight and
        # the launch are all that counts
        _linear("linear_token", 1, 4096, 4096, residual=True),
        # a small ragged batch through a layer of odd sizes, biased, with an activation
        _linear("linear_ragged", 77, 1000, 1111, act="gelu", bias=True, dtype="fp16"),
        # the gated half of a prompt's feed-forward block
        _linear("linear_gated", 2048, 4096, 12288, act="silu", gated=True),
        # the other half, for a large batch of prompts
        _linear("linear_prompt", 8192, 12288, 4096, residual=True),
        # a decode step of 16 requests: rotate and append one token each
        _rope("rope_step", 16, 16, 32, 8, 128, 128, 8000),
        # the gradient of a partly rotated, interleaved head of odd length, not in a cache
        _rope("rope_inverse", 1537, 1, 20, 0, 80, 32, 6000, dtype="fp32", interleaved=True, scaling="linear",
              append=False),
        # the prompts of a long context, with scaled frequencies
        _rope("rope_prompt", 32768, 3, 32, 8, 128, 128, 200000, dtype="fp16", scaling="parts"),
        # a small decode step over a short shared prompt
        _attend("attend_step", 1, 8, 500, 60, 1, 32, 8, 128),
        # a large decode step over a long shared document
        _attend("attend_shared", 1, 96, 32768, 700, 1, 32, 8, 128, lens=2),
        # chunks of new prompt tokens behind the prompts of several tenants
        _attend("attend_chunk", 4, 6, 4000, 900, 700, 24, 8, 64, page=32, dtype="fp16", lens=3),
        # between two steps: finished requests freed, others forked, every running one grown by its next tokens
        _pages("pages_step", "step", 4096, 96, 900, 24, 2, 8, 128),
        # a fragmented pool made dense
        _pages("pages_compact", "compact", 6000, 200, 500, 0, 2, 8, 128, lens=2),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _widths(c):
    """The sizes of a case, with the widths of its rows of heads."""
    d, h, k = c.get("dim", 0), c.get("heads", 0), c.get("kv_heads", 0)
    return [v for v in c.values() if type(v) is int] + [h * d, k * d, 2 * k * d, (h + 2 * k) * d]


def draw(rng):
    c = _draw(rng)
    while 3072 in _widths(c):
        c = _draw(rng)
    return c


def _draw(rng):
    op = rng.choice(("linear", "rope", "attend", "pages"))
    if op == "linear":
        while True:
            m, k, n = _log(rng, 1, 8192), 8 * _log(rng, 8, 1536), _log(rng, 64, 12288)
            gated = rng.random() < 0.3
            if 2 * m * k * n * (2 if gated else 1) <= 2 * 8192 * 12288 * 4096:
                break
        c = _linear("", m, k, n, act=rng.choice(("none", "relu", "gelu", "silu")),
                    gated=gated, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                    dtype=rng.choice(("bf16", "fp16")))
    elif op == "rope":
        append = rng.random() < 0.7
        dim = rng.choice((64, 80, 96, 128))
        kv = rng.choice((1, 2, 4, 8)) if append else 0
        heads = kv * rng.choice((1, 4, 5, 8)) if append else rng.choice((5, 12, 20, 32))
        tokens = _log(rng, 1, 32768)
        seqs = min(tokens, _log(rng, 1, 64))
        top = max(rng.choice((6000, 40000, 200000)), 2 * (-(-tokens // seqs)))
        c = _rope("", tokens, seqs, heads, kv, dim, rng.choice((dim, dim // 2, 32)),
                  top, dtype=rng.choice(("bf16", "fp16")),
                  interleaved=rng.random() < 0.5, scaling=rng.choice(("none", "linear", "parts")), append=append,
                  page=rng.choice((16, 32, 64)))
        if not append and rng.random() < 0.5:
            c["dtype"] = "fp32"
    elif op == "attend":
        while True:
            groups, members = _log(rng, 1, 6), _log(rng, 1, 96)
            prefix, suffix = _log(rng, 16, 32768), _log(rng, 4, 1000)
            q_max = 1 if rng.random() < 0.6 else _log(rng, 2, 700)
            tokens = groups * members * q_max
            if groups * members <= 128 and tokens * (prefix + suffix) <= 50_000_000 and groups * prefix <= 65536:
                break
        kv = rng.choice((1, 2, 8))
        c = _attend("", groups, members, prefix, suffix, q_max, kv * rng.choice((1, 4, 5, 8)), kv,
                    rng.choice((64, 80, 128)), page=rng.choice((16, 32, 64)), dtype=rng.choice(("bf16", "fp16")),
                    lens=rng.randrange(1 << 30))
    else:
        action = rng.choice(("step", "compact"))
        page = rng.choice((16, 32))
        seqs = _log(rng, 12, 200)
        length = _log(rng, 20, 900)
        n_pages = 2 * seqs * (length // page + 2) + 64
        while n_pages * page > 6000 * 16:
            n_pages, seqs, length = n_pages // 2, max(12, seqs // 2), max(20, length * 2 // 3)
            n_pages = max(n_pages, 2 * seqs * (length // page + 2) + 64)
        c = _pages("", action, n_pages + rng.randrange(60), seqs, length, max(1, seqs // 4), rng.choice((1, 2)),
                   rng.choice((1, 4, 8)), rng.choice((64, 128)), page=page, lens=rng.randrange(1 << 30))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Lengths and tables of a case: from its plain values alone
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


def _page_rows(c):
    """Host tables of a pages case: table, lens, refs; requests 0, 4, 8, ... share their neighbours' first pages."""
    r = random.Random(c["lens"])
    S, P, page = c["seqs"], c["n_pages"], c["page"]
    cols = (c["length"] + c["length"] // 2) // page + 4
    ids = list(range(P))
    r.shuffle(ids)
    table, lens, refs = np.full((S, cols), -1, np.int32), np.zeros(S, np.int32), np.zeros(P, np.int32)
    live = S if c["action"] == "compact" else S - c["moved"]
    for s in range(live):
        n = r.randint(max(1, c["length"] // 2), c["length"])
        shared = 0
        if s % 4:
            shared = min(int(lens[s - s % 4]), n) // page
            table[s, :shared] = table[s - s % 4, :shared]
        need = -(-n // page)
        for k in range(shared, need):
            table[s, k] = ids.pop()
        lens[s] = n
        np.add.at(refs, table[s, :need], 1)
    return table, lens, refs, live


def _step(c, live):
    """The requests that finish, those forked (source, new), and those that grow by how many tokens."""
    r = random.Random(c["lens"] + 1)
    order = list(range(live))
    r.shuffle(order)
    done, kept = order[:c["moved"] // 2], order[c["moved"] // 2:]
    dst = list(range(live, c["seqs"]))
    src = [r.choice(kept) for _ in dst]
    grown = kept + dst
    r.shuffle(grown)
    return done, src, dst, grown, [r.choice((1, 1, 1, 1, c["page"] + 5)) for _ in grown]


def _freqs(c):
    """The angle of one position for each pair, in 64 bits, and the factor of the magnitude."""
    half = c["rotary"] // 2
    f = 10000.0 ** (-2.0 * np.arange(half) / c["rotary"])
    if c["scaling"] == "linear":
        return f / 4.0, 1.0
    if c["scaling"] == "parts":
        turns = 8192 * f / (2 * math.pi)
        g = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        return f * (1 - g) / 16.0 + f * g, 0.1 * math.log(16.0) + 1.0
    return f, 1.0


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
    c, dt = case, DTYPES.get(case.get("dtype", "bf16"))

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dt)

    if c["op"] == "linear":
        m, k, n = c["tokens"], c["k"], c["n"]
        s.update(x=normal(m, k), w=normal(n, k, scale=k ** -0.5), bias=normal(n) if c["bias"] else None,
                 gate=normal(n, k, scale=k ** -0.5) if c["gated"] else None,
                 gate_bias=normal(n) if c["gated"] and c["bias"] else None,
                 residual=normal(m, n) if c["residual"] else None)
        if own:
            from paper_2608_15762_gb300 import gmgop
            s["ws"] = gmgop.Workspace(DEV)
        return s
    if c["op"] == "rope":
        T, H, Hk, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        # tokens of each request follow one another; the heads lie in one row, as the product before leaves them
        per = -(-T // c["seqs"])
        seq = np.arange(T) // per
        first = np.random.default_rng(seed).integers(0, c["top"] - per, c["seqs"])
        pos = first[seq] + np.arange(T) % per
        s.update(row=normal(T, (H + 2 * Hk) * D), pos=torch.from_numpy(pos.astype(np.int32)).to(DEV),
                 seq=torch.from_numpy(seq.astype(np.int32)).to(DEV))
        f, s["factor"] = _freqs(c)
        s["freqs"] = f
        if c["append"]:
            page = c["page"]
            cols = -(-c["top"] // page) + 1
            table = np.full((c["seqs"], cols), -1, np.int32)
            used = [np.unique(pos[seq == b] // page) for b in range(c["seqs"])]
            n = sum(len(u) for u in used)
            ids = np.random.default_rng(seed + 1).permutation(n + 3).astype(np.int32)
            at = 0
            for b, u in enumerate(used):
                table[b, u] = ids[at:at + len(u)]
                at += len(u)
            s["table"] = torch.from_numpy(table).to(DEV)
            s["pool"] = normal(n + 3, 1, 2, Hk, page, D)
        if own:
            from paper_2608_15762_gb300 import gmgop
            s["rope"] = gmgop.Rope(c["rotary"], freqs=f, factor=s["factor"], interleaved=c["interleaved"], device=DEV)
            if c["append"]:
                s["cache"] = gmgop.PageCache(s["pool"], table=s["table"])
        else:
            # a program without the operator keeps the angles' cosines and sines
            a = torch.arange(c["top"], device=DEV, dtype=torch.float64)[:, None] * torch.from_numpy(f).to(DEV)
            s["cos"], s["sin"] = (torch.cos(a) * s["factor"]).float(), (torch.sin(a) * s["factor"]).float()
        return s
    if c["op"] == "attend":
        prefix, group, q, kv = _attend_lens(c)
        B, page, Hk, D = len(q), c["page"], c["kv_heads"], c["dim"]
        cols = max(-(-n // page) for n in kv)
        table, at = np.full((B, cols), -1, np.int32), 0
        total = sum(p // page for p in prefix) + sum(-(-kv[b] // page) - prefix[group[b]] // page for b in range(B))
        ids = np.random.default_rng(seed).permutation(total + 2).astype(np.int32)
        for b in range(B):
            full, need = prefix[group[b]] // page, -(-kv[b] // page)
            if b % c["members"]:
                table[b, :full] = table[b - b % c["members"], :full]
                full_from = full
            else:
                full_from = 0
            table[b, full_from:need] = ids[at:at + need - full_from]
            at += need - full_from
        pool = normal(total + 2, 1, 2, Hk, page, D)
        # a page that the prefix ends in was copied when the requests were forked
        for b in range(B):
            lead, tail = b - b % c["members"], prefix[group[b]] % page
            if tail and b != lead:
                k = prefix[group[b]] // page
                pool[int(table[b, k]), :, :, :, :tail] = pool[int(table[lead, k]), :, :, :, :tail]
        s.update(q=normal(sum(q), c["heads"], D), pool=pool, table=torch.from_numpy(table).to(DEV),
                 scale=D ** -0.5, lens=(prefix, group, q, kv))
        if own:
            from paper_2608_15762_gb300 import gmgop
            s["cache"] = gmgop.PageCache(pool, table=s["table"])
            off = [g * c["members"] for g in range(c["groups"] + 1)]
            s["plan"] = gmgop.AttendPlan(q, kv, c["heads"], Hk, D, page, group_off=off, prefix=prefix, device=DEV)
        else:
            first = np.cumsum([0] + q)[:-1]
            b_of = np.repeat(np.arange(B), q)
            qi = np.arange(sum(q)) - first[b_of]
            g_of = np.asarray(group)[b_of]
            g_first = np.asarray([first[g * c["members"]] for g in range(c["groups"])])
            up = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).to(DEV)  # noqa: E731
            s.update(b_of=up(b_of), qi=up(qi), g_of=up(g_of), gi=up(np.arange(sum(q)) - g_first[g_of]),
                     kv=up(np.asarray(kv)), n_q=up(np.asarray(q)), pre=up(np.asarray(prefix)), grp=up(np.asarray(group)),
                     lead=up(np.arange(c["groups"]) * c["members"]))
        return s
    # pages
    table, lens, refs, live = _page_rows(c)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)  # noqa: E731
    dt = torch.bfloat16
    s.update(pool=normal(c["n_pages"], c["layers"], 2, c["kv_heads"], c["page"], c["dim"]),
             table0=up(table), lens0=up(lens), refs0=up(refs))
    s.update(table=s["table0"].clone(), lens=s["lens0"].clone(), refs=s["refs0"].clone())
    if c["action"] == "step":
        s.update(zip(("done", "src", "dst", "grown", "add"), map(up, _step(c, live))))
    if own:
        from paper_2608_15762_gb300 import gmgop
        s["cache"] = gmgop.PageCache(s["pool"], table=s["table"], lens=s["lens"], refs=s["refs"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _act(x, act):
    if act == "relu":
        return x.clamp(min=0)
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return x


def _plain_linear(s):
    c, x = s["case"], s["x"].float()

    def product(w, b):
        y = x @ w.float().t()
        return y if b is None else y + b.float()

    y = product(s["w"], s["bias"])
    y = _act(product(s["gate"], s["gate_bias"]), c["act"]) * y if c["gated"] else _act(y, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _turn(s, x, inverse):
    """The rotated heads of x [T, heads, dim], in 32 bits."""
    c, R = s["case"], s["case"]["rotary"]
    pos = s["pos"].long()
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    if inverse:
        sin = -sin
    x = x.float()
    if c["interleaved"]:
        u, v = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((u * cos - v * sin, u * sin + v * cos), -1).flatten(-2)
    else:
        u, v = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _heads(s):
    c = s["case"]
    T, H, Hk, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
    row = s["row"]
    return (row[:, :H * D].view(T, H, D), row[:, H * D:(H + Hk) * D].view(T, Hk, D),
            row[:, (H + Hk) * D:].view(T, Hk, D))


def _plain_rope(s):
    c = s["case"]
    q, k, v = _heads(s)
    dt = q.dtype
    if not c["append"]:
        return _turn(s, q, True).to(dt)
    pos, page = s["pos"].long(), c["page"]
    at = s["table"][s["seq"].long(), pos // page].long()
    s["pool"][at, 0, 0, :, pos % page] = _turn(s, k, False).to(dt)
    s["pool"][at, 0, 1, :, pos % page] = v
    return _turn(s, q, False).to(dt), s["pool"]


def _plain_attend(s):
    c = s["case"]
    H, Hk, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    G, pool, q = H // Hk, s["pool"], s["q"]
    prefix, _, n_q, kv = s["lens"]
    ng, B, T = c["groups"], len(n_q), sum(n_q)
    # the prefix: all queries of a group against its keys
    Pm = max(prefix)
    np_ = -(-Pm // page)
    rows = s["table"][s["lead"]][:, :np_].long().clamp(min=0)
    kp, vp = (pool[rows, 0, i].float().transpose(1, 2).reshape(ng, Hk, np_ * page, D) for i in (0, 1))
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
    ks, vs = (pool[pages, 0, i, :, at % page].float().masked_fill_(~here[..., None, None], 0).transpose(1, 2)
              for i in (0, 1))
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


def _restore(s):
    s["table"].copy_(s["table0"])
    s["lens"].copy_(s["lens0"])
    s["refs"].copy_(s["refs0"])


def _plain_pages(s):
    c, page = s["case"], s["case"]["page"]
    table, lens, refs, pool = s["table"], s["lens"], s["refs"], s["pool"]
    P, cols = c["n_pages"], torch.arange(s["table"].shape[1], device=DEV)

    def count(rows, by):
        """Add `by` to the references of every page in rows."""
        more = torch.zeros(P + 1, dtype=torch.int32, device=DEV)
        at = torch.where(rows >= 0, rows, P).reshape(-1).long()
        refs.add_(more.index_add_(0, at, torch.full_like(at, by, dtype=torch.int32))[:P])

    if c["action"] == "compact":
        used = refs > 0
        n = used.sum()
        ids = torch.arange(P, device=DEV)
        frm, to = ids[used & (ids >= n)], ids[~used & (ids < n)]
        pool[to] = pool[frm]
        new = torch.arange(P, dtype=torch.int32, device=DEV)
        new[frm] = to.int()
        table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()], table))
        refs[to] = refs[frm]
        refs[frm] = 0
        return table, lens, refs, pool
    done, src, dst = s["done"].long(), s["src"].long(), s["dst"].long()
    count(table[done], -1)
    table[done] = -1
    lens[done] = 0
    table[dst] = table[src]
    lens[dst] = lens[src]
    count(table[dst], 1)
    seq, add = s["grown"].long(), s["add"]
    old = lens[seq]
    have, want = (old + page - 1) // page, (old + add + page - 1) // page
    rows = table[seq]
    tail = rows.gather(1, (have - 1).clamp(min=0).long()[:, None])[:, 0]
    copied = (old % page != 0) & (add > 0) & (refs[tail.clamp(min=0).long()] > 1)
    need = want - have + copied.int()
    off = torch.cumsum(need, 0) - need
    free = torch.sort(torch.where(refs == 0, 0, 1), stable=True)[1].int()
    fresh = (cols >= have[:, None]) & (cols < want[:, None])
    which = (off + copied.int() - have)[:, None] + cols
    mine = free[off.long()]
    rows = torch.where(fresh, free[which.clamp(0, P - 1).long()], rows)
    rows = torch.where(copied[:, None] & (cols == (have - 1)[:, None]), mine[:, None], rows)
    pool[torch.where(copied, mine, tail).long()] = pool[tail.long()]
    count(torch.where(copied, tail, -1), -1)
    count(torch.where(fresh, rows, -1), 1)
    count(torch.where(copied, mine, -1), 1)
    table[seq] = rows
    lens[seq] = old + add
    return table, lens, refs, pool


def run(state):
    s, c = state, state["case"]
    if c["op"] == "linear":
        if not own:
            return _plain_linear(s)
        from paper_2608_15762_gb300 import gmgop
        return gmgop.linear(s["x"], s["w"], bias=s["bias"], act=c["act"], gate=s["gate"], gate_bias=s["gate_bias"],
                            residual=s["residual"], ws=s["ws"])
    if c["op"] == "rope":
        if not own:
            return _plain_rope(s)
        from paper_2608_15762_gb300 import gmgop
        q, k, v = _heads(s)
        if not c["append"]:
            return gmgop.rope(s["rope"], q, s["pos"], backward=True)
        return gmgop.rope_append(s["rope"], q, k, v, s["pos"], s["seq"], s["cache"], 0), s["pool"]
    if c["op"] == "attend":
        if not own:
            return _plain_attend(s)
        from paper_2608_15762_gb300 import gmgop
        return gmgop.attend(s["plan"], s["q"], s["cache"], 0, scale=s["scale"], lse=True)
    _restore(s)
    if not own:
        return _plain_pages(s)
    cache = s["cache"]
    if c["action"] == "compact":
        cache.compact()
    else:
        cache.free(s["done"])
        cache.fork(s["src"], s["dst"])
        cache.grow(s["grown"], s["add"])
    return s["table"], s["lens"], s["refs"], s["pool"]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _page_moves(c):
    """Pages whose data a pass copies."""
    table, lens, refs, live = _page_rows(c)
    if c["action"] == "compact":
        n = int((refs > 0).sum())
        return int((refs[n:] > 0).sum())
    # a request that grows out of a page that others hold too takes a copy of it
    done, src, dst, grown, _ = _step(c, live)
    for b in done:
        np.add.at(refs, table[b][table[b] >= 0], -1)
        table[b], lens[b] = -1, 0
    for a, b in zip(src, dst):
        table[b], lens[b] = table[a], lens[a]
        np.add.at(refs, table[b][table[b] >= 0], 1)
    return sum(int(lens[b] % c["page"] != 0 and refs[table[b, lens[b] // c["page"]]] > 1) for b in grown)


def work(case):
    c = case
    e = 4 if c.get("dtype") == "fp32" else 2
    if c["op"] == "linear":
        m, k, n, w = c["tokens"], c["k"], c["n"], 2 if c["gated"] else 1
        return {"bytes": e * (m * k + w * n * k + m * n * (2 if c["residual"] else 1) + (w * n if c["bias"] else 0)),
                "flops": 2 * m * n * k * w}
    if c["op"] == "rope":
        T, H, Hk, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        return {"bytes": 2 * e * T * (H + 2 * Hk) * D + 4 * T * (2 if c["append"] else 1),
                "flops": 3 * T * (H + Hk) * c["rotary"]}
    if c["op"] == "attend":
        prefix, group, q, kv = _attend_lens(c)
        own_keys = sum(kv[b] - prefix[group[b]] for b in range(len(q)))
        pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(q, kv))
        return {"bytes": 2 * e * (sum(prefix) + own_keys) * c["kv_heads"] * c["dim"]
                + 2 * e * sum(q) * c["heads"] * c["dim"] + 4 * sum(q) * c["heads"],
                "flops": 4 * pairs * c["heads"] * c["dim"]}
    table, lens, refs, _ = _page_rows(c)
    data = c["layers"] * 2 * c["kv_heads"] * c["page"] * c["dim"] * 2
    return {"bytes": 2 * _page_moves(c) * data + 2 * 4 * (table.size + lens.size + refs.size), "flops": 0}


# ---------------------------------------------------------------------------
# The definition, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "pages":
        return None     # whole numbers and copies
    c, s = case, prepare(case, seed)
    if c["op"] == "linear":
        if 2 * c["tokens"] * c["k"] * c["n"] > 9e11:
            return None
        x = s["x"].double()

        def product(w, b):
            y = torch.mm(x, w.double().t())
            return y if b is None else y + b.double()[None, :]

        def bent(y):
            if c["act"] == "relu":
                return torch.where(y > 0, y, torch.zeros_like(y))
            if c["act"] == "silu":
                return y * torch.special.expit(y)
            if c["act"] == "gelu":
                return y * torch.special.ndtr(y)
            return y

        y = product(s["w"], s["bias"])
        y = bent(product(s["gate"], s["gate_bias"])) * y if c["gated"] else bent(y)
        return y if s["residual"] is None else y + s["residual"].double()
    if c["op"] == "rope":
        R, f = c["rotary"], torch.from_numpy(s["freqs"]).to(DEV)
        turn = torch.polar(torch.full((c["tokens"], R // 2), float(s["factor"]), dtype=torch.float64, device=DEV),
                           s["pos"].double()[:, None] * f * (1.0 if c["append"] else -1.0))[:, None]

        def turned(x):
            x = x.double().clone()
            if c["interleaved"]:
                z = torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) * turn
                x[..., :R] = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * turn
                x[..., :R // 2], x[..., R // 2:R] = z.real, z.imag
            return x

        q, k, v = _heads(s)
        if not c["append"]:
            return turned(q)
        pool, k = s["pool"].double(), turned(k)
        pos = s["pos"].long()
        slot = s["table"].long()[s["seq"].long(), torch.div(pos, c["page"], rounding_mode="floor")]
        pool[slot, 0, 0, :, pos % c["page"]] = k
        pool[slot, 0, 1, :, pos % c["page"]] = v.double()
        return turned(q), pool
    # attention: request by request, over all its cached tokens
    prefix, group, n_q, kv = s["lens"]
    H, Hk, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    o = torch.empty(sum(n_q), H, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(sum(n_q), H, dtype=torch.float64, device=DEV)
    if 4 * H * D * sum(n * t for n, t in zip(n_q, kv)) > 6e12:
        return None
    at = 0
    for b, n in enumerate(n_q):
        t = kv[b]
        pages = s["table"][b, :-(-t // page)].long()
        k, v = (s["pool"][pages, 0, i].permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :t].double() for i in (0, 1))
        x = s["q"][at:at + n].double()
        sees = torch.arange(t, device=DEV)[None] <= torch.arange(t - n, t, device=DEV)[:, None]
        for h in range(H):
            z = (x[:, h] @ k[h * Hk // H].t() * s["scale"]).masked_fill(~sees, -math.inf)
            lse[at:at + n, h] = torch.logsumexp(z, -1)
            o[at:at + n, h] = torch.softmax(z, -1) @ v[h * Hk // H]
        at += n
    return o, lse
