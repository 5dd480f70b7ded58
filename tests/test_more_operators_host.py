"""The C ABI of the norms around a block and of the operators on a cache in 8 bits: the refusals that need no GPU
(arguments are checked before any launch), and the work that a plan lists."""
import ctypes as C
import random

import numpy as np
import pytest

from paper_2608_15762_gb300 import build, gmgop as P, gmgsim as G
from test_operators_host import _On, _Untouched


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


# ---------------------------------------------------------------------------
# Norms
# ---------------------------------------------------------------------------

def _norm(**kw):
    a = dict(dtype=P.BF16, stream_dtype=P.F32, kind=0, after=1, m=4, n=8, x=256, y=512, y_weight=768, y_bias=1024, weight=256,
             bias=256, gate=256, r=2048, h=4096, x_row=8, y_row=8, gate_row=0, gate_col=1, r_row=8, h_row=8, scale=1.0, eps=1e-6)
    a.update(kw)
    s = P._Norm()
    for k, v in a.items():
        setattr(s, k, v)
    return P.lib().op_norm(C.addressof(s), None)


@pytest.mark.parametrize("kw", [dict(dtype=7), dict(dtype=P.E4M3), dict(stream_dtype=P.F16), dict(stream_dtype=5), dict(kind=2), dict(kind=-1),
                                dict(m=-1), dict(n=-1), dict(m=2 ** 31), dict(n=32769), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(scale=float("nan")), dict(shift=float("nan")), dict(x=0), dict(x_row=7), dict(y_row=7),
                                dict(r_row=7), dict(h_row=7), dict(gate_col=2), dict(gate_col=-1), dict(gate_row=7), dict(gate_row=-1),
                                dict(y=0), dict(y=0, after=0, gate=0, r=0), dict(after=0), dict(h=0), dict(h=0, weight=0),
                                dict(h=0, weight=0, bias=0, r=0)])
def test_norm_refuses(kw):
    assert _norm(**kw) == G.GMG_EINVAL


def test_norm_of_nothing_is_done():
    assert _norm(m=0, x=0) == _norm(n=0, x_row=0, weight=0) == G.GMG_OK
    assert P.lib().op_norm(None, None) == G.GMG_EINVAL


# ---------------------------------------------------------------------------
# A cache in 8 bits
# ---------------------------------------------------------------------------

def _cache8(**kw):
    a = dict(pool=256, table=256, lens=256, refs=256, status=256, dtype=P.E4M3, n_pages=10, n_layers=2, n_kv_heads=2,
             page_tokens=16, head_dim=64, n_seq=4, max_pages=6)
    a.update(kw)
    s = P._Cache()
    for k, v in a.items():
        setattr(s, k, v)
    return s


BAD = [dict(pool=0), dict(pool=8), dict(table=0), dict(lens=0), dict(refs=0), dict(status=0), dict(dtype=P.F32), dict(dtype=4),
       dict(n_pages=0), dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=512), dict(head_dim=8), dict(head_dim=72),
       dict(head_dim=144), dict(head_dim=0), dict(n_seq=0), dict(max_pages=0), dict(n_layers=0), dict(n_kv_heads=0)]


def test_bytes_of_a_page():
    L = P.lib()
    # codes, a scale for 16 tokens of each head, up to 128 bytes
    assert L.op_page8_bytes(1, 1, 16, 16) == 512 + 128
    assert L.op_page8_bytes(2, 8, 64, 128) == 2 * 2 * 8 * (64 * 128 + 4 * 4)
    assert L.op_page8_bytes(3, 5, 32, 80) == -(-3 * 2 * 5 * (32 * 80 + 2 * 4) // 128) * 128
    for a in ((0, 1, 16, 16), (1, 0, 16, 16), (1, 1, 8, 16), (1, 1, 48, 16), (1, 1, 16, 24), (1, 1, 16, 256), (-1, 1, 16, 16)):
        assert L.op_page8_bytes(*a) == 0
        with pytest.raises(ValueError):
            P.page8_bytes(*a)


@pytest.mark.parametrize("kw", BAD)
def test_calls_refuse_a_bad_cache(kw):
    L, c = P.lib(), _cache8(**kw)
    r = C.addressof(c)
    assert L.op_page_scratch_bytes(r) == 0
    assert L.op_free(r, 256, 1, 256, 1 << 30, None) == G.GMG_EINVAL
    assert _append(c) == G.GMG_EINVAL
    assert _attend(c) == G.GMG_EINVAL


def test_page_calls_take_it():
    L, c = P.lib(), _cache8()
    r = C.addressof(c)
    assert L.op_page_scratch_bytes(r) > 0
    assert L.op_grow(r, 256, 256, 1, 0, 0, None) == G.GMG_EWS


def _append(cache, layer=0, dtype=P.BF16, tokens=3, heads=2, q=256, k=256, v=256, pos=256, seq=256, out=256, rotary=64, freq=256):
    p = P._Rope(freq, rotary, 0, 1.0)
    return P.lib().op_rope_append8(C.addressof(p), C.addressof(cache), layer, dtype, tokens, heads, q, 128, 64, k, 128, 64, v,
                                   128, 64, pos, seq, out, 128, 64, None)


def test_append8_refuses():
    for kw in (dict(layer=2), dict(layer=-1), dict(dtype=P.F32), dict(dtype=P.E4M3), dict(tokens=-1), dict(tokens=2 ** 31), dict(heads=-1),
               dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(seq=None), dict(out=None), dict(rotary=63),
               dict(rotary=66), dict(rotary=-2), dict(freq=None), dict(heads=2 ** 20)):
        assert _append(_cache8(), **kw) == G.GMG_EINVAL, kw
    assert _append(_cache8(), tokens=0) == G.GMG_OK
    assert _append(_cache8(dtype=P.BF16)) == G.GMG_EINVAL                    # a cache of 16-bit values
    p, c = P._Rope(256, 64, 0, 1.0), _cache8()                               # and the call for those refuses codes
    assert P.lib().op_rope_append(C.addressof(p), C.addressof(c), 0, 3, 2, 256, 128, 64, 256, 128, 64, 256, 128, 64, 256, 256,
                                  256, 128, 64, None) == G.GMG_EINVAL


def _attend(cache, layer=0, dtype=P.F16, q=256, out=256, work=256, size=1 << 40, strides=(512, 64, 512, 64), items=256, scale=1.0):
    plan, _ = P.attend_items([1, 2], [5, 90], 8, 2, 64, 16, bits=8)
    return P.lib().op_attend8(C.addressof(plan), items, C.addressof(cache), layer, dtype, q, strides[0], strides[1], scale, out,
                              strides[2], strides[3], None, work, size, None)


def test_attend8_refuses():
    for kw in (dict(layer=2), dict(layer=-1), dict(dtype=P.F32), dict(dtype=P.E4M3), dict(q=None), dict(q=264), dict(out=None), dict(out=8),
               dict(items=None), dict(items=8), dict(strides=(513, 64, 512, 64)), dict(strides=(512, 60, 512, 64)),
               dict(strides=(512, 64, 500, 64)), dict(scale=float("nan"))):
        assert _attend(_cache8(), **kw) == G.GMG_EINVAL, kw
    assert _attend(_cache8(), work=0) == _attend(_cache8(), work=128) == _attend(_cache8(), size=0) == G.GMG_EWS
    for kw in (dict(head_dim=80), dict(n_kv_heads=4), dict(page_tokens=32), dict(n_seq=1), dict(max_pages=5)):
        assert _attend(_cache8(**kw)) == G.GMG_EINVAL, kw
    (plan, _), c = P.attend_items([1, 2], [5, 90], 8, 2, 64, 16), _cache8()
    assert P.lib().op_attend(C.addressof(plan), 256, C.addressof(c), 0, 256, 512, 64, 1.0, 256, 512, 64, None, 256, 1 << 40,
                             None) == G.GMG_EINVAL


def test_attend8_plan_refuses():
    ok = dict(q_len=[1, 2], kv_len=[5, 9], n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, bits=8)
    P.attend_items(**ok)
    for kw in (dict(q_len=[1, -1]), dict(kv_len=[-5, 9]), dict(n_heads=7), dict(n_heads=258), dict(head_dim=72), dict(head_dim=144),
               dict(page_tokens=8), dict(page_tokens=24), dict(seq=[0, -1]), dict(kv_len=[5, 2 ** 30 + 1]), dict(n_sm=0),
               dict(group_off=[0, 2], prefix=[5]), dict(group_off=[1, 2], prefix=[3])):
        with pytest.raises(G.GmgError) as e:
            P.attend_items(**dict(ok, **kw))
        assert e.value.code == G.GMG_EINVAL, kw


def _covered8(q, kv, heads, kv_heads, groups=None, prefix=None):
    """Every (query, key) of a batch lies in one item, and joins list the parts of exactly those."""
    plan, items = P.attend_items(q, kv, heads, kv_heads, 64, 16, group_off=groups, prefix=prefix, bits=8)
    g, n = heads // kv_heads, plan.n_items
    cover, joined, used = {t: [] for t in range(sum(q))}, {}, set()
    for tok0, n_tok, row, lo, hi, pos0, part, _ in items[:8 * n].reshape(n, 8).tolist():
        assert 0 < n_tok * g <= (16 if plan.few else 128)
        for t in range(tok0, tok0 + n_tok):
            cover[t].append((lo, hi, row, pos0 + t - tok0, part + (t - tok0) * g if part >= 0 else -1))
    for tok0, n_tok, b0, b1, s0, s1, n0, n1 in items[8 * n:].reshape(-1, 8).tolist():
        assert n_tok <= plan.join_tokens
        for t in range(tok0, tok0 + n_tok):
            assert t not in joined
            joined[t] = [b0 + i * s0 + (t - tok0) * g for i in range(n0)] + [b1 + i * s1 + (t - tok0) * g for i in range(n1)]
    t = 0
    for b in range(len(q)):
        for i in range(q[b]):
            runs, pos, at = sorted(cover[t]), kv[b] - q[b] + i, 0
            if t in joined:
                assert sorted(joined[t]) == sorted(r[4] for r in runs)
                assert all(0 <= x and x + g <= plan.part_rows and x not in used for x in joined[t])
                used.update(joined[t])
            else:
                assert len(runs) == 1 and runs[0][4] == -1
            for lo, hi, row, p, _ in runs:
                if hi:
                    assert lo == at and (p == pos or p >= 0x7f000000)
                    at = hi
                    if row != b:
                        k = [k for k in range(len(prefix)) if groups[k] <= b < groups[k + 1]][0]
                        assert hi <= prefix[k] and groups[k] <= row < groups[k + 1]
            assert at >= max(0, pos + 1)
            t += 1
    return bool(plan.few)


def test_attend8_plan_covers_every_key_once():
    r = random.Random(0)
    kinds = set()
    for _ in range(150):
        n, g, hk = r.randint(1, 40), r.choice([1, 2, 3, 4, 8, 16, 40, 128]), r.choice([1, 2, 8])
        groups = [0] + sorted(r.randint(0, n) for _ in range(r.randint(0, 4))) + [n]
        prefix = [r.choice([0, 1, 64, 100, 3000]) for _ in groups[1:]]
        q = [r.choice([0, 1, 1, 1, 2, 9, 200]) for _ in range(n)]
        kv = [prefix[k] + q[b] + r.choice([0, 0, 5, 70, 5000]) for k in range(len(prefix)) for b in range(groups[k], groups[k + 1])]
        kinds.add(_covered8(q, kv, g * hk, hk, groups, prefix))
        kinds.add(_covered8([min(x, 1) for x in q], kv, g * hk, hk))
        kinds.add(_covered8(q, [max(0, t - r.choice([0, 0, 3, 10 ** 6])) for t in kv], g * hk, hk))
    assert kinds == {False, True}


# ---------------------------------------------------------------------------
# The binding
# ---------------------------------------------------------------------------

def test_calls_refuse_what_does_not_fit_together(monkeypatch):
    """Before anything is launched: the library must not be reached."""
    import torch
    P.lib()
    monkeypatch.setattr(P, "_LIB", _Untouched())
    monkeypatch.setattr(P, "lib", _Untouched())
    monkeypatch.setattr(P, "_current", lambda: 0)
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32

    class Stream:
        def __init__(self, index):
            self.device_index, self.cuda_stream = index, 0

    def cache(index, dtype=torch.uint8):
        c = object.__new__(P.PageCache8)
        c.device, c._index, c.dtype, c.n_kv_heads, c.head_dim = torch.device("cuda", index), index, dtype, 2, 64
        c.ref, c._work = 256, (256, 256)
        return c

    def rope(index):
        p = object.__new__(P.Rope)
        p.index, p.ref = index, 256
        return p

    def plan(index, kind=P.AttendPlan8):
        p = object.__new__(kind)
        p.index, p.ref, p.shape, p.work, p._ptr, p.head_dim, p.work_bytes = index, 256, (3, 2, 64), {0: 256}, 256, 64, 256
        return p

    def heads(index, n=2, dtype=bf, tokens=3):
        return _On(index, tokens, n, 64, dtype=dtype)

    def ints(index, n=3):
        return _On(index, n, dtype=i32)

    def append(at=0, of=0, stream=None, q=None, k=None, v=None, pos=None, seq=None, c=None):
        P.rope_append8(rope(of), q or heads(at), k or heads(at), v or heads(at), pos or ints(at), seq or ints(at), c or cache(at), 0,
                       out=heads(at), stream=stream)

    def attend(at=0, of=0, stream=None, q=None, c=None, p=None):
        P.attend8(p or plan(of), q or heads(at), c or cache(at), 0, out=heads(at), stream=stream)

    for call in (lambda: append(1, 1), lambda: append(1, 0), lambda: append(0, 1), lambda: append(0, -1), lambda: append(stream=Stream(1)),
                 lambda: append(k=heads(0, 3)), lambda: append(v=heads(0, tokens=2)), lambda: append(k=heads(0, dtype=torch.float16)),
                 lambda: append(q=heads(0, dtype=f32), k=heads(0, dtype=f32), v=heads(0, dtype=f32)), lambda: append(pos=ints(0, 2)),
                 lambda: append(seq=ints(1)), lambda: append(k=heads(1)), lambda: append(c=cache(0, bf)),
                 lambda: attend(1, 1), lambda: attend(1, 0), lambda: attend(0, 1), lambda: attend(q=heads(0, 3)),
                 lambda: attend(q=heads(0, dtype=f32)), lambda: attend(c=cache(0, bf)), lambda: attend(p=plan(0, P.AttendPlan)),
                 lambda: P.attend(plan(0), heads(0), cache(0, bf), 0, out=heads(0))):
        with pytest.raises(ValueError):
            call()

    def mat(index=0, m=4, n=8, dtype=bf):
        return _On(index, m, n, dtype=dtype)

    def vec(index=0, n=8, dtype=bf):
        return _On(index, n, dtype=dtype)

    x = mat()
    for kw in (dict(x=mat(1), out=mat(1)), dict(x=mat(-1), out=mat(-1)), dict(kind="max"), dict(w=vec(n=7)), dict(w=vec(1)), dict(w=vec(dtype=f32)),
               dict(bias=vec(n=9)), dict(out=mat(n=9)), dict(out=mat(dtype=f32)), dict(out=mat(1)), dict(x=mat(dtype=torch.float16), w=vec()),
               dict(x=mat(dtype=torch.float64)), dict(after=True), dict(gate=vec()), dict(x_out=mat()), dict(only_x=True), dict(y_w=vec()),
               dict(y=mat(m=3)), dict(y=mat(1)), dict(y=mat(dtype=f32)), dict(y=mat(), y_w=vec()), dict(y=mat(), y_bias=vec()),
               dict(y=mat(), after=True, y_w=vec(n=7)), dict(y=mat(), gate=vec(n=4)), dict(y=mat(), gate=mat(m=3)), dict(y=mat(), gate=mat(1)),
               dict(y=mat(), gate=vec(dtype=f32)), dict(y=mat(), x_out=mat(dtype=f32)), dict(y=mat(), only_x=True, w=vec()),
               dict(y=mat(), only_x=True, out=mat()), dict(stream=Stream(1))):
        a = dict(dict(x=x, out=mat()), **kw)
        if kw.get("only_x") and "out" not in kw:
            a["out"] = None
        if "y" in a and "x_out" not in a:
            a["x_out"] = mat()
        with pytest.raises(ValueError):
            monkeypatch.setattr(torch.cuda, "stream", lambda s: __import__("contextlib").nullcontext())
            P.norm(**a)


def test_pool_of_another_shape_is_refused():
    import torch
    n = P.page8_bytes(1, 2, 16, 64)
    for pool in (torch.zeros(3, n, dtype=torch.uint8), torch.zeros(3, n + 128, dtype=torch.uint8), torch.zeros(3, n)):   # (none on a GPU)
        with pytest.raises(ValueError):
            P.PageCache8(pool, 1, 2, 16, 64, 2, 2)
    assert P._AttendPlan8._fields_[:len(P._AttendPlan._fields_)] == P._AttendPlan._fields_
    assert np.dtype(np.int32).itemsize * 8 == 32 and C.sizeof(P._AttendPlan8) >= C.sizeof(P._AttendPlan) + 8
