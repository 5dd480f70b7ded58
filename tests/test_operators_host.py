"""The decoder-layer operators' C ABI: exported symbols and the refusals that need no GPU
(arguments are checked before any launch)."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from paper_2608_15762_gb300 import build, gmgop as P, gmgsim as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "gmgop.h")).read()
    hdr = re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)
    assert set(re.findall(r"\b(op_\w+)\s*\(", hdr)) == set(P.EXPORTED)
    for n in P.EXPORTED:
        assert hasattr(P.lib(), n), n


def _linear(**kw):
    a = dict(dtype=P.BF16, act=0, gated=0, m=4, n=8, k=16, x=256, w=512, y=1024, x_row=16, w_row=16, gate_row=16,
             residual_row=8, y_row=8)
    a.update(kw)
    s = P._Linear()
    for k, v in a.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("kw", [dict(dtype=P.F32), dict(dtype=7), dict(act=9), dict(act=-1), dict(m=-1), dict(k=-3),
                                dict(x=0), dict(w=0), dict(y=0), dict(x_row=15), dict(w_row=8), dict(y_row=7),
                                dict(residual=256, residual_row=4), dict(gated=1, gate=0), dict(gate_bias=256),
                                dict(m=2 ** 31)])
def test_linear_refuses(kw):
    a = _linear(**kw)
    assert P.lib().op_linear_work_bytes(C.addressof(a)) == 0
    assert P.lib().op_linear(C.addressof(a), 256, 1 << 30, None) == G.GMG_EINVAL


def test_linear_refuses_a_short_workspace():
    a = _linear()
    assert P.lib().op_linear_work_bytes(C.addressof(a)) >= 4096
    for work, size in ((0, 1 << 30), (128, 1 << 30), (256, 64)):
        assert P.lib().op_linear(C.addressof(a), work, size, None) == G.GMG_EWS


def _cache(**kw):
    a = dict(pool=256, table=256, lens=256, refs=256, status=256, dtype=P.BF16, n_pages=10, n_layers=2, n_kv_heads=2,
             page_tokens=16, head_dim=64, n_seq=4, max_pages=6)
    a.update(kw)
    s = P._Cache()
    for k, v in a.items():
        setattr(s, k, v)
    return s


BAD_CACHES = [dict(pool=0), dict(pool=8), dict(table=0), dict(dtype=P.F32), dict(n_pages=0), dict(page_tokens=12),
              dict(page_tokens=4), dict(page_tokens=512), dict(head_dim=129), dict(head_dim=12), dict(head_dim=136),
              dict(n_seq=0), dict(max_pages=0), dict(n_layers=0), dict(n_kv_heads=0)]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_page_calls_refuse_a_bad_cache(kw):
    L, r = P.lib(), C.addressof(_cache(**kw))
    assert L.op_page_scratch_bytes(r) == 0
    assert L.op_free(r, 256, 1, 256, 1 << 30, None) == G.GMG_EINVAL
    assert L.op_fork(r, 256, 256, None, 1, 256, 1 << 30, None) == G.GMG_EINVAL
    assert L.op_grow(r, 256, 256, 1, 256, 1 << 30, None) == G.GMG_EINVAL
    assert L.op_compact(r, 256, 1 << 30, None) == G.GMG_EINVAL


def test_page_calls_refuse_bad_lists_and_scratch():
    c = _cache()
    L, r = P.lib(), C.addressof(c)
    need = L.op_page_scratch_bytes(r)
    assert need > 0
    assert L.op_free(r, 256, -1, 256, need, None) == G.GMG_EINVAL
    assert L.op_free(r, 256, 5, 256, need, None) == G.GMG_EINVAL
    assert L.op_free(r, None, 2, 256, need, None) == G.GMG_EINVAL
    assert L.op_fork(r, 256, None, None, 2, 256, need, None) == G.GMG_EINVAL
    assert L.op_grow(r, 256, None, 2, 256, need, None) == G.GMG_EINVAL
    for work, size in ((0, need), (64, need), (256, need - 1)):
        assert L.op_grow(r, 256, 256, 1, work, size, None) == G.GMG_EWS
        assert L.op_compact(r, work, size, None) == G.GMG_EWS


def test_rope_refuses():
    L = P.lib()

    def rope(rotary=64, freq=256, dtype=P.BF16, tokens=3, heads=2, dim=64, x=256, pos=256, out=256):
        p = P._Rope(freq, rotary, 0, 1.0)
        return L.op_rope(C.addressof(p), dtype, tokens, heads, dim, x, 128, 64, pos, 0, out, 128, 64, None)

    for kw in (dict(rotary=63), dict(rotary=66), dict(rotary=-2), dict(freq=None), dict(dtype=5), dict(tokens=-1),
               dict(heads=-1), dict(dim=0), dict(x=None), dict(pos=None), dict(out=None), dict(rotary=258, dim=300)):
        assert rope(**kw) == G.GMG_EINVAL, kw
    assert rope(tokens=0) == G.GMG_OK
    p = P._Rope(256, 64, 0, 1.0)

    def append(cache, layer=0, k=256, seq=256):
        return L.op_rope_append(C.addressof(p), C.addressof(cache), layer, 3, 2, 256, 128, 64, k, 128, 64, 256, 128, 64,
                                256, seq, 256, 128, 64, None)

    assert append(_cache(), layer=2) == append(_cache(), layer=-1) == append(_cache(), k=None) == G.GMG_EINVAL
    assert append(_cache(), seq=None) == append(_cache(head_dim=32)) == G.GMG_EINVAL
    for kw in BAD_CACHES:
        assert append(_cache(**kw)) == G.GMG_EINVAL


def _refuses(*a, **kw):
    with pytest.raises(G.GmgError) as e:
        P.attend_items(*a, **kw)
    assert e.value.code == G.GMG_EINVAL


def test_attend_plan_refuses():
    ok = dict(q_len=[1, 2], kv_len=[5, 9], n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16)
    P.attend_items(**ok)
    for kw in (dict(q_len=[1, -1]), dict(kv_len=[-5, 9]), dict(n_heads=7), dict(n_heads=0), dict(n_kv_heads=0),
               dict(n_heads=258, n_kv_heads=2), dict(head_dim=136), dict(head_dim=60), dict(page_tokens=24),
               dict(seq=[0, -1]), dict(q_len=[2 ** 30, 1]), dict(n_sm=0),
               dict(group_off=[0, 1], prefix=[3]), dict(group_off=[1, 2], prefix=[3]),
               dict(group_off=[0, 2], prefix=[5]), dict(group_off=[0, 2], prefix=[-1]),
               dict(group_off=[0, 2, 1, 2], prefix=[0, 0, 0])):
        _refuses(**dict(ok, **kw))
    for kw in (dict(kv_len=[5]), dict(seq=[1]), dict(group_off=[0, 2]), dict(group_off=[0, 2], prefix=[1, 1])):
        with pytest.raises(ValueError):
            P.attend_items(**dict(ok, **kw))


def test_attend_refuses():
    L = P.lib()
    plan, items = P.attend_items([1, 2], [5, 90], 8, 2, 64, 16)

    def call(cache, layer=0, q=256, out=256, work=256, size=1 << 40, strides=(512, 64, 512, 64), items=256):
        return L.op_attend(C.addressof(plan), items, C.addressof(cache), layer, q, strides[0], strides[1], 1.0, out,
                           strides[2], strides[3], None, work, size, None)

    for kw in (dict(layer=2), dict(layer=-1), dict(q=None), dict(q=264), dict(out=None), dict(out=8), dict(items=None),
               dict(strides=(513, 64, 512, 64)), dict(strides=(512, 60, 512, 64)), dict(strides=(512, 64, 500, 64))):
        assert call(_cache(), **kw) == G.GMG_EINVAL, kw
    assert call(_cache(), work=0) == call(_cache(), work=128) == call(_cache(), size=0) == G.GMG_EWS
    for kw in BAD_CACHES + [dict(head_dim=72), dict(n_kv_heads=4), dict(page_tokens=32), dict(n_seq=1), dict(max_pages=5)]:
        assert call(_cache(**kw)) == G.GMG_EINVAL, kw


def test_rope_freqs_refuses():
    for a, kw in (((63,), {}), ((0,), {}), ((64,), dict(base=1.0)), ((64,), dict(scaling="none", scale=0.5)),
                  ((64,), dict(scaling="other")), ((64,), dict(scaling="parts", scale=2.0)), ((2,), dict(scaling="base"))):
        with pytest.raises(ValueError):
            P.rope_freqs(*a, **kw)


def test_rope_fractions_are_the_rounded_frequencies():
    f = P.rope_freqs(128)[0]
    p = P.Rope(128, freqs=f, device="cpu")
    got = p.freq.numpy().view(np.uint64).astype(object)
    for a, b in zip(got, f):
        assert abs(int(a) - b / (2 * np.pi) * 2.0 ** 64) <= 2.0 ** 64 * b / (2 * np.pi) * 2.0 ** -51 + 1


def _covered(q, kv, heads, kv_heads, groups=None, prefix=None):
    """Every (query, key) of a batch lies in one item, and joins list the parts of exactly those."""
    plan, items = P.attend_items(q, kv, heads, kv_heads, 64, 16, group_off=groups, prefix=prefix)
    g, n = heads // kv_heads, plan.n_items
    cover, joined, used = {t: [] for t in range(sum(q))}, {}, set()
    for tok0, n_tok, row, lo, hi, pos0, part, _ in items[:8 * n].reshape(n, 8).tolist():
        assert 0 < n_tok * g <= 128
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


def test_attend_plan_covers_every_key_once():
    import random
    r = random.Random(0)
    for _ in range(150):
        n, g, hk = r.randint(1, 40), r.choice([1, 2, 3, 4, 8, 40]), r.choice([1, 2, 8])
        groups = [0] + sorted(r.randint(0, n) for _ in range(r.randint(0, 4))) + [n]
        prefix = [r.choice([0, 1, 64, 100, 3000]) for _ in groups[1:]]
        q = [r.choice([0, 1, 1, 1, 2, 9, 200]) for _ in range(n)]
        kv = [prefix[k] + q[b] + r.choice([0, 0, 5, 70, 5000]) for k in range(len(prefix)) for b in range(groups[k], groups[k + 1])]
        _covered(q, kv, g * hk, hk, groups, prefix)
        _covered(q, [max(0, t - r.choice([0, 0, 3, 10 ** 6])) for t in kv], g * hk, hk)


def test_a_workspace_keeps_what_it_has_outgrown():
    """A captured call writes to the buffer that it was captured with whenever it is replayed."""
    import gc
    import weakref
    ws = P.Workspace("cpu")
    sizes = [4096, 5000, 20000, 20001, 10 ** 6]
    held = []
    for n in sizes:
        held.append(weakref.ref(ws.get(n)))
        assert ws.size >= n and ws.ptr % 256 == 0 and ws.ptr == ws.buf.data_ptr()
    gc.collect()
    assert all(h() is not None for h in held)
    assert sum(b.numel() for b in {h().data_ptr(): h() for h in held}.values()) <= 2 * ws.size
    held[0]()[:4] = 1                        # waits that gave up are counted wherever they were noted
    assert ws.gave_up() == 0x01010101


def test_waits_that_gave_up_on_default_workspaces_can_be_asked_for(monkeypatch):
    made = {(0, h): P.Workspace("cpu") for h in (0, 7)}
    monkeypatch.setattr(P, "_WORK", made)
    assert P.gave_up() == 0
    for ws in made.values():
        ws.get(4096)
    assert P.gave_up() == 0
    made[(0, 7)].buf[:4] = 1
    made[(0, 0)].buf[0] = 2
    assert P.gave_up() == 0x01010103


class _On:
    """What the binding asks of a tensor, of one that lies on GPU ``index``."""

    def __init__(self, index, *shape, dtype):
        import torch
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.device = torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def get_device(self):
        return self.index

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


class _Untouched:
    def __getattr__(self, name):
        def called(*a):
            raise AssertionError("called " + name)
        return called


def test_calls_refuse_what_is_not_on_the_current_gpu(monkeypatch):
    """Before anything is launched: the library must not be reached."""
    import torch
    P.lib()
    monkeypatch.setattr(P, "_LIB", _Untouched())
    monkeypatch.setattr(P, "lib", _Untouched())
    monkeypatch.setattr(P, "_current", lambda: 0)
    bf, i32 = torch.bfloat16, torch.int32

    class Stream:
        def __init__(self, index):
            self.device_index, self.cuda_stream = index, 0

    def plan(index, **kw):
        p = object.__new__(P.Rope if not kw else P.AttendPlan)
        p.index, p.ref = index, 256
        for k, v in kw.items():
            setattr(p, k, v)
        return p

    def cache(index):
        c = object.__new__(P.PageCache)
        c.device, c._index, c.dtype, c.n_kv_heads, c.head_dim = torch.device("cuda", index), index, bf, 2, 64
        c.ref, c._work = 256, (256, 256)
        return c

    def heads(index, n=2):
        return _On(index, 3, n, 64, dtype=bf)

    def ints(index, n=3):
        return _On(index, n, dtype=i32)

    def attend_plan(index):
        return plan(index, shape=(3, 2, 64), work={0: 256}, _ptr=256, head_dim=64, work_bytes=256)

    def rope(at, of, stream=None):
        P.rope(plan(of), heads(at), ints(at), out=heads(at), stream=stream)

    def append(at, of, stream=None):
        P.rope_append(plan(of), heads(at), heads(at), heads(at), ints(at), ints(at), cache(at), 0, out=heads(at), stream=stream)

    def attend(at, of, stream=None):
        P.attend(attend_plan(of), heads(at), cache(at), 0, out=heads(at), stream=stream)

    def linear(at, of, stream=None):
        ws = P.Workspace("cpu")
        ws.get(4096)
        ws.index = of
        P.linear(_On(at, 4, 64, dtype=bf), _On(at, 8, 64, dtype=bf), out=_On(at, 4, 8, dtype=bf), ws=ws, stream=stream)

    for call in (rope, append, attend, linear):
        for args in ((1, 1), (1, 0), (0, 1), (0, -1), (0, 0, Stream(1))):
            if call is attend and len(args) == 3 or call is linear and args != (1, 1):
                continue                     # (these ask for the stream's capture first, which takes a GPU)
            with pytest.raises(ValueError):
                call(*args)
    for call in (lambda c: c.free(ints(1, 2)), lambda c: c.fork(ints(1, 2), ints(1, 2)), lambda c: c.grow(ints(1, 2), ints(1, 2)),
                 lambda c: c.compact()):
        with pytest.raises(ValueError):
            call(cache(1))
    with pytest.raises(ValueError):
        P._handle(Stream(1), 0)
    assert P._handle(Stream(0), 0) == 0


def test_the_library_needs_no_cuda_runtime_beside_it():
    """It loads where no toolkit is installed, the simulator with it."""
    import subprocess
    import sys
    code = ("import ctypes, sys\n"
            "L = ctypes.CDLL(sys.argv[1])\n"
            "assert L.gmg_strerror and L.op_linear\n"
            "assert 'libcudart' not in open('/proc/self/maps').read()\n")
    subprocess.check_call([sys.executable, "-c", code, G.LIB_PATH])


def test_rope_fractions_are_rounded_once():
    """freq is f / (2 pi) * 2^64 to within half a unit, as the header says, for 64-bit f."""
    from decimal import Decimal, getcontext
    getcontext().prec = 80
    pi = Decimal("3.1415926535897932384626433832795028841971693993751058209749445923078164062862089986")
    top = float(np.nextafter(2 * np.pi, 0))
    for f in (P.rope_freqs(128)[0], P.rope_freqs(96, base=5e5, scaling="parts", scale=8.0, length=8192)[0],
              np.array([0.0, 1e-300, 5e-324, 1.0, 3.0, top])):
        got = P.Rope(2 * len(f), freqs=f, device="cpu").freq.numpy().view(np.uint64)
        for a, b in zip(got, f):
            assert abs(int(a) - min(Decimal(float(b)) * 2 ** 64 / (2 * pi), Decimal(2 ** 64 - 1))) <= Decimal("0.5000001")


def test_attend_plan_refuses_lengths_that_no_cache_holds():
    """Rounded up to whole steps or tiles they would pass 32 bits."""
    for q, kv in (([1], [2 ** 31 - 1]), ([1], [2 ** 30 + 1]), ([0], [2 ** 31 - 1]), ([2 ** 30 + 1], [5])):
        _refuses(q, kv, 1, 1, 64, 16)
    plan, items = P.attend_items([1], [2 ** 30], 8, 1, 64, 256)
    runs = sorted(items[:8 * plan.n_items].reshape(-1, 8)[:, 3:5].tolist())
    assert runs[0][0] == 0 and runs[-1][1] == 2 ** 30 and all(a[1] == b[0] for a, b in zip(runs, runs[1:]))
