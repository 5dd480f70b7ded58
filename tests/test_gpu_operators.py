"""GPU parity of the decoder-layer operators (include/gmgop.h) with plain implementations
in 64 bits (op_ref.py); whole numbers and copies exactly."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import op_ref as R  # noqa: E402
from paper_2608_15762_gb300 import gmgop as P  # noqa: E402
from paper_2608_15762_gb300 import gmgsim as G  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_15762_gb300 import build
    build.build()
    assert torch.cuda.is_available()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype=BF, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# Products
# ---------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 64, 128), (1, 4096, 256), (2, 72, 130), (7, 1000, 33), (16, 128, 128), (17, 520, 257),
         (33, 64, 1), (64, 2048, 96), (100, 136, 640), (128, 8, 128), (129, 200, 300), (256, 512, 512), (300, 1024, 777),
         (513, 264, 1025), (1500, 640, 130)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear_sizes(m, k, n, dtype):
    g = _gen(m + 3 * k + 7 * n)
    x, w = _rand(g, m, k, dtype=dtype), _rand(g, n, k, dtype=dtype, scale=k ** -0.5)
    for kw in (dict(), dict(bias=_rand(g, n, dtype=dtype), act="gelu", residual=_rand(g, m, n, dtype=dtype)),
               dict(gate=_rand(g, n, k, dtype=dtype, scale=k ** -0.5), act="silu"),
               dict(gate=_rand(g, n, k, dtype=dtype, scale=k ** -0.5), act="relu", bias=_rand(g, n, dtype=dtype),
                    gate_bias=_rand(g, n, dtype=dtype), residual=_rand(g, m, n, dtype=dtype))):
        want, tol = R.linear(x, w, **kw)
        R.within(P.linear(x, w, **kw), want, tol, "linear %s" % sorted(kw))


@pytest.mark.parametrize("act", sorted(P.ACTS))
def test_linear_activations_over_their_range(act):
    # one input per row picks a value from the weight: every output is the activation of one number
    v = torch.linspace(-30, 30, 512, device="cuda").to(HF)
    x, w = torch.zeros(3, 8, dtype=HF, device="cuda"), torch.zeros(512, 8, dtype=HF, device="cuda")
    x[:, 0], w[:, 0] = torch.tensor([1.0, 0.5, -1.0], device="cuda").to(HF), v
    want, tol = R.linear(x, w, act=act)
    R.within(P.linear(x, w, act=act), want, tol, act)


@pytest.mark.parametrize("off,ld,k", [(0, 72, 64), (8, 136, 100), (1, 80, 64), (0, 77, 70), (4, 65, 65)])
@pytest.mark.parametrize("m", [3, 150])
def test_linear_strides_and_alignment(m, off, ld, k):
    g = _gen(ld)
    n = 90
    x = _rand(g, m, ld + 16)[:, off:off + k]
    w, gate = _rand(g, n, ld, scale=0.1)[:, :k], _rand(g, n, ld, scale=0.1)[:, :k]
    out = torch.full((m, n + 5), 7.0, dtype=BF, device="cuda")
    res = _rand(g, m, n + 3)[:, 1:n + 1]
    kw = dict(gate=gate, act="silu", residual=res)
    want, tol = R.linear(x, w, **kw)
    P.linear(x, w, out=out[:, 2:n + 2], **kw)
    R.within(out[:, 2:n + 2], want, tol)
    assert bool((out[:, :2] == 7).all()) and bool((out[:, n + 2:] == 7).all())


@pytest.mark.parametrize("m", [5, 200])
def test_linear_into_its_residual(m):
    g = _gen(m)
    x, w, y = _rand(g, m, 256), _rand(g, 384, 256, scale=1 / 16), _rand(g, m, 384)
    want, tol = R.linear(x, w, residual=y)
    assert P.linear(x, w, residual=y, out=y) is y
    R.within(y, want, tol)


@pytest.mark.parametrize("m,k,n", [(0, 64, 32), (4, 64, 0), (4, 0, 32), (1, 0, 9)])
def test_linear_empty(m, k, n):
    g = _gen(5)
    x, w, b = _rand(g, m, k), _rand(g, n, k), _rand(g, n)
    res = _rand(g, m, n)
    want, tol = R.linear(x, w, bias=b, act="silu", residual=res)
    y = P.linear(x, w, bias=b, act="silu", residual=res)
    assert y.shape == (m, n)
    R.within(y, want, tol)
    want, tol = R.linear(x, w, bias=b, act="silu", gate=w, gate_bias=b)
    R.within(P.linear(x, w, bias=b, act="silu", gate=w, gate_bias=b), want, tol)


@pytest.mark.parametrize("m", [2, 140])
def test_linear_infinities_and_nan_stay_in_their_rows(m):
    g = _gen(11)
    x, w = _rand(g, m, 512), _rand(g, 200, 512, scale=1 / 16)
    x[0, 3], x[1, 500] = math.inf, math.nan
    y = P.linear(x, w)
    assert not bool(torch.isfinite(y[0]).any()) and bool(torch.isnan(y[1]).all())
    want, tol = R.linear(x[2:], w)
    R.within(y[2:], want, tol)


def test_linear_same_bits_every_time():
    g = _gen(12)
    for m, k, n in ((1, 8192, 512), (40, 4096, 384), (700, 1024, 600)):
        x, w, r = _rand(g, m, k), _rand(g, n, k, scale=k ** -0.5), _rand(g, m, n)
        first = P.linear(x, w, residual=r)
        for _ in range(5):
            assert torch.equal(P.linear(x, w, residual=r), first)


def test_linear_on_another_stream_and_in_a_graph():
    g = _gen(13)
    x, w = _rand(g, 9, 2048), _rand(g, 640, 2048, scale=2048 ** -0.5)
    want, tol = R.linear(x, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y = P.linear(x, w, stream=st)
    st.synchronize()
    R.within(y, want, tol)
    ws = P.Workspace()
    P.linear(x, w, ws=ws)
    torch.cuda.synchronize()
    out = torch.empty(9, 640, dtype=BF, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.linear(x, w, out=out, ws=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        R.within(out, want, tol)


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, HF, FF])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 8, 8), (5, 3, 64, 64), (3, 7, 80, 32), (130, 4, 128, 128), (2, 5, 33, 6),
                                       (9, 2, 96, 96), (4, 3, 128, 0), (17, 40, 72, 36), (1, 1, 256, 256)])
def test_rope(T, H, D, rot, inter, dtype):
    g = _gen(T * 100 + D)
    f = P.rope_freqs(rot)[0] if rot else np.zeros(0)
    plan = P.Rope(rot, freqs=f, factor=1.25, interleaved=inter)
    x = _rand(g, T, H, D, dtype=dtype)
    pos = torch.randint(0, 300000, (T,), generator=g, device="cuda", dtype=torch.int32)
    for back in (False, True):
        want, tol = R.rope(x, pos, f, 1.25, inter, back)
        R.within(P.rope(plan, x, pos, backward=back), want, tol)


def test_rope_far_positions():
    f = P.rope_freqs(128)[0]
    pos = _ints([0, 1, -1, -77777, 2 ** 20 + 1, 2 ** 31 - 1, -2 ** 31])
    x = _rand(_gen(3), 7, 2, 128, dtype=FF)
    want, tol = R.rope(x, pos, f)
    R.within(P.rope(P.Rope(128, freqs=f), x, pos), want, tol)


def test_rope_strides_in_place_and_odd_alignment():
    g = _gen(4)
    f = P.rope_freqs(64)[0]
    plan = P.Rope(64, freqs=f)
    pos = torch.arange(11, dtype=torch.int32, device="cuda")
    buf = _rand(g, 11, 3 * 64 + 3)
    for off in (0, 1):
        row = buf.clone()
        view = row[:, off:off + 192].view(11, 3, 64) if off == 0 else row[:, off:off + 192].unflatten(1, (3, 64))
        want, tol = R.rope(view, pos, f)
        P.rope(plan, view, pos, out=view)
        R.within(view, want, tol)
        assert torch.equal(row[:, off + 192:], buf[:, off + 192:]) and torch.equal(row[:, :off], buf[:, :off])
    x = _rand(g, 3, 11, 64).transpose(0, 1)     # heads outside
    want, tol = R.rope(x, pos, f)
    R.within(P.rope(plan, x, pos), want, tol)
    assert P.rope(plan, _rand(g, 0, 3, 64), pos[:0]).shape == (0, 3, 64)


def test_rope_backward_is_the_gradient():
    """By differences: the map is linear, so (f(x + d) - f(x)) . g = d . back(g) to rounding."""
    g = _gen(6)
    for inter in (False, True):
        plan = P.Rope(48, interleaved=inter, scaling="parts", scale=8.0, length=4096)
        x, d, y = (_rand(g, 21, 3, 64, dtype=FF) for _ in range(3))
        pos = torch.arange(5000, 5021, dtype=torch.int32, device="cuda")
        step = P.rope(plan, x + d, pos).double() - P.rope(plan, x, pos).double()
        a, b = (step * y.double()).sum(), (d.double() * P.rope(plan, y, pos, backward=True).double()).sum()
        size = (d.double().abs() * y.double().abs()).sum() + 21 * 3 * 64
        assert abs(float(a - b)) <= 2e-6 * plan.factor * float(size)


def test_rope_scalings():
    f, m = P.rope_freqs(64, 10000.0, "linear", 4.0)
    assert np.allclose(f * 4, P.rope_freqs(64)[0]) and m == 1.0
    f, _ = P.rope_freqs(64, 10000.0, "base", 4.0)
    assert f[0] == 1.0 and np.isclose(f[-1] * 4, P.rope_freqs(64)[0][-1])
    f, m = P.rope_freqs(64, 10000.0, "parts", 4.0, length=8192)
    b = P.rope_freqs(64)[0]
    assert f[0] == b[0] and np.isclose(f[-1] * 4, b[-1]) and np.all(np.diff(f) < 0) and np.isclose(m, 1 + 0.1 * math.log(4))


def _cache(g, n_pages, layers, hk, page, dim, n_seq, cols, dtype=BF):
    return P.PageCache(_rand(g, n_pages, layers, 2, hk, page, dim, dtype=dtype), n_seq, cols)


@pytest.mark.parametrize("T,H,Hk,D,rot,page,dtype", [(1, 4, 1, 64, 64, 16, BF), (50, 8, 2, 80, 40, 8, HF),
                                                     (33, 0, 3, 128, 128, 32, BF), (200, 5, 5, 24, 12, 256, HF)])
def test_rope_append(T, H, Hk, D, rot, page, dtype):
    g = _gen(T + D)
    n_seq, cols = 4, -(-T // page) + 2
    c = _cache(g, n_seq * cols + 3, 2, Hk, page, D, n_seq, cols, dtype)
    ids = torch.randperm(n_seq * cols + 3, generator=g, device="cuda")[:n_seq * cols].int()
    c.table.copy_(ids.view(n_seq, cols))
    plan = P.Rope(rot, base=500.0)
    row = _rand(g, T, (H + 2 * Hk) * D, dtype=dtype)
    q, k, v = row[:, :H * D].unflatten(1, (H, D)) if H else row.new_zeros(T, 0, D), \
        row[:, H * D:(H + Hk) * D].unflatten(1, (Hk, D)), row[:, (H + Hk) * D:].unflatten(1, (Hk, D))
    # tokens of the rows one after another, some padded (-1), one beyond its row's pages
    seq = torch.arange(T, device="cuda", dtype=torch.int32) % n_seq
    pos = torch.arange(T, device="cuda", dtype=torch.int32) // n_seq
    dropped = 0
    if T > 10:
        seq[3], seq[7], pos[5], dropped = -1, n_seq, cols * page, 2
    before = c.pool.clone()
    out = P.rope_append(plan, q, k, v, pos, seq, c, 1)
    f = P.rope_freqs(rot, 500.0)[0]
    want, tol = R.rope(q, pos, f)
    R.within(out, want, tol)
    kw, kt = R.rope(k, pos, f)
    expect, bound = before.double().cpu(), torch.zeros(before.shape, dtype=torch.float64)
    for t in range(T):
        r, p = int(seq[t]), int(pos[t])
        if 0 <= r < n_seq and p < cols * page:
            at = int(c.table[r, p // page])
            expect[at, 1, 0, :, p % page], bound[at, 1, 0, :, p % page] = kw[t], kt[t]
            expect[at, 1, 1, :, p % page] = v[t].double().cpu()
    R.within(c.pool, expect, bound)
    assert c.status.tolist()[4] == dropped


# ---------------------------------------------------------------------------
# Pages
# ---------------------------------------------------------------------------

def _same(c, ref, label):
    torch.cuda.synchronize()
    assert c.table.tolist() == ref.table(), label
    assert c.lens.tolist() == ref.lens, label
    assert c.refs.tolist() == ref.refs, label
    used = [p for p, n in enumerate(ref.refs) if n]
    first = c.pool[:, 0, 0, 0, 0, 0].float().long().tolist()
    assert [first[p] for p in used] == [ref.data[p] % 251 for p in used], label


def _labelled(n_pages, layers, hk, page, dim, n_seq, cols):
    pool = (torch.arange(n_pages, device="cuda") % 251).to(BF).view(-1, 1, 1, 1, 1, 1)
    return P.PageCache(pool.expand(n_pages, layers, 2, hk, page, dim).contiguous(), n_seq, cols)


@pytest.mark.parametrize("n_pages,page,n_seq,cols,seed", [(37, 8, 9, 12, 1), (900, 16, 40, 30, 2), (4096, 8, 300, 20, 3),
                                                          (9001, 32, 120, 64, 4), (1, 16, 2, 3, 5)])
def test_pages_random_walk(n_pages, page, n_seq, cols, seed):
    r = random.Random(seed)
    c = _labelled(n_pages, 2, 1, page, 8, n_seq, cols)
    ref = R.Pages(n_pages, page, n_seq, cols)
    done = 0
    for step in range(60):
        what = r.choice(("grow", "grow", "fork", "free", "compact"))
        some = r.sample(range(n_seq), r.randint(1, n_seq))
        if what == "grow":
            most = max(1, 2 * n_pages * page // (3 * len(some) * 4))
            add = [r.choice((0, 1, 1, 2, page, r.randint(0, min(most, cols * page // 3)))) for _ in some]
            ok = ref.grow(some, add)
            c.grow(_ints(some), _ints(add))
        elif what == "fork":
            empty = [b for b in range(n_seq) if not ref.lens[b] and not ref.rows[b]]
            dst = r.sample(empty, r.randint(0, len(empty)))
            full = [b for b in range(n_seq) if b not in dst]
            if not full:
                continue
            src = [r.choice(full) for _ in dst]
            keep = [r.randint(0, ref.lens[a]) for a in src] if r.random() < 0.5 else None
            ok = ref.fork(src, dst, keep)
            c.fork(_ints(src), _ints(dst), None if keep is None else _ints(keep))
        elif what == "free":
            some = some[:max(1, len(some) // 3)]
            ok = ref.free(some)
            c.free(_ints(some))
        else:
            ok = True
            moved = ref.compact()
            c.compact()
            assert tuple(c.status.tolist()[2:4]) == moved
        assert (c.code()[0] == P.PAGE_OK) == ok, (step, what, c.code())
        done += ok
        _same(c, ref, (step, what))
    assert done > 20


def test_pages_copy_every_byte():
    g = _gen(8)
    c = _cache(g, 50, 3, 2, 16, 72, 6, 8)
    c.grow(_ints([0]), _ints([21]))
    c.fork(_ints([0, 0, 0]), _ints([1, 2, 3]), _ints([21, 18, 16]))
    row = c.table[0].tolist()
    old = c.pool.clone()
    c.grow(_ints([1, 2, 3]), _ints([1, 3, 1]))
    t = c.table.tolist()
    assert t[0] == row and t[1][0] == t[2][0] == t[3][0] == row[0]
    assert len({t[0][1], t[1][1], t[2][1], t[3][1]}) == 4 and c.refs[row[1]] == 1
    for a in (1, 2):
        assert torch.equal(c.pool[t[a][1]], old[row[1]])
    keep = [p for p in range(50) if p not in (t[1][1], t[2][1])]
    assert torch.equal(c.pool[keep], old[keep])
    c.free(_ints([0, 2]))
    held = {r: [c.pool[p].clone() for p in c.table[r].tolist() if p >= 0] for r in (1, 3)}
    c.compact()
    for r, pages in held.items():
        now = [p for p in c.table[r].tolist() if p >= 0]
        assert all(torch.equal(c.pool[p], d) for p, d in zip(now, pages))
    assert int((c.refs > 0).sum()) == int((c.refs[:4] > 0).sum())


def test_references_are_counted_from_a_table():
    pool = torch.zeros(9, 1, 2, 1, 8, 8, dtype=BF, device="cuda")
    table = torch.tensor([[3, 5, -1], [3, 7, 5], [-1, 99, -1]], dtype=torch.int32, device="cuda")
    c = P.PageCache(pool, table=table, lens=_ints([16, 24, 0]))
    assert c.refs.tolist() == [0, 0, 0, 2, 0, 2, 0, 1, 0]
    c.grow(_ints([0]), _ints([8]))
    assert c.code() == (P.PAGE_OK, 0) and c.table[0].tolist() == [3, 5, 0]


def test_page_calls_refuse_without_change():
    c = _labelled(10, 1, 1, 8, 8, 5, 4)
    c.grow(_ints([0, 1]), _ints([20, 9]))
    before = [t.clone() for t in (c.table, c.lens, c.refs, c.pool)]
    calls = [(lambda: c.grow(_ints([2, 3]), _ints([8, 40])), (P.PAGE_LONG, 1)),
             (lambda: c.grow(_ints([2, 3]), _ints([32, 32])), (P.PAGE_FULL, 3)),
             (lambda: c.grow(_ints([2, 5]), _ints([1, 1])), (P.PAGE_SEQ, 1)),
             (lambda: c.grow(_ints([-1]), _ints([1])), (P.PAGE_SEQ, 0)),
             (lambda: c.grow(_ints([2, 3, 2]), _ints([1, 1, 1])), (P.PAGE_TWICE, None)),
             (lambda: c.grow(_ints([2]), _ints([-1])), (P.PAGE_LONG, 0)),
             (lambda: c.grow(_ints([0]), _ints([2 ** 31 - 1])), (P.PAGE_LONG, 0)),
             (lambda: c.fork(_ints([0]), _ints([1])), (P.PAGE_USED, 0)),
             (lambda: c.fork(_ints([0, 2]), _ints([2, 3])), (P.PAGE_TWICE, 1)),
             (lambda: c.fork(_ints([0]), _ints([2]), _ints([21])), (P.PAGE_LONG, 0)),
             (lambda: c.fork(_ints([7]), _ints([2])), (P.PAGE_SEQ, 0)),
             (lambda: c.fork(_ints([0, 1]), _ints([2, 2])), (P.PAGE_TWICE, None)),
             (lambda: c.free(_ints([0, 0])), (P.PAGE_TWICE, None)),
             (lambda: c.free(_ints([1, 9])), (P.PAGE_SEQ, 1))]
    for call, (code, entry) in calls:
        call()
        got = c.code()
        assert got[0] == code and (entry is None or got[1] == entry), (got, code, entry)
        assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.lens, c.refs, c.pool)))
    c.free(_ints([]))
    assert c.code() == (0, 0)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def _filled(g, kv, hk, dim, page, dtype=BF, shared=(), layers=2, spare=3, poison=True):
    """A cache whose rows hold kv tokens, pages in random order; rows of a shared entry
    (first, last, tokens) hold the same first tokens, in the same full pages.  Slots that
    hold no token, and pages that no row lists, are NaN."""
    B, cols = len(kv), max(1, max(-(-n // page) for n in kv) if kv else 1)
    total = sum(-(-n // page) for n in kv) + spare
    pool = torch.full((total, layers, 2, hk, page, dim), math.nan if poison else 0.0, dtype=dtype, device="cuda")
    ids = torch.randperm(total, generator=g, device="cuda").tolist()
    table = torch.full((B, cols), -1, dtype=torch.int32)
    keys, vals = [], []
    lead = {}
    for first, last, tokens in shared:
        for b in range(first + 1, last):
            lead[b] = (first, tokens)
    for b, n in enumerate(kv):
        k, v = _rand(g, n, hk, dim, dtype=dtype), _rand(g, n, hk, dim, dtype=dtype)
        skip = 0
        if b in lead:
            a, tokens = lead[b]
            k[:tokens], v[:tokens] = keys[a][:tokens], vals[a][:tokens]
            skip = tokens // page
            table[b, :skip] = table[a, :skip]
        for j in range(skip, -(-n // page)):
            p = table[b, j] = ids.pop()
            part = slice(j * page, min(n, (j + 1) * page))
            pool[int(p), 1, 0, :, :part.stop - part.start] = k[part].transpose(0, 1)
            pool[int(p), 1, 1, :, :part.stop - part.start] = v[part].transpose(0, 1)
        keys.append(k)
        vals.append(v)
    return P.PageCache(pool, table=table.cuda()), keys, vals


def _check_attend(q_len, kv, H, Hk, D, page, dtype=BF, groups=None, prefix=None, seed=0, scale=None, q=None):
    g = _gen(seed + sum(kv) + D)
    shared = [] if groups is None else [(groups[i], groups[i + 1], prefix[i]) for i in range(len(prefix))]
    cache, keys, vals = _filled(g, kv, Hk, D, page, dtype, shared)
    q = _rand(g, sum(q_len), H, D, dtype=dtype) if q is None else q
    scale = D ** -0.5 if scale is None else scale
    plan = P.AttendPlan(q_len, kv, H, Hk, D, page, group_off=groups, prefix=prefix)
    o, lse = P.attend(plan, q, cache, 1, scale=scale, lse=True)
    at = 0
    for b, n in enumerate(q_len):
        if n:
            wo, to, wl, tl = R.attend(q[at:at + n], keys[b], vals[b], n, scale)
            R.within(o[at:at + n], wo, to, "request %d" % b)
            R.within(lse[at:at + n], wl, tl, "lse of request %d" % b)
        at += n
    assert cache.status.tolist()[5] == 0
    return cache, plan, q, o, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,Hk,D,page", [(8, 2, 128, 16), (4, 4, 64, 64), (6, 2, 80, 8), (7, 1, 24, 256), (40, 8, 128, 32),
                                         (64, 1, 64, 128)])
def test_attend_lengths(H, Hk, D, page, dtype):
    kv = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1000]
    _check_attend([1] * len(kv), kv, H, Hk, D, page, dtype)
    _check_attend([min(n, 7) for n in kv], kv, H, Hk, D, page, dtype, seed=1)
    _check_attend(kv[:11], kv[:11], H, Hk, D, page, dtype, seed=2)


def test_attend_rows_that_see_nothing():
    # no cached tokens; more queries than tokens; no queries
    cache, plan, q, o, lse = _check_attend([3, 5, 0, 1, 2], [0, 2, 70, 0, 2], 4, 2, 64, 16)
    assert bool((o[:3] == 0).all()) and bool((lse[:3] == -math.inf).all())
    assert bool((o[3:6] == 0).all()) and bool((lse[3:6] == -math.inf).all())
    empty = P.AttendPlan([], [], 4, 2, 64, 16)
    assert P.attend(empty, q[:0], cache, 1).shape == (0, 4, 64)
    empty = P.AttendPlan([0, 0], [5, 0], 4, 2, 64, 16)
    assert P.attend(empty, q[:0], cache, 1).shape == (0, 4, 64)


@pytest.mark.parametrize("H,Hk,D,page,dtype", [(8, 2, 128, 16, BF), (8, 8, 64, 32, HF), (5, 1, 80, 64, BF), (12, 4, 128, 8, HF)])
@pytest.mark.parametrize("pre", [[64], [100], [1], [513]])
def test_attend_shared_prefix(H, Hk, D, page, dtype, pre):
    n = 21
    kv = [pre[0] + 1 + (7 * b) % 90 for b in range(n)]
    _check_attend([1] * n, kv, H, Hk, D, page, dtype, groups=[0, n], prefix=pre)
    q = [1 + (5 * b) % 9 for b in range(n)]
    kv = [pre[0] + q[b] + (11 * b) % 70 for b in range(n)]
    _check_attend(q, kv, H, Hk, D, page, dtype, groups=[0, n], prefix=pre, seed=1)


def test_attend_groups_of_every_kind():
    # no prefix; a long one with one member; one with many; an empty group; long queries in a group
    groups, prefix = [0, 2, 3, 3, 20, 24, 25], [0, 300, 50, 777, 130, 0]
    r = random.Random(3)
    q, kv = [], []
    for i, p in enumerate(prefix):
        for b in range(groups[i], groups[i + 1]):
            n = r.choice((0, 1, 2, 3)) if i != 4 else r.choice((1, 90, 200))
            q.append(n)
            kv.append(p + n + r.randint(0, 100))
    for H, Hk, D, page in ((8, 2, 128, 16), (3, 3, 64, 32), (16, 1, 96, 16)):
        _check_attend(q, kv, H, Hk, D, page, groups=groups, prefix=prefix)


@pytest.mark.parametrize("q_len,kv_len,D", [(1, 20000, 128), (3, 9001, 64), (900, 2500, 128), (1, 64 * 1024 + 3, 64)])
def test_attend_long(q_len, kv_len, D):
    _check_attend([q_len], [kv_len], 8, 2, D, 64)


def test_attend_long_shared():
    n = 70
    kv = [8192 + 1 + 3 * b for b in range(n)]
    _check_attend([1] * n, kv, 16, 2, 128, 32, groups=[0, n], prefix=[8192])


def test_attend_large_scores_and_scales():
    g = _gen(77)
    for scale in (8.0, 0.0, -1.0, 1e-3):
        _check_attend([2, 40], [300, 150], 4, 2, 64, 16, scale=scale, seed=5)
    q = _rand(g, 3, 4, 64, scale=40.0)      # one key takes nearly everything
    _check_attend([3], [500], 4, 2, 64, 16, q=q, seed=6)


def test_attend_infinities_and_nan_stay_with_their_rows():
    """A query that is not finite spoils its own row only; a value that is not finite, the
    rows that see it only."""
    g = _gen(31)
    kv, n = 200, 150
    cache, keys, vals = _filled(g, [kv], 2, 64, 16)
    q = _rand(g, n, 4, 64)
    q[7, 1, 5] = math.nan
    plan = P.AttendPlan([n], [kv], 4, 2, 64, 16)
    o = P.attend(plan, q, cache, 1)
    clean = q.clone()
    clean[7, 1] = 0
    wo, to, _, _ = R.attend(clean, keys[0], vals[0], n, 0.125)
    assert bool(torch.isnan(o[7, 1]).all())
    o[7, 1] = wo[7, 1].to(BF)
    R.within(o, wo, to)
    for bad in (math.nan, math.inf):
        at = 120                              # of the tokens; query i sees it from i = at - (kv - n) on
        p = int(cache.table[0, at // 16])
        old = cache.pool[p].clone()
        cache.pool[p, 1, 1, 0, at % 16, 3] = bad
        cache.pool[p, 1, 0, 1, at % 16, 3] = bad
        o = P.attend(plan, clean, cache, 1)
        first = at - (kv - n)
        R.within(o[:first], wo[:first], to[:first], str(bad))
        assert not bool(torch.isfinite(o[first:, :2, 3]).any()) and not bool(torch.isfinite(o[first:, 2:]).any(-1).all())
        cache.pool[p] = old


def test_attend_strides_streams_and_graph():
    g = _gen(41)
    q_len, kv = [1, 4, 1], [100, 37, 65]
    cache, keys, vals = _filled(g, kv, 2, 64, 16)
    row = _rand(g, 6, (8 + 4) * 64)
    q = row[:, :8 * 64].unflatten(1, (8, 64))
    plan = P.AttendPlan(q_len, kv, 8, 2, 64, 16)
    want = P.attend(plan, q.contiguous(), cache, 1)
    assert torch.equal(P.attend(plan, q, cache, 1), want)
    out = torch.full((6, 10, 64), 3.0, dtype=BF, device="cuda")
    P.attend(plan, q, cache, 1, out=out[:, 1:9])
    assert torch.equal(out[:, 1:9], want) and bool((out[:, 0] == 3).all()) and bool((out[:, 9] == 3).all())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y = P.attend(plan, q, cache, 1, stream=st)
    st.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.attend(plan, q, cache, 1)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_attend_heads_outside_tokens_and_wide_groups():
    """Queries and results laid out head by head; 128 query heads on one key/value head."""
    g = _gen(42)
    for H, Hk, D in ((6, 2, 64), (128, 1, 128), (100, 1, 72)):
        q_len, kv = [3, 1, 40], [77, 300, 41]
        cache, keys, vals = _filled(g, kv, Hk, D, 32)
        q = _rand(g, H, sum(q_len), D).transpose(0, 1)
        out = torch.empty(H, sum(q_len), D, dtype=BF, device="cuda").transpose(0, 1)
        plan = P.AttendPlan(q_len, kv, H, Hk, D, 32)
        o, lse = P.attend(plan, q, cache, 1, out=out, lse=True)
        at = 0
        for b, n in enumerate(q_len):
            wo, to, wl, tl = R.attend(q[at:at + n], keys[b], vals[b], n, D ** -0.5)
            R.within(o[at:at + n], wo, to)
            R.within(lse[at:at + n], wl, tl)
            at += n


def test_attend_one_plan_on_two_streams():
    g = _gen(44)
    kv = [900] * 6
    cache, keys, vals = _filled(g, kv, 2, 64, 16)
    plan = P.AttendPlan([1] * 6, kv, 16, 2, 64, 16)
    assert plan.c.n_joins > 0
    qs = [_rand(g, 6, 16, 64) for _ in range(2)]
    want = [P.attend(plan, q, cache, 1) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            got[i].append(P.attend(plan, qs[i], cache, 1, stream=st))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_attend_table_with_missing_pages():
    """A page number outside the pool reads as no token's, never outside the pool's memory."""
    g = _gen(43)
    cache, keys, vals = _filled(g, [64], 1, 64, 16, poison=False)
    cache.table[0, 1] = 10 ** 6
    cache.table[0, 2] = -1
    plan = P.AttendPlan([1], [64], 1, 1, 64, 16)
    o = P.attend(plan, _rand(g, 1, 1, 64), cache, 1)
    assert o.shape == (1, 1, 64)
    torch.cuda.synchronize()


def test_a_step_of_requests_end_to_end():
    """Prompt, fork, two steps: the cache that the operators build gives the attention of the
    tokens themselves."""
    g = _gen(51)
    H, Hk, D, page = 8, 2, 64, 16
    cache = P.PageCache(torch.full((64, 1, 2, Hk, page, D), math.nan, dtype=BF, device="cuda"), 6, 12)
    plan = P.Rope(D)
    f = P.rope_freqs(D)[0]
    toks = {0: []}

    def step(rows, n, groups=None, prefix=None):
        T = len(rows) * n
        qkv = _rand(g, T, (H + 2 * Hk) * D)
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([H * D, Hk * D, Hk * D], 1))
        old = [len(toks[r]) for r in rows]
        pos = _ints(o + i for o in old for i in range(n))
        seq = _ints(r for r in rows for _ in range(n))
        cache.grow(_ints(rows), _ints([n] * len(rows)))
        rot = P.rope_append(plan, q, k, v, pos, seq, cache, 0)
        for i, r in enumerate(rows):
            for j in range(n):
                toks[r].append((k[i * n + j], v[i * n + j], old[i] + j))
        a = P.AttendPlan([n] * len(rows), [o + n for o in old], H, Hk, D, page, seq=rows, group_off=groups, prefix=prefix)
        o = P.attend(a, rot, cache, 0)
        for i, r in enumerate(rows):
            kk = torch.stack([t[0] for t in toks[r]])
            kp = _ints(t[2] for t in toks[r])
            kr = P.rope(plan, kk, kp)
            vv = torch.stack([t[1] for t in toks[r]])
            wo, to, _, _ = R.attend(rot[i * n:(i + 1) * n], kr, vv, n, D ** -0.5)
            R.within(o[i * n:(i + 1) * n], wo, to)

    step([0], 45)
    cache.fork(_ints([0, 0, 0]), _ints([1, 2, 3]))
    for r in (1, 2, 3):
        toks[r] = list(toks[0])
    step([0, 1, 2, 3], 1, [0, 4], [45])
    step([3, 1], 2, [0, 2], [45])
    cache.free(_ints([0, 1]))
    cache.compact()
    step([2, 3], 1, [0, 2], [45])
    assert cache.code()[0] == 0


# ---------------------------------------------------------------------------
# Offsets beyond 32 bits
# ---------------------------------------------------------------------------

def test_linear_and_rope_beyond_2_31_elements():
    g = _gen(61)
    m, n, k = 70_001, 32_768, 64
    x, w = _rand(g, m, k), _rand(g, n, k, scale=1 / 8)
    ws = P.Workspace()
    y = P.linear(x, w, ws=ws)
    assert y.numel() > 2 ** 31 and ws.gave_up() == 0
    for part in (slice(0, 2), slice(65_530, 65_540), slice(m - 3, m)):
        want, tol = R.linear(x[part], w)
        R.within(y[part], want, tol)
    heads = y.view(m, n // 128, 128)
    pos = torch.arange(m, dtype=torch.int32, device="cuda")
    last = heads[m - 2:].clone()
    P.rope(P.Rope(128), heads, pos, out=heads)
    want, tol = R.rope(last, pos[m - 2:], P.rope_freqs(128)[0])
    R.within(heads[m - 2:], want, tol)


def test_cache_beyond_2_31_elements():
    """The last pages of a pool of more than 2^31 elements: appended to, copied, read."""
    g = _gen(62)
    hk, page, D, n_pages = 8, 64, 128, 17_000
    pool = torch.empty(n_pages, 1, 2, hk, page, D, dtype=BF, device="cuda")
    assert pool.numel() > 2 ** 31
    c = P.PageCache(pool, n_seq=3, max_pages=6)
    c.refs.fill_(1)                      # only pages at the far end, and one in front, are free
    c.refs[n_pages - 8:] = 0
    c.refs[3] = 0
    c.grow(_ints([0]), _ints([150]))
    assert c.table[0].tolist()[:3] == [3, n_pages - 8, n_pages - 7]
    k, v = _rand(g, 150, hk, D), _rand(g, 150, hk, D)
    none = torch.empty(150, 0, D, dtype=BF, device="cuda")
    at = torch.arange(150, dtype=torch.int32, device="cuda")
    P.rope_append(P.Rope(0), none, k, v, at, torch.zeros_like(at), c, 0)
    c.fork(_ints([0]), _ints([1]))
    c.grow(_ints([1, 0]), _ints([1, 1]))
    new = [torch.cat((t, _rand(g, 1, hk, D))) for t in (k, v)]
    P.rope_append(P.Rope(0), none[:1], new[0][150:], new[1][150:], _ints([150]), _ints([1]), c, 0)
    q = _rand(g, 1, 16, D)
    o, lse = P.attend(P.AttendPlan([1], [151], 16, hk, D, page, seq=[1]), q, c, 0, lse=True)
    wo, to, wl, tl = R.attend(q, *new, 1, D ** -0.5)
    R.within(o, wo, to)
    R.within(lse, wl, tl)
    assert c.code()[0] == P.PAGE_OK and c.table[1].tolist()[2] == n_pages - 6
    c.free(_ints([0]))
    c.compact()
    assert c.status.tolist()[2] == 0 or int(c.refs[n_pages - 1]) == 0
    o2 = P.attend(P.AttendPlan([1], [151], 16, hk, D, page, seq=[1]), q, c, 0)
    assert torch.equal(o2, o)


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("pre", [[200], [321], [1001]])
@pytest.mark.parametrize("H,Hk,D,page,dtype", [(8, 2, 128, 16, BF), (5, 1, 80, 64, HF), (6, 6, 64, 8, BF)])
def test_attend_pooled_prefix_of_odd_lengths(pre, H, Hk, D, page, dtype):
    """Prefixes that end inside a step and a page, read once for all requests (the plan joins)."""
    n = 304 // Hk + 5                        # more than one round of blocks takes apart
    kv = [pre[0] + 1 + (13 * b) % 150 for b in range(n)]
    _, plan, *_ = _check_attend([1] * n, kv, H, Hk, D, page, dtype, groups=[0, n], prefix=pre)
    assert plan.c.n_joins >= n
    q = [1 + b % 3 for b in range(n)]
    _check_attend(q, [pre[0] + q[b] + (7 * b) % 60 for b in range(n)], H, Hk, D, page, dtype, groups=[0, n], prefix=pre)


def test_attend_many_parts():
    """More than eight parts a head, and few: both ways of joining them."""
    _check_attend([1], [30011], 2, 1, 128, 16)
    _check_attend([1, 2], [3000, 900], 2, 1, 64, 32)


def test_executor_example():
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(__file__), "..", "examples"))
    import executor_feedback as E
    lines = []
    r = E.main(layers=2, hidden=256, heads=4, kv_heads=2, ffn=320, requests=8, prompt=210, steps=5, n_dev=4, candidates=64,
               say=lines.append)
    ex = r["executor"]
    assert ex.cache.status.tolist()[0] == 0 and ex.cache.status.tolist()[4:6] == [0, 0]
    assert ex.cache.lens.tolist() == ex.len
    refs = torch.zeros_like(ex.cache.refs)
    used = ex.cache.table[ex.cache.table >= 0].long()
    refs.index_add_(0, used, torch.ones_like(used, dtype=torch.int32))
    assert torch.equal(refs, ex.cache.refs) and int((refs > 0).sum()) == int((refs[:int((refs > 0).sum())] > 0).sum())
    assert all(len(s) for s in ex.samples.values()) and any("t = " in s for s in lines)
    assert r["best"] >= 0 and r["makespan"] > 0 and bool((r["desc"].dur >= 1).all())


# ---------------------------------------------------------------------------
# Values that are not finite, in steps that follow one another
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("D,dtype", [(128, BF), (64, HF)])
def test_attend_values_that_are_not_finite_in_consecutive_steps(D, dtype):
    """A head each, so that a tile's 128 queries end in two steps of keys or three, with values that are
    not finite in the second, the third or all of them: only the rows that see one get it, and the
    keys of one step are never taken for another's.  Many requests, so that the warps' pace differs."""
    g = _gen(71)
    n, page, H = 60, 16, 2
    q_len = [128] * n
    kv = [128 + (7 * b) % 100 for b in range(n)]
    cache, keys, vals = _filled(g, kv, H, D, page, dtype)
    q = _rand(g, sum(q_len), H, D, dtype=dtype)
    want, tol, spoilt = [], [], torch.zeros(sum(q_len), H, D, dtype=torch.bool)
    for b in range(n):
        before = kv[b] - q_len[b]
        clean = vals[b].clone()
        # keys of the steps that the tile's queries end in: each step's, some steps' or one's
        for step in range(before // 64 + 1, (kv[b] - 1) // 64 + 1):
            if b % 3 == 1 and step % 2:
                continue
            for k in (64 * step + b % 5, 64 * step + 63 - b % 7)[:1 + b % 2]:
                if before < k < kv[b]:
                    h, d = k % H, (5 * k + b) % D
                    cache.pool[int(cache.table[b, k // page]), 1, 1, h, k % page, d] = (math.nan, math.inf, -math.inf)[k % 3]
                    clean[k, h, d] = 0
                    spoilt[128 * b + k - before:128 * (b + 1), h, d] = True
        w, t, _, _ = R.attend(q[128 * b:128 * (b + 1)], keys[b], clean, q_len[b], D ** -0.5)
        want.append(w)
        tol.append(t)
    want, tol = torch.cat(want).cpu(), torch.cat(tol).cpu()
    assert bool(spoilt.any()) and not bool(spoilt.all())
    plan = P.AttendPlan(q_len, kv, H, H, D, page)
    first = None
    for _ in range(40):
        o = P.attend(plan, q, cache, 1).cpu()
        assert not bool(torch.isfinite(o[spoilt]).any())
        o[spoilt] = want[spoilt].to(dtype)
        if first is None:
            R.within(o, want, tol)
            first = o
        assert torch.equal(o, first)
    assert cache.status.tolist()[5] == 0


# ---------------------------------------------------------------------------
# Workspaces and captured calls
# ---------------------------------------------------------------------------

def _work_bytes(m, k, n, gated=0):
    import ctypes as C
    a = P._Linear(P.BF16, 0, gated, 0, m, n, k, 256, 256, 256 if gated else 0, 0, 0, 0, 256, k, k, k if gated else 0, 0, n)
    return P.lib().op_linear_work_bytes(C.addressof(a))


def test_linear_captured_before_its_workspace_grew():
    """The replay's partial sums go where they were captured to go, not to memory that others have now."""
    g = _gen(81)
    m, k, n = 1270, 2056, 4001                     # 80 tiles: four are dealt out by steps, and joined
    x, w = _rand(g, m, k), _rand(g, n, k, scale=k ** -0.5)
    need, more = _work_bytes(m, k, n), _work_bytes(2560, 4096, 4096)
    assert 4096 < need < more
    want, tol = R.linear(x, w)
    ws = P.Workspace()
    R.within(P.linear(x, w, ws=ws), want, tol)
    out = torch.empty(m, n, dtype=BF, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.linear(x, w, out=out, ws=ws)
    P.linear(_rand(g, 2560, 4096), _rand(g, 4096, 4096), ws=ws)
    torch.cuda.synchronize()
    others = [torch.full((need // 4,), 7.0, device="cuda") for _ in range(4)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        R.within(out, want, tol)
    assert all(bool((t == 7).all()) for t in others) and ws.gave_up() == 0


def _captured(fn, stream):
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out = fn()
    return graph, out


def _replayed_side_by_side(fns, wants):
    """Graphs captured on one stream, then replayed on streams of their own, with eager calls beside them."""
    capture = torch.cuda.Stream()
    made = [_captured(fn, capture) for fn in fns]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    eager = []
    for _ in range(30):
        for (graph, _), st in zip(made, streams):
            with torch.cuda.stream(st):
                graph.replay()
        with torch.cuda.stream(capture):
            eager.append(fns[0]())
    torch.cuda.synchronize()
    for (_, out), want in zip(made, wants):
        assert torch.equal(out, want)
    assert all(torch.equal(t, wants[0]) for t in eager)


def test_linear_graphs_of_one_stream_do_not_share_a_workspace():
    g = _gen(82)
    m, k, n = 1270, 2056, 4001
    w = _rand(g, n, k, scale=k ** -0.5)
    xs = [_rand(g, m, k) for _ in range(3)]
    wants = [P.linear(x, w) for x in xs]
    kept = {key: ws.size for key, ws in P._WORK.items()}
    _replayed_side_by_side([lambda x=x: P.linear(x, w) for x in xs], wants)
    new = set(P._WORK) - set(kept)
    assert len(new) == 1 and P._WORK[new.pop()].gave_up() == 0      # the eager calls' stream, made outside a capture
    # a workspace that is too small, or has not been used, is left as it is
    ws = P.Workspace()
    graph, out = _captured(lambda: P.linear(xs[0], w, ws=ws), torch.cuda.Stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, wants[0]) and ws.buf is None and ws.gave_up() == 0


def test_attend_graphs_of_one_plan_do_not_share_a_workspace():
    g = _gen(83)
    kv = [1500] * 6
    cache, keys, vals = _filled(g, kv, 2, 64, 16)
    plan = P.AttendPlan([1] * 6, kv, 16, 2, 64, 16)
    assert plan.c.n_joins > 0
    qs = [_rand(g, 6, 16, 64) for _ in range(3)]
    wants = [P.attend(plan, q, cache, 1) for q in qs]
    assert len(plan.work) == 1
    _replayed_side_by_side([lambda q=q: P.attend(plan, q, cache, 1) for q in qs], wants)
    assert len(plan.work) == 2


def test_calls_refuse_plans_and_workspaces_of_other_devices():
    g = _gen(84)
    x, pos = _rand(g, 3, 2, 64), _ints([0, 1, 2])
    cache = _cache(g, 4, 1, 2, 16, 64, 2, 2)
    cpu = P.Rope(64, device="cpu")
    ws = P.Workspace("cpu")
    for call in (lambda: P.rope(cpu, x, pos), lambda: P.rope_append(cpu, x, x, x, pos, pos, cache, 0),
                 lambda: P.linear(x[0], x[1], ws=ws)):
        with pytest.raises(ValueError):
            call()
    plan = P.AttendPlan([3], [3], 2, 2, 64, 16)
    plan.index = -1
    with pytest.raises(ValueError):
        P.attend(plan, x, cache, 0)


@pytest.mark.parametrize("n_seq", [40, 3000])
def test_a_row_listed_twice_is_reported_at_its_second_entry(n_seq):
    """Whatever the order in which the threads run: the smallest entry that an earlier one equals."""
    r = random.Random(n_seq)
    c = _labelled(64, 1, 1, 8, 8, n_seq + 1, 20)
    c.grow(_ints([n_seq]), _ints([5]))
    for _ in range(12):
        rows = r.sample(range(n_seq), n_seq // 2)
        for _ in range(r.randint(1, 6)):
            rows[r.randrange(len(rows))] = r.choice(rows)
        seen, first = set(), None
        for i, row in enumerate(rows):
            if row in seen and first is None:
                first = i
            seen.add(row)
        want = (P.PAGE_TWICE, first) if first is not None else None
        for call in (lambda: c.free(_ints(rows)), lambda: c.grow(_ints(rows), _ints([0] * len(rows))),
                     lambda: c.fork(_ints([n_seq] * len(rows)), _ints(rows), _ints([0] * len(rows)))):
            call()
            if want is not None:
                assert c.code() == want
            else:
                assert c.code()[0] == P.PAGE_OK
    c.grow(_ints([3, 5, 5, 3]), _ints([1, 1, 1, 1]))
    assert c.code() == (P.PAGE_TWICE, 2)
    c.free(_ints([7, 7]))
    assert c.code() == (P.PAGE_TWICE, 1)


# ---------------------------------------------------------------------------
# Products over pairs of blocks: more tiles than fill half of the SMs
# ---------------------------------------------------------------------------

def _pair_sizes():
    # one round and a part, odd columns and rows; several tiles dealt out by steps and joined, odd and even;
    # a last tile of one row and one column; columns of x that are no whole step
    return [(1300, 520, 5001, False), (1270, 2056, 4001, True), (1537, 1544, 3500, False), (2305, 264, 2561, False),
            (640, 4104, 6600, True), (20000, 72, 300, False)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,k,n,joined", _pair_sizes())
def test_linear_over_pairs(m, k, n, joined, dtype):
    g = _gen(m + k + n)
    x, w, gate = _rand(g, m, k, dtype=dtype), _rand(g, n, k, dtype=dtype, scale=k ** -0.5), _rand(g, n, k, dtype=dtype, scale=k ** -0.5)
    bias, gate_bias, res = _rand(g, n, dtype=dtype), _rand(g, n, dtype=dtype), _rand(g, m, n, dtype=dtype)
    assert 2 * -(-n // 256) * -(-m // 256) > 76
    if joined:
        assert _work_bytes(m, k, n) > 4096 and _work_bytes(m, k, n, 1) > 4096
    for kw in (dict(), dict(bias=bias, act="gelu", residual=res), dict(act="relu", residual=res), dict(bias=bias, act="silu"),
               dict(gate=gate, act="silu"), dict(gate=gate, act="relu", bias=bias, gate_bias=gate_bias, residual=res),
               dict(gate=gate, act="gelu", gate_bias=gate_bias), dict(gate=gate, act="none", bias=bias, residual=res)):
        want, tol = R.linear(x, w, **kw)
        ws = P.Workspace()
        y = P.linear(x, w, ws=ws, **kw)
        R.within(y, want, tol, "linear %s" % sorted(kw))
        assert torch.equal(P.linear(x, w, ws=ws, **kw), y) and ws.gave_up() == 0


@pytest.mark.parametrize("m,k,n", [(1300, 520, 5001), (1270, 2056, 4001)])
def test_linear_over_pairs_strides_and_in_place(m, k, n):
    g = _gen(m)
    x, w, gate = _rand(g, m, k + 24)[:, 8:8 + k], _rand(g, n, k + 8, scale=k ** -0.5)[:, :k], _rand(g, n, k + 16, scale=k ** -0.5)[:, 8:8 + k]
    out = torch.full((m, n + 9), 7.0, dtype=BF, device="cuda")
    res = _rand(g, m, n + 3)[:, 1:n + 1]
    for kw in (dict(act="silu", residual=res), dict(gate=gate, act="silu", residual=res)):
        want, tol = R.linear(x, w, **kw)
        P.linear(x, w, out=out[:, 5:n + 5], **kw)
        R.within(out[:, 5:n + 5], want, tol)
        assert bool((out[:, :5] == 7).all()) and bool((out[:, n + 5:] == 7).all())
        y = res.clone()
        P.linear(x, w, out=y, **dict(kw, residual=y))
        R.within(y, want, tol)


@pytest.mark.parametrize("m,k,n", [(1300, 520, 5001), (1270, 2056, 4001)])
def test_linear_over_pairs_infinities_and_nan_stay_in_their_rows_and_columns(m, k, n):
    g = _gen(n)
    x, w = _rand(g, m, k), _rand(g, n, k, scale=k ** -0.5)
    want, tol = R.linear(x, w)
    rows, cols = (0, 255, 256, m - 1), (1, 127, 128, n - 1)
    for i, r in enumerate(rows):
        x[r, (5 * i) % k] = (math.nan, math.inf)[i % 2]
    for i, c in enumerate(cols):
        w[c, (k - 1 - i)] = (math.nan, -math.inf)[i % 2]
    y = P.linear(x, w)
    clean = torch.ones(m, n, dtype=torch.bool, device="cuda")
    clean[list(rows)] = False
    clean[:, list(cols)] = False
    assert not bool(torch.isfinite(y[list(rows)]).any()) and not bool(torch.isfinite(y[:, list(cols)]).any())
    R.within(y[clean], want[clean], tol[clean])


def test_linear_clusters_of_every_tile():
    """Fewer tiles: each height of a tile, gated and not, with every activation and both types."""
    g = _gen(91)
    for i, m in enumerate((3, 16, 17, 31, 32, 33, 64, 65, 128, 129, 255, 256, 257)):
        k, n, dtype = 1032 + 8 * i, 384 + 37 * i, (BF, HF)[i % 2]
        x, w, gate = _rand(g, m, k, dtype=dtype), _rand(g, n, k, dtype=dtype, scale=k ** -0.5), _rand(g, n, k, dtype=dtype, scale=k ** -0.5)
        bias, res = _rand(g, n, dtype=dtype), _rand(g, m, n, dtype=dtype)
        for act in sorted(P.ACTS):
            for kw in (dict(bias=bias, act=act, residual=res), dict(gate=gate, act=act, gate_bias=bias, residual=res)):
                want, tol = R.linear(x, w, **kw)
                R.within(P.linear(x, w, **kw), want, tol, "%d rows, %s" % (m, sorted(kw)))


# ---------------------------------------------------------------------------
# What a table without a page, and a compaction, come to
# ---------------------------------------------------------------------------

def test_attend_missing_pages_read_as_zeros():
    g = _gen(43)
    for D, page, n in ((64, 16, 64), (128, 8, 200)):
        cache, keys, vals = _filled(g, [n], 1, D, page)
        gone = {1: 10 ** 6, 2: -1, 5: len(cache.refs), (n - 1) // page: -2 ** 31}
        for j, p in gone.items():
            if j < -(-n // page):
                cache.table[0, j] = p
                keys[0][j * page:(j + 1) * page] = 0
                vals[0][j * page:(j + 1) * page] = 0
        q = _rand(g, 3, 2, D)
        o, lse = P.attend(P.AttendPlan([3], [n], 2, 1, D, page), q, cache, 1, lse=True)
        wo, to, wl, tl = R.attend(q, keys[0], vals[0], 3, D ** -0.5)
        R.within(o, wo, to)
        R.within(lse, wl, tl)


def test_compact_moves_the_last_pages_of_a_large_pool():
    g = _gen(92)
    hk, page, D, n_pages = 8, 64, 128, 17_000
    pool = torch.empty(n_pages, 1, 2, hk, page, D, dtype=BF, device="cuda")
    c = P.PageCache(pool, n_seq=3, max_pages=6)
    c.refs.fill_(1)
    c.refs[n_pages - 8:] = 0
    c.refs[3] = 0
    c.grow(_ints([0]), _ints([150]))         # pages 3, n - 8, n - 7
    c.grow(_ints([1]), _ints([10]))          # n - 6
    assert c.table[:2, :3].tolist() == [[3, n_pages - 8, n_pages - 7], [n_pages - 6, -1, -1]]
    for p in (3, n_pages - 8, n_pages - 7, n_pages - 6):
        pool[p] = _rand(g, 1, 2, hk, page, D)
    held, still = pool[n_pages - 6].clone(), pool[n_pages - 9].clone()
    c.free(_ints([0]))
    c.compact()
    assert c.status.tolist()[:4] == [P.PAGE_OK, 0, 1, n_pages - 8]
    assert c.table.tolist() == [[-1] * 6, [3] + [-1] * 5, [-1] * 6] and c.lens.tolist() == [0, 10, 0]
    refs = c.refs.tolist()
    assert refs[:n_pages - 8] == [1] * (n_pages - 8) and refs[n_pages - 8:] == [0] * 8
    assert torch.equal(pool[3], held) and torch.equal(pool[n_pages - 9], still)
    # two pages move, in order
    c.grow(_ints([0, 2]), _ints([64, 128]))
    assert c.table[:, :2].tolist() == [[n_pages - 8, -1], [3, -1], [n_pages - 7, n_pages - 6]]
    for p in (n_pages - 7, n_pages - 6):
        pool[p] = _rand(g, 1, 2, hk, page, D)
    held = [pool[n_pages - 7].clone(), pool[n_pages - 6].clone()]
    c.free(_ints([0, 1]))
    c.compact()
    assert c.status.tolist()[:4] == [P.PAGE_OK, 0, 2, n_pages - 7]
    assert c.table[2, :2].tolist() == [3, n_pages - 8]
    assert torch.equal(pool[3], held[0]) and torch.equal(pool[n_pages - 8], held[1])
    assert c.refs[n_pages - 9:].tolist() == [1, 1] + [0] * 7
