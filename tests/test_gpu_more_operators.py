"""GPU parity of the norms around a block and of the operators on a cache in 8 bits (include/gmgop.h) with
plain implementations in 64 bits (op8_ref.py)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import op8_ref as R8  # noqa: E402
import op_ref as R  # noqa: E402
from paper_2608_15762_gb300 import gmgop as P  # noqa: E402
from paper_2608_15762_gb300 import gmgsim as G  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
F8 = torch.float8_e4m3fn


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
# Norms
# ---------------------------------------------------------------------------

def _norm_case(g, m, n, dt, xt, kind, after, gate, bias, block=True):
    kw = dict(kind=kind, w=1 + _rand(g, n, dtype=dt, scale=0.2), bias=_rand(g, n, dtype=dt) if bias else None)
    if block:
        kw.update(y=_rand(g, m, n, dtype=dt) + 0.5, after=after, scale=0.375,
                  gate={None: None, "column": _rand(g, n, dtype=dt), "row": _rand(g, m, 1, dtype=dt),
                        "full": _rand(g, m, n, dtype=dt)}[gate])
        if after:
            kw.update(y_w=_rand(g, n, dtype=dt), y_bias=_rand(g, n, dtype=dt) if bias else None)
    return _rand(g, m, n, dtype=xt, scale=3.0) + 1, kw


def _check_norm(got, x, kw, what=""):
    (h, th), r = R8.norm(x, **kw)
    if r is None:
        R.within(got, h, th, what)
    else:
        R.within(got[0], h, th, what + " h")
        R.within(got[1], r[0], r[1], what + " r")


@pytest.mark.parametrize("dt,xt", [(BF, BF), (BF, FF), (HF, HF), (HF, FF), (FF, FF)])
@pytest.mark.parametrize("m,n", [(1, 1), (3, 7), (5, 8), (1, 256), (9, 257), (4, 264), (33, 1000), (6, 1024), (2, 1032),
                                 (7, 4096), (3, 5003), (2, 8192), (3, 8200), (1, 16384), (2, 16400), (2, 20001), (1, 32768)])
def test_norm_sizes(m, n, dt, xt):
    g = _gen(m + 3 * n)
    for kind, after, gate, bias in (("rms", False, None, False), ("layer", True, "column", True), ("rms", True, "row", False),
                                    ("layer", False, "full", True)):
        x, kw = _norm_case(g, m, n, dt, xt, kind, after, gate, bias)
        _check_norm(P.norm(x, **kw), x, kw, "%s %s" % (kind, gate))
        x, kw = _norm_case(g, m, n, dt, xt, kind, after, gate, bias, block=False)
        _check_norm(P.norm(x, **kw), x, kw, kind)


@pytest.mark.parametrize("dt,xt", [(BF, BF), (HF, FF), (FF, FF)])
@pytest.mark.parametrize("m,n", [(152, 4096), (153, 4096), (200, 264), (153, 2040), (304, 5003), (305, 5003), (310, 301), (160, 16384),
                                 (257, 129), (1027, 8)])
def test_norm_many_rows(m, n, dt, xt):
    g = _gen(m + 3 * n)
    for kind, after, gate, bias in (("rms", True, "column", False), ("layer", False, "row", True)):
        x, kw = _norm_case(g, m, n, dt, xt, kind, after, gate, bias)
        _check_norm(P.norm(x, **kw), x, kw, "%s %s" % (kind, gate))


def test_norm_without_weights_and_with_shifted_ones():
    g = _gen(2)
    x, y = _rand(g, 5, 640, dtype=FF), _rand(g, 5, 640)
    for kw in (dict(y=y), dict(y=y, after=True, eps=0.1), dict(y=y, w=_rand(g, 640), shift=1.0),
               dict(y=y, after=True, y_w=_rand(g, 640), shift=1.0, kind="layer", scale=-2.0)):
        _check_norm(P.norm(x, **kw), x, kw)
    r = P.norm(x, y=y, scale=0.5, only_x=True)
    _, (want, tol) = R8.norm(x, y=y, scale=0.5)
    R.within(r, want, tol)
    out = torch.empty(5, 640, dtype=BF, device="cuda")
    assert P.norm(x, out=out) is out
    (want, tol), _ = R8.norm(x, w=torch.ones(640, dtype=BF, device="cuda"))
    R.within(out, want, tol)


@pytest.mark.parametrize("off,ld", [(0, 72), (8, 88), (1, 80), (4, 77)])
@pytest.mark.parametrize("xt", [BF, FF])
def test_norm_strides_and_alignment(off, ld, xt):
    g = _gen(ld)
    m, n = 11, 64
    x, y = _rand(g, m, ld + 16, dtype=xt)[:, off:off + n], _rand(g, m, ld)[:, :n]
    gate = _rand(g, m, ld + 16)[:, off:off + n]
    kw = dict(y=y, w=_rand(g, n), gate=gate, after=True, y_w=_rand(g, n))
    out, x_out = torch.full((m, n + 5), 7.0, dtype=BF, device="cuda"), torch.full((m, n + 3), 7.0, dtype=xt, device="cuda")
    got = P.norm(x, out=out[:, 2:n + 2], x_out=x_out[:, 1:n + 1], **kw)
    _check_norm(got, x, kw)
    assert bool((out[:, :2] == 7).all()) and bool((out[:, n + 2:] == 7).all())
    assert bool((x_out[:, :1] == 7).all()) and bool((x_out[:, n + 1:] == 7).all())
    kw["gate"] = _rand(g, m, 5)[:, 3:4]
    _check_norm(P.norm(x, **kw), x, kw)


@pytest.mark.parametrize("dt,xt", [(BF, BF), (HF, FF), (FF, FF)])
@pytest.mark.parametrize("m,n", [(5, 100), (9, 300), (4, 3001), (3, 5003), (306, 5003), (2, 16384), (2, 20001), (2, 32753), (2, 32755), (2, 32768)])
def test_norm_rows_that_lie_alike_and_anyhow(m, n, dt, xt):
    g = _gen(n)
    x, kw = _norm_case(g, m, n, dt, xt, "layer", True, "full", True)
    want = P.norm(x, **kw)
    _check_norm(want, x, kw)

    def strided(t, more, off=0):                       # the same numbers in longer rows
        b = torch.full((m, n + more + off), 7.0, dtype=t.dtype, device="cuda")
        b[:, off:off + n] = t
        return b[:, off:off + n]
    for more, off in (((1,) * 5, 0), ((3, 11, 3, 3, 19), 0), ((1, 2, 3, 4, 5), 0), ((1,) * 5, 1)):
        a, b = dict(kw, y=strided(kw["y"], more[1], off), gate=strided(kw["gate"], more[2], off)), strided(x, more[0], off)
        h, r = strided(torch.zeros(m, n, dtype=dt, device="cuda"), more[3], off), strided(x, more[4], off)
        P.norm(b, out=h, x_out=r, **a)
        _check_norm((h, r), x, kw)
        for t, k in ((h, more[3]), (r, more[4])):      # nothing beside the rows is written
            whole = t.as_strided((m, n + k + off), t.stride(), t.storage_offset() - off)
            assert bool((whole[:, :off] == 7).all()) and bool((whole[:, off + n:] == 7).all())


@pytest.mark.parametrize("n", [96, 4096, 5003, 32768])
def test_norm_in_place(n):
    g = _gen(n)
    x, kw = _norm_case(g, 6, n, BF, BF, "layer", True, "full", True)
    was, block = x.clone(), kw["y"].clone()
    h, r = P.norm(x, x_out=x, **kw)
    assert r is x
    _check_norm((h, r), was, kw)
    x.copy_(was)
    h, r = P.norm(x, out=kw["y"], x_out=x, **kw)       # the block's result is no longer needed
    _check_norm((h, r), was, dict(kw, y=block))
    kw["y"] = block.clone()
    h, r = P.norm(was, x_out=kw["y"], **kw)
    _check_norm((h, r), was, dict(kw, y=block))
    y = was.clone()
    assert P.norm(y, kw["w"], out=y) is y
    _check_norm(y, was, dict(w=kw["w"]))


def test_norm_rows_do_not_touch_each_other():
    g = _gen(7)
    for n in (512, 3000):
        x, kw = _norm_case(g, 9, n, BF, BF, "rms", True, None, False)
        x[2, 5], kw["y"][4, 0], x[6, 1] = math.nan, math.inf, math.inf
        h, r = P.norm(x, **kw)
        good = [0, 1, 3, 5, 7, 8]
        kw2 = dict(kw, y=kw["y"][good])
        _check_norm((h[good], r[good]), x[good], kw2)
        assert bool(torch.isnan(h[2]).all()) and not bool(torch.isfinite(h[4]).any())
    x = torch.zeros(3, 640, dtype=BF, device="cuda")
    assert bool((P.norm(x, _rand(g, 640)) == 0).all())          # a row of zeros, by eps
    assert bool((P.norm(x + 5, _rand(g, 640), kind="layer") == 0).all())


def test_norm_empty_streams_and_graph():
    g = _gen(8)
    w = _rand(g, 64)
    assert P.norm(_rand(g, 0, 64), w).shape == (0, 64)
    assert P.norm(_rand(g, 3, 0), torch.empty(0, dtype=BF, device="cuda")).shape == (3, 0)
    x, kw = _norm_case(g, 20, 2048, BF, FF, "rms", True, "column", True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = P.norm(x, stream=st, **kw)
    st.synchronize()
    _check_norm(got, x, kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, r = P.norm(x, **kw)
    x.copy_(_rand(g, 20, 2048, dtype=FF))
    graph.replay()
    _check_norm((h, r), x, kw)
    assert all(torch.equal(a, b) for a, b in zip(P.norm(x, **kw), (h, r)))     # the same bits


def test_norm_beyond_2_31_elements():
    n, m = 32768, 65600
    x = torch.empty(m, n, dtype=BF, device="cuda")
    x.view(-1)[:] = 1.0
    x[-1] = torch.arange(n, device="cuda").to(BF)
    last = x[-3:].clone()
    P.norm(x, out=x)
    (want, tol), _ = R8.norm(last)
    R.within(x[-3:], want, tol)
    assert bool((x[0] == 1).all())
    del x


# ---------------------------------------------------------------------------
# Appending in 8 bits
# ---------------------------------------------------------------------------

def _cache8(g, n_pages, layers, hk, page, dim, n_seq, cols):
    """Pages in random order, with random codes and scales."""
    pool = torch.zeros(n_pages, P.page8_bytes(layers, hk, page, dim), dtype=torch.uint8, device="cuda")
    c = P.PageCache8(pool, layers, hk, page, dim, n_seq, cols)
    c.codes.view(torch.uint8).copy_((torch.randn(c.codes.shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(F8).view(torch.uint8))
    c.scales.copy_(torch.exp2(torch.randint(-9, -3, c.scales.shape, generator=g, device="cuda").float()))
    c.table.copy_(torch.randperm(n_pages, generator=g, device="cuda")[:n_seq * cols].int().view(n_seq, cols))
    return c


def _in_range(want, dtype):
    """A pair of numbers can be turned to 1.41 times the larger: what is beyond the type's range (by half a step: of
    3e38 turned to 4.2e38 in bf16, whose largest is 3.39e38) is an infinity there."""
    most = float(torch.finfo(dtype).max) * (1 + R.U[dtype] / 2)
    return torch.where(want.abs() >= most, torch.sign(want) * math.inf, want)


def _check_append(c, layer, T, H, pos, seq, plan, freqs, inter, dtype, g, factor=1.0, row=None, scale=1.0):
    Hk, D = c.n_kv_heads, c.head_dim
    row = _rand(g, T, (H + 2 * Hk) * D, dtype=dtype, scale=scale) if row is None else row
    q, k, v = (row[:, a:b].unflatten(1, (-1, D)) if b > a else row.new_zeros(T, 0, D)
               for a, b in ((0, H * D), (H * D, (H + Hk) * D), ((H + Hk) * D, (H + 2 * Hk) * D)))
    ref, before = R8.Blocks(c), c.pool.clone()
    first = c.codes.clone()
    out = P.rope_append8(plan, q, k, v, pos, seq, c, layer)
    want, tol = R.rope(q, pos, freqs, factor, inter)
    R.within(out, _in_range(want, dtype), tol)
    kw = _in_range(R.rope(k, pos, freqs, factor, inter)[0], FF)
    p, s = pos.tolist(), seq.tolist()
    old_scales = ref.scales.clone()
    touched = ref.append(kw, 0, layer, p, s)
    assert touched == ref.append(v.double().cpu(), 1, layer, p, s)
    got_codes, got_scales = c.codes.cpu().double(), c.scales.cpu().double()
    # scales: equal but where the largest key lies so near a power of two times 448 that its error decides
    same = got_scales == ref.scales
    assert bool(same[:, :, 1].all())
    assert float((~same).sum()) <= 2
    # what was not touched keeps its bytes
    mine = torch.zeros_like(old_scales, dtype=torch.bool)
    for page, block in touched:
        mine[page, layer, :, :, block] = True
    assert torch.equal(got_scales[~mine], old_scales[~mine])
    keep = ~mine.repeat_interleave(16, -1)
    assert torch.equal(got_codes[keep], first.cpu().double()[keep])
    after = c.codes.shape[1:].numel()
    scales_end = after + c.scales.shape[1:].numel() * 4
    assert torch.equal(c.pool[:, scales_end:], before[:, scales_end:])
    # values: exactly the reference's, kept ones too; keys within one step where their error moves the rounding
    assert torch.equal(got_codes[:, :, 1].nan_to_num(777), ref.codes[:, :, 1].nan_to_num(777))
    differ = (got_codes != ref.codes) & ~(got_codes.isnan() & ref.codes.isnan()) & same.repeat_interleave(16, -1)[..., None]
    assert float(differ.double().mean()) <= 1e-4
    # neighbours in e4m3 are at most 2^-3 of the larger, or 2^-9, apart
    a, b = got_codes[differ], ref.codes[differ]
    assert bool(((a - b).abs() <= torch.maximum(torch.maximum(a.abs(), b.abs()) * 2.0 ** -3, torch.tensor(2.0 ** -9).double())).all())
    return c, ref, out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,H,Hk,D,rot,page,inter", [(1, 4, 1, 64, 64, 16, False), (50, 8, 2, 80, 32, 16, True), (33, 0, 3, 128, 128, 32, False),
                                                     (200, 5, 5, 48, 16, 256, False), (77, 6, 2, 16, 6, 64, True), (40, 4, 4, 96, 96, 32, True),
                                                     (5000, 2, 1, 128, 64, 64, False), (64, 3, 1, 32, 0, 16, False), (29, 2, 2, 112, 50, 128, False)])
def test_append8(T, H, Hk, D, rot, page, inter, dtype):
    g = _gen(T + D)
    n_seq = 4
    per = -(-T // n_seq)
    cols = -(-(per + 37) // page) + 1
    c = _cache8(g, n_seq * cols + 3, 2, Hk, page, D, n_seq, cols)
    f = P.rope_freqs(rot, 500.0)[0] if rot else np.zeros(0)
    plan = P.Rope(rot, freqs=f, factor=1.25, interleaved=inter)
    seq = [t // per for t in range(T)]
    pos = [(0, 5, 16, 31)[s] + t % per for t, s in enumerate(seq)]      # from the start of a block and from inside
    dropped = 0
    if T > 20:
        seq[3], seq[7], pos[5], dropped = -1, n_seq, cols * page, 2       # padding, no such row, beyond the row's pages
        c.table[seq[T - 1], pos[T - 1] // page] = -1
        dropped += sum(s == seq[T - 1] and p // page == pos[T - 1] // page for s, p in zip(seq, pos))
    _check_append(c, 1, T, H, _ints(pos), _ints(seq), plan, f, inter, dtype, g, 1.25)
    assert c.status.tolist()[4] == dropped


@pytest.mark.parametrize("T,n_seq,H,Hk,D,rot,page,inter", [(608, 38, 5, 1, 128, 128, 16, False), (607, 3, 4, 2, 64, 64, 32, False),
                                                           (777, 2, 5, 3, 80, 32, 64, True), (1300, 100, 4, 1, 48, 16, 16, False),
                                                           (4000, 5, 17, 1, 64, 64, 16, False), (4900, 700, 9, 1, 96, 96, 16, False),
                                                           (4400, 3, 30, 1, 128, 128, 16, False)])
def test_append8_tokens_in_sixteens_and_queries_apart(T, n_seq, H, Hk, D, rot, page, inter):
    g = _gen(T + D)
    per = -(-T // n_seq)
    cols = -(-(per + 20) // page) + 1
    c = _cache8(g, n_seq * cols + 3, 1, Hk, page, D, n_seq, cols)
    f = P.rope_freqs(rot, 500.0)[0]
    seq = [t // per for t in range(T)]
    pos = [s % 19 + t % per for t, s in enumerate(seq)]
    for t in range(5, T, 40):
        seq[t] = -1
    _check_append(c, 0, T, H, _ints(pos), _ints(seq), P.Rope(rot, freqs=f, interleaved=inter), f, inter, BF, g)
    assert c.status.tolist()[4] == 0


def test_append8_one_token_at_a_time():
    """A block whose scale grows as tokens come, from the least that there is."""
    g = _gen(5)
    c = _cache8(g, 8, 1, 2, 32, 64, 2, 3)
    f = P.rope_freqs(64)[0]
    plan = P.Rope(64, freqs=f)
    sizes = [0.0, 1e-30, 1e-6, 0.01, 0.01, 3.0, 500.0, 1.0, 448.0, 449.0, 30000.0, 1.0, 1e5, 3e38, 2.0, 0.0, 1.0, 5.0, 0.0]
    for t, size in enumerate(sizes):
        x = _rand(g, 2, 6 * 64) * 0 + torch.sign(_rand(g, 2, 6 * 64)) * size
        _check_append(c, 0, 2, 2, _ints([t, 20 + t]), _ints([0, 1]), plan, f, False, BF, g, row=x.to(BF))


def test_append8_values_that_are_not_finite():
    g = _gen(6)
    c = _cache8(g, 8, 1, 1, 16, 32, 2, 3)
    plan = P.Rope(0)
    row = _rand(g, 7, 3 * 32)
    row[1, 40], row[2, 70], row[3, 66], row[4, 64 + 5] = math.nan, math.inf, -math.inf, math.nan
    _check_append(c, 0, 7, 1, _ints([3, 4, 5, 6, 7, 8, 9]), _ints([1] * 7), plan, np.zeros(0), False, BF, g, row=row)
    v = c.codes[int(c.table[1, 0]), 0, 1, 0].float()
    assert float(v[5, 6]) == 448 and float(v[6, 2]) == -448 and math.isnan(float(v[7, 5]))
    row[:, 32:] = math.nan                                         # nothing finite: the least scale
    P.rope_append8(plan, row[:, :32].unflatten(1, (1, 32)), row[:, 32:64].unflatten(1, (1, 32)), row[:, 64:].unflatten(1, (1, 32)),
                   _ints(range(7)), _ints([0] * 7), c, 0)
    assert float(c.scales[int(c.table[0, 0]), 0, 0, 0, 0]) == 2.0 ** -60


def test_append8_reads_any_scale():
    """Scales that are no powers of two, and some that are none at all, in blocks that are partly filled."""
    g = _gen(9)
    c = _cache8(g, 8, 1, 1, 16, 32, 6, 1)
    c.scales[c.table[:, 0].long(), 0, :, 0, 0] = torch.tensor([0.003, 0.0, -1.0, math.nan, math.inf, 1e-30], device="cuda")[:, None]
    ref = R8.Blocks(c)
    row = _rand(g, 6, 3 * 32)
    P.rope_append8(P.Rope(0), *(row[:, i * 32:(i + 1) * 32].unflatten(1, (1, 32)) for i in range(3)), _ints([9] * 6), _ints(range(6)), c, 0)
    for i, old in enumerate((0.003, 2.0 ** -60, 2.0 ** -60, 2.0 ** -60, 2.0 ** 60, 2.0 ** -60)):
        page = int(c.table[i, 0])
        for which in (0, 1):
            x = row[i, 32 + 32 * which:64 + 32 * which].double().cpu()
            old32 = float(torch.tensor(old, dtype=FF))
            s = max(old32, R8.need(float(x.abs().max())))
            assert float(c.scales[page, 0, which, 0, 0]) == s
            got = c.codes[page, 0, which, 0].cpu().double()
            by = float(torch.tensor(old32, dtype=FF) / torch.tensor(s, dtype=FF))
            if s > old32:
                assert torch.equal(got[:9], R8.rounded((ref.codes[page, 0, which, 0, :9].float() * by).double()))
            else:
                assert torch.equal(got[:9], ref.codes[page, 0, which, 0, :9])
            inv = torch.tensor(1.0, dtype=FF) / torch.tensor(s, dtype=FF)
            assert torch.equal(got[9], R8.rounded((x.float() * inv).double()))
            assert torch.equal(got[10:], ref.codes[page, 0, which, 0, 10:])


def test_append8_strides_streams_and_graph():
    g = _gen(10)
    f = P.rope_freqs(64)[0]
    plan = P.Rope(64, freqs=f)
    pos, seq = _ints(range(3, 43)), _ints([1] * 40)
    c = _cache8(g, 12, 1, 2, 16, 64, 2, 4)
    for off in (0, 1, 8):                                          # (unaligned: an element at a time)
        buf = _rand(g, 40, 8 * 64 + 9)
        _check_append(c, 0, 40, 4, pos, seq, plan, f, False, BF, g, row=buf[:, off:off + 8 * 64])
    x = _rand(g, 2, 40, 64).transpose(0, 1)                        # heads outside, queries in place
    start = c.pool.clone()
    plain = P.rope_append8(plan, x.contiguous(), x.contiguous(), x.contiguous(), pos, seq, c, 0)
    wrote = c.pool.clone()
    c.pool.copy_(start)
    q = x.clone()
    assert P.rope_append8(plan, q, x, x, pos, seq, c, 0, out=q) is q
    assert torch.equal(q, plain) and torch.equal(c.pool, wrote)
    st = torch.cuda.Stream()
    c.pool.copy_(start)
    st.wait_stream(torch.cuda.current_stream())
    got = P.rope_append8(plan, x, x, x, pos, seq, c, 0, stream=st)
    st.synchronize()
    assert torch.equal(got, plain) and torch.equal(c.pool, wrote)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.rope_append8(plan, x, x, x, pos, seq, c, 0)
    c.pool.copy_(start)
    for _ in range(2):                                             # again: the same tokens, the same bytes
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, plain) and torch.equal(c.pool, wrote)
    assert P.rope_append8(plan, x[:0], x[:0], x[:0], pos[:0], seq[:0], c, 0).shape == (0, 2, 64)


def test_append8_many_tokens_of_many_rows():
    """More tokens than one a block; rows that begin and end anywhere; the same as a few tokens at a time."""
    g = _gen(11)
    n_seq, page, Hk, D = 37, 32, 2, 64
    lens = [int(x) for x in torch.randint(1, 400, (n_seq,), generator=torch.Generator().manual_seed(3))]
    first = [int(x) for x in torch.randint(0, 60, (n_seq,), generator=torch.Generator().manual_seed(4))]
    cols = 500 // page + 1
    a = _cache8(g, n_seq * cols, 1, Hk, page, D, n_seq, cols)
    b = P.PageCache8(a.pool.clone(), 1, Hk, page, D, table=a.table.clone())
    plan = P.Rope(64, base=500.0)
    pos = [first[s] + i for s in range(n_seq) for i in range(lens[s])]
    seq = [s for s in range(n_seq) for _ in range(lens[s])]
    T = len(pos)
    assert T > 152 * 32
    x = [_rand(g, T, Hk, D) for _ in range(3)]
    whole = P.rope_append8(plan, *x, _ints(pos), _ints(seq), a, 0)
    parts, t = [], 0
    while t < T:      # cut where a block begins, or a row
        e = min(T, t + 900)
        while e < T and pos[e] % 16 and seq[e] == seq[e - 1]:
            e += 1
        parts.append(P.rope_append8(plan, *(y[t:e] for y in x), _ints(pos[t:e]), _ints(seq[t:e]), b, 0))
        t = e
    assert torch.equal(torch.cat(parts), whole) and torch.equal(a.pool, b.pool)


# ---------------------------------------------------------------------------
# Pages in 8 bits
# ---------------------------------------------------------------------------

def test_pages8_move_codes_and_scales():
    g = _gen(12)
    c = _cache8(g, 50, 3, 2, 16, 80, 6, 8)
    c.table.fill_(-1)
    c.grow(_ints([0]), _ints([21]))
    c.fork(_ints([0, 0, 0]), _ints([1, 2, 3]), _ints([21, 18, 16]))
    old = c.pool.clone()
    c.grow(_ints([1, 2, 3]), _ints([1, 3, 1]))
    t = c.table.tolist()
    assert c.code()[0] == P.PAGE_OK
    for r in (1, 2):
        assert t[r][1] != t[0][1] and torch.equal(c.pool[t[r][1]], old[t[0][1]])
    c.free(_ints([0]))
    rows = {r: [c.pool[p].clone() for p in c.table[r].tolist() if p >= 0] for r in (1, 2, 3)}
    c.compact()
    assert c.code()[0] == P.PAGE_OK
    for r, pages in rows.items():
        now = [p for p in c.table[r].tolist() if p >= 0]
        assert all(p < int(c.status[3]) for p in now) and all(torch.equal(c.pool[p], was) for p, was in zip(now, pages))


# ---------------------------------------------------------------------------
# Attention over a cache in 8 bits
# ---------------------------------------------------------------------------

def _filled8(g, kv, hk, dim, page, shared=(), layers=2, spare=3, scales=None):
    """A cache in 8 bits whose rows hold kv tokens, pages in random order; rows of a shared entry (first, last, tokens)
    hold the same first tokens, in the same full pages.  Slots that hold no token, and pages that no row lists, are
    NaN, and so are their scales.  (cache, and for each row codes and scales [tokens, 2, heads, ...])"""
    B, cols = len(kv), max(1, max(-(-n // page) for n in kv) if kv else 1)
    total = sum(-(-n // page) for n in kv) + spare
    c = P.PageCache8(torch.full((total, P.page8_bytes(layers, hk, page, dim)), 0x7f, dtype=torch.uint8, device="cuda"),
                     layers, hk, page, dim, B, cols)
    c.scales.fill_(math.nan)
    ids = torch.randperm(total, generator=g, device="cuda").tolist()
    table = torch.full((B, cols), -1, dtype=torch.int32)
    held, lead = [], {}
    for first, last, tokens in shared:
        for b in range(first + 1, last):
            lead[b] = (first, tokens)
    for b, n in enumerate(kv):
        blocks = -(-n // 16)
        codes = (torch.randn(n, 2, hk, dim, generator=g, device="cuda") * 100).clamp(-448, 448).to(F8).view(torch.uint8)
        sc = torch.exp2(torch.randint(-8, -5, (blocks, 2, hk), generator=g, device="cuda").float()) if scales is None else scales(blocks)
        skip = 0
        if b in lead:
            a, tokens = lead[b]
            codes[:tokens] = held[a][0][:tokens]
            sc[:-(-tokens // 16)] = held[a][1][:-(-tokens // 16)]
            skip = tokens // page
            table[b, :skip] = table[a, :skip]
        for j in range(skip, -(-n // page)):
            p = table[b, j] = ids.pop()
            part = slice(j * page, min(n, (j + 1) * page))
            c.codes.view(torch.uint8)[int(p), 1, :, :, :part.stop - part.start] = codes[part].permute(1, 2, 0, 3)
            m = -(-(part.stop - part.start) // 16)
            c.scales[int(p), 1, :, :, :m] = sc[j * page // 16:j * page // 16 + m].permute(1, 2, 0)
        held.append((codes, sc))
    c.table.copy_(table)
    return c, held


def _kv8(codes, sc):
    """(keys, values, the values' scales) of a row, in 64 bits."""
    s = sc.double().clamp(2.0 ** -60, 2.0 ** 60).repeat_interleave(16, 0)[:codes.shape[0]]
    v = codes.view(F8).double() * s[..., None]
    return v[:, 0], v[:, 1], s[:, 1]


def _check_attend8(q_len, kv, H, Hk, D, page, dtype=BF, groups=None, prefix=None, seed=0, scale=None, q=None, scales=None):
    g = _gen(seed + sum(kv) + D)
    shared = [] if groups is None else [(groups[i], groups[i + 1], prefix[i]) for i in range(len(prefix))]
    cache, held = _filled8(g, kv, Hk, D, page, shared, scales=scales)
    q = _rand(g, sum(q_len), H, D, dtype=dtype) if q is None else q
    scale = D ** -0.5 if scale is None else scale
    plan = P.AttendPlan8(q_len, kv, H, Hk, D, page, group_off=groups, prefix=prefix)
    o, lse = P.attend8(plan, q, cache, 1, scale=scale, lse=True)
    assert cache.status.tolist()[5] == 0
    at = 0
    for b, n in enumerate(q_len):
        if n:
            wo, to, wl, tl = R8.attend(q[at:at + n], *_kv8(*held[b]), n, scale)
            R.within(o[at:at + n], wo, to, "request %d" % b)
            R.within(lse[at:at + n], wl, tl, "lse of request %d" % b)
        at += n
    return cache, plan, q, o, lse, held


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,Hk,D,page", [(8, 2, 128, 16), (4, 4, 64, 64), (6, 2, 80, 16), (7, 1, 16, 256), (40, 8, 128, 32),
                                         (64, 1, 64, 128), (33, 1, 112, 32), (3, 3, 48, 16)])
def test_attend8_lengths(H, Hk, D, page, dtype):
    kv = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1000]
    _check_attend8([1] * len(kv), kv, H, Hk, D, page, dtype)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,Hk,D,page", [(128, 1, 64, 16), (128, 1, 128, 64), (16, 1, 128, 256), (17, 1, 80, 16), (32, 2, 64, 16), (1, 1, 16, 16)])
def test_attend8_the_largest_and_the_smallest_groups(H, Hk, D, page, dtype):
    _check_attend8([1, 2, 1], [1, 4097, 700], H, Hk, D, page, dtype)


def test_attend8_two_streams_at_once():
    first = _check_attend8([1, 2], [20000, 9000], 8, 2, 128, 16)
    second = _check_attend8([1] * 5, [3000, 7000, 1, 900, 12000], 8, 1, 64, 32, seed=1)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(6):
        for one, other in ((first, second), (second, first)):        # each plan on both streams
            for case, s in zip((one, other), streams):
                cache, plan, q, o, lse, _ = case
                got.append((P.attend8(plan, q, cache, 1, lse=True, stream=s), (o, lse)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for pair, want in got for a, b in zip(pair, want))


def test_attend8_rows_that_see_nothing():
    _, _, _, o, lse, _ = _check_attend8([3, 1, 0, 5, 2], [0, 0, 7, 3, 2], 8, 2, 64, 16)
    assert bool((o[:4] == 0).all()) and bool(torch.isinf(lse[:4]).all()) and bool((o[4:6] == 0).all())
    plan = P.AttendPlan8([0, 0], [0, 5], 8, 2, 64, 16)
    cache, _ = _filled8(_gen(0), [5, 5], 2, 64, 16)
    assert P.attend8(plan, _rand(_gen(1), 0, 8, 64), cache, 1).shape == (0, 8, 64)


@pytest.mark.parametrize("H,Hk,D,page,dtype", [(8, 2, 128, 16, BF), (5, 1, 64, 32, HF), (12, 12, 80, 64, BF), (40, 1, 96, 16, HF)])
def test_attend8_many_queries(H, Hk, D, page, dtype):
    _check_attend8([1, 7, 64, 130, 200, 33], [400, 7, 300, 130, 777, 64], H, Hk, D, page, dtype)


@pytest.mark.parametrize("H,Hk,D,page,dtype", [(8, 2, 128, 16, BF), (16, 2, 64, 32, HF), (5, 5, 80, 16, BF)])
@pytest.mark.parametrize("pre", [1, 129, 1000, 4100])
def test_attend8_shared_prefix(H, Hk, D, page, dtype, pre):
    n = 24
    q = [1 + b % 3 for b in range(n)]
    kv = [pre + q[b] + (b * 7) % 90 for b in range(n)]
    _check_attend8(q, kv, H, Hk, D, page, dtype, [0, n], [pre])


def test_attend8_groups_of_every_kind():
    q = [1, 1, 5, 0, 2, 1, 1, 1, 9, 1, 1, 1]
    pre = [0, 2000, 64, 700]
    groups = [0, 2, 6, 6, 12]
    kv = [30 + 40 * b for b in range(2)] + [2000 + x + (3 * b) for b, x in enumerate(q[2:6])] + [
        700 + x + 17 * b for b, x in enumerate(q[6:])]
    _check_attend8(q, kv, 8, 2, 64, 16, BF, groups, pre)


@pytest.mark.parametrize("q_len,kv_len,D", [(1, 65536, 128), (4, 40001, 64), (3, 20000, 80)])
def test_attend8_long(q_len, kv_len, D):
    _check_attend8([q_len], [kv_len], 8, 2, D, 64)


def test_attend8_large_scores_and_scales():
    for i, scale in enumerate((4.0, -0.5, 0.0, 1e-6, 30.0)):
        for dtype in (BF, HF):
            _check_attend8([5, 1], [300, 900], 8, 2, 64, 16, dtype, seed=i, scale=scale)
    g = _gen(3)
    for size in (2.0 ** -30, 2.0 ** 20, 2.0 ** 60):               # queries beyond fp16's range: the tile's largest decides
        q = (torch.randn(6, 8, 64, generator=g, device="cuda") * size).to(BF)
        _check_attend8([5, 1], [300, 900], 8, 2, 64, 16, BF, scale=0.125 / size, q=q)


def test_attend8_scales_far_apart():
    """Blocks whose values' scales differ by up to 2^110; a key's weight must not be lost for its value's size."""
    for lo, hi in ((-60, 60), (-12, 12), (-60, -40)):
        def some(blocks):
            g = _gen(blocks + hi)
            s = torch.full((blocks, 2, 2), 2.0 ** -7, device="cuda")
            s[:, 1] = torch.exp2(torch.randint(lo, hi + 1, (blocks, 2), generator=g, device="cuda").float())
            return s
        _check_attend8([1, 3, 40], [700, 300, 500], 8, 2, 64, 16, BF if hi < 10 else torch.bfloat16, scales=some)


def test_attend8_scales_that_are_no_powers_of_two():
    def some(blocks):
        return torch.rand(blocks, 2, 2, generator=_gen(blocks), device="cuda") * 0.02 + 1e-4
    _check_attend8([1, 3, 70], [700, 300, 500], 8, 2, 128, 32, scales=some)


def test_attend8_scales_out_of_range():
    """As the nearer bound, NaN as the lower: the values of such blocks are next to nothing."""
    odd = torch.tensor([0.0, -1.0, 1e-30, math.nan, 0.01, 0.01], device="cuda")
    g = _gen(5)
    cache, held = _filled8(g, [90], 1, 64, 16, scales=lambda n: odd[:n, None, None].expand(n, 2, 1).clone())
    q = _rand(g, 1, 4, 64)
    o, lse = P.attend8(P.AttendPlan8([1], [90], 4, 1, 64, 16), q, cache, 1, lse=True)
    codes, sc = held[0]
    wo, to, wl, tl = R8.attend(q, *_kv8(codes, sc.nan_to_num(0.0)), 1, 0.125)
    R.within(o, wo, to)
    R.within(lse, wl, tl)


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, HF)])
def test_attend8_values_that_are_not_finite_stay_with_those_that_see_them(D, dtype):
    g = _gen(21)
    n, t, H, Hk, page = 200, 700, 4, 2, 16
    cache, held = _filled8(g, [t, t], Hk, D, page)
    codes, sc = held[0]
    spots = [(t - 1, 0, 3), (t - 50, 1, 0), (t - 128, 0, 5), (t - 129, 1, 7), (t - 199, 0, 9)]     # values: (token, head, dim)
    for at, h, d in spots:
        cache.codes.view(torch.uint8)[int(cache.table[0, at // page]), 1, 1, h, at % page, d] = 0xff
        codes[at, 1, h, d] = 0xff
    k_spot = t - 77                                                                                # a key
    cache.codes.view(torch.uint8)[int(cache.table[0, k_spot // page]), 1, 0, 1, k_spot % page, 2] = 0x7f
    q = _rand(g, n + 1, H, D, dtype=dtype)
    q[5, 1, 0], q[6, 0, 1] = math.nan, math.inf
    plan = P.AttendPlan8([n, 1], [t, t], H, Hk, D, page)
    o, lse = P.attend8(plan, q, cache, 1, lse=True)
    k, v, vs = _kv8(codes, sc)
    clean = torch.where(v.isnan(), 0.0, v)
    wo, to, wl, tl = R8.attend(q[:n], k, clean, vs, n, D ** -0.5)
    bad = torch.zeros(n, H, D, dtype=torch.bool, device="cuda")
    row = torch.zeros(n, H, dtype=torch.bool, device="cuda")
    for at, h, d in spots:
        bad[max(0, at - (t - n)):, 2 * h:2 * h + 2, d] = True
    row[k_spot - (t - n):, 2:] = True
    row[5, 1] = row[6, 0] = True
    got = o[:n].clone()
    assert bool(torch.isnan(got[bad]).all()) and not bool(torch.isfinite(got[row]).any())
    fine = ~(bad | row[..., None])
    assert bool(torch.isfinite(got[fine]).all())
    R.within(torch.where(fine, got, 0), torch.where(fine, wo, 0), to)
    R.within(torch.where(row, 0, lse[:n]), torch.where(row, 0, wl), tl)
    assert not bool(torch.isfinite(lse[:n][row]).any())
    wo, to, _, _ = R8.attend(q[n:], *_kv8(*held[1]), 1, D ** -0.5)                                 # the other request
    R.within(o[n:], wo, to)


def test_attend8_missing_pages_read_as_zeros():
    g = _gen(23)
    kv, page = [300, 70], 32
    cache, held = _filled8(g, kv, 2, 64, page)
    cache.table[0, 3], cache.table[1, 0] = -1, cache.pool.shape[0] + 5
    held[0][0][96:128], held[1][0][:32] = 0, 0
    held[0][1][6:8], held[1][1][:2] = 1.0, 1.0
    q = _rand(g, 3, 8, 64)
    o, lse = P.attend8(P.AttendPlan8([1, 2], kv, 8, 2, 64, page), q, cache, 1, lse=True)
    for a, b, i in ((0, 1, 0), (1, 3, 1)):
        wo, to, wl, tl = R8.attend(q[a:b], *_kv8(*held[i]), b - a, 0.125)
        R.within(o[a:b], wo, to)
        R.within(lse[a:b], wl, tl)


def test_attend8_strides_streams_and_graphs():
    g = _gen(24)
    kv, q_len = [900, 40, 3000], [1, 3, 2]
    cache, plan, q, o, lse, _ = _check_attend8(q_len, kv, 8, 2, 64, 16)
    wide = torch.zeros(6, 3 * 8, 80, dtype=BF, device="cuda")
    wide[:, 8:16, 8:72] = q
    out = torch.full((6, 8, 72), 7.0, dtype=BF, device="cuda")
    P.attend8(plan, wide[:, 8:16, 8:72], cache, 1, out=out[..., :64])
    assert torch.equal(out[..., :64], o) and bool((out[..., 64:] == 7).all())
    outside = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(P.attend8(plan, outside, cache, 1), o)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got, z = P.attend8(plan, q, cache, 1, lse=True, stream=st)
    st.synchronize()
    assert torch.equal(got, o) and torch.equal(z, lse)
    graphs, outs = [], []
    for _ in range(2):                                             # each with a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(P.attend8(plan, q, cache, 1))
        graphs.append(graph)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, o) for x in outs)
    for _ in range(3):
        assert torch.equal(P.attend8(plan, q, cache, 1), o)        # the same bits


def test_cache8_beyond_2_31_bytes():
    g = _gen(25)
    page, Hk, D, layers = 64, 8, 128, 4
    nbytes = P.page8_bytes(layers, Hk, page, D)
    n = 2 ** 32 // nbytes + 40
    pool = torch.zeros(n, nbytes, dtype=torch.uint8, device="cuda")
    c = P.PageCache8(pool, layers, Hk, page, D, 2, 8)
    c.table.copy_(torch.arange(n - 16, n, device="cuda").int().flip(0).view(2, 8))
    f = P.rope_freqs(D)[0]
    plan = P.Rope(D, freqs=f)
    T = 300
    x = [_rand(g, T, h, D) for h in (16, Hk, Hk)]
    pos, seq = _ints(range(T)), _ints([1] * T)
    q = P.rope_append8(plan, *x, pos, seq, c, 3)
    o, lse = P.attend8(P.AttendPlan8([T], [T], 16, Hk, D, page, seq=[1]), q, c, 3, lse=True)
    at = c.table[1, :-(-T // page)].long()
    codes = c.codes.view(torch.uint8)[at, 3].permute(0, 3, 1, 2, 4).reshape(-1, 2, Hk, D)[:T]
    sc = c.scales[at, 3].permute(0, 3, 1, 2).reshape(-1, 2, Hk)[:-(-T // 16)]
    k, v, vs = _kv8(codes, sc)
    assert float((v - x[2].double()).abs().max()) <= float(x[2].abs().max()) * 2.0 ** -4
    wo, to, wl, tl = R8.attend(q, k, v, vs, T, D ** -0.5)
    R.within(o, wo, to)
    R.within(lse, wl, tl)
    assert not bool(pool[:n - 16].any()) if n < 3000 else not bool(pool[::97][:-1].any())


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

def test_a_layer_on_a_cache_in_8_bits():
    """Steps of requests that fork: norm, qkv, rotation into the cache, attention, projection with its norm and residual.
    Each operator against 64 bits on its own inputs, the cache against what was appended."""
    g = _gen(31)
    H, Hk, D, page, hidden = 8, 2, 64, 16, 512
    cache = P.PageCache8(torch.zeros(200, P.page8_bytes(2, Hk, page, D), dtype=torch.uint8, device="cuda"), 2, Hk, page, D, 6, 30)
    freqs = P.rope_freqs(D)[0]
    rope = P.Rope(D, freqs=freqs)
    w = dict(qkv=_rand(g, (H + 2 * Hk) * D, hidden, scale=hidden ** -0.5), o=_rand(g, hidden, H * D, scale=(H * D) ** -0.5),
             n1=_rand(g, hidden) + 1, n2=_rand(g, hidden) + 1, n3=_rand(g, hidden) + 1)
    kept = {}                                                       # (row, layer) -> keys, values as appended

    def step(rows, n, lens, groups=None, prefix=None):
        cache.grow(_ints(rows), _ints([n] * len(rows)))
        T = len(rows) * n
        pos, seq = _ints(l + i for l in lens for i in range(n)), _ints(r for r in rows for _ in range(n))
        plan = P.AttendPlan8([n] * len(rows), [l + n for l in lens], H, Hk, D, page, seq=rows, group_off=groups, prefix=prefix)
        x = _rand(g, T, hidden, dtype=FF)
        h = P.norm(x, w["n1"])
        for layer in (0, 1):
            kw = dict(w=w["n1"])
            if layer == 0:
                _check_norm(h, x, kw)
            row = P.linear(h, w["qkv"])
            q, k, v = (t.unflatten(1, (-1, D)) for t in row.split([H * D, Hk * D, Hk * D], 1))
            turned, _ = R.rope(k, pos, freqs)
            q = P.rope_append8(rope, q, k, v, pos, seq, cache, layer)
            for i, r in enumerate(rows):
                a, b = kept.get((r, layer), (torch.zeros(0, Hk, D).double(),) * 2)
                part = slice(i * n, (i + 1) * n)
                kept[r, layer] = torch.cat((a, turned[part])), torch.cat((b, v[part].double().cpu()))
            o = P.attend8(plan, q, cache, layer)
            for i, r in enumerate(rows):
                t = lens[i] + n
                at = cache.table[r, :-(-t // page)].long()
                codes = cache.codes.view(torch.uint8)[at, layer].permute(0, 3, 1, 2, 4).reshape(-1, 2, Hk, D)[:t]
                sc = cache.scales[at, layer].permute(0, 3, 1, 2).reshape(-1, 2, Hk)[:-(-t // 16)]
                kk, vv, vs = _kv8(codes, sc)
                wo, to, _, _ = R8.attend(q[i * n:(i + 1) * n], kk, vv, vs, n, D ** -0.5)
                R.within(o[i * n:(i + 1) * n], wo, to)
                for got, want, s in ((kk, kept[r, layer][0], sc[:, 0]), (vv, kept[r, layer][1], sc[:, 1])):
                    # rounded once, again where the block's scale has grown (then to multiples of 2^-9 of it: up to 15 times,
                    # each to half a step), of values that were off by the rotation's 1e-6
                    s = s.double().repeat_interleave(16, 0)[:t, :, None].cpu()
                    assert bool(((got.cpu() - want).abs() <= want.abs() * (2.0 ** -4 + 1e-6) + 16 * s * 2.0 ** -10 + 1e-6).all())
            y = P.linear(o.flatten(1), w["o"])
            kw = dict(y=y, w=w["n2"], after=True, y_w=w["n3"], scale=0.5)
            was = x.clone()
            h, x = P.norm(x, x_out=x, **kw)
            _check_norm((h, x), was, kw)

    step([0], 203, [0])
    cache.fork(_ints([0] * 4), _ints([1, 2, 3, 4]), _ints([203, 203, 150, 16]))
    for layer in (0, 1):
        for r, t in ((1, 203), (2, 203), (3, 150), (4, 16)):
            kept[r, layer] = tuple(a[:t] for a in kept[0, layer])
    step([1, 2], 1, [203, 203], [0, 2], [203])
    step([3, 4, 0], 5, [150, 16, 203])
    step([1, 2, 3, 4], 2, [204, 204, 155, 21])
    cache.free(_ints([0, 3]))
    cache.compact()
    step([4, 1], 40, [23, 206])
    assert cache.code()[0] == P.PAGE_OK and cache.status.tolist()[4:6] == [0, 0]


def test_executor_example_in_8_bits():
    """The example's layers on a cache in 8 bits: it runs, its operators are timed, a graph is placed on their times."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "executor_feedback.py")
    spec = importlib.util.spec_from_file_location("executor_feedback_8", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    out = m.main(layers=2, hidden=256, heads=4, kv_heads=1, ffn=512, requests=8, prompt=200, steps=3, n_dev=4, candidates=64,
                 say=lambda *_: None, bits=8)
    ex = out["executor"]
    assert ex.cache.status.tolist()[4:6] == [0, 0] and all(len(v) > 0 for v in ex.samples.values())
    assert out["makespan"] > 0 and bool((ex.cache.scales >= 0).all())
