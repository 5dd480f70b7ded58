"""GPU parity of the operators on a cache in 8 bits (include/gmgop.h) at the ends of their ranges: rows of attention
in which one key has most of the weight."""
import math

import pytest

torch = pytest.importorskip("torch")

import op8_ref as R8  # noqa: E402
import op_ref as R  # noqa: E402
from paper_2608_15762_gb300 import gmgop as P  # noqa: E402
from test_gpu_more_operators import _check_attend8, _kv8  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
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


def _codes(x):
    return x.clamp(-448, 448).to(F8).view(torch.uint8)


def _one_row(keys, values, ks, vs, page=64, tail=0):
    """A cache of one request: codes [tokens, heads, dim] under one scale for keys and one for values."""
    t, hk, dim = keys.shape
    n = -(-t // page)
    c = P.PageCache8(torch.zeros(n, P.page8_bytes(1, hk, page, dim), dtype=torch.uint8, device="cuda"), 1, hk, page, dim, 1, n)
    c.table.copy_(torch.randperm(n, generator=_gen(t), device="cuda").int()[None])
    c.scales[:, 0, 0], c.scales[:, 0, 1] = ks, vs
    for which, x in ((0, keys), (1, values)):
        whole = torch.zeros(n * page, hk, dim, dtype=torch.uint8, device="cuda")
        whole[:t] = x
        c.codes.view(torch.uint8)[c.table[0].long(), 0, which] = whole.view(n, page, hk, dim).transpose(1, 2)
    return c


def _exact(q, keys, values, ks, vs, n, scale, floor):
    """(o, bound) in 64 bits.  A score is off by d + 8 roundings of its magnitudes (two each), a weight by that of its own
    score and of the row's others, by 2^-11 of itself where it is rounded, and by `floor` of the row's largest; sums
    over t keys are off by t / 16 + 16 roundings."""
    t, hk, dim = keys.shape
    H = q.shape[1]
    k = (keys.view(F8).double() * ks).transpose(0, 1)
    v = (values.view(F8).double() * vs).transpose(0, 1)
    o, tol = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape, dtype=torch.float64, device="cuda")
    sees = torch.arange(t, device="cuda")[None] <= torch.arange(t - n, t, device="cuda")[:, None]
    for h in range(H):
        x, kh, vh = q[:, h].double(), k[h * hk // H], v[h * hk // H]
        z = (x @ kh.t() * scale).masked_fill(~sees, -math.inf)
        worst = (2 * (dim + 8) * R.U32 * scale * (x.abs() @ kh.t().abs())).masked_fill(~sees, 0).amax(-1, keepdim=True)
        p = torch.softmax(z, -1)
        o[:, h] = p @ vh
        rel = 2.0 ** -11 + 4 * worst + 2e-5 + 2 * (t / 16 + 16) * R.U32
        tol[:, h] = (rel * (p @ vh.abs()) + floor * p.amax(-1, keepdim=True) * vh.abs().sum(0) + R.U[q.dtype] * o[:, h].abs()
                     + R.TINY[q.dtype])
    return o, tol


# What a weight is off by where it is far below a row's largest, of which it is a share: half of the last code's least
# step, 2^-26, where the largest is at least 2^11; half of fp16's, 2^-25, where it is at least 2^8.
FLOOR = {1: 2.0 ** -37, 0: 2.0 ** -33}
# (keys, how far the first key's score is ahead, the others' deviation)
PEAKS = [(300, 17.0, 0.0), (8992, 14.0, 0.2), (16000, 15.0, 0.2), (32000, 16.0, 0.2), (131072, 12.0, 0.0), (131072, 16.0, 1.0),
         (131072, 17.0, 0.0), (131072, 20.0, 0.0)]


def _peaked(t, ahead, spread, H, hk, dim, n, dtype):
    """Heads whose first key is `ahead` of the others, with a value of a fiftieth of theirs, whose mean is 0.5: the
    result is what very many small weights give."""
    g = _gen(int(t + ahead))
    ks, vs, scale = 2.0 ** -5, 2.0 ** -6, dim ** -0.5
    sign = torch.randint(0, 2, (hk, dim), generator=g, device="cuda") * 2.0 - 1
    keys = torch.randn(t, hk, dim, generator=g, device="cuda") * spread
    keys[0] = sign * (ahead * dim ** -0.5)
    values = torch.randn(t, hk, dim, generator=g, device="cuda") + 0.5
    values[0] = 0.01
    by = 1 + 0.02 * torch.rand(n, H, 1, generator=g, device="cuda")
    q = (sign.repeat_interleave(H // hk, 0) * by).to(dtype)
    return q, _codes(keys / ks), _codes(values / vs), ks, vs, scale


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("t,ahead,spread", PEAKS)
@pytest.mark.parametrize("H,hk,dim", [(4, 1, 128), (16, 1, 64)])
def test_attend8_one_key_with_most_of_the_weight(t, ahead, spread, H, hk, dim, dtype, monkeypatch):
    q, keys, values, ks, vs, scale = _peaked(t, ahead, spread, H, hk, dim, 1, dtype)
    c = _one_row(keys, values, ks, vs)
    for sms in (1, 152):                                 # all its keys one item's; cut into many
        monkeypatch.setattr(P, "_n_sm", lambda device: sms)
        plan = P.AttendPlan8([1], [t], H, hk, dim, 64)
        assert plan.c.few == (t > 1000) and (sms > 1 or plan.c.n_items <= 2)
        want, tol = _exact(q, keys, values, ks, vs, 1, scale, FLOOR[plan.c.few])
        R.within(P.attend8(plan, q, c, 0, scale=scale), want, tol, "%d items" % plan.c.n_items)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("t,ahead,spread", PEAKS)
@pytest.mark.parametrize("H,hk,dim", [(4, 1, 128), (40, 1, 64)])
def test_attend8_one_key_with_most_of_the_weight_of_many_rows(t, ahead, spread, H, hk, dim, dtype, monkeypatch):
    n = 160 // H
    q, keys, values, ks, vs, scale = _peaked(t, ahead, spread, H, hk, dim, n, dtype)
    c = _one_row(keys, values, ks, vs)
    want, tol = _exact(q, keys, values, ks, vs, n, scale, FLOOR[0])
    for sms in (1, 152):
        monkeypatch.setattr(P, "_n_sm", lambda device: sms)
        plan = P.AttendPlan8([n], [t], H, hk, dim, 64)
        assert not plan.c.few
        R.within(P.attend8(plan, q, c, 0, scale=scale), want, tol, "%d items" % plan.c.n_items)


@pytest.mark.parametrize("dtype,size,scale", [(BF, 2.0 ** 30, 0.125), (BF, 2.0 ** 100, 0.125), (HF, 2.0 ** 20, 16.0)])
@pytest.mark.parametrize("B", [1, 4, 24])
def test_attend8_rows_of_very_different_size(B, dtype, size, scale):
    """A tile's rows may be several requests' and heads': what one of them holds is not lost for another's size."""
    g = _gen(41)
    H, hk, dim, pre = 8, 2, 64, 4000
    q = torch.randn(B, H, dim, generator=g, device="cuda") * (0.125 / scale)
    big = torch.zeros(B, H, dtype=torch.bool, device="cuda")
    big[1::4], big[::3, 1], big[2::4, 4:7] = True, True, True
    q = torch.where(big[..., None], (q * size).clamp(-6e4, 6e4) if dtype is HF else q * size, q).to(dtype)
    kv = [pre + 1 + 3 * b for b in range(B)]
    keys = _codes(torch.randn(max(kv), hk, dim, generator=g, device="cuda") * 80)
    values = _codes(torch.randn(max(kv), hk, dim, generator=g, device="cuda") * 80)
    c = _one_row(keys, values, 2.0 ** -6, 2.0 ** -6, page=16)
    c = P.PageCache8(c.pool, 1, hk, 16, dim, table=c.table.expand(B, -1).contiguous())
    plan = P.AttendPlan8([1] * B, kv, H, hk, dim, 16, group_off=[0, B], prefix=[pre])
    assert plan.c.few == (B < 24)
    got = P.attend8(plan, q, c, 0, scale=scale)
    for b in range(B):
        want, tol = _exact(q[b:b + 1], keys[:kv[b]], values[:kv[b]], 2.0 ** -6, 2.0 ** -6, 1, scale, FLOOR[plan.c.few])
        small = ~big[b:b + 1]
        R.within(got[b:b + 1][small], want[small], tol[small], "request %d" % b)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,H", [(1, 4), (1, 16), (4, 4), (40, 4), (13, 40)])
@pytest.mark.parametrize("t", [300, 7001, 65536])
def test_attend8_every_part_counts(n, H, t, dtype):
    """64 keys, anywhere, share the weight, and each has a dimension of its own: where one is lost, or a part of the keys is
    joined with another weight, that dimension shows it."""
    dim, ks, vs, scale = 128, 2.0 ** -4, 2.0 ** -6, 128 ** -0.5
    g = _gen(t + n)
    sign = torch.randint(0, 2, (1, dim), generator=g, device="cuda") * 2.0 - 1
    keys = torch.zeros(t, 1, dim, device="cuda")
    values = torch.randn(t, 1, dim, generator=g, device="cuda") * 0.01
    spots = torch.randperm(t - n, generator=g, device="cuda")[:64]
    keys[spots] = sign * (20 * dim ** -0.5)
    values[spots] = 0
    values[spots, 0, torch.arange(64, device="cuda") * 2] = 1 + torch.rand(64, generator=g, device="cuda")
    q = (sign[None] * (1 + 0.02 * torch.rand(n, H, 1, generator=g, device="cuda"))).to(dtype)
    keys, values = _codes(keys / ks), _codes(values / vs)
    plan = P.AttendPlan8([n], [t], H, 1, dim, 64)
    got = P.attend8(plan, q, _one_row(keys, values, ks, vs), 0, scale=scale)
    want, tol = _exact(q, keys, values, ks, vs, n, scale, FLOOR[plan.c.few])
    assert bool((want[..., ::2].abs() > 0.01).all()) and bool((tol[..., ::2] < 0.01 * want[..., ::2].abs()).all())
    R.within(got, want, tol)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("q_len,H,few", [([1], 8, 1), ([4], 8, 1), ([64], 8, 0)])
def test_attend8_long_as_a_whole(q_len, H, few, dtype):
    """The whole result's error, beside each element's bound: weights that are rounded to 2^-11 or less, independently, and one
    rounding to the result's type."""
    t = [50000 + q_len[0]]
    _, plan, q, o, _, held = _check_attend8(q_len, t, H, 2, 64, 32, dtype, seed=q_len[0])
    assert plan.c.few == few
    k, v, _ = _kv8(*held[0])
    G = H // 2
    want = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    hide = torch.arange(t[0], device="cuda")[None] > torch.arange(t[0] - q_len[0], t[0], device="cuda")[:, None]
    for h in range(H):
        z = (q[:, h].double() @ k[:, h // G].t() * 64 ** -0.5).masked_fill(hide, -math.inf)
        want[:, h] = torch.softmax(z, -1) @ v[:, h // G]
    assert float((o.double() - want).norm() / want.norm()) <= R.U[dtype] + 2.0 ** -10


@pytest.mark.parametrize("lo,hi", [(-60, -40), (-30, 4), (-12, 4)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attend8_scales_of_values_far_apart(lo, hi, dtype):
    """In both types, through tiles of few rows and of many."""
    def some(blocks):
        g = _gen(blocks + hi)
        s = torch.full((blocks, 2, 2), 2.0 ** -7, device="cuda")
        s[:, 1] = torch.exp2(torch.randint(lo, hi + 1, (blocks, 2), generator=g, device="cuda").float())
        return s
    kinds = [_check_attend8(q, kv, 8, 2, 64, 16, dtype, scales=some)[1].c.few
             for q, kv in (([1, 3], [4000, 3000]), ([1, 3, 140], [700, 300, 5000]))]
    assert kinds == [1, 0]


# ---------------------------------------------------------------------------
# Appending
# ---------------------------------------------------------------------------

def _near_middles(freq, dtype, seed, want=400):
    """Pairs (u, w), positions and pair numbers whose turn, in 64 bits, lies within one last bit of fp32 of the middle
    between two codes (of any scale that is a power of two), from below and from above: (u, w, pos, pair, which)."""
    g = _gen(seed)
    n = 1 << 24
    found = []
    for _ in range(40):
        u, w = (torch.randn(n, generator=g, device="cuda").to(dtype) for _ in range(2))
        pos = torch.randint(0, 200000, (n,), generator=g, device="cuda")
        pair = torch.randint(0, freq.numel(), (n,), generator=g, device="cuda")
        x, y = _turned(u.double(), w.double(), pos, freq[pair])
        for which, v in ((0, x), (1, y)):
            m, e = torch.frexp(v.abs())                        # v = m 2^e, m from 0.5 to 1: 4 bits are multiples of 1 / 16
            off = m * 16 - torch.floor(m * 16) - 0.5           # in steps of codes; a last bit is 2^-20 of one
            # (where pairs cancel, the error in 32 bits is more last bits than are looked at)
            ok = (off.abs() < 2.0 ** -20) & (off != 0) & (v.abs() > 0.7 * torch.maximum(u.abs(), w.abs())) & (v.abs() > 0.05)
            i = ok.nonzero()[:, 0]
            found.append(torch.stack((u[i].double(), w[i].double(), pos[i].double(), pair[i].double(),
                                      torch.full_like(u[i], which, dtype=torch.float64), torch.sign(off[i]))))
        if sum(f.shape[1] for f in found) >= want:
            break
    f = torch.cat(found, 1)[:, :want]
    assert f.shape[1] == want and min(int((f[5] < 0).sum()), int((f[5] > 0).sum())) > want // 4
    return f[0].to(dtype), f[1].to(dtype), f[2].int(), f[3].long()


def _turned(u, w, pos, freq):
    """In 64 bits, by angles that are whole 64-bit fractions of a turn."""
    a = (freq * pos.long()).double() * (math.pi * 2.0 ** -63)      # (the product wraps)
    return u * torch.cos(a) - w * torch.sin(a), u * torch.sin(a) + w * torch.cos(a)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D,rotary,inter", [(64, 64, False), (64, 64, True), (80, 32, False), (128, 64, True), (32, 8, True), (48, 6, False),
                                            (16, 10, True)])
@pytest.mark.parametrize("off", [0, 1])
def test_append8_keys_near_the_middle_of_two_codes(D, rotary, inter, off, dtype):
    """The code is the nearer one, wherever the keys lie in memory."""
    freqs, _ = P.rope_freqs(rotary, 10000.0 if rotary > 8 else 100.0)
    plan = P.Rope(rotary, freqs=freqs, interleaved=inter)
    u, w, pos, pair = _near_middles(plan.freq, dtype, D + rotary)
    # a token each, in blocks of their own
    T, half = u.numel(), rotary // 2
    order = torch.argsort(pos // 16, stable=True)
    keep = torch.cat((torch.ones(1, dtype=torch.bool, device="cuda"), (pos[order] // 16).diff() != 0))
    order = order[keep]
    u, w, pos, pair = u[order], w[order], pos[order], pair[order]
    T = order.numel()
    assert T > 300
    g = _gen(3)
    x = torch.randn(T, 1, D, generator=g, device="cuda").to(dtype)
    i, j = (2 * pair, 2 * pair + 1) if inter else (pair, pair + half)
    rows = torch.arange(T, device="cuda")
    x[rows, 0, i], x[rows, 0, j] = u, w
    cols = int(pos.max()) // 16 + 1
    cache = P.PageCache8(torch.zeros(T, P.page8_bytes(1, 1, 16, D), dtype=torch.uint8, device="cuda"), 1, 1, 16, D, 1, cols)
    cache.table[0, (pos // 16).long()] = torch.randperm(T, generator=g, device="cuda").int()
    buf = torch.zeros(T, D + 16, dtype=dtype, device="cuda")
    buf[:, off:off + D] = x[:, 0]
    k = buf[:, off:off + D].unflatten(1, (1, D))
    P.rope_append8(plan, x[:, :0], k, x, pos, torch.zeros_like(pos), cache, 0)
    page = cache.table[0, (pos // 16).long()].long()
    code = cache.codes[page, 0, 0, 0, (pos % 16).long()].double()
    scale = cache.scales[page, 0, 0, 0, 0].double()[:, None]
    want = x[:, 0].double().clone()
    p = torch.arange(half, device="cuda")
    a, b = (2 * p, 2 * p + 1) if inter else (p, p + half)
    want[:, a], want[:, b] = _turned(want[:, a], want[:, b], pos[:, None], plan.freq[None])
    assert bool((want.abs() <= 448 * scale).all()) and bool((want.abs().amax(1, keepdim=True) > 224 * scale).all())
    # of the pairs that were looked for both, of the others all but what lies within 32 bits' error of a middle
    near = torch.zeros_like(want, dtype=torch.bool)
    near[rows, i], near[rows, j] = True, True
    wrong = code != R8.rounded((want / scale).cpu()).cuda()
    assert not bool(wrong[near].any()), "%d of %d" % (int(wrong[near].sum()), int(near.sum()))
    assert float(wrong.double().mean()) < 1e-4


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D,rotary,inter", [(64, 64, False), (80, 32, True), (128, 128, False), (96, 16, False), (64, 8, True)])
def test_append8_codes_do_not_depend_on_where_tensors_lie(D, rotary, inter, dtype):
    g = _gen(D)
    T, H, hk, page = 6000, 2, 2, 32
    plan = P.Rope(rotary, freqs=P.rope_freqs(rotary)[0], interleaved=inter)
    pos, seq = torch.arange(37, 37 + T, device="cuda").int(), torch.zeros(T, dtype=torch.int32, device="cuda")
    row = torch.randn(T, (H + 2 * hk) * D, generator=g, device="cuda").to(dtype)
    row[::7, 3 * D:3 * D + 9] = -0.0
    start = torch.randint(0, 120, ((T + 37) // page + 1, P.page8_bytes(1, hk, page, D)), generator=g, device="cuda").to(torch.uint8)
    got = []
    for off in (0, 1, 3):
        buf = torch.zeros(T, row.shape[1] + 8, dtype=dtype, device="cuda")
        buf[:, off:off + row.shape[1]] = row
        at = buf[:, off:off + row.shape[1]]
        q, k, v = (at[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, H), (H, H + hk), (H + hk, H + 2 * hk)))
        pool = start.clone()
        cache = P.PageCache8(pool, 1, hk, page, D, 1, pool.shape[0], table=torch.arange(pool.shape[0], device="cuda").int()[None])
        cache.scales.fill_(2.0 ** -8)
        P.rope_append8(plan, q, k, v, pos, seq, cache, 0)
        got.append(pool)
    assert all(torch.equal(pool, got[0]) for pool in got[1:])
    # and each code stands for its value: rounded once, of keys that are off by the rotation's error in 32 bits
    exact = row[:, H * D:].double().unflatten(1, (2, hk, D)).clone()
    p = torch.arange(rotary // 2, device="cuda")
    i, j = (2 * p, 2 * p + 1) if inter else (p, p + rotary // 2)
    exact[:, 0][..., i], exact[:, 0][..., j] = _turned(exact[:, 0][..., i], exact[:, 0][..., j], pos[:, None, None], plan.freq)
    flat = lambda x: x[:, 0].permute(1, 2, 0, 3, *range(4, x.dim() - 1)).flatten(2, 3)  # noqa: E731
    codes, scales = flat(cache.codes)[:, :, :T + 37], flat(cache.scales)
    want = torch.zeros(2, hk, T + 37, D, dtype=torch.float64, device="cuda")
    want[:, :, 37:] = exact.permute(1, 2, 0, 3)
    scales = scales[:, :, :-(-(T + 37) // 16)]
    pad = scales.shape[2] * 16 - (T + 37)
    codes, want = torch.nn.functional.pad(codes.float(), (0, 0, 0, pad)), torch.nn.functional.pad(want, (0, 0, 0, pad))
    assert bool(R8.near(codes, scales, None, want, 2e-6)[:, :, 37:].all())


def _append_in_order(entries, n_seq=40, page=16):
    """(seq, pos) entries, in their order, into an empty cache: (cache, what was appended, seq, pos)."""
    g = _gen(len(entries))
    T, D = len(entries), 32
    cache = P.PageCache8(torch.zeros(n_seq * 4, P.page8_bytes(1, 1, page, D), dtype=torch.uint8, device="cuda"), 1, 1, page, D,
                         n_seq, 4, table=torch.arange(n_seq * 4, device="cuda").int().view(n_seq, 4))
    x = torch.randn(T, 1, D, generator=g, device="cuda").to(BF)
    seq, pos = (torch.tensor([e[i] for e in entries], dtype=torch.int32, device="cuda") for i in (0, 1))
    P.rope_append8(P.Rope(0), x, x, x, pos, seq, cache, 0)
    return cache, x, seq, pos


@pytest.mark.parametrize("lead", [0, 3, 15, 16, 700])
def test_append8_counts_tokens_out_of_order(lead):
    """Tokens that break the lists' order within 32 entries are seen, wherever thread blocks begin."""
    none = (-1, 0)
    before = [(1 + t // 64, t % 64) for t in range(lead)]
    unseen = [(0, 0)] + [none] * 31 + [(0, 1)] + [none] * 29 + [(0, 2)]             # two runs of a block, too far apart
    cases = [([(0, 0), (0, 1), (0, 2)], 0),
             ([(0, 0)] + [none] * 9 + [(0, 1)] + [none] * 20 + [(0, 2)], 0),        # 31 entries from the first to the last
             ([(0, 0)] + [none] * 9 + [(0, 1)] + [none] * 21 + [(0, 2)], 1),        # one too far
             ([(0, 0)] + [none] * 19 + [(0, 1)] + [none] * 19 + [(0, 2)] + [none] * 19 + [(0, 3)], 2),
             ([(0, 17)] + [none] * 24 + [(0, 1)] + [none] * 24 + [(0, 2)], 0),      # the one before is another block's
             ([(0, 0)] + [none] * 30 + [(0, 1)] + [none] * 30 + [(0, 2)], 1),
             (unseen, 0),
             ([(0, t) for t in range(40)], 0),
             ([(0, 5), (0, 4), (0, 3)], 2),                                         # backwards
             ([(0, 5), (0, 5)], 1),                                                 # the same token twice
             ([(0, 3), (0, 4), (0, 30), (0, 5), (0, 6), (0, 31)], 3),               # a block, another one, the first again
             ([(r, t) for t in range(8) for r in (0, 39)], 14),                     # two rows in turn
             ([(r, 16 * t + 2) for t in range(4) for r in (0, 39)], 0)]             # but blocks of their own
    for entries, count in cases:
        cache, x, seq, pos = _append_in_order(before + entries)
        assert cache.status.tolist()[4:7] == [0, 0, count], entries
        if count == 0 and entries is not unseen:
            on = seq >= 0
            at = cache.table[seq[on].long(), (pos[on] // 16).long()].long()
            for which in (0, 1):
                code = cache.codes[at, 0, which, 0, (pos[on] % 16).long()].double()
                s = cache.scales[at, 0, which, 0, 0].double()[:, None]
                assert torch.equal(code.cpu(), R8.rounded((x[on, 0].double() / s).cpu()))
