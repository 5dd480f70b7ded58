"""Plain implementations of the decoder-layer operators in 64 bits, for their tests, and
the bounds on a kernel's error that follow from the types it rounds to."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # unit roundoff
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
U32 = 2.0 ** -24


def within(got, want, tol, what=""):
    """got within tol of want, element by element; equal where want is not finite."""
    got, want = got.double().cpu(), want.cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what + ": infinities differ"
    d = (got - want).abs()[fine]
    t = tol.cpu().expand(want.shape)[fine]
    bad = d > t
    assert not bool(bad.any()), "%s: %d of %d outside, worst %.3g times the bound" % (
        what, int(bad.sum()), bad.numel(), float((d / t.clamp(min=1e-300)).max()))


def bent(v, act):
    if act == "relu":
        return torch.where(v < 0, torch.zeros_like(v), v)
    if act == "silu":
        return v * torch.special.expit(v)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))
    return v


def linear(x, w, bias=None, act="none", gate=None, gate_bias=None, residual=None):
    """(result, bound): sums of k products held in 32 bits are off by at most k + 8
    roundings of the sum of magnitudes (two for each, as a tensor core may cut off
    instead of rounding); an activation's slope is at most 1.13 and it is computed to
    within 4 roundings and 1e-6 of its argument; then one rounding to the output's type."""
    u = U[x.dtype]
    x64 = x.double()

    def product(w, b):
        y, mag = x64 @ w.double().t(), x64.abs() @ w.double().abs().t()
        if b is not None:
            y, mag = y + b.double(), mag + b.double().abs()
        return y, 2 * (x.shape[1] + 8) * U32 * mag

    v, e = product(w, bias)
    if gate is not None:
        g, eg = product(gate, gate_bias)
        a = bent(g, act)
        ea = 1.13 * eg + 2e-6 * g.abs()
        v, e = a * v, ea * (v.abs() + e) + a.abs() * e
    else:
        v, e = bent(v, act), 1.13 * e + 2e-6 * v.abs() * (act != "none")
    if residual is not None:
        v = v + residual.double()
        e = e + U32 * v.abs()
    return v, e * (1 + u) + (u + 2 * U32) * v.abs() + TINY[x.dtype]


def rope(x, pos, freqs, factor=1.0, interleaved=False, backward=False):
    """(result, bound): the angle is off by at most pi 2^-25 + pos 2^-62, sine and cosine by
    2 roundings more, three roundings in the products, then one to the output's type."""
    half = freqs.shape[0]
    R = 2 * half
    a = pos.double().cpu()[:, None, None] * torch.from_numpy(np.asarray(freqs))
    c, s = torch.cos(a) * factor, torch.sin(a) * factor * (-1 if backward else 1)
    y = x.double().cpu().clone()
    mag = y.abs().clone()
    one, two = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, half), slice(half, R))
    u, v = y[..., one].clone(), y[..., two].clone()
    y[..., one], y[..., two] = u * c - v * s, u * s + v * c
    mag[..., one] = mag[..., two] = (u.abs() + v.abs()) * factor
    # 64-bit sines of large angles are themselves off by the rounding of the angle
    err = (math.pi * 2 ** -25 + 8 * U32) * mag + float(pos.abs().max() if pos.numel() else 0) * 7 * 2 ** -53 * mag
    err[..., R:] = 0
    return y, err + U[x.dtype] * y.abs() * (torch.arange(y.shape[-1]) < R) + TINY[x.dtype]


def attend(q, keys, values, n_q, scale):
    """One request: q [n, heads, dim], keys and values [tokens, kv_heads, dim].  (o, bound, lse,
    bound): a score is off by d + 8 roundings of its magnitudes (two each), which moves a
    probability by that much; probabilities are rounded once to the values' type."""
    n, H, D = q.shape
    t, Hk = keys.shape[0], keys.shape[1]
    G = H // Hk
    k, v = (a.double().repeat_interleave(G, 1).transpose(0, 1) for a in (keys, values))   # [H, t, D]
    x = q.double().transpose(0, 1)
    sees = torch.arange(t, device=q.device)[None] <= torch.arange(t - n, t, device=q.device)[:, None]
    z = (x @ k.transpose(1, 2) * scale).masked_fill(~sees, -math.inf)
    ds = (2 * (D + 8) * U32 * abs(scale) * (x.abs() @ k.abs().transpose(1, 2))).masked_fill(~sees, 0)
    none = ~sees.any(1)
    lse = torch.logsumexp(z, -1) if t else torch.full((H, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(z - lse[..., None]).masked_fill(~sees, 0)
    p[:, none] = 0
    o, mag = p @ v, p @ v.abs()
    worst = ds.amax(-1) if t else torch.zeros_like(lse)
    rel = 4 * worst + 1e-5
    u = U[q.dtype]
    tol = (u + rel)[..., None] * mag + u * o.abs() + TINY[q.dtype]
    ltol = worst + 1e-5 + 4 * U32 * lse.abs().masked_fill(lse.isinf(), 0)
    return o.transpose(0, 1), tol.transpose(0, 1), lse.transpose(0, 1), ltol.transpose(0, 1)


class Pages:
    """The page calls, one step after another, on lists and a dict of page contents."""

    def __init__(self, n_pages, page, n_seq, max_pages):
        self.page, self.max_pages = page, max_pages
        self.rows, self.lens, self.refs = [[] for _ in range(n_seq)], [0] * n_seq, [0] * n_pages
        self.data = list(range(n_pages))      # what each page holds, as a label
        self.code = 0

    def _bad(self, *lists):
        for rows in lists:
            if any(not 0 <= r < len(self.rows) for r in rows):
                return True
        return False

    def free(self, seq):
        if self._bad(seq) or len(set(seq)) < len(seq):
            return False
        for r in seq:
            for p in self.rows[r]:
                self.refs[p] -= 1
            self.rows[r], self.lens[r] = [], 0
        return True

    def fork(self, src, dst, keep=None):
        if self._bad(src, dst) or len(set(dst)) < len(dst) or set(src) & set(dst):
            return False
        keep = [self.lens[a] for a in src] if keep is None else keep
        if any(not 0 <= k <= self.lens[a] for a, k in zip(src, keep)) or any(self.rows[b] or self.lens[b] for b in dst):
            return False
        for a, b, k in zip(src, dst, keep):
            self.rows[b] = self.rows[a][:-(-k // self.page)]
            self.lens[b] = k
            for p in self.rows[b]:
                self.refs[p] += 1
        return True

    def grow(self, seq, add):
        if self._bad(seq) or len(set(seq)) < len(seq):
            return False
        if any(a < 0 or -(-(self.lens[r] + a) // self.page) > self.max_pages for r, a in zip(seq, add)):
            return False
        free = [p for p, n in enumerate(self.refs) if n == 0]
        plan, shared = [], {r: bool(self.rows[r]) and self.lens[r] % self.page != 0 and self.refs[self.rows[r][-1]] > 1
                            for r in seq}
        for r, a in zip(seq, add):
            copy = a > 0 and shared[r]
            more = -(-(self.lens[r] + a) // self.page) - len(self.rows[r]) + copy
            plan.append((r, a, copy, [free.pop(0) if free else None for _ in range(more)]))
        if any(p is None for _, _, _, new in plan for p in new):
            return False
        old = list(self.data)
        for r, a, copy, new in plan:
            for p in new:
                self.refs[p] = 1
            if copy:
                tail = self.rows[r][-1]
                self.refs[tail] -= 1
                self.rows[r][-1] = new[0]
                self.data[new[0]] = old[tail]
                new = new[1:]
            self.rows[r] = self.rows[r] + new
            self.lens[r] += a
        return True

    def compact(self):
        used = sum(n > 0 for n in self.refs)
        frm = [p for p in range(used, len(self.refs)) if self.refs[p]]
        to = [p for p in range(used) if not self.refs[p]]
        new = dict(zip(frm, to))
        for a, b in new.items():
            self.data[b] = self.data[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[new.get(p, p) for p in row] for row in self.rows]
        return len(frm), used

    def table(self):
        return [row + [-1] * (self.max_pages - len(row)) for row in self.rows]
