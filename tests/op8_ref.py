"""Plain implementations in 64 bits of the norms around a block and of a cache in 8 bits, for their
tests, and the bounds on a kernel's error that follow from the types it rounds to."""
import math

import torch

from op_ref import TINY, U, U32, rope

F8 = torch.float8_e4m3fn


def norm(x, w=None, bias=None, kind="rms", eps=1e-6, shift=0.0, y=None, after=False, y_w=None, y_bias=None, gate=None,
         scale=1.0, **_):
    """((h, bound), (r, bound) or None).  Sums of n terms by shares of threads are off by at most
    n / 32 + 16 roundings of their magnitudes; a mean of squares moves its inverse root by half of that; four
    roundings more on the way."""
    n = x.shape[1]
    e_sum = (n / 32 + 16) * U32
    dt = y.dtype if y is not None else w.dtype if w is not None else x.dtype

    def normed(v, dv, w, b):
        """dv: what v itself may be off by."""
        mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        dm = (e_sum * v.abs() + dv).mean(1, keepdim=True) if kind == "layer" else 0.0
        c = v - mean
        dc = dv + dm + U32 * c.abs()
        square = (c * c).mean(1, keepdim=True)
        ds = (2 * c.abs() * dc + dc * dc).mean(1, keepdim=True) + e_sum * square
        inv = 1 / torch.sqrt(square + eps)
        # 1 / sqrt moves by at most what it does where the square is the least that it may be
        least = (square - ds).clamp(min=0) + eps
        di = (1 / torch.sqrt(least.clamp(min=1e-300)) - inv) + 4 * U32 * inv
        by = 1.0 if w is None else w.double() + shift
        o = c * inv * by
        do = (dc * (inv + di) + c.abs() * di) * (by if w is None else by.abs()) + 4 * U32 * o.abs()
        if b is not None:
            o = o + b.double()
            do = do + U32 * o.abs()
        return o, do

    r, dr = x.double(), torch.zeros_like(x, dtype=torch.float64)
    if y is not None:
        z, dz = y.double(), torch.zeros_like(y, dtype=torch.float64)
        if after:
            z, dz = normed(z, dz, y_w, y_bias)
        by = scale if gate is None else gate.double() * scale
        r = r + z * by
        dr = dz * (abs(by) if gate is None else by.abs()) + 3 * U32 * (z * by).abs() + U32 * r.abs()
    h, dh = normed(r, dr, w, bias)
    out = h, dh * (1 + U[dt]) + U[dt] * h.abs() + TINY[dt]
    return out, None if y is None else (r, dr * (1 + U[x.dtype]) + U[x.dtype] * r.abs() + TINY[x.dtype])


def rounded(x):
    """To the nearest e4m3 number (4 significant bits, or a multiple of 2^-9), ties to even, NaN kept."""
    m, e = torch.frexp(x.abs().clamp(min=2.0 ** -6))
    step = torch.tensor([2.0 ** i for i in range(-12, 12)], dtype=torch.float64)[(e - 1 - 3).clamp(-12, 11).long() + 12]
    return (torch.round(x / step) * step).clamp(-448, 448)


def need(top):
    """The least power of two from 2^-60 to 2^60 that brings top to at most 448."""
    return next((2.0 ** i for i in range(-60, 61) if top <= 448 * 2.0 ** i), 2.0 ** 60)


class Blocks:
    """A cache in 8 bits as codes and scales in 64 bits, on the CPU; ``append`` token by token in plain Python."""

    def __init__(self, cache):
        self.codes, self.scales = cache.codes.cpu().to(torch.float64), cache.scales.cpu().double()
        self.table, self.page = cache.table.cpu(), cache.page_tokens

    def written(self, r, p):
        if not 0 <= r < self.table.shape[0] or not 0 <= p < self.table.shape[1] * self.page:
            return False
        return 0 <= int(self.table[r, p // self.page]) < self.codes.shape[0]

    def append(self, x, which, layer, pos, seq):
        """x [tokens, kv_heads, dim] in 64 bits; the runs one after another; returns {(page, block)} touched."""
        t, n = 0, len(pos)
        touched = []
        while t < n:
            if not self.written(seq[t], pos[t]):
                t += 1
                continue
            run, u = [t], t + 1
            while u < n and (not self.written(seq[u], pos[u]) or (
                    seq[u] == seq[t] and pos[u] > pos[run[-1]] and pos[u] // 16 == pos[t] // 16)):
                run += [u] if self.written(seq[u], pos[u]) else []
                u += 1
            t = u
            page = int(self.table[seq[run[0]], pos[run[0]] // self.page])
            slot = pos[run[0]] % self.page
            block, f = slot // 16, slot % 16
            for h in range(x.shape[1]):
                v = x[run, h]
                fine = v[torch.isfinite(v)].abs()
                s = need(float(fine.max()) if fine.numel() else 0.0)
                old = float(self.scales[page, layer, which, h, block])
                if f:
                    s = max(s, min(max(old, 2.0 ** -60), 2.0 ** 60))
                    here = self.codes[page, layer, which, h, block * 16:block * 16 + f]
                    here.copy_(rounded(here * (min(max(old, 2.0 ** -60), 2.0 ** 60) / s)))
                self.scales[page, layer, which, h, block] = s
                for i, a in enumerate(run):
                    self.codes[page, layer, which, h, pos[a] % self.page] = rounded(v[i] / s)
            touched.append((page, block))
        return touched

    def values(self):
        return self.codes * self.scales.repeat_interleave(16, -1)[..., None]


def near(got_codes, got_scales, want, exact, dtol):
    """Codes within one rounding of the exact values that they stand for: the value is off by dtol before it
    is rounded, to 4 significant bits or a multiple of 2^-9 of its scale."""
    value = got_codes.double() * got_scales.double().repeat_interleave(16, -1)[..., None]
    s = got_scales.double().repeat_interleave(16, -1)[..., None]
    return (value - exact).abs() <= dtol + exact.abs() * 2.0 ** -4 + s * 2.0 ** -10


def attend(q, keys, values, v_scales, n_q, scale):
    """One request: q [n, heads, dim]; keys, values [tokens, kv_heads, dim] in 64 bits (code times scale),
    v_scales [tokens, kv_heads].  (o, bound, lse, bound): a score is off by d + 8 roundings of its magnitudes
    (two each, as a tensor core may cut off), and so is its exponent; the weights w = p v_scale, of which the largest is
    at least 2^4, are rounded to 11 bits or more, the smaller ones to multiples of 2^-17 (bf16: three codes, the last a
    256th of what it says, of at least 2^-9) or 2^-21 (fp16: four, a 4096th; fp16 itself has 2^-24); sums over t keys are
    off by t / 16 + 16 roundings."""
    n, H, D = q.shape
    t, Hk = keys.shape[0], keys.shape[1]
    G = H // Hk
    k, v = (a.double().repeat_interleave(G, 1).transpose(0, 1) for a in (keys, values))   # [H, t, D]
    vs = v_scales.double().repeat_interleave(G, 1).t()[:, None]                            # [H, 1, t]
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
    rel = 4 * worst + 2e-5 + 2 * (t / 16 + 16) * U32
    u = U[q.dtype]
    tol = (2.0 ** -11 + rel)[..., None] * mag + u * o.abs() + TINY[q.dtype]
    if t:
        w = p * vs
        most = w.amax(-1, keepdim=True)                        # at least 2^4 in the kernel's units
        half = 2.0 ** (-18 if q.dtype is torch.bfloat16 else -22)
        tol = tol + half * 2.0 ** -4 * (most * ((v.abs() / vs.transpose(1, 2)).masked_fill(vs.transpose(1, 2) == 0, 0)
                                                      ).nansum(1, keepdim=True))
    ltol = worst + 2e-5 + 2 * (t / 16 + 16) * U32 + 4 * U32 * lse.abs().masked_fill(lse.isinf(), 0)
    return o.transpose(0, 1), tol.transpose(0, 1), lse.transpose(0, 1), ltol.transpose(0, 1)


__all__ = ["Blocks", "F8", "attend", "near", "need", "norm", "rope", "rounded"]
