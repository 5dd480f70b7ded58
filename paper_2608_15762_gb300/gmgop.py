"""Thin Python binding of the decoder-layer operators in ``include/gmgop.h``.

The operators are what an executor runs of a placed graph: products with their
epilogue (``linear``), rotary positions (``rope``, ``rope_append``), a paged cache
(``PageCache``) and attention over shared prefixes (``AttendPlan``, ``attend``).
Argument marshalling only; PyTorch provides device memory and streams.  Calls
are asynchronous on the current stream, or on ``stream``, where their results'
memory then belongs (and which the memory of their inputs, plans and caches has to
outlive).  Operands, plans, workspaces and stream are on the current GPU.  What the C ABI
refuses raises ``GmgError``; tensors of the wrong shape, type or device raise ``ValueError``.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import struct
from typing import Optional, Sequence

import numpy as np
import torch

from . import gmgsim as G
from .gmgsim import GmgError, _aligned_empty, _check

EXPORTED = ("op_page_scratch_bytes", "op_free", "op_fork", "op_grow", "op_compact", "op_rope", "op_rope_append",
            "op_attend_plan", "op_attend", "op_linear_work_bytes", "op_linear")

F32, BF16, F16 = 0, 1, 2
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
PAGE_OK, PAGE_FULL, PAGE_SEQ, PAGE_TWICE, PAGE_LONG, PAGE_USED = range(6)


class _Cache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pool", "table", "lens", "refs", "status")] + [
        (n, C.c_int32) for n in ("dtype", "n_pages", "n_layers", "n_kv_heads", "page_tokens", "head_dim", "n_seq",
                                 "max_pages")]


class _Rope(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rotary", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float)]


class _AttendDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_batch", "n_heads", "n_kv_heads", "head_dim", "page_tokens",
                                         "n_groups")] + [
        (n, C.c_void_p) for n in ("q_len", "kv_len", "seq", "group_off", "prefix")]


class _AttendPlan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_batch", "n_heads", "n_kv_heads", "head_dim", "page_tokens", "n_items",
                                         "n_joins", "max_seq", "max_kv", "join_tokens")] + [
        ("n_tokens", C.c_int64), ("part_rows", C.c_int64), ("plan_bytes", C.c_size_t), ("work_bytes", C.c_size_t)]


class _Linear(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "act", "gated", "reserved")] + [
        (n, C.c_int64) for n in ("m", "n", "k")] + [
        (n, C.c_void_p) for n in ("x", "w", "gate", "bias", "gate_bias", "residual", "y")] + [
        (n, C.c_int64) for n in ("x_row", "w_row", "gate_row", "residual_row", "y_row")]


# _Linear's bytes: packing them is quicker than filling a ctypes structure.
_LINEAR = struct.Struct("@4i3q7P5q")
assert _LINEAR.size == C.sizeof(_Linear)
_LIB = None


def lib():
    global _LIB
    if _LIB is None:
        L = G.lib()
        vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
        sig = {
            "op_page_scratch_bytes": ([vp], sz),
            "op_free": ([vp, vp, i32, vp, sz, vp], C.c_int),
            "op_fork": ([vp, vp, vp, vp, i32, vp, sz, vp], C.c_int),
            "op_grow": ([vp, vp, vp, i32, vp, sz, vp], C.c_int),
            "op_compact": ([vp, vp, sz, vp], C.c_int),
            "op_rope": ([vp, i32, i64, i32, i32, vp, i64, i64, vp, i32, vp, i64, i64, vp], C.c_int),
            "op_rope_append": ([vp, vp, i32, i64, i32] + [vp, i64, i64] * 3 + [vp, vp, vp, i64, i64, vp], C.c_int),
            "op_attend_plan": ([vp, i32, vp, vp, sz], C.c_int),
            "op_attend": ([vp, vp, vp, i32, vp, i64, i64, f32, vp, i64, i64, vp, vp, sz, vp], C.c_int),
            "op_linear_work_bytes": ([vp], sz),
            "op_linear": ([vp, vp, sz, vp], C.c_int),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _LIB = L
    return _LIB


# A call of a small operator takes the GPU a few microseconds, so the host's part is kept short:
# checks are plain comparisons, and a range is pushed only where the environment asks for it.
_traced = G._traced if G.NVTX else lambda name: lambda fn: fn
_I32 = torch.int32
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_RAW = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _handle(stream, device_index):
    """The stream's handle, by default that of the current stream.  The library launches on the current
    GPU, so operands and stream have to be there."""
    if _current() != device_index:
        raise ValueError("operands on GPU %d, which is not the current one" % device_index)
    if stream is not None:
        if stream.device_index != device_index:
            raise ValueError("stream: on the operands' GPU")
        return stream.cuda_stream
    if _RAW is not None:
        return _RAW(device_index)
    return torch.cuda.current_stream(device_index).cuda_stream


def _dtype(t) -> int:
    d = _TYPES.get(t.dtype)
    if d is None:
        raise ValueError("element type %s: fp32, bf16 or fp16" % t.dtype)
    return d


def _need(ok, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _fail(rc: int, what: str):
    raise GmgError(rc, what)


def _on(stream):
    """Memory allocated inside belongs to `stream`."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _capturing(stream) -> bool:
    """Whether the stream's calls are being captured into a graph."""
    with _on(stream):
        return torch.cuda.is_current_stream_capturing()


def _list(t, device, what: str) -> int:
    """The length of a list on the GPU."""
    if t.dtype is not _I32 or t.dim() != 1 or t.device != device or not t.is_contiguous():
        raise ValueError("%s: a contiguous int32 list on the operands' GPU" % what)
    return t.shape[0]


# ---------------------------------------------------------------------------
# Pages of a cache
# ---------------------------------------------------------------------------

class PageCache:
    """A paged cache of keys and values: pool [n_pages, n_layers, 2, n_kv_heads,
    page_tokens, head_dim] and, int32, table [n_seq, max_pages] (-1: no page), lens
    [n_seq] and refs [n_pages].  What is not given starts empty, but references are
    counted from a given table (which has to come with its lens where rows are to grow).
    It is set up on the current stream, which calls on others have to wait for.
    The page calls take int32 lists on the GPU and do not synchronise; ``code()`` does,
    and says how the last one went."""

    def __init__(self, pool, n_seq: int = 0, max_pages: int = 0, table=None, lens=None, refs=None):
        _need(pool.is_cuda and pool.dim() == 6 and pool.shape[2] == 2 and pool.is_contiguous(),
              "pool: contiguous, [n_pages, n_layers, 2, n_kv_heads, page_tokens, head_dim], on a GPU")
        dev, i32 = pool.device, torch.int32
        if table is None:
            table = torch.full((n_seq, max_pages), -1, dtype=i32, device=dev)
        n_seq, max_pages = table.shape
        lens = torch.zeros(n_seq, dtype=i32, device=dev) if lens is None else lens
        _need(table.dtype == i32 and table.is_contiguous() and table.device == dev, "table: contiguous int32")
        if refs is None:
            refs = torch.zeros(pool.shape[0], dtype=i32, device=dev)
            used = table[(table >= 0) & (table < pool.shape[0])].long()
            refs.index_add_(0, used, torch.ones_like(used, dtype=i32))
        _list(lens, dev, "lens")
        _list(refs, dev, "refs")
        _need(lens.numel() == n_seq and refs.numel() == pool.shape[0], "lens, refs: one entry a row, one a page")
        self.pool, self.table, self.lens, self.refs = pool, table, lens, refs
        self.status = torch.zeros(8, dtype=i32, device=dev)
        p = pool.shape
        self.n_layers, self.n_kv_heads, self.page_tokens, self.head_dim = p[1], p[3], p[4], p[5]
        self.device, self.dtype, self._index = dev, pool.dtype, pool.get_device()
        self.c = _Cache(pool.data_ptr(), table.data_ptr(), lens.data_ptr(), refs.data_ptr(), self.status.data_ptr(),
                        _dtype(pool), p[0], p[1], p[3], p[4], p[5], n_seq, max_pages)
        self.ref = C.addressof(self.c)
        nbytes = (_LIB or lib()).op_page_scratch_bytes(self.ref)
        if nbytes == 0:
            raise GmgError(G.GMG_EINVAL, "op_page_scratch_bytes")
        self.scratch = _aligned_empty(nbytes, dev)
        self.scratch.zero_()
        self._work = self.scratch.data_ptr(), nbytes

    def code(self):
        """(PAGE_* code of the last page call, the list entry or the missing pages)."""
        return tuple(self.status[:2].tolist())

    @_traced("op_free")
    def free(self, seq, stream=None):
        """Empty the listed rows and drop their references."""
        n = _list(seq, self.device, "seq")
        rc = (_LIB or lib()).op_free(self.ref, seq.data_ptr(), n, *self._work, _handle(stream, self._index))
        if rc:
            _fail(rc, "op_free")

    @_traced("op_fork")
    def fork(self, src, dst, keep=None, stream=None):
        """The empty rows dst get the first ``keep`` tokens (all) of rows src by reference."""
        n = _list(src, self.device, "src")
        if _list(dst, self.device, "dst") != n or (keep is not None and _list(keep, self.device, "keep") != n):
            raise ValueError("src, dst, keep: one length")
        rc = (_LIB or lib()).op_fork(self.ref, src.data_ptr(), dst.data_ptr(), None if keep is None else keep.data_ptr(), n,
                           *self._work, _handle(stream, self._index))
        if rc:
            _fail(rc, "op_fork")

    @_traced("op_grow")
    def grow(self, seq, add, stream=None):
        """Room for ``add`` more tokens in the listed rows, whose lengths grow by them; a
        partly filled last page that others hold too is copied first."""
        n = _list(seq, self.device, "seq")
        if _list(add, self.device, "add") != n:
            raise ValueError("seq, add: one length")
        rc = (_LIB or lib()).op_grow(self.ref, seq.data_ptr(), add.data_ptr(), n, *self._work, _handle(stream, self._index))
        if rc:
            _fail(rc, "op_grow")

    @_traced("op_compact")
    def compact(self, stream=None):
        """Move the pages in use to the lowest page numbers."""
        rc = (_LIB or lib()).op_compact(self.ref, *self._work, _handle(stream, self._index))
        if rc:
            _fail(rc, "op_compact")


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

def rope_freqs(rotary: int, base: float = 10000.0, scaling: str = "none", scale: float = 1.0, length: int = 0,
               low: float = 1.0, high: float = 32.0):
    """(angle per position of each pair in 64 bits, factor of the magnitude).

    none: f_i = base^(-2i / rotary).  linear: f_i / scale.  base: the base grown to
    base * scale^(rotary / (rotary - 2)), which divides the lowest frequency by scale.
    parts: pairs that turn ``high`` times or more over ``length`` positions keep their
    frequency, those that turn ``low`` times or less have it divided by scale, a
    linear mix between; the factor is 0.1 ln(scale) + 1."""
    _need(rotary % 2 == 0 and rotary > 0 and base > 1.0 and scale >= 1.0, "rotary even, base > 1, scale >= 1")
    i = np.arange(rotary // 2, dtype=np.float64)
    if scaling == "base":
        _need(rotary > 2, "scaling the base takes more than one pair")
        base = base * scale ** (rotary / (rotary - 2))
    f = base ** (-2.0 * i / rotary)
    if scaling in ("none", "base"):
        return f, 1.0
    if scaling == "linear":
        return f / scale, 1.0
    _need(scaling == "parts", "scaling: none, linear, base or parts")
    _need(length > 0 and high > low, "parts: length > 0, high > low")
    keep = np.clip((length * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
    return f * (keep + (1.0 - keep) / scale), 0.1 * math.log(scale) + 1.0


def _pi(bits: int) -> int:
    """pi 2^bits in whole numbers: 16 arctan(1/5) - 4 arctan(1/239), by their series."""
    def arctan(x):
        power = total = (1 << (bits + 16)) // x
        n = 1
        while power:
            power //= -x * x
            n += 2
            total += power // n
        return total
    return (16 * arctan(5) - 4 * arctan(239)) >> 16


_PI = _pi(256)


def _turns(f: float) -> int:
    """f / (2 pi) * 2^64, rounded (f is 64-bit: the quotient in 64 bits would be up to 2^10 off)."""
    n, d = f.as_integer_ratio()
    return min((n << (64 + 256)) // (d * _PI) + 1 >> 1, 2 ** 64 - 1)


class Rope:
    """The frequencies of rotary positions, on the GPU: fractions of a turn per
    position in 64 bits.  freqs (64-bit, 0 <= f < 2 pi) and factor as from
    ``rope_freqs``, or its arguments."""

    def __init__(self, rotary: int, freqs=None, factor: float = 1.0, interleaved: bool = False, device="cuda", **kw):
        if freqs is None:   # (no rotation at all where rotary is 0)
            freqs, factor = rope_freqs(rotary, **kw) if rotary else (np.zeros(0), factor)
        freqs = np.asarray(freqs, np.float64)
        _need(freqs.shape == (rotary // 2,) and rotary % 2 == 0, "freqs: one per pair")
        _need(bool(np.all((freqs >= 0) & (freqs < 2 * math.pi))), "freqs: 0 <= f < 2 pi")
        turns = np.array([_turns(float(f)) for f in freqs], np.uint64)
        self.rotary, self.factor, self.interleaved = int(rotary), float(factor), bool(interleaved)
        self.freq = torch.from_numpy(turns.view(np.int64).copy()).to(device)
        self.c = _Rope(self.freq.data_ptr(), self.rotary, int(self.interleaved), self.factor)
        self.ref, self.index = C.addressof(self.c), self.freq.get_device()


def _heads(t, what: str):
    """(pointer, stride of a token, of a head) of a tensor [tokens, heads, head_dim]."""
    s = t.stride()
    if len(s) != 3 or (s[2] != 1 and t.shape[2] > 1):
        raise ValueError("%s: [tokens, heads, head_dim], contiguous in head_dim" % what)
    return t.data_ptr(), s[0], s[1]


def _like(x, out, stream):
    """`out`, checked against x, or a new tensor of its shape."""
    if out is None:
        if stream is None:
            return torch.empty(x.shape, dtype=x.dtype, device=x.device)
        with torch.cuda.stream(stream):
            return torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if out.shape != x.shape or out.dtype is not x.dtype or out.device != x.device:
        raise ValueError("out: of the input's shape, type and GPU")
    return out


@_traced("op_rope")
def rope(plan: Rope, x, pos, backward: bool = False, out=None, stream=None):
    """x [tokens, heads, head_dim] rotated by pos (int32, one a token); ``backward``: by
    minus the angle, which takes the gradient of the result to that of x.  out may be x."""
    kind = _dtype(x)
    ptr, s0, s1 = _heads(x, "x")
    T, H, D = x.shape
    index = x.get_device()
    if index < 0 or _list(pos, x.device, "pos") != T:
        raise ValueError("x on a GPU, pos: one entry a token")
    if plan.index != index:
        raise ValueError("plan: on x's GPU")
    out = _like(x, out, stream)
    rc = (_LIB or lib()).op_rope(plan.ref, kind, T, H, D, ptr, s0, s1, pos.data_ptr(), 1 if backward else 0, *_heads(out, "out"),
                       _handle(stream, index))
    if rc:
        _fail(rc, "op_rope")
    return out


@_traced("op_rope_append")
def rope_append(plan: Rope, q, k, v, pos, seq, cache: PageCache, layer: int, out=None, stream=None):
    """q rotated by pos (returned); k rotated and v written to ``layer`` of the cache as
    token pos[t] of row seq[t] (a negative seq: not written)."""
    T, H, D = q.shape
    kv, dt, dev = (T, cache.n_kv_heads, D), cache.dtype, cache.device
    if D != cache.head_dim or k.shape != kv or v.shape != kv:
        raise ValueError("q [tokens, heads, head_dim], k and v [tokens, n_kv_heads, head_dim]")
    if q.dtype is not dt or k.dtype is not dt or v.dtype is not dt or q.device != dev or k.device != dev or v.device != dev:
        raise ValueError("q, k, v: the cache's type, on its GPU")
    if plan.index != cache._index:
        raise ValueError("plan: on the cache's GPU")
    if _list(pos, dev, "pos") != T or _list(seq, dev, "seq") != T:
        raise ValueError("pos, seq: one entry a token")
    out = _like(q, out, stream)
    rc = (_LIB or lib()).op_rope_append(plan.ref, cache.ref, layer, T, H, *_heads(q, "q"), *_heads(k, "k"), *_heads(v, "v"),
                              pos.data_ptr(), seq.data_ptr(), *_heads(out, "out"), _handle(stream, cache._index))
    if rc:
        _fail(rc, "op_rope_append")
    return out


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

_SMS = {}


def _n_sm(device) -> int:
    if device not in _SMS:
        _SMS[device] = torch.cuda.get_device_properties(device).multi_processor_count
    return _SMS[device]


def attend_items(q_len, kv_len, n_heads, n_kv_heads, head_dim, page_tokens, seq=None, group_off=None, prefix=None,
                 n_sm: int = 152):
    """(plan, its int32 array on the host): the work of ``attend`` for these lengths."""
    arr = [None if a is None else np.ascontiguousarray(a, np.int32) for a in (q_len, kv_len, seq, group_off, prefix)]
    q, kv, sq, off, pre = arr
    _need(q.ndim == 1 and kv.shape == q.shape and (sq is None or sq.shape == q.shape),
          "q_len, kv_len, seq: one entry a request")
    _need((off is None) == (pre is None) and (off is None or off.shape == (pre.size + 1,)),
          "group_off: one entry more than prefix")
    ptr = [None if a is None else a.ctypes.data for a in arr]
    d = _AttendDesc(q.size, n_heads, n_kv_heads, head_dim, page_tokens, 0 if pre is None else pre.size, *ptr)
    plan = _AttendPlan()
    items = np.empty(1 << 14, np.int32)      # most plans are shorter; longer ones are made again
    call = (_LIB or lib()).op_attend_plan
    rc = call(C.addressof(d), n_sm, C.addressof(plan), items.ctypes.data, items.nbytes)
    if rc == G.GMG_EWS:
        _check(call(C.addressof(d), n_sm, C.addressof(plan), None, 0), "op_attend_plan")
        items = np.empty(plan.plan_bytes // 4, np.int32)
        rc = call(C.addressof(d), n_sm, C.addressof(plan), items.ctypes.data, items.nbytes)
    _check(rc, "op_attend_plan")
    return plan, items[:plan.plan_bytes // 4].copy()


class AttendPlan:
    """The work of ``attend`` for requests of q_len new and kv_len cached tokens (the
    new ones among them), for every layer of a step (a graph captured with it serves these
    lengths, and has a workspace of its own).  seq: their table rows (0, 1,
    ...).  group_off, prefix: requests group_off[g] .. group_off[g + 1] share their
    first prefix[g] tokens."""

    def __init__(self, q_len: Sequence[int], kv_len: Sequence[int], n_heads: int, n_kv_heads: int, head_dim: int,
                 page_tokens: int, seq: Optional[Sequence[int]] = None, group_off: Optional[Sequence[int]] = None,
                 prefix: Optional[Sequence[int]] = None, device="cuda", stream=None):
        dev = torch.device(device)
        self.c, items = attend_items(q_len, kv_len, n_heads, n_kv_heads, head_dim, page_tokens, seq, group_off, prefix,
                                     _n_sm(dev))
        self.ref = C.addressof(self.c)
        self.n_tokens, self.n_heads, self.head_dim = int(self.c.n_tokens), n_heads, head_dim
        self.shape = (self.n_tokens, n_heads, head_dim)
        self.work_bytes = int(self.c.work_bytes)
        with _on(stream):
            self.items = torch.from_numpy(items).to(dev)
        self._ptr, self.index = self.items.data_ptr() if items.size else None, self.items.get_device()
        self.work, self._kept = {}, []       # a workspace per stream that the plan has been used on

    def empty_work(self):
        return _aligned_empty(self.work_bytes, self.items.device)

    def new_work(self, handle):
        self._kept.append(self.empty_work())
        self.work[handle] = self._kept[-1].data_ptr()
        return self.work[handle]


@_traced("op_attend")
def attend(plan: AttendPlan, q, cache: PageCache, layer: int, scale: Optional[float] = None, out=None, lse=False,
           stream=None):
    """Attention of q [tokens, heads, head_dim] (the requests' new tokens, one request
    after another) over the cache; with ``lse`` also log sum exp [tokens, heads], fp32."""
    if q.shape != plan.shape or q.dtype is not cache.dtype or q.device != cache.device:
        raise ValueError("q: [tokens, heads, head_dim] of the plan, the cache's type, on its GPU")
    if plan.index != cache._index:
        raise ValueError("plan: on the cache's GPU")
    h = _handle(stream, cache._index)
    work = plan.work.get(h)
    if stream is None:
        out = _like(q, out, None)
        z = torch.empty(plan.shape[:2], dtype=torch.float32, device=q.device) if lse else None
        if torch.cuda.is_current_stream_capturing():
            own = plan.empty_work()          # the graph's memory, free for its later calls
            work = own.data_ptr()
        elif work is None:
            work = plan.new_work(h)
    else:
        with torch.cuda.stream(stream):
            out = _like(q, out, None)
            z = torch.empty(plan.shape[:2], dtype=torch.float32, device=q.device) if lse else None
            if torch.cuda.is_current_stream_capturing():
                own = plan.empty_work()
                work = own.data_ptr()
            elif work is None:
                work = plan.new_work(h)
    rc = (_LIB or lib()).op_attend(plan.ref, plan._ptr, cache.ref, layer, *_heads(q, "q"),
                                   plan.head_dim ** -0.5 if scale is None else scale, *_heads(out, "out"),
                                   None if z is None else z.data_ptr(), work, plan.work_bytes, h)
    if rc:
        _fail(rc, "op_attend")
    return (out, z) if lse else out


# ---------------------------------------------------------------------------
# Products
# ---------------------------------------------------------------------------

class Workspace:
    """A workspace of ``linear``: grown on demand, its head zeroed when it is made.
    Calls that share one must be ordered (one stream), replays of captured ones among them.
    What it has outgrown stays allocated, as a captured call writes there whenever it is replayed;
    it doubles at least, so that this is no more than the workspace itself."""

    def __init__(self, device="cuda"):
        self.device, self.buf, self.ptr, self.size, self._kept = device, None, 0, 0, []
        self.index = None                    # its GPU, once it has memory

    def get(self, nbytes: int, stream=None):
        if self.buf is None or self.size < nbytes:
            if self.buf is not None:
                self._kept.append(self.buf)
            with _on(stream):
                self.buf = _aligned_empty(max(nbytes, 2 * self.size, 4096), self.device)
                self.buf[:4096].zero_()
            self.ptr, self.size, self.index = self.buf.data_ptr(), self.buf.numel(), self.buf.get_device()
        return self.buf

    def gave_up(self) -> int:
        """Blocks of ``linear`` with a wait that gave up (0 unless the GPU is at fault); synchronises."""
        return sum(int(b[:4].view(torch.int32).item()) for b in self._kept + [self.buf] if b is not None)


_WORK = {}      # the default workspaces, by GPU and stream


def gave_up() -> int:
    """Blocks of ``linear`` on its default workspaces with a wait that gave up (0 unless the GPU is at fault: what a
    call with such a block wrote is not its result); synchronises."""
    return sum(ws.gave_up() for ws in list(_WORK.values()))


def _rows(t, n, k, dt, dev, what: str):
    """(pointer, stride of a row) of a matrix [n, k]."""
    if t.shape != (n, k) or t.dtype is not dt or t.device != dev:
        raise ValueError("%s: [%d, %d], of x's type and on its GPU" % (what, n, k))
    s = t.stride()
    if s[1] != 1 and k > 1:
        raise ValueError("%s: rows contiguous" % what)
    return t.data_ptr(), s[0] if n > 1 or s[0] > k else k


def _column(t, n, dt, dev, what: str):
    if t.shape != (n,) or t.dtype is not dt or t.device != dev or not t.is_contiguous():
        raise ValueError("%s: [%d], contiguous, of x's type and on its GPU" % (what, n))
    return t.data_ptr()


def _captured_linear(a, ws, out, dev, stream, h):
    """A call into a graph, whose replays may run beside the stream's other work, or another graph's.
    (The head of the graph's own workspace is not zeroed: nobody can ask for its count.)"""
    L = _LIB or lib()
    need = L.op_linear_work_bytes(a)
    if ws is not None and ws.size >= need and ws.index == out.get_device():
        ptr, size = ws.ptr, ws.size
    else:
        with _on(stream):
            own = _aligned_empty(need, dev)
        ptr, size = own.data_ptr(), need
    rc = L.op_linear(a, ptr, size, h)
    if rc:
        _fail(rc, "op_linear")
    return out


@_traced("op_linear")
def linear(x, w, bias=None, act: str = "none", gate=None, gate_bias=None, residual=None, out=None,
           ws: Optional[Workspace] = None, stream=None):
    """act(x w^T + bias) + residual or, with a gate, act(x gate^T + gate_bias) * (x w^T +
    bias) + residual, for x [m, k], w and gate [n, k], biases [n], residual [m, n].
    act: none, relu, silu, gelu.  out may be residual.  ws: kept per stream by default; a captured
    call has one in its graph's memory, unless it is given one that is large enough."""
    m, k = x.shape
    n, dt, dev, index = w.shape[0], x.dtype, x.device, x.get_device()
    kind, how = _TYPES.get(dt), ACTS.get(act)
    if kind is None or how is None or index < 0:
        raise ValueError("x: bf16 or fp16, on a GPU; act: one of %s" % ", ".join(ACTS))
    if gate_bias is not None and gate is None:
        raise ValueError("gate_bias without a gate")
    if out is None:
        if stream is None:
            out = torch.empty((m, n), dtype=dt, device=dev)
        else:
            with torch.cuda.stream(stream):
                out = torch.empty((m, n), dtype=dt, device=dev)
    xp, xs = _rows(x, m, k, dt, dev, "x")
    wp, wrow = _rows(w, n, k, dt, dev, "w")
    yp, ys = _rows(out, m, n, dt, dev, "out")
    gp, gs = (0, 0) if gate is None else _rows(gate, n, k, dt, dev, "gate")
    rp, rs = (0, 0) if residual is None else _rows(residual, m, n, dt, dev, "residual")
    a = _LINEAR.pack(kind, how, 0 if gate is None else 1, 0, m, n, k, xp, wp, gp,
                     0 if bias is None else _column(bias, n, dt, dev, "bias"),
                     0 if gate_bias is None else _column(gate_bias, n, dt, dev, "gate_bias"), rp, yp, xs, wrow, gs, rs, ys)
    h = _handle(stream, index)
    if (torch.cuda.is_current_stream_capturing() if stream is None else _capturing(stream)):
        return _captured_linear(a, ws, out, dev, stream, h)
    if ws is None:
        ws = _WORK.get((index, h))
        if ws is None:
            ws = _WORK[(index, h)] = Workspace(dev)
    if ws.ptr == 0:
        ws.get(4096, stream)
    if ws.index != index:
        raise ValueError("ws: on x's GPU")
    L = _LIB or lib()
    rc = L.op_linear(a, ws.ptr, ws.size, h)
    if rc == G.GMG_EWS:      # it refuses a short workspace before it does anything
        ws.get(L.op_linear_work_bytes(a), stream)
        rc = L.op_linear(a, ws.ptr, ws.size, h)
    if rc:
        _fail(rc, "op_linear")
    return out
