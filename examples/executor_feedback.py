"""From running operators to placing them: an executor on one GPU runs the decoder layers of a batch
of requests with ``gmgop`` and times each operator; the online estimators are fitted on these times;
the what-if simulation then places a graph whose durations they predict.

The requests share a prompt: one request runs it, the others are forked from it (their pages are the
same until they write), and every step's attention reads the shared pages once.  Weights and inputs
are random.

    python examples/executor_feedback.py [--layers 4 --hidden 2048 --requests 24 --prompt 1500 --steps 6]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2608_15762_gb300 import gmgop as P  # noqa: E402
from paper_2608_15762_gb300 import gmgsim as G  # noqa: E402
from paper_2608_15762_gb300 import workloads as W  # noqa: E402

KIND = {name: i for i, name in enumerate(W.LAYER_OPS)}
# Nodes of the layer that a call covers along with its own.
COVERS = {"kvw": "rope", "add1": "oproj", "silu": "gateup", "add2": "down"}


class Executor:
    """The layers' weights, a paged cache, and the times of the operators that have run."""

    def __init__(self, layers, hidden, heads, kv_heads, ffn, n_seq, tokens, page=16, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.layers, self.hidden, self.heads, self.kv_heads, self.dim = layers, hidden, heads, kv_heads, hidden // heads
        self.page, self.dtype, self.gen = page, dtype, g
        D = self.dim

        def weight(n, k):
            return (torch.randn(n, k, generator=g, device="cuda") * k ** -0.5).to(dtype)

        self.w = [dict(qkv=weight((heads + 2 * kv_heads) * D, hidden), o=weight(hidden, heads * D),
                       gate=weight(ffn, hidden), up=weight(ffn, hidden), down=weight(hidden, ffn))
                  for _ in range(layers)]
        cols = -(-tokens // page) + 1
        pool = torch.zeros(n_seq * cols, layers, 2, kv_heads, page, D, dtype=dtype, device="cuda")
        self.cache = P.PageCache(pool, n_seq=n_seq, max_pages=cols)
        self.rope = P.Rope(D, device="cuda")
        self.len = [0] * n_seq
        self.ahead = torch.randn(4096, 4096, generator=g, device="cuda").to(dtype)
        self.samples = {k: [] for k in ("qkv", "rope", "attn", "oproj", "gateup", "down")}
        self.timed = []

    def ints(self, v):
        return torch.tensor(list(v), dtype=torch.int32, device="cuda")

    def call(self, kind, features, fn):
        """Run an operator between two events."""
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        out = fn()
        b.record()
        self.timed.append((kind, features, a, b))
        return out

    def step(self, rows, n, group=None, keep_times=True):
        """n new tokens of every row, through all layers; group: tokens that all rows share."""
        B, T, H, Hk, D = len(rows), len(rows) * n, self.heads, self.kv_heads, self.dim
        old = [self.len[r] for r in rows]
        self.cache.grow(self.ints(rows), self.ints([n] * B))
        pos, seq = self.ints(o + i for o in old for i in range(n)), self.ints(r for r in rows for _ in range(n))
        kv = [o + n for o in old]
        plan = P.AttendPlan([n] * B, kv, H, Hk, D, self.page, seq=rows,
                            group_off=None if group is None else [0, B], prefix=None if group is None else [group])
        first = torch.randn(T, self.hidden, generator=self.gen, device="cuda").to(self.dtype)
        pairs = float(sum(n * (t - n) + n * (n + 1) // 2 for t in kv))
        read = float(sum(kv) - (B - 1) * (group or 0))

        def product(kind, a, weight, **kw):
            m, k = a.shape
            return self.call(kind, (float(m) * weight.shape[0] * k, 1.0), lambda: P.linear(a, weight, **kw))

        # twice: the first pass brings memory and code, the second is timed, behind enough other work that
        # the host has issued it when the GPU comes to it
        for timed in (False, True):
            x, self.timed = first, []
            for _ in range(20 * self.layers if timed else 0):
                P.linear(self.ahead, self.ahead)
            for layer, w in enumerate(self.w):
                qkv = product("qkv", norm(x), w["qkv"])
                q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([H * D, Hk * D, Hk * D], 1))
                q = self.call("rope", (float(T), 1.0),
                              lambda: P.rope_append(self.rope, q, k, v, pos, seq, self.cache, layer))
                o = self.call("attn", (pairs, read, 1.0), lambda: P.attend(plan, q, self.cache, layer))
                x = product("oproj", o.flatten(1), w["o"], residual=x)
                h = product("gateup", norm(x), w["up"], gate=w["gate"], act="silu")
                x = product("down", h, w["down"], residual=x)
        for r in rows:
            self.len[r] += n
        torch.cuda.synchronize()
        if keep_times:
            for kind, features, a, b in self.timed:
                self.samples[kind].append((features, a.elapsed_time(b) * 1e3))
        self.timed = []
        return x

    def fork(self, src, dst):
        self.cache.fork(self.ints([src] * len(dst)), self.ints(dst))
        for r in dst:
            self.len[r] = self.len[src]

    def free(self, rows):
        self.cache.free(self.ints(rows))
        self.cache.compact()
        for r in rows:
            self.len[r] = 0


def norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def fit(samples):
    """Estimators by number of features, over the operators with such samples."""
    fitted = []
    for n_feat in (2, 3):
        kinds = [k for k, s in samples.items() if s and len(s[0][0]) == n_feat]
        off = np.cumsum([0] + [len(samples[k]) for k in kinds]).astype(np.int32)
        x = np.array([f for k in kinds for f, _ in samples[k]], np.float64)
        y = np.array([t for k in kinds for _, t in samples[k]], np.float64)
        est = G.Estimators(len(kinds), n_feat)
        est.update(*(torch.from_numpy(a).cuda() for a in (off, x, y)))
        fitted.append((est, kinds))
    return fitted


def durations(fitted, kinds, features, default):
    """Predicted microseconds of graph nodes: their kinds (indexes of a layer's nodes) and each
    kind's features; nodes that a call covers take the shortest time, the others `default`."""
    n = len(kinds)
    names = [W.LAYER_OPS[k] if k >= 0 else None for k in kinds]
    dur = torch.tensor([1 if name in COVERS else default for name in names], dtype=torch.int64, device="cuda")
    for est, of in fitted:
        place = np.array([of.index(name) if name in of else -1 for name in names], np.int32)
        x = np.array([features.get(name, (0.0,) * est.n_feat) if name in of else (0.0,) * est.n_feat for name in names],
                     np.float64)
        dur = est.predict_durations(torch.from_numpy(place).cuda()[:, None], torch.from_numpy(x).cuda(), dur)[:, 0].clone()
    return dur.cpu().numpy().reshape(n)


def graph(layers, requests, n_dev, dur_of, out_bytes):
    """One step of `requests` requests, each a chain of decoder layers, on n_dev accelerators."""
    t = W.prefill_template(layers)
    n = t.n
    off = np.concatenate([t.pred_off[:-1] + r * t.pred_off[-1] for r in range(requests)] + [[requests * t.pred_off[-1]]])
    idx = np.concatenate([t.pred_idx + r * n for r in range(requests)])
    return W.GmgDesc(n_dev=n_dev, pred_off=off.astype(np.int32), pred_idx=idx.astype(np.int32),
                     dur=np.tile(dur_of(t.kind), requests).astype(np.int64),
                     out_bytes=np.full(requests * n, out_bytes, np.int64), release=np.zeros(requests * n, np.int64),
                     req_id=np.repeat(np.arange(requests), n).astype(np.int32),
                     scored=np.ones(requests * n, np.uint8), deadline=np.full(requests, 10 ** 9, np.int64),
                     cap=np.full(n_dev, 1 << 40, np.int64), base=np.zeros(n_dev, np.int64),
                     avail0=np.zeros(n_dev, np.int64), bw=np.full(n_dev * n_dev, 400_000, np.int64),
                     lat=np.full(n_dev * n_dev, 10, np.int64)).normalized()


def main(layers=4, hidden=2048, heads=16, kv_heads=2, ffn=5632, requests=24, prompt=1500, steps=6, n_dev=8,
         candidates=1024, say=print):
    ex = Executor(layers, hidden, heads, kv_heads, ffn, requests, prompt + 16 * steps + 64)
    ex.step([0], prompt, keep_times=False)                    # the shared prompt (and the first run of everything)
    others = list(range(1, requests))
    ex.fork(0, others)
    for i in range(steps):
        n = (1, 2, 1, 4, 1, 8)[i % 6]                         # steps of one token, and of drafted ones
        some = list(range(requests if i % 2 == 0 else max(2, requests // 2)))
        ex.step(some, n, group=prompt, keep_times=i > 0 or steps == 1)
    ex.free(others[len(others) // 2:])
    ex.step(list(range(1 + len(others) // 2)), 1, group=prompt)
    fitted = fit(ex.samples)
    for est, kinds in fitted:
        beta, ok = est.coefficients()
        for k, b, good in zip(kinds, beta.tolist(), ok.tolist()):
            t = [y for _, y in ex.samples[k]]
            say("%-7s %3d samples, %8.1f us on average, %s" % (k, len(t), sum(t) / len(t),
                                                             "t = " + " + ".join("%.3g x%d" % (v, i) for i, v in enumerate(b))
                                                             if good else "not fitted"))
    T, D = requests, hidden // heads
    sizes = dict(qkv=(heads + 2 * kv_heads) * D * hidden, oproj=hidden * hidden, gateup=ffn * hidden, down=hidden * ffn)
    features = {k: (float(T) * v, 1.0) for k, v in sizes.items()}
    features["rope"] = (float(T), 1.0)
    features["attn"] = (float(T * (prompt + 20)), float(prompt + 20 * T), 1.0)
    desc = graph(layers, requests // 4, n_dev, lambda kind: durations(fitted, list(kind), features, 5), T * hidden * 2)
    gmg = G.gmg_create(desc)
    place = torch.from_numpy(W.random_rows(3, range(candidates), desc.n_ops, n_dev)).cuda()
    out = G.sim_batch(gmg, place)
    best, score = G.select_best(out).tolist()
    say("best of %d placements of %d operators on %d accelerators: %d, %d us" % (
        candidates, desc.n_ops, n_dev, best, int(out.makespan[best])))
    return dict(executor=ex, fitted=fitted, best=best, score=score, makespan=int(out.makespan[best]), desc=desc)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 4), ("hidden", 2048), ("heads", 16), ("kv-heads", 2), ("ffn", 5632), ("requests", 24),
                        ("prompt", 1500), ("steps", 6)):
        ap.add_argument("--" + name, type=int, default=value)
    main(**{k.replace("-", "_"): v for k, v in vars(ap.parse_args()).items()})
