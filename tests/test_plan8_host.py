"""Host side of the plans of attention over a cache in 8 bits (include/gmgop.h): how a batch is cut, and what that costs."""
import ctypes as C
import heapq
import random
import time

import numpy as np
import pytest

from paper_2608_15762_gb300 import build, gmgop as P, gmgsim as G


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


# keys of a step, rows of a tile, and in steps: the shortest part, what a block takes alone, an item's and a join's cost
FEW, MANY = (128, 16, 4, 8, 4, 5), (64, 128, 6, 12, 4, 8)


def _cut(q, kv, group, kv_heads, n_sm, cut):
    """(parts of every run, all steps with the items' cost), block by block: the longest first, on the place that is free first."""
    keys, rows, shortest, alone, item, join = cut
    tile, runs = rows // group, []
    for n, t in zip(q, kv):
        for a in range(0, n, tile):
            hi = max(t - n + min(n, a + tile), 0)
            runs.append(-(-hi // keys))
    tiles = sum(-(-n // tile) for n in q)
    longest = max([-(-t // keys) for n, t in zip(q, kv) if n], default=0)
    small = tiles * kv_heads <= 2 * n_sm and longest <= alone
    most = max(alone if small else shortest, -(-sum(n + item for n in runs) * kv_heads // (2 * n_sm)))
    parts = lambda m: [max(1, -(-n // m)) for n in runs]  # noqa: E731
    if not small:
        best = None
        for k in range(1, 7):
            m = max(shortest, -(-most // k))
            sizes = sorted((n * (i + 1) // p - n * i // p + item for n, p in zip(runs, parts(m)) for i in range(p)), reverse=True)
            if len(sizes) * kv_heads > 40 * 2 * n_sm:
                break
            places = [0] * (2 * n_sm)
            for s in sizes:
                for _ in range(kv_heads):
                    heapq.heapreplace(places, places[0] + s)
            end = max(places) + (join if max(parts(m), default=1) > 1 else 0)
            if best is None or end < best[0]:
                best = end, m
            if m == shortest:
                break
        most = best[1] if best else most
    return parts(most), sum(runs) + item * sum(parts(most))


def test_attend8_plan_is_cut_as_block_by_block():
    r = random.Random(2)
    kinds = set()
    for i in range(120):
        n, group, hk = r.randint(1, 60), r.choice([1, 4, 5, 8, 16, 40]), r.choice([1, 2, 8])
        q = [1] * n if i % 2 else [r.choice([0, 1, 3, 60, 200]) for _ in range(n)]
        kv = [x + r.choice([0, 40, 700, 5000, r.randint(0, 20000)]) for x in q]
        n_sm = r.choice([152, 152, 40, 3])
        plan, items = P.attend_items(q, kv, group * hk, hk, 64, 16, n_sm=n_sm, bits=8)
        many = _cut(q, kv, group, hk, n_sm, MANY)
        few = _cut(q, kv, group, hk, n_sm, FEW) if group <= 16 else None
        is_few = few is not None and few[1] * 1900 <= many[1] * 1300
        assert bool(plan.few) == is_few
        assert plan.n_items == sum((few if is_few else many)[0])
        kinds.add(is_few)
    assert kinds == {False, True}


def test_attend8_plan_costs_little_more_than_the_16_bit_one():
    """A decode step makes a plan: the search for an even cut must not outweigh the step."""
    r = random.Random(3)
    for kw in (dict(q_len=[1] * 64, kv_len=[r.randint(7000, 9300) for _ in range(64)], n_heads=32, n_kv_heads=8),
               dict(q_len=[4], kv_len=[131072], n_heads=40, n_kv_heads=8),
               dict(q_len=[1] * 1024, kv_len=[r.randint(2000, 4000) for _ in range(1024)], n_heads=32, n_kv_heads=8)):
        best = {}
        for _ in range(25):
            for bits in (16, 8):
                t = time.perf_counter()
                P.attend_items(head_dim=128, page_tokens=16, bits=bits, **kw)
                best[bits] = min(best.get(bits, 1e9), time.perf_counter() - t)
        assert best[8] <= 6 * best[16], best


@pytest.mark.parametrize("name,kind", [("op_attend_plan", P._AttendPlan), ("op_attend8_plan", P._AttendPlan8)])
def test_a_short_buffer_is_told_what_is_needed(name, kind):
    q, kv = np.ones(30, np.int32), np.full(30, 20000, np.int32)
    d = P._AttendDesc(30, 8, 2, 64, 16, 0, q.ctypes.data, kv.ctypes.data, None, None, None)
    call, plan, want = getattr(P.lib(), name), kind(), kind()
    assert call(C.addressof(d), 152, C.addressof(want), None, 0) == G.GMG_OK
    items = np.full(want.plan_bytes // 4 + 8, 7, np.int32)
    assert call(C.addressof(d), 152, C.addressof(plan), items.ctypes.data, want.plan_bytes - 4) == G.GMG_EWS
    assert bytes(plan) == bytes(want) and bool((items == 7).all())
    assert call(C.addressof(d), 152, C.addressof(plan), items.ctypes.data, want.plan_bytes) == G.GMG_OK
    assert bytes(plan) == bytes(want) and bool((items[-8:] == 7).all())
