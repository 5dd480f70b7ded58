// What the attention kernels share: work items and how a batch is cut into them, and the join of
// partial results.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <functional>
#include <map>
#include <utility>
#include <vector>

#include "../../include/gmgop.h"
#include "gmgop_pairs.cuh"

namespace gop {
namespace {

constexpr int32_t kSeesAll = 0x7f000000;
constexpr int32_t kMaxLen = 1 << 30;   // of a request: no cache holds more, and lengths rounded up to steps stay in 32 bits

struct Item {
  int32_t tok0, n_tok;                 // queries
  int32_t row;                         // of the table
  int32_t lo, hi;                      // keys
  int32_t pos0;                        // position of the first query; kSeesAll: no query is before a key
  int32_t part;                        // first row of its partial results, or -1: the result itself
  int32_t reserved;
};

// Queries whose results are joined from n[i] parts of step[i] rows each, from row base[i] on:
// those of the prefix (0) and of what follows it (1).
struct Join {
  int32_t tok0, n_tok;
  int32_t base[2], step[2], n[2];
};

struct AttendArgs {
  const Item* items;
  const Join* joins;
  const int32_t* table;
  int32_t* status;
  int32_t max_pages, page_tokens, n_pages, planes, plane;   // planes of the pool: a page's layers and K, V
  int32_t n_heads, n_kv, group, dim;
  float scale2;                        // |scale| log2 e, > 0
  int32_t negative;                    // the products take -Q
  void* out;
  int64_t o_tok, o_head;
  float* lse;
  float *part_o, *part_lse;            // [n_kv][part_rows][dim], [n_kv][part_rows], log2
  int64_t part_rows;
};

// Joins the parts of a query head: o = sum_i 2^(lse_i - L) o_i with L = log2 sum_i 2^lse_i.  A
// warp takes one head of a token, a lane four elements; with more than 8 parts a block does: its
// four warps every fourth part, and their sums are then added in order (us a call, a warp / a block:
// one request of 32,000 tokens, 42 parts, 31.7 / 26.6; 96 requests of nine parts 72.6 / 72.2; 32 requests
// of eight drafted tokens, few parts, 29.1 / 33.4).
template <class T>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float4 sums[3][32];
  __shared__ float weights[3];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const Join j = a.joins[blockIdx.x];
  const int32_t all = j.n_tok * a.n_heads, n = j.n[0] + j.n[1];
  const bool wide = n > 8;
  for (int32_t w0 = blockIdx.y * (wide ? 1 : 4); w0 < all; w0 += gridDim.y * (wide ? 1 : 4)) {
    const int32_t w = wide ? w0 : w0 + warp;
    if (w >= all) break;
    const int32_t tok = w / a.n_heads, h = w - tok * a.n_heads, hk = h / a.group;
    const int32_t r = tok * a.group + h - hk * a.group;
    auto row_of = [&](int32_t i) {
      return hk * a.part_rows + r +
             (i < j.n[0] ? j.base[0] + (int64_t)i * j.step[0] : j.base[1] + (int64_t)(i - j.n[0]) * j.step[1]);
    };
    float top = -INFINITY;
    for (int32_t i = lane; i < n; i += 32) top = fmaxf(top, __ldcg(a.part_lse + row_of(i)));
#pragma unroll
    for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float ref = top == -INFINITY ? 0.f : top;
    float4 o = {};
    float sum = 0.f;
#pragma unroll 4
    for (int32_t i = wide ? warp : 0; i < n; i += wide ? 4 : 1) {
      const int64_t row = row_of(i);
      const float f = exp2f(__ldcg(a.part_lse + row) - ref);
      sum += f;
      if (lane * 4 < a.dim) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part_o + row * a.dim + lane * 4));
        o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      }
    }
    if (wide) {
      if (warp > 0) {
        sums[warp - 1][lane] = o;
        if (lane == 0) weights[warp - 1] = sum;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const float4 v = sums[i][lane];
        o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
        sum += weights[i];
      }
      __syncthreads();
    }
    if (!wide || warp == 0) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int64_t t = j.tok0 + tok;
      if (lane * 4 < a.dim) {
        uint2 v;
        v.x = pack(T(), o.x * inv, o.y * inv);
        v.y = pack(T(), o.z * inv, o.w * inv);
        *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head + lane * 4) = v;
      }
      if (a.lse && lane == 0) a.lse[t * a.n_heads + h] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
    }
  }
}

inline bool desc_ok(const op_attend_desc_t* d, int32_t rows) {
  if (!d || d->n_batch < 0 || d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads || d->n_groups < 0)
    return false;
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8) return false;
  if (d->page_tokens < 8 || d->page_tokens > 256 || (d->page_tokens & (d->page_tokens - 1))) return false;
  if (d->n_heads / d->n_kv_heads > rows) return false;
  if (d->n_batch > 0 && (!d->q_len || !d->kv_len)) return false;
  int64_t total = 0;
  for (int32_t b = 0; b < d->n_batch; ++b) {
    if (d->q_len[b] < 0 || d->kv_len[b] < 0 || (d->seq && d->seq[b] < 0)) return false;
    if (d->q_len[b] > kMaxLen || d->kv_len[b] > kMaxLen) return false;
    total += d->q_len[b];
  }
  if (total > 0x7fffffff / d->n_heads) return false;
  if (d->n_groups > 0) {
    if (!d->group_off || !d->prefix || d->group_off[0] != 0 || d->group_off[d->n_groups] != d->n_batch) return false;
    for (int32_t g = 0; g < d->n_groups; ++g) {
      if (d->group_off[g + 1] < d->group_off[g] || d->prefix[g] < 0) return false;
      for (int32_t b = d->group_off[g]; b < d->group_off[g + 1]; ++b)
        if (d->prefix[g] > 0 && d->prefix[g] > d->kv_len[b] - d->q_len[b]) return false;
    }
  }
  return true;
}

// The work items of a batch, cut so that they fill the SMs (two blocks each).
struct Work {
  std::vector<Item> items;
  std::vector<Join> joins;
  int64_t part_rows = 0;
};

// A run of queries against a run of keys, before it is cut along the keys.
struct Run {
  int32_t tok0, n_tok, row, lo, hi, pos0;
  bool pooled;        // over the requests of a group
};

// How a kernel's work is cut: the keys of a step and the rows of a tile, and, in steps:
struct Cutting {
  int32_t keys, rows;
  int64_t min_steps;     // of an item that is cut
  int64_t alone_steps;   // up to so many a block takes alone, where one round of blocks is enough
  int64_t item_steps;    // what an item costs beyond its steps
  int64_t join_steps;    // what writing and joining a tile's partial results costs
  bool balanced;         // cut so that the blocks' rounds come out even, not only into as many items as blocks run at once
};

inline int64_t steps_of(const Run& r, const Cutting& cut) {
  return r.hi > r.lo ? (r.hi + cut.keys - 1) / cut.keys - r.lo / cut.keys : 0;
}
inline int64_t parts_of(int64_t steps, int64_t most) { return std::max<int64_t>(1, (steps + most - 1) / most); }

// Of some lengths up to `most`, the one with which blocks that start one after another, the longest first, on
// `slots` places end first.  Equal blocks and places that are free at the same time are taken together: a decode
// step of 64 requests is a few dozen moves and not 500 (a plan 40 us where block by block it took 529).
inline int64_t even_cut(const std::vector<Run>& runs, int32_t heads, int64_t slots, int64_t most, const Cutting& cut) {
  int64_t best = most, best_end = -1;
  bool pooled = false;
  std::vector<int64_t> lengths;
  lengths.reserve(runs.size());
  for (const Run& r : runs) lengths.push_back(steps_of(r, cut)), pooled |= r.pooled;
  std::sort(lengths.begin(), lengths.end(), std::greater<int64_t>());
  std::vector<std::pair<int64_t, int64_t>> sizes;                // and how many there are
  std::map<int64_t, int64_t> places;                             // when they are free, and how many then
  for (int64_t k = 1; k <= 6; ++k) {
    const int64_t most_k = std::max(cut.min_steps, (most + k - 1) / k);
    sizes.clear();
    bool joins = pooled;
    int64_t blocks = 0;
    for (size_t i = 0; i < lengths.size();) {
      const int64_t n = lengths[i], parts = parts_of(n, most_k);
      int64_t same = 0;
      for (; i < lengths.size() && lengths[i] == n; ++i) ++same;
      joins |= parts > 1;
      blocks += same * parts;
      if (n % parts) sizes.emplace_back(n / parts + 1 + cut.item_steps, same * (n % parts));
      sizes.emplace_back(n / parts + cut.item_steps, same * (parts - n % parts));
    }
    if (blocks * heads > 40 * slots) break;                      // (so many come out even by themselves)
    std::sort(sizes.begin(), sizes.end(), std::greater<std::pair<int64_t, int64_t>>());
    places.clear();
    places[0] = slots;
    for (const auto& size : sizes)
      for (int64_t left = size.second * heads; left > 0;) {
        const auto first = places.begin();
        const int64_t now = first->first, n = std::min(left, first->second);
        if (n == first->second) places.erase(first);
        else first->second -= n;
        places[now + size.first] += n;
        left -= n;
      }
    const int64_t end = places.rbegin()->first + (joins ? cut.join_steps : 0);
    if (best_end < 0 || end < best_end) best = most_k, best_end = end;
    if (most_k == cut.min_steps) break;
  }
  return best;
}

// A batch's runs and the longest part that they are cut into.
struct Runs {
  std::vector<Run> runs;
  int64_t most;
};

inline void list_runs(const op_attend_desc_t& d, int64_t n_sm, const Cutting& cut, Runs* to) {
  const int32_t keys = cut.keys, tile = cut.rows / (d.n_heads / d.n_kv_heads);
  // a small step, which one round of blocks takes with a few steps each: apart and uncut, so that
  // nothing is left to join
  int64_t alone = 0, longest = 0;
  for (int32_t b = 0; b < d.n_batch; ++b) {
    alone += (d.q_len[b] + tile - 1) / tile;
    if (d.q_len[b] > 0) longest = std::max<int64_t>(longest, (d.kv_len[b] + keys - 1) / keys);
  }
  const bool small = alone * d.n_kv_heads <= 2 * n_sm && longest <= cut.alone_steps;
  std::vector<Run>& runs = to->runs;
  const int32_t ng = d.n_groups > 0 ? d.n_groups : 1;
  int32_t tok = 0;
  for (int32_t g = 0; g < ng; ++g) {
    const int32_t b0 = d.n_groups > 0 ? d.group_off[g] : 0, b1 = d.n_groups > 0 ? d.group_off[g + 1] : d.n_batch;
    const int32_t prefix = d.n_groups > 0 ? d.prefix[g] : 0;
    int64_t tokens = 0, apart = 0;
    int32_t lead = -1;
    for (int32_t b = b0; b < b1; ++b) {
      tokens += d.q_len[b];
      apart += (d.q_len[b] + tile - 1) / tile;
      if (lead < 0 && d.q_len[b] > 0) lead = b;
    }
    // together, the prefix is read once a tile of all queries; apart, once a tile of each request's
    // (at the price of partial results to join: the steps that it saves have to outweigh them)
    const int64_t together = (tokens + tile - 1) / tile;
    const bool pool = !small && (apart - together) * (prefix / keys) > cut.join_steps * together + apart;
    if (pool)
      for (int64_t t = 0; t < tokens; t += tile)
        runs.push_back(Run{int32_t(tok + t), int32_t(std::min<int64_t>(tile, tokens - t)), d.seq ? d.seq[lead] : lead, 0,
                           prefix, kSeesAll, true});
    for (int32_t b = b0; b < b1; ++b) {
      const int32_t q = d.q_len[b], before = d.kv_len[b] - q;
      for (int32_t t = 0; t < q; t += tile) {
        const int32_t n = std::min(tile, q - t), lo = pool ? prefix : 0;
        runs.push_back(Run{tok + t, n, d.seq ? d.seq[b] : b, lo, std::max(before + t + n, lo), before + t, false});
      }
      tok += q;
    }
  }
  int64_t steps = 0;
  for (const Run& r : runs) steps += steps_of(r, cut) + cut.item_steps;
  to->most = std::max(small ? cut.alone_steps : cut.min_steps, (steps * d.n_kv_heads + 2 * n_sm - 1) / (2 * n_sm));
  if (cut.balanced && !small) to->most = even_cut(runs, d.n_kv_heads, 2 * n_sm, to->most, cut);
}

// What they come to in steps, with what the items cost beyond theirs.
inline int64_t all_steps(const Runs& from, const Cutting& cut) {
  int64_t steps = 0;
  for (const Run& r : from.runs) steps += steps_of(r, cut) + parts_of(steps_of(r, cut), from.most) * cut.item_steps;
  return steps;
}

inline void cut_runs(const op_attend_desc_t& d, const Runs& from, const Cutting& cut, Work* w) {
  const std::vector<Run>& runs = from.runs;
  const int32_t keys = cut.keys, group = d.n_heads / d.n_kv_heads, tile = cut.rows / group;
  // cut; then longest first, so that short items fill the end (equal ones keep their order:
  // tiles that read the same keys stay together)
  struct Cut {
    int32_t run, part, parts;
  };
  std::vector<int32_t> parts(runs.size()), base(runs.size(), -1), joined(runs.size(), 0);
  for (size_t i = 0; i < runs.size(); ++i) parts[i] = int32_t(parts_of(steps_of(runs[i], cut), from.most));
  // a request's queries are joined where a pooled run covers them too, or where they are cut
  size_t pooled = 0, pooled_end = 0;   // runs of the current group's pool
  for (size_t i = 0; i < runs.size(); ++i) {
    if (runs[i].pooled) {
      if (i == 0 || !runs[i - 1].pooled) pooled = i;
      pooled_end = i + 1;
      base[i] = int32_t(w->part_rows);
      w->part_rows += (int64_t)parts[i] * runs[i].n_tok * group;
      continue;
    }
    const Run& r = runs[i];
    const bool covered = pooled_end > pooled && r.lo > 0 && r.tok0 >= runs[pooled].tok0 &&
                         r.tok0 < runs[pooled_end - 1].tok0 + runs[pooled_end - 1].n_tok;
    if (!covered && parts[i] == 1) continue;
    base[i] = int32_t(w->part_rows);
    w->part_rows += (int64_t)parts[i] * r.n_tok * group;
    for (int32_t t = r.tok0; t < r.tok0 + r.n_tok;) {
      Join jn{};
      jn.tok0 = t;
      jn.n_tok = r.tok0 + r.n_tok - t;
      if (covered) {
        const size_t q = pooled + (t - runs[pooled].tok0) / tile;
        jn.n_tok = std::min(jn.n_tok, runs[q].tok0 + runs[q].n_tok - t);
        jn.base[0] = base[q] + (t - runs[q].tok0) * group;
        jn.step[0] = runs[q].n_tok * group;
        jn.n[0] = parts[q];
      }
      jn.base[1] = base[i] + (t - r.tok0) * group;
      jn.step[1] = r.n_tok * group;
      jn.n[1] = parts[i];
      w->joins.push_back(jn);
      t += jn.n_tok;
    }
  }
  std::vector<Cut> cuts;
  for (size_t i = 0; i < runs.size(); ++i) {
    if (runs[i].pooled && i > 0 && runs[i - 1].pooled && runs[i - 1].row == runs[i].row && parts[i - 1] == parts[i]) continue;
    size_t last = i + 1;    // tiles of one pool: part by part, so that those of one part meet in the L2 cache
    while (runs[i].pooled && last < runs.size() && runs[last].pooled && runs[last].row == runs[i].row && parts[last] == parts[i]) ++last;
    for (int32_t p = 0; p < parts[i]; ++p)
      for (size_t k = i; k < last; ++k) cuts.push_back(Cut{int32_t(k), p, parts[k]});
  }
  std::stable_sort(cuts.begin(), cuts.end(), [&](const Cut& x, const Cut& y) {
    return steps_of(runs[x.run], cut) / x.parts > steps_of(runs[y.run], cut) / y.parts;
  });
  for (const Cut& c : cuts) {
    const Run& r = runs[c.run];
    const int64_t s0 = r.lo / keys, n = steps_of(r, cut);
    const int64_t a = s0 + n * c.part / c.parts, b = s0 + n * (c.part + 1) / c.parts;
    Item it{};
    it.tok0 = r.tok0, it.n_tok = r.n_tok, it.row = r.row, it.pos0 = r.pos0;
    it.lo = std::max(r.lo, int32_t(a * keys));
    it.hi = int32_t(std::min<int64_t>(r.hi, b * keys));
    if (n == 0) it.lo = it.hi = 0;
    it.part = base[c.run] < 0 ? -1 : base[c.run] + c.part * r.n_tok * group;
    w->items.push_back(it);
  }
}

inline int fill_plan(const op_attend_desc_t* d, const Work& w, op_attend_plan_t* plan, int32_t* items, size_t item_bytes) {
  if (w.part_rows > 0x7fffffff || (int64_t)w.items.size() * d->n_kv_heads > 0x7fffffff) return GMG_ERANGE;
  op_attend_plan_t p{};
  p.n_batch = d->n_batch;
  p.n_heads = d->n_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.head_dim = d->head_dim;
  p.page_tokens = d->page_tokens;
  p.n_items = int32_t(w.items.size());
  p.n_joins = int32_t(w.joins.size());
  for (int32_t b = 0; b < d->n_batch; ++b) {
    p.n_tokens += d->q_len[b];
    p.max_seq = std::max(p.max_seq, d->seq ? d->seq[b] : b);
    p.max_kv = std::max(p.max_kv, d->kv_len[b]);
  }
  for (const Join& j : w.joins) p.join_tokens = std::max(p.join_tokens, j.n_tok);
  p.part_rows = w.part_rows;
  p.plan_bytes = sizeof(Item) * w.items.size() + sizeof(Join) * w.joins.size();
  p.work_bytes = 256 + size_t(w.part_rows) * d->n_kv_heads * (d->head_dim + 1) * 4;
  *plan = p;
  if (items) {
    if (item_bytes < p.plan_bytes) return GMG_EWS;
    Item* to = reinterpret_cast<Item*>(items);
    std::copy(w.items.begin(), w.items.end(), to);
    std::copy(w.joins.begin(), w.joins.end(), reinterpret_cast<Join*>(to + w.items.size()));
  }
  return GMG_OK;
}

}  // namespace
}  // namespace gop
