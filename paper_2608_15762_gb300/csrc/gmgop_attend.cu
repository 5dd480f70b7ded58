// Attention over a paged cache.  The C ABI is declared in include/gmgop.h.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/gmgop.h"
#include "gmgop_host.h"

namespace gop {
namespace {

// A request of the plan.
struct Item {
  int32_t tok0, n_q, row, kv;
};

__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
__device__ __forceinline__ void down(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void down(float v, __half* o) { *o = __float2half_rn(v); }

struct AttendArgs {
  op_cache_t cache;
  const Item* items;
  int32_t n_items, n_heads;
  int64_t n_tokens;
  const void* q;
  void* out;
  float* lse;
  int64_t q_tok, q_head, o_tok, o_head, page_stride, layer_at;
  float scale;
};

// A warp takes one query head: its lanes hold four elements each and go through the
// keys one by one, with the running maximum and sum.
template <class T>
__global__ void __launch_bounds__(128) attend_kernel(AttendArgs a) {
  const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (w >= a.n_tokens * a.n_heads) return;
  const int64_t t = w / a.n_heads;
  const int32_t h = int32_t(w % a.n_heads), hk = h / (a.n_heads / a.cache.n_kv_heads), D = a.cache.head_dim;
  int32_t lo = 0, hi = a.n_items - 1;   // the last item that starts at or before t (those without queries share a start)
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) / 2;
    if (a.items[mid].tok0 <= t) lo = mid;
    else hi = mid - 1;
  }
  const Item it = a.items[lo];
  const int64_t see = (int64_t)it.kv - it.n_q + (t - it.tok0) + 1;
  float q[4], o[4] = {}, m = -INFINITY, l = 0.f;
  for (int j = 0; j < 4; ++j) {
    const int d = lane * 4 + j;
    q[j] = d < D ? up(static_cast<const T*>(a.q)[t * a.q_tok + h * a.q_head + d]) * a.scale : 0.f;
  }
  for (int64_t k = 0; k < see; ++k) {
    const int32_t page = a.cache.table[int64_t(it.row) * a.cache.max_pages + k / a.cache.page_tokens];
    if (page < 0 || page >= a.cache.n_pages) continue;
    const T* key = static_cast<const T*>(a.cache.pool) + page * a.page_stride + a.layer_at +
                   (int64_t(hk) * a.cache.page_tokens + k % a.cache.page_tokens) * D;
    const T* val = key + int64_t(a.cache.n_kv_heads) * a.cache.page_tokens * D;
    float s = 0.f, v[4];
    for (int j = 0; j < 4; ++j) {
      const int d = lane * 4 + j;
      s += d < D ? q[j] * up(key[d]) : 0.f;
      v[j] = d < D ? up(val[d]) : 0.f;
    }
    for (int x = 16; x; x /= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
    const float n = fmaxf(m, s), f = m == n ? 1.f : expf(m - n), p = expf(s - n);
    l = l * f + p;
    for (int j = 0; j < 4; ++j) o[j] = o[j] * f + p * v[j];
    m = n;
  }
  for (int j = 0; j < 4; ++j) {
    const int d = lane * 4 + j;
    if (d < D) down(l == 0.f ? 0.f : o[j] / l, static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head + d);
  }
  if (a.lse && lane == 0) a.lse[t * a.n_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

bool desc_ok(const op_attend_desc_t* d) {
  if (!d || d->n_batch < 0 || d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads || d->n_groups < 0)
    return false;
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8) return false;
  if (d->page_tokens < 8 || d->page_tokens > 256 || (d->page_tokens & (d->page_tokens - 1))) return false;
  if (d->n_heads / d->n_kv_heads > 128) return false;
  if (d->n_batch > 0 && (!d->q_len || !d->kv_len)) return false;
  int64_t total = 0;
  for (int32_t b = 0; b < d->n_batch; ++b) {
    if (d->q_len[b] < 0 || d->kv_len[b] < 0 || (d->seq && d->seq[b] < 0)) return false;
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

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

int op_attend_plan(const op_attend_desc_t* d, int32_t n_sm, op_attend_plan_t* plan, int32_t* items,
                   size_t item_bytes) {
  if (!desc_ok(d) || !plan || n_sm < 1) return GMG_EINVAL;
  op_attend_plan_t p{};
  p.n_batch = d->n_batch;
  p.n_heads = d->n_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.head_dim = d->head_dim;
  p.page_tokens = d->page_tokens;
  p.n_items = d->n_batch;
  p.plan_bytes = sizeof(Item) * size_t(d->n_batch);
  for (int32_t b = 0; b < d->n_batch; ++b) {
    const int32_t row = d->seq ? d->seq[b] : b;
    if (items && item_bytes >= p.plan_bytes)
      reinterpret_cast<Item*>(items)[b] = Item{int32_t(p.n_tokens), d->q_len[b], row, d->kv_len[b]};
    p.n_tokens += d->q_len[b];
    if (row > p.max_seq) p.max_seq = row;
    if (d->kv_len[b] > p.max_kv) p.max_kv = d->kv_len[b];
  }
  p.work_bytes = 256;
  if (items && item_bytes < p.plan_bytes) return GMG_EWS;
  *plan = p;
  return GMG_OK;
}

int op_attend(const op_attend_plan_t* plan, const int32_t* d_items, const op_cache_t* cache, int32_t layer,
              const void* q, int64_t q_tok, int64_t q_head, float scale, void* out, int64_t out_tok, int64_t out_head,
              float* lse, void* work, size_t work_bytes, gmg_stream_t stream) {
  if (!plan || !cache_ok(cache) || layer < 0 || layer >= cache->n_layers) return GMG_EINVAL;
  if (plan->head_dim != cache->head_dim || plan->n_kv_heads != cache->n_kv_heads ||
      plan->page_tokens != cache->page_tokens || plan->max_seq >= cache->n_seq ||
      plan->max_kv > int64_t(cache->max_pages) * cache->page_tokens)
    return GMG_EINVAL;
  if (plan->n_tokens == 0) return GMG_OK;
  if (!d_items || !q || !out || !aligned(q, q_tok, q_head, 2) || !aligned(out, out_tok, out_head, 2)) return GMG_EINVAL;
  if (!work || (reinterpret_cast<uintptr_t>(work) & 255) || work_bytes < plan->work_bytes) return GMG_EWS;
  AttendArgs a{};
  a.cache = *cache;
  a.items = reinterpret_cast<const Item*>(d_items);
  a.n_items = plan->n_items;
  a.n_heads = plan->n_heads;
  a.n_tokens = plan->n_tokens;
  a.q = q, a.q_tok = q_tok, a.q_head = q_head;
  a.out = out, a.o_tok = out_tok, a.o_head = out_head;
  a.lse = lse;
  a.scale = scale;
  const int64_t plane = int64_t(cache->n_kv_heads) * cache->page_tokens * cache->head_dim;
  a.page_stride = 2 * cache->n_layers * plane;
  a.layer_at = 2 * layer * plane;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = (plan->n_tokens * plan->n_heads + 3) / 4;
  if (cache->dtype == GMG_OP_BF16) attend_kernel<__nv_bfloat16><<<(unsigned)blocks, 128, 0, st>>>(a);
  else attend_kernel<__half><<<(unsigned)blocks, 128, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // extern "C"
