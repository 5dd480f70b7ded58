// Rotary positions, dense or with keys and values written into a paged cache.
// The C ABI is declared in include/gmgop.h.
//
// An angle in turns is pos * f / (2 pi).  With f / (2 pi) as a 64-bit fraction, the
// low 64 bits of the integer product are the angle's fraction of a turn: the fraction's
// rounding, half a unit, is all that grows with the position, to 2^-34 turns at the last one,
// and no table of angles is read.  The top 32 bits are kept and rounded to fp32, 2^-26 turns.  One block
// serves one token (or a share of its heads): its threads take the sines and cosines
// of the token's pairs into shared memory once, then every head uses them.
//
// Bound by memory: 32,768 tokens of 32 + 8 + 8 heads of 128 into a cache 123 us, 6.5 TB/s
// (floor 121).  16 tokens 2.8 us, a launch; 1,537 x 20 heads of 80, fp32, 7.2 us (floor 3.0): the launch
// and a block's chain of position, frequencies, sines and only then its first load of x.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gmgop.h"
#include "gmgop_host.h"
#include "gmgop_rope.cuh"

namespace gop {
namespace {

constexpr int kThreads = 128;

struct RopeArgs {
  const uint64_t* freq;
  int32_t half;                  // pairs
  float factor, sign;
  int64_t n_tokens;
  int32_t n_heads, n_kv, dim;
  const void *q, *k, *v;
  void* out;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
  const int32_t *pos, *seq;
  op_cache_t cache;
  int64_t page_stride, layer_at;  // elements: from page to page, of the layer's keys in a page
};

template <class T, int N, bool kInter, bool kAppend>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a) {
  using V = Vec<T, N>;
  __shared__ float2 cs[kMaxPairs];
  const int64_t t = blockIdx.x;
  const int32_t pos = a.pos[t];
  for (int32_t i = threadIdx.x; i < a.half; i += kThreads) {
    cs[i] = turn_of(a.freq[i], pos, a.factor, a.factor * a.sign);
  }
  T *key = nullptr, *value = nullptr;   // this token's slot of head 0 in the cache
  if (kAppend) {
    const int32_t r = a.seq[t];
    if (r >= 0) {
      const int32_t col = pos >= 0 ? pos / a.cache.page_tokens : -1;
      int32_t page = -1;
      if (r < a.cache.n_seq && col >= 0 && col < a.cache.max_pages) page = a.cache.table[int64_t(r) * a.cache.max_pages + col];
      if (page >= 0 && page < a.cache.n_pages) {
        key = static_cast<T*>(a.cache.pool) + page * a.page_stride + a.layer_at +
              int64_t(pos % a.cache.page_tokens) * a.dim;
        value = key + int64_t(a.n_kv) * a.cache.page_tokens * a.dim;
      } else if (threadIdx.x == 0 && blockIdx.y == 0) {
        atomicAdd(&a.cache.status[4], 1);
      }
    }
  }
  __syncthreads();
  const int32_t turns = kInter ? (N == 1 ? a.half : 2 * a.half / N) : a.half / N;
  const int32_t passes = (a.dim - 2 * a.half) / N, each = turns + passes;
  const int32_t all = (a.n_heads + a.n_kv) * each;
  const int32_t copies = a.dim / N;
  const int32_t end = all + a.n_kv * copies;
  for (int32_t w = blockIdx.y * kThreads + threadIdx.x; w < end; w += gridDim.y * kThreads) {
    if (w < all) {
      const int32_t h = w / each, step = w - h * each;
      const T* x;
      T* y;
      if (h < a.n_heads) {
        x = static_cast<const T*>(a.q) + t * a.q_tok + h * a.q_head;
        y = static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head;
      } else {
        if (!key) continue;
        x = static_cast<const T*>(a.k) + t * a.k_tok + (h - a.n_heads) * a.k_head;
        y = key + int64_t(h - a.n_heads) * a.cache.page_tokens * a.dim;
      }
      if (step < turns) {
        turn_step<T, N, kInter>(x, y, step, a.half, cs);
      } else {
        const int32_t o = 2 * a.half + (step - turns) * N;
        *reinterpret_cast<V*>(y + o) = *reinterpret_cast<const V*>(x + o);
      }
    } else if (value) {
      const int32_t h = (w - all) / copies, o = (w - all - h * copies) * N;
      *reinterpret_cast<V*>(value + int64_t(h) * a.cache.page_tokens * a.dim + o) =
          *reinterpret_cast<const V*>(static_cast<const T*>(a.v) + t * a.v_tok + h * a.v_head + o);
    }
  }
}

template <class T, int N, bool kInter>
cudaError_t launch(const RopeArgs& a, bool append, cudaStream_t st) {
  // enough blocks for every SM where there are few tokens: shares of a token's heads (us, a block a
  // token / shares, 32 + 8 + 8 heads: 16 tokens 4.5 / 3.1, 200 tokens 4.6 / 4.0, 500 5.5 / 5.1)
  const int64_t steps = int64_t(a.n_heads + 2 * a.n_kv) * ((a.dim + N - 1) / N);
  int64_t split = (152 * 4 + a.n_tokens - 1) / a.n_tokens;
  if (split > (steps + kThreads - 1) / kThreads) split = (steps + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)a.n_tokens, (unsigned)(split < 1 ? 1 : split));
  if (append) rope_kernel<T, N, kInter, true><<<grid, kThreads, 0, st>>>(a);
  else rope_kernel<T, N, kInter, false><<<grid, kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_type(const RopeArgs& a, bool inter, bool append, bool wide, cudaStream_t st) {
  constexpr int N = 16 / sizeof(T);
  if (wide) return inter ? launch<T, N, true>(a, append, st) : launch<T, N, false>(a, append, st);
  return inter ? launch<T, 1, true>(a, append, st) : launch<T, 1, false>(a, append, st);
}

int run(const op_rope_t* rope, int32_t dtype, bool append, RopeArgs& a, cudaStream_t st) {
  if (!rope || (rope->rotary > 0 && !rope->freq) || rope->rotary < 0 || rope->rotary % 2 || rope->rotary > a.dim ||
      rope->rotary > 2 * kMaxPairs)
    return GMG_EINVAL;
  if (a.n_tokens < 0 || a.n_tokens > 0x7fffffff || a.n_heads < 0 || a.n_kv < 0) return GMG_EINVAL;
  if (int64_t(a.n_heads + int64_t(2) * a.n_kv) * a.dim > (1 << 30)) return GMG_EINVAL;
  if (a.n_tokens == 0 || (a.n_heads == 0 && a.n_kv == 0)) return GMG_OK;
  if (!a.pos || (a.n_heads > 0 && (!a.q || !a.out))) return GMG_EINVAL;
  a.freq = rope->freq;
  a.half = rope->rotary / 2;
  a.factor = rope->factor;
  // 16 bytes a step where every head starts on 16 bytes and the halves are whole steps, else an
  // element a step (the 32,768 tokens above: 123 us / 340)
  const int e = dtype == GMG_OP_F32 ? 4 : 2, n = 16 / e;
  const bool whole = a.dim % n == 0 && rope->rotary % (rope->interleaved ? n : 2 * n) == 0;
  bool wide = whole;
  if (a.n_heads > 0)
    wide = wide && aligned(a.q, a.q_tok, a.q_head, e) && aligned(a.out, a.o_tok, a.o_head, e);
  if (append && a.n_kv > 0) wide = wide && aligned(a.k, a.k_tok, a.k_head, e) && aligned(a.v, a.v_tok, a.v_head, e);
  cudaError_t rc;
  if (dtype == GMG_OP_F32) rc = launch_type<float>(a, rope->interleaved, append, wide, st);
  else if (dtype == GMG_OP_BF16) rc = launch_type<__nv_bfloat16>(a, rope->interleaved, append, wide, st);
  else rc = launch_type<__half>(a, rope->interleaved, append, wide, st);
  return rc == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

int op_rope(const op_rope_t* rope, int32_t dtype, int64_t n_tokens, int32_t n_heads, int32_t head_dim, const void* x,
            int64_t x_tok, int64_t x_head, const int32_t* pos, int32_t backward, void* out, int64_t out_tok,
            int64_t out_head, gmg_stream_t stream) {
  if (dtype != GMG_OP_F32 && dtype != GMG_OP_BF16 && dtype != GMG_OP_F16) return GMG_EINVAL;
  if (head_dim < 1) return GMG_EINVAL;
  RopeArgs a{};
  a.n_tokens = n_tokens;
  a.n_heads = n_heads;
  a.dim = head_dim;
  a.q = x;
  a.q_tok = x_tok;
  a.q_head = x_head;
  a.out = out;
  a.o_tok = out_tok;
  a.o_head = out_head;
  a.pos = pos;
  a.sign = backward ? -1.f : 1.f;
  return run(rope, dtype, false, a, reinterpret_cast<cudaStream_t>(stream));
}

int op_rope_append(const op_rope_t* rope, const op_cache_t* cache, int32_t layer, int64_t n_tokens, int32_t n_heads,
                   const void* q, int64_t q_tok, int64_t q_head, const void* k, int64_t k_tok, int64_t k_head,
                   const void* v, int64_t v_tok, int64_t v_head, const int32_t* pos, const int32_t* seq, void* q_out,
                   int64_t o_tok, int64_t o_head, gmg_stream_t stream) {
  if (!cache_ok(cache) || layer < 0 || layer >= cache->n_layers) return GMG_EINVAL;
  if (n_tokens > 0 && (!k || !v || !seq)) return GMG_EINVAL;
  RopeArgs a{};
  a.n_tokens = n_tokens;
  a.n_heads = n_heads;
  a.n_kv = cache->n_kv_heads;
  a.dim = cache->head_dim;
  a.q = q, a.q_tok = q_tok, a.q_head = q_head;
  a.k = k, a.k_tok = k_tok, a.k_head = k_head;
  a.v = v, a.v_tok = v_tok, a.v_head = v_head;
  a.out = q_out, a.o_tok = o_tok, a.o_head = o_head;
  a.pos = pos;
  a.seq = seq;
  a.sign = 1.f;
  a.cache = *cache;
  const int64_t plane = int64_t(cache->n_kv_heads) * cache->page_tokens * cache->head_dim;
  a.page_stride = 2 * cache->n_layers * plane;
  a.layer_at = 2 * layer * plane;
  return run(rope, cache->dtype, true, a, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
