// Keys and values into a paged cache in 8 bits, with the rotation applied on the way.  The C ABI is
// declared in include/gmgop.h.
//
// The unit is a run: the tokens of the call that one block of 16 takes, one after another in the
// lists (what is not written may lie between).  Its first token speaks for it.  A warp takes a run of one head's keys or values: up to
// 16 tokens lie in its registers while their largest magnitude is found, the block's scale
// follows, and the codes are written once.  Scales are powers of two, so a block whose scale grows
// is rounded again only where its codes become subnormal, and x / scale is exact.
// A thread block serves a share of `chunk` tokens' heads: sines and cosines once for all of them, as
// in the cache of 16-bit values.  A run that reaches past its block's tokens is taken whole by the
// block that it begins in.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gmgop.h"
#include "gmgop_host.h"
#include "gmgop_rope.cuh"

namespace gop {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;          // tokens of a block where there are many
constexpr int kBlock = kScaleTokens;
constexpr int kReach = 32;          // entries of the lists that a run lies in
constexpr int kWindow = kChunk + 2 * kReach;
constexpr int kSteps = kBlock * 128 / 8 / 32;   // 8 elements each, of a lane

struct AppendArgs {
  const uint64_t* freq;
  int32_t half;                     // pairs
  int32_t interleaved;
  float factor;
  int64_t n_tokens;
  int32_t chunk, n_heads, n_kv, dim;
  const void *q, *k, *v;
  void* out;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
  const int32_t *pos, *seq;
  op_cache_t cache;
  int64_t page_bytes, codes_at, scales_at;   // of a page; of the layer's codes and scales in it
};

// The least power of two, from 2^-60 to 2^60, that brings `top` (>= 0, finite) to at most 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float top) {
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000);
  return __uint_as_float((uint32_t)(127 + (e < -60 ? -60 : e > 60 ? 60 : e)) << 23);
}

// Two values to codes, rounded to nearest even; beyond 448 the largest, NaN stays.
__device__ __forceinline__ uint16_t narrow2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 narrow8(const float* v, float by) {
  uint2 r;
  r.x = narrow2(v[0] * by, v[1] * by) | (uint32_t)narrow2(v[2] * by, v[3] * by) << 16;
  r.y = narrow2(v[4] * by, v[5] * by) | (uint32_t)narrow2(v[6] * by, v[7] * by) << 16;
  return r;
}
__device__ __forceinline__ void wide8(uint2 c, float* v) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t two;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"((uint16_t)(w[i / 2] >> (16 * (i % 2)))));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&two));
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}

template <class T, bool kWide>
__device__ __forceinline__ void load8(const T* x, float* v) {
  if (kWide) {
    const Vec<T, 8> a = *reinterpret_cast<const Vec<T, 8>*>(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = up(a.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = up(x[i]);
  }
}

// Elements at .. at + 7 of a head x, rotated.
template <class T, bool kWide>
__device__ __forceinline__ void turned8(const T* x, int at, int half, bool inter, const float2* cs, float* v) {
  load8<T, kWide>(x + at, v);
  if (at >= 2 * half) return;
  if (kWide) {
    if (inter) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 t = cs[at / 2 + i];
        const float u = v[2 * i], w = v[2 * i + 1];
        v[2 * i] = u * t.x - w * t.y, v[2 * i + 1] = u * t.y + w * t.x;
      }
    } else {
      const bool second = at >= half;
      float o[8];
      load8<T, true>(x + (second ? at - half : at + half), o);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 t = cs[(second ? at - half : at) + i];
        v[i] = second ? o[i] * t.y + v[i] * t.x : v[i] * t.x - o[i] * t.y;
      }
    }
  } else {
    for (int i = 0; i < 8; ++i) {
      const int e = at + i;
      if (e >= 2 * half) break;
      const bool second = inter ? e & 1 : e >= half;
      const int pair = inter ? e / 2 : second ? e - half : e;
      const float o = up(x[inter ? e ^ 1 : second ? e - half : e + half]);
      const float2 t = cs[pair];
      v[i] = second ? o * t.y + v[i] * t.x : v[i] * t.x - o * t.y;
    }
  }
}

template <class T, bool kWide, bool kInter>
__global__ void __launch_bounds__(kThreads) append8_kernel(const __grid_constant__ AppendArgs a) {
  extern __shared__ float2 cs[];          // [chunk + 15][half]: of the block's own tokens, then of those that its last run takes beyond
  __shared__ int32_t pos[kWindow], seq[kWindow];   // from kReach entries before the block's first; seq -1: not written
  __shared__ int32_t run_n[kChunk], n_runs, n_more, more[kBlock];
  __shared__ unsigned char run_at[kChunk][kBlock], run_cs[kChunk][kBlock];   // a run's tokens: their entries, their rows of cs
  const int64_t t0 = (int64_t)blockIdx.x * a.chunk;
  const int own = a.n_tokens - t0 < a.chunk ? int(a.n_tokens - t0) : a.chunk;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int32_t page = a.cache.page_tokens;
  if (threadIdx.x < own + 2 * kReach) {
    const int64_t t = t0 + threadIdx.x - kReach;
    int32_t p = 0, r = -1;
    if (t >= 0 && t < a.n_tokens) {
      p = a.pos[t], r = a.seq[t];
      if (r >= 0) {
        const int32_t col = p >= 0 ? p / page : -1;
        int32_t at = -1;
        if (r < a.cache.n_seq && col >= 0 && col < a.cache.max_pages) at = a.cache.table[int64_t(r) * a.cache.max_pages + col];
        if (at < 0 || at >= a.cache.n_pages) {
          r = -1;
          if (blockIdx.y == 0 && t >= t0 && t < t0 + own) atomicAdd(&a.cache.status[4], 1);
        }
      }
    }
    pos[threadIdx.x] = p;
    seq[threadIdx.x] = r;
  }
  if (threadIdx.x == 0) n_more = 0;
  __syncthreads();
  if (warp == 0) {
    // the tokens with which a run begins: the one written before them is another block's
    const int i = lane + kReach;
    bool head = lane < own && seq[i] >= 0;
    auto joined = [&](int x, int y) { return seq[x] == seq[y] && pos[x] < pos[y] && pos[x] / kBlock == pos[y] / kBlock; };
    if (head) {
      int x = i - 1;
      while (x > i - kReach && seq[x] < 0) --x;
      if (seq[x] >= 0 && joined(x, i)) head = false;
    }
    const uint32_t heads = __ballot_sync(0xffffffffu, head);
    if (head) {
      const int r = __popc(heads & ((1u << lane) - 1));
      int n = 0, beyond = 0;
      for (int x = i, y = i; y < i + kReach && n < kBlock; ++y) {
        if (seq[y] < 0) continue;
        if (y > i && !joined(x, y)) break;
        run_at[r][n] = (unsigned char)y;
        if (y - kReach < own) {
          run_cs[r][n] = (unsigned char)(y - kReach);
        } else {   // (the block's last run alone comes here)
          more[beyond] = y;
          run_cs[r][n] = (unsigned char)(own + beyond++);
        }
        ++n;
        x = y;
      }
      run_n[r] = n;
      if (beyond) n_more = beyond;
    }
    if (lane == 0) n_runs = __popc(heads);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (own + n_more) * a.half; i += kThreads) {
    const int t = i / a.half, p = i - t * a.half;
    // (a token that is not written is turned all the same: its query)
    cs[i] = turn_of(a.freq[p], pos[t < own ? t + kReach : more[t - own]], a.factor, a.factor);
  }
  __syncthreads();

  // runs: a warp a head's keys or values
  const int vecs = a.dim / 8, units = n_runs * 2 * a.n_kv;
  for (int u = blockIdx.y * (kThreads / 32) + warp; u < units; u += gridDim.y * (kThreads / 32)) {
    const int run = u / (2 * a.n_kv), x = u - run * 2 * a.n_kv, is_v = x / a.n_kv, h = x - is_v * a.n_kv;
    const int at = run_at[run][0], n = run_n[run] * vecs;
    const int32_t p0 = pos[at];
    const int64_t p = a.cache.table[int64_t(seq[at]) * a.cache.max_pages + p0 / page];
    unsigned char* in = static_cast<unsigned char*>(a.cache.pool) + p * a.page_bytes;
    const int head = is_v * a.n_kv + h, slot0 = p0 % page / kBlock * kBlock;
    float* scale_at = reinterpret_cast<float*>(in + a.scales_at) + head * (page / kBlock) + slot0 / kBlock;
    unsigned char* codes = in + a.codes_at + (int64_t(head) * page + slot0) * a.dim;
    const int kept = p0 % kBlock;
    float old = kept ? *scale_at : 0.f;
    const T* from = is_v ? static_cast<const T*>(a.v) + (t0 - kReach) * a.v_tok + h * a.v_head
                         : static_cast<const T*>(a.k) + (t0 - kReach) * a.k_tok + h * a.k_head;
    const int64_t row = is_v ? a.v_tok : a.k_tok;
    float v[kSteps][8], top = 0.f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int i = lane + 32 * s, tok = i / vecs, c = i - tok * vecs;
      if (32 * s >= n) break;
      if (i < n) {
        const T* x = from + run_at[run][tok] * row;
        if (is_v) load8<T, kWide>(x + c * 8, v[s]);
        else turned8<T, kWide>(x, c * 8, a.half, kInter, cs + run_cs[run][tok] * a.half, v[s]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float m = fabsf(v[s][k]);
          if (m <= 3.402823466e38f) top = fmaxf(top, m);   // (infinities and NaN do not count)
        }
      }
    }
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    float scale = scale_for(top);
    if (kept) {
      old = fminf(fmaxf(old, 8.67361738e-19f), 1.15292150e18f);   // 2^-60 .. 2^60, NaN the least
      if (scale > old) {   // what the block holds before this run is rounded to the larger scale
        const float by = old / scale;
        for (int i = lane; i < kept * vecs; i += 32) {
          float w[8];
          uint2* c = reinterpret_cast<uint2*>(codes + i * 8);
          wide8(*c, w);
          *c = narrow8(w, by);
        }
      } else {
        scale = old;
      }
    }
    const float by = 1.f / scale;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int i = lane + 32 * s, tok = i / vecs, c = i - tok * vecs;
      if (32 * s >= n) break;
      if (i < n)
        *reinterpret_cast<uint2*>(codes + (pos[run_at[run][tok]] % kBlock) * a.dim + c * 8) = narrow8(v[s], by);
    }
    if (lane == 0) *scale_at = scale;
  }

  // queries: as dense ones
  constexpr int N = kWide ? 8 : 1;
  using V = Vec<T, N>;
  const int turns = kInter ? (N == 1 ? a.half : 2 * a.half / N) : a.half / N;
  const int each = turns + (a.dim - 2 * a.half) / N, per = a.n_heads * each;
  for (int w = blockIdx.y * kThreads + threadIdx.x; w < own * per; w += gridDim.y * kThreads) {
    const int tok = w / per, y = w - tok * per, h = y / each, step = y - h * each;
    const T* from = static_cast<const T*>(a.q) + (t0 + tok) * a.q_tok + h * a.q_head;
    T* to = static_cast<T*>(a.out) + (t0 + tok) * a.o_tok + h * a.o_head;
    if (step < turns) {
      turn_step<T, N, kInter>(from, to, step, a.half, cs + tok * a.half);
    } else {
      const int o = 2 * a.half + (step - turns) * N;
      *reinterpret_cast<V*>(to + o) = *reinterpret_cast<const V*>(from + o);
    }
  }
}

template <class T, bool kWide, bool kInter>
cudaError_t launch(AppendArgs a, cudaStream_t st) {
  // where there are many tokens a block takes 16 of them, so that most runs' sines are those of its
  // queries too; else one, in shares
  a.chunk = a.n_tokens >= 152 * 2 * kChunk ? kChunk : 1;
  const int64_t blocks = (a.n_tokens + a.chunk - 1) / a.chunk;
  const int64_t steps = int64_t(a.chunk) * (a.n_heads + 2 * a.n_kv) * (a.dim / 8);
  int64_t split = (152 * 4 + blocks - 1) / blocks;
  if (split > (steps + kThreads - 1) / kThreads) split = (steps + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)blocks, (unsigned)(split < 1 ? 1 : split));
  append8_kernel<T, kWide, kInter><<<grid, kThreads, (a.chunk + kBlock - 1) * a.half * sizeof(float2), st>>>(a);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_type(const AppendArgs& a, bool wide, cudaStream_t st) {
  if (wide) return a.interleaved ? launch<T, true, true>(a, st) : launch<T, true, false>(a, st);
  return a.interleaved ? launch<T, false, true>(a, st) : launch<T, false, false>(a, st);
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" int op_rope_append8(const op_rope_t* rope, const op_cache_t* cache, int32_t layer, int32_t dtype,
                               int64_t n_tokens, int32_t n_heads, const void* q, int64_t q_tok, int64_t q_head,
                               const void* k, int64_t k_tok, int64_t k_head, const void* v, int64_t v_tok,
                               int64_t v_head, const int32_t* pos, const int32_t* seq, void* q_out, int64_t o_tok,
                               int64_t o_head, gmg_stream_t stream) {
  if (!cache8_ok(cache) || layer < 0 || layer >= cache->n_layers) return GMG_EINVAL;
  if (dtype != GMG_OP_BF16 && dtype != GMG_OP_F16) return GMG_EINVAL;
  if (!rope || (rope->rotary > 0 && !rope->freq) || rope->rotary < 0 || rope->rotary % 2 || rope->rotary > cache->head_dim)
    return GMG_EINVAL;
  if (n_tokens < 0 || n_tokens > 0x7fffffff || n_heads < 0) return GMG_EINVAL;
  if ((n_heads + int64_t(2) * cache->n_kv_heads) * cache->head_dim > (1 << 24)) return GMG_EINVAL;
  if (n_tokens == 0) return GMG_OK;
  if (!pos || !seq || !k || !v || (n_heads > 0 && (!q || !q_out))) return GMG_EINVAL;
  AppendArgs a{};
  a.freq = rope->freq;
  a.half = rope->rotary / 2;
  a.interleaved = rope->interleaved;
  a.factor = rope->factor;
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
  a.cache = *cache;
  a.page_bytes = page8_bytes(*cache);
  a.codes_at = int64_t(layer) * 2 * a.n_kv * cache->page_tokens * a.dim;
  a.scales_at = page8_scales(*cache) + int64_t(layer) * 2 * a.n_kv * (cache->page_tokens / kScaleTokens) * 4;
  // 16 bytes a step where every head starts on 16 bytes and the halves are whole steps
  bool wide = rope->rotary % (rope->interleaved ? 8 : 16) == 0 && aligned(k, k_tok, k_head, 2) && aligned(v, v_tok, v_head, 2);
  if (n_heads > 0) wide = wide && aligned(q, q_tok, q_head, 2) && aligned(q_out, o_tok, o_head, 2);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t rc = dtype == GMG_OP_BF16 ? launch_type<__nv_bfloat16>(a, wide, st) : launch_type<__half>(a, wide, st);
  return rc == cudaSuccess ? GMG_OK : GMG_ECUDA;
}
