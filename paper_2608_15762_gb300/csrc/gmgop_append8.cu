// Keys and values into a paged cache in 8 bits, with the rotation applied on the way.  The C ABI is
// declared in include/gmgop.h.
//
// The unit is a run: the tokens of the call that one block of 16 takes, one after another in the
// lists (what is not written may lie between).  Its first token speaks for it.  A warp takes a run of
// one head's keys or values: up to 16 tokens lie in its registers while their largest magnitude is
// found, the block's scale follows, and the codes are written once.  Scales are powers of two, so a block whose scale grows
// is rounded again only where its codes become subnormal, and x / scale is exact.
// What bounds it is memory, as far as the few registers allow that keep a run's loads in flight (a prompt of 32,768
// tokens, 32 + 8 + 8 heads of 128: 150 us, of them 68 for keys and values, 201 MB at 3.0 TB/s, and
// 82 for queries), and where tokens are few the chain of loads from a token's position to
// its block's scale (16 tokens 4.9 us).
// A thread block serves a share of `chunk` tokens' heads: sines and cosines once for all of them, as
// in the cache of 16-bit values.  A run that reaches past its block's tokens is taken whole by the
// block that it begins in.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/gmgop.h"
#include "gmgop_host.h"
#include "gmgop_rope.cuh"

namespace gop {
namespace {

constexpr int kThreads = 128;       // (blocks of 256: a prompt 142 us for 136, 304 requests' tokens 10.1 for 7.6)
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

__device__ __forceinline__ uint2 narrow8(const float* v, float by) {
  uint2 r;
  r.x = codes2(v[0] * by, v[1] * by) | (uint32_t)codes2(v[2] * by, v[3] * by) << 16;
  r.y = codes2(v[4] * by, v[5] * by) | (uint32_t)codes2(v[6] * by, v[7] * by) << 16;
  return r;
}
// The same of four pairs.
__device__ __forceinline__ uint2 narrow8(const uint64_t* v, uint64_t by2) {
  uint16_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x, y;
    halves(fma2(v[i], by2, 0ull), &x, &y);
    c[i] = codes2(x, y);
  }
  return uint2{c[0] | (uint32_t)c[1] << 16, c[2] | (uint32_t)c[3] << 16};
}
__device__ __forceinline__ void wide8(uint2 c, float* v) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = wide2((uint16_t)(w[i / 2] >> (16 * (i % 2))));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&two));
    v[2 * i] = f.x, v[2 * i + 1] = f.y;
  }
}

template <class T>
__device__ __forceinline__ void load8(const T* x, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = up(x[i]);
}

// Turned in 32 bits, a number may lie on the wrong side of the middle between two codes: not where it is more than
// kNear of its last bits from it (its error is about three of them, more where a pair cancels).  Looking for such numbers
// and turning them again costs a prompt of 32,768 tokens 12 us of 148 (18 with a kNear of 16), and leaves codes 50 times
// nearer to the exact ones': 8e-7 of their norm for 4e-5.
constexpr uint32_t kNear = 4, kNearTop = 2 * kNear << 12;
__device__ __forceinline__ uint32_t from_middle(float x) {   // below kNearTop: near one (codes have the first 3 of the 23 bits)
  return (__float_as_uint(x) << 12) + ((0x80000 + kNear) << 12);
}
// Those pairs of the eight that have a number near the middle of two codes, again in 64 bits.  x: as turned, to be put
// right; from: as they came; halves: their elements are 8 apart (else neighbours).  (Out of line: few warps come here.
// And short, as it is fetched then: with a function for a pair in it, 304 requests' tokens took 17.4 us for 16.4.)
__device__ __noinline__ void turn_exactly(float* x, const float* from, bool halves, int32_t pair, int32_t half,
                                          const uint64_t* freq, int32_t pos, float factor) {
#pragma unroll 1
  for (int p = 0; p < 8 && pair + p < half; ++p) {
    const int i = halves ? p : 2 * p, j = halves ? p + 8 : 2 * p + 1;
    if (from_middle(x[i]) >= kNearTop && from_middle(x[j]) >= kNearTop) continue;
    const uint64_t turn = freq[pair + p] * (uint64_t)(int64_t)pos;
    double s, c;
    sincospi((double)(int64_t)turn * 1.0842021724855044e-19, &s, &c);   // 2^-63: half turns
    const double u = from[i], w = from[j], v[2] = {(u * c - w * s) * factor, (u * s + w * c) * factor};
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      float f = (float)v[k];
      // a middle itself that was rounded to goes back to its side
      if ((__float_as_uint(f) & 0xfffff) == 0x80000 && (double)f != v[k])
        f = __uint_as_float(__float_as_uint(f) + (fabs(v[k]) > fabs((double)f) ? 1 : -1));
      x[k ? j : i] = f;
    }
  }
}

// Elements at .. at + 7 of a head x, rotated, one by one: in the same steps as whole pieces, so that codes do not depend on
// where a tensor lies.  exactly: those near a middle as above.
template <class T>
__device__ __forceinline__ void turned8(const T* x, int at, int half, bool inter, const float2* cs, bool exactly, const uint64_t* freq,
                                        int32_t pos, float factor, float* v) {
  load8(x + at, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = at + i;
    if (e >= 2 * half) break;
    const bool second = inter ? e & 1 : e >= half;
    const int pair = inter ? e / 2 : second ? e - half : e;
    const float o = up(x[inter ? e ^ 1 : second ? e - half : e + half]);
    const float u = second ? o : v[i], w = second ? v[i] : o;
    const float2 t = cs[pair];
    float r[2] = {__fmaf_rn(u, t.x, __fmul_rn(w, -t.y)),
                  inter ? __fmaf_rn(w, t.x, __fmul_rn(u, t.y)) : __fmaf_rn(u, t.y, __fmul_rn(w, t.x))};
    if (exactly && (from_middle(r[0]) < kNearTop || from_middle(r[1]) < kNearTop)) {
      const float from[2] = {u, w};
      turn_exactly(r, from, false, pair, pair + 1, freq, pos, factor);
    }
    v[i] = second ? r[1] : r[0];
  }
}

__device__ __forceinline__ float most_of(const float* v, float top) {
#pragma unroll
  for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(v[k]));   // (NaN does not count)
  return top;
}
__device__ __forceinline__ float most_finite(const float* v, float top) {
  for (int k = 0; k < 8; ++k) {
    const float m = fabsf(v[k]);
    if (m <= 3.402823466e38f) top = fmaxf(top, m);
  }
  return top;
}

template <class T, bool kWide, bool kInter>
__global__ void __launch_bounds__(kThreads, 5) append8_kernel(const __grid_constant__ AppendArgs a) {
  // [chunk + 15][half] for the keys of the block's runs, then [chunk][half] for its queries (which are turned as dense
  // ones are)
  extern __shared__ __align__(16) float2 cs[];
  // from kReach entries before the block's first; seq -1: not written
  __shared__ int32_t pos[kWindow], seq[kWindow], page_at[kWindow];
  __shared__ uint32_t written[4], heads[4];        // of the window's entries, by bit: those written, and those that begin a run
  __shared__ int32_t run_n[kChunk], run_cs[kChunk], n_runs, n_turned, turned_at[kChunk + kBlock];
  __shared__ unsigned char run_at[kChunk][kBlock];   // a run's entries
  const int64_t t0 = (int64_t)blockIdx.x * a.chunk;
  const int own = a.n_tokens - t0 < a.chunk ? int(a.n_tokens - t0) : a.chunk;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int32_t page = a.cache.page_tokens;
  int32_t my_pos = 0, my_seq = -1, my_page = -1;
  // the page that an entry is written to, or -1
  auto page_of = [&](int32_t p, int32_t row) {
    const int32_t col = p >= 0 ? p / page : -1;
    if (row < 0 || row >= a.cache.n_seq || col < 0 || col >= a.cache.max_pages) return -1;
    const int32_t x = a.cache.table[int64_t(row) * a.cache.max_pages + col];
    return x < a.cache.n_pages ? x : -1;
  };
  if (warp < 3) {
    const int64_t t = t0 + threadIdx.x - kReach;
    if (threadIdx.x < own + 2 * kReach && t >= 0 && t < a.n_tokens) {
      my_pos = a.pos[t], my_seq = a.seq[t];
      if (my_seq >= 0) {
        my_page = page_of(my_pos, my_seq);
        if (my_page < 0) {
          my_seq = -1;
          if (blockIdx.y == 0 && t >= t0 && t < t0 + own) atomicAdd(&a.cache.status[4], 1);
        }
      }
    }
    if (threadIdx.x < kWindow) pos[threadIdx.x] = my_pos, seq[threadIdx.x] = my_seq, page_at[threadIdx.x] = my_page;
    const uint32_t bits = __ballot_sync(0xffffffffu, my_seq >= 0);
    if (lane == 0) written[warp] = bits;
  } else if (threadIdx.x == 96) {
    written[3] = heads[3] = 0;
  }
  __syncthreads();
  // 32 of the window's bits from entry i on
  auto bits_at = [](const uint32_t* words, int i) { return __funnelshift_r(words[i / 32], words[i / 32 + 1], i % 32); };
  if (warp < 3) {
    // an entry goes with the one written before it where that is an earlier token of its block
    bool head = my_seq >= 0;
    if (head && threadIdx.x > 0) {
      const int from = threadIdx.x < 31 ? 0 : threadIdx.x - 31;
      const uint32_t before = bits_at(written, from) & ((1u << (threadIdx.x - from)) - 1);
      if (before) {
        const int x = from + 31 - __clz(before);
        head = !(seq[x] == my_seq && pos[x] < my_pos && pos[x] / kBlock == my_pos / kBlock);
      }
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, head);
    if (lane == 0) heads[warp] = bits;
  }
  __syncthreads();
  {
    // a run is what is written from its head to the next, within kReach entries; a warp lists every fourth
    const uint32_t mine = bits_at(heads, kReach) & ((1u << own) - 1);   // (own <= 16)
    const int n = __popc(mine);
    uint32_t rest = mine;
    int before = 0;
    for (int r = 0; r < n; ++r, rest &= rest - 1) {
      const int i = kReach + __ffs(rest) - 1;
      const uint32_t next = bits_at(heads, i) & ~1u;
      const uint32_t run = bits_at(written, i) & (next ? (1u << (__ffs(next) - 1)) - 1 : ~0u);
      const int tokens = __popc(run);    // at most kBlock, of one block and in increasing order
      if (r % (kThreads / 32) == warp) {
        if (run >> lane & 1) {
          const int k = __popc(run & ((1u << lane) - 1));
          run_at[r][k] = (unsigned char)(i + lane);
          turned_at[before + k] = i + lane;
        }
        if (lane == 0) run_n[r] = tokens, run_cs[r] = before;
        // out of order: an entry of the kReach up to this one is in the same block
        const int e = i - 1 - lane;
        const bool twice = lane < kReach - 1 && seq[e] == seq[i] && pos[e] / kBlock == pos[i] / kBlock;
        if (__any_sync(0xffffffffu, twice) && lane == 0 && blockIdx.y == 0) atomicAdd(&a.cache.status[6], tokens);
      }
      before += tokens;
    }
    if (threadIdx.x == 0) n_runs = n, n_turned = before;
    // or too far behind its run's head, and in no run: none of the entries up to kReach - 1 before it is a head.  (Only of the
    // first that the window shows is it not certain that it is one: what it may follow lies before the window.)
    if (blockIdx.y == 0 && threadIdx.x < own && seq[kReach + threadIdx.x] >= 0 && !(mine >> threadIdx.x & 1)) {
      const uint32_t shown = written[0] & ~1u, near = bits_at(heads, threadIdx.x + 1) & ~(1u << (kReach - 1));
      const int x = __ffs(shown) - 1;      // (entry 0 is before those)
      bool lost = near == 0;
      if (!lost && !(written[0] & 1) && x > (int)threadIdx.x && near == 1u << (x - 1 - threadIdx.x))
        for (int64_t t = t0 - kReach + x - 1; t >= 0 && t > t0 - 2 * kReach + x; --t)
          if (page_of(a.pos[t], a.seq[t]) >= 0) {
            lost = a.seq[t] == seq[x] && a.pos[t] < pos[x] && a.pos[t] / kBlock == pos[x] / kBlock;
            break;
          }
      if (lost) atomicAdd(&a.cache.status[6], 1);
    }
  }
  __syncthreads();
  // in halves: eight pairs a lane, both elements of each
  const int eights = kWide && !kInter ? a.half / 8 : 0;
  float2* const cs_q = cs + (a.chunk + kBlock - 1) * a.half;
  const int q_rows = a.n_heads > 0 ? own : 0;
  for (int i = threadIdx.x; i < (n_turned + q_rows) * a.half; i += kThreads) {
    const int t = i / a.half, p = i - t * a.half;
    if (t < n_turned) {
      const float2 turn = near_turn_of(a.freq[p], pos[turned_at[t]], a.factor);
      // for eight pairs a lane: two pairs' cosines, then their sines, and neighbouring lanes' next to each other; else in
      // order
      float* at = reinterpret_cast<float*>(cs + t * a.half);
      at += eights ? (p % 8 / 2 * eights + p / 8) * 4 + p % 2 : 2 * p;
      at[0] = turn.x, at[eights ? 2 : 1] = turn.y;
    } else cs_q[i - n_turned * a.half] = turn_of(a.freq[p], pos[kReach + t - n_turned], a.factor, a.factor);
  }
  __syncthreads();

  // runs: a warp a head's keys or values
  const int vecs = a.dim / 8, units = n_runs * 2 * a.n_kv;
  const int doubles = a.dim / 16;      // of a token
  const uint32_t per_vec = 65536 / vecs + 1, per_double = 65536 / doubles + 1;   // i * per_x >> 16 is i / x, for i below 256
  for (int u = blockIdx.y * (kThreads / 32) + warp; u < units; u += gridDim.y * (kThreads / 32)) {
    const int run = u / (2 * a.n_kv), x = u - run * 2 * a.n_kv, is_v = x / a.n_kv, h = x - is_v * a.n_kv;
    const int at = run_at[run][0], n = run_n[run];
    const float2* turns = cs + run_cs[run] * a.half;
    const int32_t p0 = pos[at];
    const int64_t p = page_at[at];
    unsigned char* in = static_cast<unsigned char*>(a.cache.pool) + p * a.page_bytes;
    const int head = is_v * a.n_kv + h, slot0 = p0 % page / kBlock * kBlock;
    float* scale_at = reinterpret_cast<float*>(in + a.scales_at) + head * (page / kBlock) + slot0 / kBlock;
    unsigned char* codes = in + a.codes_at + (int64_t(head) * page + slot0) * a.dim;
    const int kept = p0 % kBlock;
    float old = kept ? *scale_at : 0.f;
    const T* from = is_v ? static_cast<const T*>(a.v) + (t0 - kReach) * a.v_tok + h * a.v_head
                         : static_cast<const T*>(a.k) + (t0 - kReach) * a.k_tok + h * a.k_head;
    const int64_t row = is_v ? a.v_tok : a.k_tok;
    // step s of a lane: elements from .. on of a token; two steps of keys are eight pairs' elements, or 16 one after another
    const bool paired = kWide && !is_v;
    auto place = [&](int s, int* tok, int* elem) {
      const int i = lane + 32 * (paired ? s / 2 : s);
      *tok = i * (paired ? per_double : per_vec) >> 16;
      const int d = i - *tok * (paired ? doubles : vecs);
      *elem = !paired ? d * 8 : d < eights ? d * 8 + (s % 2 ? a.half : 0) : d * 16 + s % 2 * 8;
      return *tok < n;
    };
    float scale, by;
    // the block's scale for values of up to top; what it holds before this run is rounded to it where it is larger
    auto settle = [&](float top) {
      scale = scale_for(top);
      if (kept) {
        old = fminf(fmaxf(old, 8.67361738e-19f), 1.15292150e18f);   // 2^-60 .. 2^60, NaN the least
        if (scale > old) {
          const float to = old / scale;
          for (int i = lane; i < kept * vecs; i += 32) {
            float w[8];
            uint2* c = reinterpret_cast<uint2*>(codes + i * 8);
            wide8(*c, w);
            *c = narrow8(w, to);
          }
        } else {
          scale = old;
        }
      }
      by = 1.f / scale;
    };
    auto most = [](float top) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))); };
    auto put = [&](int tok, int e, const float* v) {
      const uint64_t w[4] = {two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])};
      *reinterpret_cast<uint2*>(codes + (pos[run_at[run][tok]] % kBlock) * a.dim + e) = narrow8(w, two(by, by));
    };
    // Twice over the values: for their largest, and for their codes (with infinities, which do not count, thrice).
    // (Where loads are of 16 bytes they lie in registers as they came, else they are read again.)
    auto twice = [&](auto&& each) {
      float top = 0.f;
      each([&](int, int, const float* v) { top = most_of(v, top); }, false);
      top = most(top);
      if (!(top <= 3.402823466e38f)) {
        top = 0.f;
        each([&](int, int, const float* v) { top = most_finite(v, top); }, false);
        top = most(top);
      }
      settle(top);
      each(put, true);
    };
    if (kWide) {
      uint4 raw[kSteps];
      int32_t to[kSteps];                // in codes; negative: nothing
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        int tok, e;
        to[s] = -1;
        if (place(s, &tok, &e)) {
          const int x = run_at[run][tok];
          raw[s] = *reinterpret_cast<const uint4*>(from + x * row + e);
          to[s] = (pos[x] % kBlock) * a.dim + e;
        }
      }
      auto word = [&](int s, int i) { return i == 0 ? raw[s].x : i == 1 ? raw[s].y : i == 2 ? raw[s].z : raw[s].w; };
      auto as_two = [](uint32_t w) { return two(unpack(T(), w, 0), unpack(T(), w, 1)); };
      if (is_v) {
        uint32_t both = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          if (to[s] >= 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) both = most_of(T(), both, word(s, i) & 0x7fff7fff);
        float top = most(fmaxf(unpack(T(), both, 0), unpack(T(), both, 1)));
        if (!(top <= 3.402823466e38f)) {   // infinities do not count
          top = 0.f;
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            for (int i = 0; i < 8; ++i) {
              const float m = fabsf(unpack(T(), word(s, i / 2), i % 2));
              if (to[s] >= 0 && m <= 3.402823466e38f) top = fmaxf(top, m);
            }
          top = most(top);
        }
        settle(top);
        const uint64_t by2 = two(by, by);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if (to[s] < 0) continue;
          const uint64_t v[4] = {as_two(raw[s].x), as_two(raw[s].y), as_two(raw[s].z), as_two(raw[s].w)};
          *reinterpret_cast<uint2*>(codes + to[s]) = narrow8(v, by2);
        }
      } else {
        // pairs: (u, w) -> (u c - w s, u s + w c)
        auto each = [&](auto&& use) {
#pragma unroll
          for (int s = 0; s < kSteps; s += 2) {
            if (to[s] < 0) continue;
            int tok, e;
            place(s, &tok, &e);
            const float2* turn = turns + tok * a.half;
            uint64_t v[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = as_two(word(s, i)), w[i] = as_two(word(s + 1, i));
            if (kInter) {
              auto turned = [&](uint64_t* x, int at) {
                if (at >= 2 * a.half) return;
                const float4* t = reinterpret_cast<const float4*>(turn + at / 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float4 cs4 = t[i / 2];
                  const float c = i % 2 ? cs4.z : cs4.x, d = i % 2 ? cs4.w : cs4.y;
                  float y, z;
                  halves(x[i], &y, &z);
                  x[i] = fma2(x[i], two(c, c), fma2(two(z, y), two(-d, d), 0ull));
                }
              };
              turned(v, e);
              turned(w, e + 8);
            } else if (e < a.half) {
              const float4* t = reinterpret_cast<const float4*>(turn) + e / 8;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float4 cs4 = t[i * eights];
                const uint64_t c = two(cs4.x, cs4.y), d = two(cs4.z, cs4.w), y = v[i], z = w[i];
                v[i] = fma2(y, c, fma2(z, two(-cs4.z, -cs4.w), 0ull));
                w[i] = fma2(y, d, fma2(z, c, 0ull));
              }
            }
            use(s, v, w);
          }
        };
        auto largest = [&](auto&& of) {
          float top = 0.f;
          each([&](int, uint64_t* v, uint64_t* w) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x0, x1, x2, x3;
              halves(v[i], &x0, &x1);
              halves(w[i], &x2, &x3);
              top = fmaxf(fmaxf(top, fmaxf(of(x0), of(x1))), fmaxf(of(x2), of(x3)));
            }
          });
          return most(top);
        };
        float top = largest([](float x) { return fabsf(x); });
        if (!(top <= 3.402823466e38f)) top = largest([](float x) { return fabsf(x) <= 3.402823466e38f ? fabsf(x) : 0.f; });
        settle(top);
        const uint64_t by2 = two(by, by);
        each([&](int s, uint64_t* v, uint64_t* w) {
          uint32_t nearest = ~0u;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x0, x1, x2, x3;
            halves(v[i], &x0, &x1);
            halves(w[i], &x2, &x3);
            nearest = min(nearest, min(min(from_middle(x0), from_middle(x1)), min(from_middle(x2), from_middle(x3))));
          }
          if (nearest < kNearTop) {
            int tok, e;
            place(s, &tok, &e);
            float x[16], from[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              halves(v[i], &x[2 * i], &x[2 * i + 1]);
              halves(w[i], &x[8 + 2 * i], &x[9 + 2 * i]);
#pragma unroll
              for (int k = 0; k < 2; ++k)
                from[2 * i + k] = unpack(T(), word(s, i), k), from[8 + 2 * i + k] = unpack(T(), word(s + 1, i), k);
            }
            turn_exactly(x, from, !kInter, kInter ? e / 2 : e, a.half, a.freq, pos[run_at[run][tok]], a.factor);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = two(x[2 * i], x[2 * i + 1]), w[i] = two(x[8 + 2 * i], x[9 + 2 * i]);
          }
          *reinterpret_cast<uint2*>(codes + to[s]) = narrow8(v, by2);
          *reinterpret_cast<uint2*>(codes + to[s + 1]) = narrow8(w, by2);
        });
      }
    } else {
      twice([&](auto&& use, bool codes_now) {
#pragma unroll 1
        for (int s = 0; s < kSteps; ++s) {
          int tok, e;
          if (!place(s, &tok, &e)) continue;
          const T* x = from + run_at[run][tok] * row;
          float v[8];
          if (is_v) load8(x + e, v);
          else turned8(x, e, a.half, kInter, turns + tok * a.half, codes_now, a.freq, pos[run_at[run][tok]], a.factor, v);
          use(tok, e, v);
        }
      });
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
      turn_step<T, N, kInter>(from, to, step, a.half, cs_q + tok * a.half);
    } else {
      const int o = 2 * a.half + (step - turns) * N;
      *reinterpret_cast<V*>(to + o) = *reinterpret_cast<const V*>(from + o);
    }
  }
}

template <class T, bool kWide, bool kInter>
cudaError_t launch(const AppendArgs& a, cudaStream_t st) {
  const int64_t blocks = (a.n_tokens + a.chunk - 1) / a.chunk;
  const int64_t steps = int64_t(a.chunk) * (a.n_heads + 2 * a.n_kv) * (a.dim / 8);
  int64_t split = (152 * 4 + blocks - 1) / blocks;
  if (split > (steps + kThreads - 1) / kThreads) split = (steps + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)blocks, (unsigned)(split < 1 ? 1 : split));
  append8_kernel<T, kWide, kInter><<<grid, kThreads, ((a.n_heads > 0 ? 2 : 1) * a.chunk + kBlock - 1) * a.half * sizeof(float2), st>>>(a);
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
  // 16 bytes a step where every head starts on 16 bytes and the halves are whole steps (else a
  // call on a prompt takes 423 us for 158)
  bool wide = rope->rotary % (rope->interleaved ? 8 : 16) == 0 && aligned(k, k_tok, k_head, 2) && aligned(v, v_tok, v_head, 2);
  if (n_heads > 0) wide = wide && aligned(q, q_tok, q_head, 2) && aligned(q_out, o_tok, o_head, 2);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  // One token a block, its queries and its runs in shares: a decode step of 16 tokens 4.5 us, with 16 a block 9.2 (these
  // without the search for numbers near a middle, which adds about a tenth to each).  Where there are many, and 16 or more for each
  // row that the cache has (which rows the tokens are of, the host does not know: of a cache of many rows a call for a few has
  // one a block up to 4,864 tokens, though 16 would be better), 16 a block, which has few runs then (with 32 + 8 + 8 heads of 128, 2,432 tokens 20.8 us,
  // one a block 26.0; 608 12.0 and 13.3; 304 11.4 and 10.5; 1,216 of as many sequences 25.5 and 20.3, 4,864 81.7 and 82.1).
  // Very many queries then as dense ones, in a launch of their own with few registers a thread (32,768 tokens 136 us, in one
  // launch 161; 4,864 32.6 and 34.8; 2,432 21.8 and 20.8; 16,384 of 8 heads of 64 21.5 and 17.3).
  a.chunk = 1;
  if (n_tokens >= 152 * 4 && n_tokens >= std::min<int64_t>(int64_t(kBlock) * cache->n_seq, 152 * 2 * kChunk)) {
    a.chunk = kChunk;
    if (n_tokens * n_heads * a.dim >= 1 << 24) {
      const int e = op_rope(rope, dtype, n_tokens, n_heads, a.dim, q, q_tok, q_head, pos, 0, q_out, o_tok, o_head, stream);
      if (e != GMG_OK) return e;
      a.n_heads = 0;
    }
  }
  const cudaError_t rc = dtype == GMG_OP_BF16 ? launch_type<__nv_bfloat16>(a, wide, st) : launch_type<__half>(a, wide, st);
  return rc == cudaSuccess ? GMG_OK : GMG_ECUDA;
}
