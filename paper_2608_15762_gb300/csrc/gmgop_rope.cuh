// What the kernels with rotary positions share: the turn of a pair at a position, and steps of a head.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gmgop_pairs.cuh"

namespace gop {
namespace {

constexpr int kMaxPairs = 128;   // rotary <= 256

// (cosine * by_c, sine * by_s) of the angle of a pair.
__device__ __forceinline__ float2 turn_of(uint64_t freq, int32_t pos, float by_c, float by_s) {
  const uint64_t turn = freq * (uint64_t)(int64_t)pos;
  // the top 32 bits, signed: half turns in [-1, 1)
  const float x = (float)(int32_t)(turn >> 32) * 4.656612873077393e-10f;   // 2^-31
  float s, c;
  sincospif(x, &s, &c);
  return make_float2(c * by_c, s * by_s);
}

// The same, nearer by what the fp32 argument leaves out (up to 2^-26 turns), to first order: to the rounding of sine and
// cosine.
__device__ __forceinline__ float2 near_turn_of(uint64_t freq, int32_t pos, float by) {
  const uint64_t turn = freq * (uint64_t)(int64_t)pos;
  const int32_t top = (int32_t)(turn >> 32);
  const float whole = (float)top;                                          // 2^31 half turns at most
  float s, c;
  sincospif(whole * 4.656612873077393e-10f, &s, &c);                       // 2^-31
  const float left = (float)((int64_t)top - (int64_t)whole) * (4.656612873077393e-10f * 3.14159265f);
  return make_float2(fmaf(-s, left, c) * by, fmaf(c, left, s) * by);
}

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ void down(float v, float* o) { *o = v; }
__device__ __forceinline__ void down(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void down(float v, __half* o) { *o = __float2half_rn(v); }

template <class T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// One head: N elements of type T a step, aligned to N elements.  Pairs of the half
// layout take a step of the first half and one of the second, interleaved ones a step.
template <class T, int N, bool kInter>
__device__ __forceinline__ void turn_step(const T* x, T* y, int32_t step, int32_t half, const float2* cs) {
  using V = Vec<T, N>;
  if (kInter) {
    if (N == 1) {   // unaligned: a pair a step
      const float u = up(x[2 * step]), w = up(x[2 * step + 1]);
      const float2 t = cs[step];
      down(u * t.x - w * t.y, &y[2 * step]);
      down(u * t.y + w * t.x, &y[2 * step + 1]);
    } else {
      const V a = *reinterpret_cast<const V*>(x + step * N);
      V b;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const float u = up(a.v[2 * j]), w = up(a.v[2 * j + 1]);
        const float2 t = cs[step * (N / 2) + j];
        down(u * t.x - w * t.y, &b.v[2 * j]);
        down(u * t.y + w * t.x, &b.v[2 * j + 1]);
      }
      *reinterpret_cast<V*>(y + step * N) = b;
    }
  } else {
    const V a = *reinterpret_cast<const V*>(x + step * N), b = *reinterpret_cast<const V*>(x + half + step * N);
    V c, d;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float u = up(a.v[j]), w = up(b.v[j]);
      const float2 t = cs[step * N + j];
      down(u * t.x - w * t.y, &c.v[j]);
      down(u * t.y + w * t.x, &d.v[j]);
    }
    *reinterpret_cast<V*>(y + step * N) = c;
    *reinterpret_cast<V*>(y + half + step * N) = d;
  }
}

}  // namespace
}  // namespace gop
