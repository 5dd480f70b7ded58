// Norms before and after a block, with its gate and residual scale.  The C ABI is declared in
// include/gmgop.h.
//
// One pass: a row lies in registers, in fp32, from its loads to its stores; a warp takes a short row, a
// block a longer one.  The mean and the mean square of what deviates from it are sums over the row,
// each by shuffles and once through shared memory, so that no cancellation hides in them.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/gmgop.h"
#include "gmgop_host.h"

namespace gop {
namespace {

constexpr int kMaxThreads = 1024;

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
__device__ __forceinline__ void down(float v, float* o) { *o = v; }
__device__ __forceinline__ void down(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void down(float v, __half* o) { *o = __float2half_rn(v); }

template <class T>
struct alignas(16) Bytes16 {
  T v[16 / sizeof(T)];
};

// A thread's share of a row: kVecs times 8 neighbouring elements or, where rows are not made of whole
// aligned 16 bytes, single elements; `threads` apart.
template <int kVecs, bool kWide>
struct Share {
  int tid, threads, n;
  __device__ int at(int i) const {       // of element i of 8 * kVecs
    return kWide ? (i / 8 * threads + tid) * 8 + i % 8 : i * threads + tid;
  }
  template <class T>
  __device__ void load(const T* x, float* v) const {
    if (kWide) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        constexpr int per = 16 / sizeof(T);
#pragma unroll
        for (int b = 0; b < 8 / per; ++b) {
          Bytes16<T> a{};
          if (at(8 * k) < n) a = *reinterpret_cast<const Bytes16<T>*>(x + at(8 * k) + b * per);
#pragma unroll
          for (int i = 0; i < per; ++i) v[8 * k + b * per + i] = up(a.v[i]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8 * kVecs; ++i) v[i] = at(i) < n ? up(x[at(i)]) : 0.f;
    }
  }
  template <class T>
  __device__ void store(T* x, const float* v) const {
    if (kWide) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        constexpr int per = 16 / sizeof(T);
#pragma unroll
        for (int b = 0; b < 8 / per; ++b) {
          Bytes16<T> a;
#pragma unroll
          for (int i = 0; i < per; ++i) down(v[8 * k + b * per + i], &a.v[i]);
          if (at(8 * k) < n) *reinterpret_cast<Bytes16<T>*>(x + at(8 * k) + b * per) = a;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8 * kVecs; ++i)
        if (at(i) < n) down(v[i], x + at(i));
    }
  }
};

// The sum over the threads of a row; `buf` in turn, so that one barrier a sum is enough.
__device__ __forceinline__ float row_sum(float v, float (*buf)[kMaxThreads / 32], int* turn) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  if (blockDim.x == 32) return v;
  float* b = buf[*turn];
  *turn ^= 1;
  if ((threadIdx.x & 31) == 0) b[threadIdx.x / 32] = v;
  __syncthreads();
  const int warps = blockDim.x / 32, lane = threadIdx.x & 31;
  v = lane < warps ? b[lane] : 0.f;
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

template <class T, class X, int kVecs, bool kWide, int kThreads>
__global__ void __launch_bounds__(kThreads, 1) norm_kernel(const __grid_constant__ op_norm_t a) {
  constexpr int N = 8 * kVecs;
  __shared__ float buf[2][kMaxThreads / 32];
  int turn = 0;
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.m) return;              // (a whole warp, where a block has several rows)
  const Share<kVecs, kWide> s{(int)threadIdx.x, (int)blockDim.x, (int)a.n};
  const float n = (float)a.n;          // (divided by, as 1 / n is rounded: a row of one number has that mean)
  // Where rows are few their last weights are loaded with them: behind the sums they would be waited for once more
  constexpr bool kAhead = kVecs == 1 && kThreads > 128;
  float w_ahead[kAhead ? N : 1], b_ahead[kAhead ? N : 1];
  if (kAhead && a.weight) s.load(static_cast<const T*>(a.weight), w_ahead);
  if (kAhead && a.bias) s.load(static_cast<const T*>(a.bias), b_ahead);
  // v <- its norm with weight and bias
  auto normed = [&](float* v, const void* weight, const void* bias, bool ahead) {
    if (a.kind == GMG_NORM_LAYER) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum += v[i];
      const float mean = row_sum(sum, buf, &turn) / n;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = s.at(i) < a.n ? v[i] - mean : 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fmaf(v[i], v[i], sum);
    const float inv = 1.f / sqrtf(row_sum(sum, buf, &turn) / n + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= inv;
    if (weight) {
      float w[N];
      if (!ahead) s.load(static_cast<const T*>(weight), w);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= (ahead ? w_ahead[kAhead ? i : 0] : w[i]) + a.shift;
    }
    if (bias) {
      float b[N];
      if (!ahead) s.load(static_cast<const T*>(bias), b);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += ahead ? b_ahead[kAhead ? i : 0] : b[i];
    }
  };
  float v[N];
  s.load(static_cast<const X*>(a.x) + row * a.x_row, v);
  if (a.y) {
    float z[N];
    s.load(static_cast<const T*>(a.y) + row * a.y_row, z);
    if (a.after) normed(z, a.y_weight, a.y_bias, false);
    if (a.gate && a.gate_col) {
      float g[N];
      s.load(static_cast<const T*>(a.gate) + row * a.gate_row, g);
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] *= g[i];
    }
    const float by = a.gate && !a.gate_col ? up(static_cast<const T*>(a.gate)[row * a.gate_row]) * a.scale : a.scale;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fmaf(by, z[i], v[i]);
    if (a.r) s.store(static_cast<X*>(a.r) + row * a.r_row, v);
  }
  if (a.h) {
    normed(v, a.weight, a.bias, kAhead);
    s.store(static_cast<T*>(a.h) + row * a.h_row, v);
  }
}

template <class T, class X, bool kWide>
cudaError_t launch(const op_norm_t& a, cudaStream_t st) {
  const int64_t vecs = (a.n + 7) / 8;
  // a warp a row up to 1,024 elements; then a block, with 8 elements a thread where rows are few, so that a row's way is
  // short, else with 16, which leaves more of them on an SM (%s)
  auto go = [&](auto kernel, int v) {
    int64_t threads = (vecs + v - 1) / v;
    threads = (threads + 31) / 32 * 32;
    const int rows = threads == 32 ? 4 : 1;
    kernel<<<(unsigned)((a.m + rows - 1) / rows), dim3((unsigned)threads, rows), 0, st>>>(a);
    return cudaGetLastError();
  };
  if (vecs <= 32) return go(norm_kernel<T, X, 1, kWide, 128>, 1);
  if (vecs <= 128) return go(norm_kernel<T, X, 4, kWide, 128>, 4);
  if (vecs <= kMaxThreads && a.m <= 1216) return go(norm_kernel<T, X, 1, kWide, kMaxThreads>, 1);
  if (vecs <= 2 * 512) return go(norm_kernel<T, X, 2, kWide, 512>, 2);
  if (vecs <= 2 * kMaxThreads) return go(norm_kernel<T, X, 2, kWide, kMaxThreads>, 2);
  return go(norm_kernel<T, X, 4, kWide, kMaxThreads>, 4);
}

template <class T, class X>
cudaError_t launch_type(const op_norm_t& a, bool wide, cudaStream_t st) {
  return wide ? launch<T, X, true>(a, st) : launch<T, X, false>(a, st);
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" int op_norm(const op_norm_t* p, gmg_stream_t stream) {
  if (!p) return GMG_EINVAL;
  op_norm_t a = *p;
  const bool types = (a.dtype == GMG_OP_F32 || a.dtype == GMG_OP_BF16 || a.dtype == GMG_OP_F16) &&
                     (a.stream_dtype == a.dtype || a.stream_dtype == GMG_OP_F32);
  if (!types || (a.kind != GMG_NORM_RMS && a.kind != GMG_NORM_LAYER)) return GMG_EINVAL;
  if (a.m < 0 || a.m > 0x7fffffff || a.n < 0 || a.n > GMG_NORM_MOST) return GMG_EINVAL;
  if (!(a.scale == a.scale) || !(a.shift == a.shift) || !(a.eps >= 0.f)) return GMG_EINVAL;
  if (a.m == 0 || a.n == 0) return GMG_OK;
  if (!a.y && (a.after || a.gate || a.r || a.y_weight || a.y_bias)) return GMG_EINVAL;
  if (!a.after && (a.y_weight || a.y_bias)) return GMG_EINVAL;
  if (!a.h && (!a.r || a.weight || a.bias)) return GMG_EINVAL;
  if (!a.x || a.x_row < a.n || (a.y && a.y_row < a.n) || (a.h && a.h_row < a.n) || (a.r && a.r_row < a.n)) return GMG_EINVAL;
  if (a.gate && ((a.gate_col != 0 && a.gate_col != 1) || (a.gate_row != 0 && a.gate_row < (a.gate_col ? a.n : 1))))
    return GMG_EINVAL;
  const int e = a.dtype == GMG_OP_F32 ? 4 : 2, ex = a.stream_dtype == GMG_OP_F32 ? 4 : 2;
  bool wide = a.n % 8 == 0 && aligned(a.x, a.x_row, 0, ex);
  for (const void* w : {a.weight, a.bias, a.y_weight, a.y_bias}) wide = wide && aligned(w, 0, 0, e);
  if (a.y) wide = wide && aligned(a.y, a.y_row, 0, e);
  if (a.h) wide = wide && aligned(a.h, a.h_row, 0, e);
  if (a.r) wide = wide && aligned(a.r, a.r_row, 0, ex);
  if (a.gate && a.gate_col) wide = wide && aligned(a.gate, a.gate_row, 0, e);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool wider = a.stream_dtype != a.dtype;
  cudaError_t rc;
  if (a.dtype == GMG_OP_F32) rc = launch_type<float, float>(a, wide, st);
  else if (a.dtype == GMG_OP_BF16)
    rc = wider ? launch_type<__nv_bfloat16, float>(a, wide, st) : launch_type<__nv_bfloat16, __nv_bfloat16>(a, wide, st);
  else rc = wider ? launch_type<__half, float>(a, wide, st) : launch_type<__half, __half>(a, wide, st);
  return rc == cudaSuccess ? GMG_OK : GMG_ECUDA;
}
