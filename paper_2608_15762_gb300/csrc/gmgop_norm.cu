// Norms before and after a block, with its gate and residual scale.  The C ABI is declared in
// include/gmgop.h.
//
// N(v; w, b) = (v - mean) / sqrt(mean((v - mean)^2) + eps) (w + shift) + b, with mean 0 for rms, of
// x + scale * gate * z, and z = N(y) or y.  What bounds it is memory (16,384 rows of 4,096, x in 32 bits:
// 126.5 us, 6.4 TB/s of the 805 MB that it has to move), and a launch's and two loads' latency where rows
// are few (one of 4,096: 2.0 us).
//
// One pass: a row lies in registers, in fp32, from its loads to its stores; a warp takes a short row, a
// block a longer one.  The mean and the mean square of what deviates from it are sums over the row,
// each by shuffles and once through shared memory, so that no cancellation hides in them.
// The last weights are loaded with the row: behind the sums they would be waited for once more.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/gmgop.h"
#include "gmgop_host.h"
#include "gmgop_pairs.cuh"

namespace gop {
namespace {

constexpr int kMaxThreads = 1024;

__device__ __forceinline__ float up(float, uint32_t w) { return __uint_as_float(w); }
template <class T>
__device__ __forceinline__ float up(T, uint32_t w) { return unpack(T(), w, 0); }
template <class T>
__device__ __forceinline__ uint32_t down(T, float v) { return pack(T(), v, 0.f); }
__device__ __forceinline__ float one(const float* x) { return *x; }
template <class T>
__device__ __forceinline__ float one(const T* x) { return gop::up(*x); }

// How rows lie: anyhow; in whole aligned 16 bytes; or of any length, but all of a row's tensors alike, so that the same
// groups of 8 elements are aligned in each of them (the first and last of which may be a part; what is one for all rows is
// loaded element by element: 4,000 rows of 5,003 39.7 us, all of it element by element 66.5, 50,000 of 1,003 87 and 177).
enum Rows { kAnyhow, kWhole, kAlike };

// A thread's share of a row, as it lies in memory: kVecs times 8 neighbouring elements, `threads` apart, or, where rows
// lie anyhow, single elements, kRow apart.
template <class T, int kVecs, int kRows, int kRow>
struct Share {
  static constexpr int N = 8 * kVecs, kEach = 4 / (int)sizeof(T), kWords = kRows == kAnyhow ? N : N / kEach;
  uint32_t w[kWords];

  static __device__ __forceinline__ int at(int i, int before) {   // of element i; `before`: elements of the first group before the row
    if (kRows == kAnyhow) return i * kRow + (int)threadIdx.x;
    return (i / 8 * (int)blockDim.x + (int)threadIdx.x) * 8 + i % 8 - (kRows == kAlike ? before : 0);
  }
  static __device__ __forceinline__ uint32_t bits(const T* x) {
    return sizeof(T) == 4 ? *reinterpret_cast<const uint32_t*>(x) : *reinterpret_cast<const unsigned short*>(x);
  }
  // (what is beyond the row is 0)
  __device__ __forceinline__ void load_each(const T* x, int n, int before) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = at(i, before);
      const uint32_t v = e >= 0 && e < n ? bits(x + e) : 0;
      if constexpr (kWords == N) w[i] = v;
      else w[i / 2] = i % 2 ? w[i / 2] | v << 16 : v;
    }
  }
  // `alike`: x is one of the row's tensors, not one for all rows
  __device__ __forceinline__ void load(const T* x, int n, int before, bool alike) {
    if constexpr (kRows == kAnyhow) {
      load_each(x, n, before);
    } else if constexpr (kRows == kWhole) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        uint4 v{};
        const int e = at(i * kEach, before);
        if (e < n) v = *reinterpret_cast<const uint4*>(x + e);
        w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
      }
    } else {
      if (!alike) return load_each(x, n, before);
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int e = at(8 * k, before);
        constexpr int kGroup = 8 / kEach;
        if (e >= 0 && e + 8 <= n) {
#pragma unroll
          for (int i = 0; i < kGroup; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(x + e + i * kEach);
            w[k * kGroup + i] = v.x, w[k * kGroup + i + 1] = v.y, w[k * kGroup + i + 2] = v.z, w[k * kGroup + i + 3] = v.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < kGroup; ++i) {
            const int d = e + i * kEach;
            uint32_t v = d >= 0 && d < n ? bits(x + d) : 0;
            if (kEach == 2 && d + 1 >= 0 && d + 1 < n) v |= bits(x + d + 1) << 16;
            w[k * kGroup + i] = v;
          }
        }
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (kRows == kAnyhow || sizeof(T) == 4) return up(T(), w[i]);
    else return unpack(T(), w[i / 2], i % 2);
  }
  static __device__ __forceinline__ void put(T* x, float v) {
    if constexpr (sizeof(T) == 4) *x = v;
    else *reinterpret_cast<unsigned short*>(x) = (unsigned short)down(T(), v);
  }
  static __device__ __forceinline__ void store(T* x, int n, int before, const float* v) {
    if constexpr (kRows == kAnyhow) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = at(i, before);
        if (e < n) put(x + e, v[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 4 * kEach) {
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (sizeof(T) == 4) o[k] = __float_as_uint(v[i + k]);
          else o[k] = pack(T(), v[i + 2 * k], v[i + 2 * k + 1]);
        }
        const int e = at(i, before);
        if (kRows == kWhole ? e < n : e >= 0 && e + 4 * kEach <= n) {
          *reinterpret_cast<uint4*>(x + e) = uint4{o[0], o[1], o[2], o[3]};
        } else if (kRows == kAlike) {
#pragma unroll
          for (int k = 0; k < 4 * kEach; ++k)
            if (e + k >= 0 && e + k < n) put(x + e + k, v[i + k]);
        }
      }
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

template <class T, class X, int kVecs, int kRows, int kRow, int kBlocks>
__global__ void __launch_bounds__(kRow == 32 ? 256 : kRow, kBlocks) norm_kernel(const __grid_constant__ op_norm_t a) {
  using ShareT = Share<T, kVecs, kRows, kRow>;
  using ShareX = Share<X, kVecs, kRows, kRow>;
  constexpr int N = 8 * kVecs;
  __shared__ float buf[2][kMaxThreads / 32];
  int turn = 0;
  const int n = (int)a.n;
  const float count = (float)n;        // (divided by, as 1 / n is rounded: a row of one number has that mean)
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.m) return;              // (a whole warp, where a block has several rows)
  const int before = kRows == kAlike ? (int)(row * a.x_row & 7) : 0;
  auto in = [&](int i) {
    const int e = ShareT::at(kRows == kWhole ? i / 8 * 8 : i, before);
    return kRows == kAlike ? (unsigned)e < (unsigned)n : e < n;
  };
  // v <- its norm, without weight and bias
  auto normed = [&](float (&v)[N]) {
    if (a.kind == GMG_NORM_LAYER) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum += v[i];
      const float mean = row_sum(sum, buf, &turn) / count;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = in(i) ? v[i] - mean : 0.f;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fmaf(v[i], v[i], sum);
    const float inv = 1.f / sqrtf(row_sum(sum, buf, &turn) / count + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= inv;
  };
  auto weighted = [&](float (&v)[N], const ShareT& w) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= w.get(i) + a.shift;
  };
  auto biased = [&](float (&v)[N], const void* bias) {
    ShareT b;
    b.load(static_cast<const T*>(bias), n, before, false);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += b.get(i);
  };
  // (where there are registers for them: 16 rows of 4,096 2.41 us, behind the sums 2.54; 2,048 of 32,768 90.5, with them 95.6)
  constexpr bool kAhead = kVecs <= 2;
  ShareX x;
  ShareT y, last;
  x.load(static_cast<const X*>(a.x) + row * a.x_row, n, before, true);
  if (a.y) y.load(static_cast<const T*>(a.y) + row * a.y_row, n, before, true);
  if (kAhead && a.weight) last.load(static_cast<const T*>(a.weight), n, before, false);
  float v[N];
  if (a.y) {
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = y.get(i);
    if (a.after) {
      normed(z);
      if (a.y_weight) {
        ShareT w;
        w.load(static_cast<const T*>(a.y_weight), n, before, false);
        weighted(z, w);
      }
      if (a.y_bias) biased(z, a.y_bias);
    }
    if (a.gate && a.gate_col) {
      ShareT g;
      g.load(static_cast<const T*>(a.gate) + row * a.gate_row, n, before, a.gate_row != 0);
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] *= g.get(i);
    }
    const float by = a.gate && !a.gate_col ? one(static_cast<const T*>(a.gate) + row * a.gate_row) * a.scale : a.scale;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = in(i) ? fmaf(by, z[i], x.get(i)) : 0.f;
    if (a.r) ShareX::store(static_cast<X*>(a.r) + row * a.r_row, n, before, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = x.get(i);
  }
  if (a.h) {
    normed(v);
    if (a.weight) {
      if (!kAhead) last.load(static_cast<const T*>(a.weight), n, before, false);
      weighted(v, last);
    }
    if (a.bias) biased(v, a.bias);
    ShareT::store(static_cast<T*>(a.h) + row * a.h_row, n, before, v);
  }
}

template <class T, class X, int kRows>
cudaError_t launch(const op_norm_t& a, cudaStream_t st) {
  auto go = [&](auto kernel, int threads, int rows) {
    kernel<<<(unsigned)((a.m + rows - 1) / rows), dim3((unsigned)threads, rows), 0, st>>>(a);
    return cudaGetLastError();
  };
  // A warp a row up to 256 elements (100,000 rows of 128 28.8 us, a block each 52.8), else a block (50,000 rows of 1,024
  // 60.9 us, a warp each 64.6), with 16 elements a thread, 32 beyond 16,384.  Where rows are few, 8 a thread make a row's
  // way shorter: 16 rows of 4,096 2.41 us, with 16 a thread 2.55, but 608 rows 4.9 against 3.9 and 16 of 8,192 2.98
  // against 2.83; of 5,003, element by element, 3.65 against 5.03, and 304 rows 6.5 against 6.75.
  // Rows that lie anyhow (16,384 x 4,096 taken so: 134 us, in 16 bytes 83) have blocks of a fixed size, which makes their
  // distances constants.
  const int n = (int)a.n;
  if constexpr (kRows == kAnyhow) {
    if (n <= 256) return go(norm_kernel<T, X, 1, kRows, 32, 1>, 32, 8);
    if (n <= 2048) return go(norm_kernel<T, X, 1, kRows, 256, 1>, 256, 1);
    if (n <= 4096) return go(norm_kernel<T, X, 2, kRows, 256, 4>, 256, 1);
    if (n <= 8192)
      return a.m <= 304 ? go(norm_kernel<T, X, 1, kRows, 1024, 1>, 1024, 1) : go(norm_kernel<T, X, 2, kRows, 512, 2>, 512, 1);
    if (n <= 16384) return go(norm_kernel<T, X, 2, kRows, 1024, 1>, 1024, 1);
    return go(norm_kernel<T, X, 4, kRows, 1024, 1>, 1024, 1);
  } else {
    const int groups = kRows == kAlike ? (n + 14) / 8 : n / 8;   // of 8 elements, wherever the first one begins
    auto round = [](int v) { return (v + 31) / 32 * 32; };
    if (groups <= 32) return go(norm_kernel<T, X, 1, kRows, 32, 1>, 32, 8);
    if (a.m <= 152 && n <= 4096) return go(norm_kernel<T, X, 1, kRows, 1024, 1>, round(groups), 1);
    if (groups <= 2048) return go(norm_kernel<T, X, 2, kRows, 1024, 1>, round((groups + 1) / 2), 1);
    return go(norm_kernel<T, X, 4, kRows, 1024, 1>, round((groups + 3) / 4), 1);
  }
}

template <class T, class X>
cudaError_t launch_type(const op_norm_t& a, int rows, cudaStream_t st) {
  return rows == kWhole ? launch<T, X, kWhole>(a, st) : rows == kAlike ? launch<T, X, kAlike>(a, st) : launch<T, X, kAnyhow>(a, st);
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
  bool whole = a.n % 8 == 0, alike = a.n <= GMG_NORM_MOST - 14;   // (a row may begin and end inside of a group)
  for (const void* w : {a.weight, a.bias, a.y_weight, a.y_bias, a.gate_col && a.gate_row == 0 ? a.gate : nullptr})
    whole = whole && aligned(w, 0, 0, e);
  auto tensor = [&](const void* x, int64_t row, int each) {
    if (!x) return;
    whole = whole && aligned(x, row, 0, each);
    alike = alike && aligned(x, 0, 0, each) && (row - a.x_row) % 8 == 0;
  };
  tensor(a.x, a.x_row, ex);
  tensor(a.y, a.y_row, e);
  tensor(a.h, a.h_row, e);
  tensor(a.r, a.r_row, ex);
  if (a.gate_col && a.gate_row != 0) tensor(a.gate, a.gate_row, e);
  const int rows = whole ? kWhole : alike ? kAlike : kAnyhow;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool wider = a.stream_dtype != a.dtype;
  cudaError_t rc;
  if (a.dtype == GMG_OP_F32) rc = launch_type<float, float>(a, rows, st);
  else if (a.dtype == GMG_OP_BF16)
    rc = wider ? launch_type<__nv_bfloat16, float>(a, rows, st) : launch_type<__nv_bfloat16, __nv_bfloat16>(a, rows, st);
  else rc = wider ? launch_type<__half, float>(a, rows, st) : launch_type<__half, __half>(a, rows, st);
  return rc == cudaSuccess ? GMG_OK : GMG_ECUDA;
}
