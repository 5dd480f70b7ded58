// Product of a batch of rows with a weight, and its epilogue: bias, activation, gate,
// residual.  The C ABI is declared in include/gmgop.h.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gmgop.h"
#include "gmgop_host.h"

namespace gop {
namespace {

__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
__device__ __forceinline__ void down(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void down(float v, __half* o) { *o = __float2half_rn(v); }

// The activations, in fp32.
__device__ __forceinline__ float act(float v, int32_t kind) {
  switch (kind) {
    case GMG_OP_RELU: return v < 0.f ? 0.f : v;   // keeps a NaN
    case GMG_OP_SILU: return v / (1.f + __expf(-v));
    case GMG_OP_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    default: return v;
  }
}

// One output element from its sums.
template <class T>
__device__ __forceinline__ void finish(const op_linear_t& a, int64_t row, int64_t col, float v, float g) {
  if (a.bias) v += up(static_cast<const T*>(a.bias)[col]);
  if (a.gated) {
    if (a.gate_bias) g += up(static_cast<const T*>(a.gate_bias)[col]);
    v *= act(g, a.act);
  } else {
    v = act(v, a.act);
  }
  if (a.residual) v += up(static_cast<const T*>(a.residual)[row * a.residual_row + col]);
  down(v, static_cast<T*>(a.y) + row * a.y_row + col);
}

// ---- operands that start or continue off 16 bytes -------------------------

// A block of 256 threads takes 64 x 64 outputs, a thread 4 x 4, from tiles of 16
// columns in shared memory.  It makes no assumption on alignment; bound by the fp32
// multiply-adds of the ordinary cores.
constexpr int kTile = 64, kDepth = 16;

template <class T, bool kGate>
__global__ void __launch_bounds__(256) linear_any_kernel(op_linear_t a) {
  __shared__ float xs[kDepth][kTile + 4], ws[kDepth][kTile + 4], gs[kGate ? kDepth : 1][kTile + 4];
  const int64_t row0 = (int64_t)blockIdx.y * kTile, col0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float v[4][4] = {}, g[4][4] = {};
  for (int64_t k0 = 0; k0 < a.k; k0 += kDepth) {
    for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
      const int r = i / kDepth, c = i % kDepth;
      const bool in = k0 + c < a.k;
      const int64_t row = row0 + r, col = col0 + r;
      xs[c][r] = in && row < a.m ? up(static_cast<const T*>(a.x)[row * a.x_row + k0 + c]) : 0.f;
      ws[c][r] = in && col < a.n ? up(static_cast<const T*>(a.w)[col * a.w_row + k0 + c]) : 0.f;
      if (kGate) gs[c][r] = in && col < a.n ? up(static_cast<const T*>(a.gate)[col * a.gate_row + k0 + c]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kDepth; ++c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = xs[c][ty * 4 + i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[i][j] = fmaf(x, ws[c][tx * 4 + j], v[i][j]);
          if (kGate) g[i][j] = fmaf(x, gs[c][tx * 4 + j], g[i][j]);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t row = row0 + ty * 4 + i, col = col0 + tx * 4 + j;
      if (row < a.m && col < a.n) finish<T>(a, row, col, v[i][j], g[i][j]);
    }
}

template <class T>
cudaError_t launch_any(const op_linear_t& a, cudaStream_t st) {
  // rows beyond the limit of a grid's second dimension take further launches
  constexpr int64_t kRows = int64_t(65535) * kTile;
  for (int64_t r = 0; r < a.m; r += kRows) {
    op_linear_t b = a;
    b.m = a.m - r < kRows ? a.m - r : kRows;
    b.x = static_cast<const T*>(a.x) + r * a.x_row;
    if (a.residual) b.residual = static_cast<const T*>(a.residual) + r * a.residual_row;
    b.y = static_cast<T*>(a.y) + r * a.y_row;
    const dim3 grid((unsigned)((a.n + kTile - 1) / kTile), (unsigned)((b.m + kTile - 1) / kTile));
    if (a.gated) linear_any_kernel<T, true><<<grid, 256, 0, st>>>(b);
    else linear_any_kernel<T, false><<<grid, 256, 0, st>>>(b);
  }
  return cudaGetLastError();
}

bool args_ok(const op_linear_t* a) {
  if (!a || (a->dtype != GMG_OP_BF16 && a->dtype != GMG_OP_F16) || a->act < GMG_OP_NONE || a->act > GMG_OP_GELU)
    return false;
  if (a->m < 0 || a->n < 0 || a->k < 0 || a->m > 0x7fffffff || a->n > 0x7fffffff || a->k > 0x7fffffff) return false;
  if (a->m == 0 || a->n == 0) return true;
  if (!a->y || a->y_row < a->n || (a->residual && a->residual_row < a->n) || (a->gate_bias && !a->gated)) return false;
  if (a->k > 0 && (!a->x || !a->w || a->x_row < a->k || a->w_row < a->k || (a->gated && (!a->gate || a->gate_row < a->k))))
    return false;
  return true;
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

size_t op_linear_work_bytes(const op_linear_t* args) { return args_ok(args) ? 4096 : 0; }

int op_linear(const op_linear_t* args, void* work, size_t work_bytes, gmg_stream_t stream) {
  if (!args_ok(args)) return GMG_EINVAL;
  if (!work || (reinterpret_cast<uintptr_t>(work) & 255) || work_bytes < op_linear_work_bytes(args)) return GMG_EWS;
  if (args->m == 0 || args->n == 0) return GMG_OK;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = args->dtype == GMG_OP_BF16 ? launch_any<__nv_bfloat16>(*args, st) : launch_any<__half>(*args, st);
  return e == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // extern "C"
