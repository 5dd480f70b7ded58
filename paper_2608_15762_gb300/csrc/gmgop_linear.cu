// Product of a batch of rows with a weight, and its epilogue: bias, activation, gate,
// residual.  The C ABI is declared in include/gmgop.h.
//
// Four kernels, by the number of rows of x and the tiles that there are (see few_tiles and
// kFewRows), and one more for operands that bulk copies cannot read.  us a call, replayed on
// weights beyond the L2 cache; in brackets the floor and what bounds it:
//   1 x 4,096 x 4,096 (rows, columns of x, outputs)   9.8 (5.0: the launch and the loads in flight; memory is at
//       35% of its rate: five blocks an SM, 82 registers a thread, so that 1,024 blocks are 1.35 rounds)
//   16 x 4,096 x 12,288                              22.5 (15: reading the weight, 4.5 TB/s)
//   77 x 1,000 x 1,111                                7.2 (0.4: launch, a chain of copy, product, sums)
//   2,048 x 4,096 x 12,288 with a gate                260 (212: 5.05 rounds of tiles; tensor cores 72%
//       busy: a tile's end is not hidden behind the next tile, as its two sums take all of TMEM)
//   8,192 x 12,288 x 4,096 and a residual             436 (424: tensor cores, 88% busy; the power limit)

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "../../include/gmgop.h"
#include "gmg_once.h"
#include "gmgop_host.h"
#include "gmgop_ptx.cuh"

namespace gop {
namespace {

__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
__device__ __forceinline__ void down(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void down(float v, __half* o) { *o = __float2half_rn(v); }

// The activations, in fp32.  (silu's exponential is the fast one: its error, a few units of 2^-24 and
// 2^-24 of the argument, is far below the output's rounding to 16 bits.)
template <int kAct>
__device__ __forceinline__ float act_of(float v) {
  if (kAct == GMG_OP_RELU) return v < 0.f ? 0.f : v;   // keeps a NaN
  if (kAct == GMG_OP_SILU) return v / (1.f + __expf(-v));
  if (kAct == GMG_OP_GELU) return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
  return v;
}
__device__ __forceinline__ float act(float v, int32_t kind) {
  switch (kind) {
    case GMG_OP_RELU: return act_of<GMG_OP_RELU>(v);
    case GMG_OP_SILU: return act_of<GMG_OP_SILU>(v);
    case GMG_OP_GELU: return act_of<GMG_OP_GELU>(v);
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

// Four neighbouring columns of a row; one 8-byte store where the row allows it.
template <class T, bool kGate>
__device__ __forceinline__ void finish4(const op_linear_t& a, int64_t row, int64_t col, const float* v, const float* g) {
  const T* bias = static_cast<const T*>(a.bias) + col;
  const T* gate_bias = static_cast<const T*>(a.gate_bias) + col;
  const T* res = static_cast<const T*>(a.residual) + row * a.residual_row + col;
  T* y = static_cast<T*>(a.y) + row * a.y_row + col;
  struct alignas(8) Four {
    T v[4];
  } old, b, gb, out;
  const int n = a.n - col < 4 ? int(a.n - col) : 4;
  if (n <= 0) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= n) break;
    if (a.residual) old.v[i] = res[i];
    if (a.bias) b.v[i] = bias[i];
    if (kGate && a.gate_bias) gb.v[i] = gate_bias[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= n) break;
    float r = v[i];
    if (a.bias) r += up(b.v[i]);
    if (kGate) r *= act(a.gate_bias ? g[i] + up(gb.v[i]) : g[i], a.act);
    else r = act(r, a.act);
    if (a.residual) r += up(old.v[i]);
    down(r, &out.v[i]);
  }
  if (n == 4 && (reinterpret_cast<uintptr_t>(y) & 7) == 0) {
    *reinterpret_cast<Four*>(y) = out;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) y[i] = out.v[i];
  }
}

// ---- operands that start or continue off 16 bytes -------------------------

// A block of 256 threads takes 64 x 64 outputs, a thread 4 x 4, from tiles of 16
// columns in shared memory.  It makes no assumption on alignment; bound by the fp32
// multiply-adds of the ordinary cores (8,192 x 12,288 x 4,096 33.8 ms, 77 x 1,000 x 1,111
// 138 us; the kernels below need rows on 16 bytes).
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

// ---- few rows of x ---------------------------------------------------------

// A warp (or four, where the weight has few and long rows) takes one row of the weight against up to
// two rows of x: 16-byte loads, kAhead of them in flight, x from the L1 cache.  No piece waits for
// another; bound by the loads that the resident blocks keep in flight (35% of the memory's rate and
// 22% of the issue slots for 4,096 x 4,096).
constexpr int kFewRows = 2;
// ... and two rows of x only with a weight of few rows (us, here / below: 6,144 x 1,024 7.2 / 8.1,
// 1,024 x 12,288 10.0 / 12.7, 12,288 x 4,096 29.9 / 24; one row 22.6 there).
constexpr int64_t kFewTwo = 8192;

template <class T>
struct alignas(16) Eight {
  T v[8];
};

template <class T, int M, bool kGate, int kWarps>
__global__ void __launch_bounds__(128) linear_few_kernel(op_linear_t a) {
  constexpr int kAhead = kGate ? 2 : 4;
  __shared__ float sums[kWarps > 1 ? 4 : 1][2 * M];
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int64_t col = kWarps > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + warp;
  if (kWarps == 1 && col >= a.n) return;
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w) + col * a.w_row;
  const T* g = kGate ? static_cast<const T*>(a.gate) + col * a.gate_row : nullptr;
  // what the end needs is on its way while the weight is read
  T old = T(), b0 = T(), b1 = T();
  if (lane < M && warp < (kWarps > 1 ? 1 : 4)) {
    if (a.residual) old = static_cast<const T*>(a.residual)[lane * a.residual_row + col];
    if (a.bias) b0 = static_cast<const T*>(a.bias)[col];
    if (kGate && a.gate_bias) b1 = static_cast<const T*>(a.gate_bias)[col];
  }
  float v[M] = {}, z[M] = {};
  const int64_t whole = a.k & ~int64_t(7), step = 256 * kWarps;
  for (int64_t k0 = (kWarps > 1 ? warp * 256 : 0) + lane * 8; k0 < whole; k0 += step * kAhead) {
    // (x with the weight, not behind it: a cold x took 3.5 us more)
    Eight<T> b[kAhead], c[kGate ? kAhead : 1], y[M][kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (k0 + j * step < whole) {
        b[j] = *reinterpret_cast<const Eight<T>*>(w + k0 + j * step);
        if (kGate) c[j] = *reinterpret_cast<const Eight<T>*>(g + k0 + j * step);
#pragma unroll
        for (int r = 0; r < M; ++r) y[r][j] = *reinterpret_cast<const Eight<T>*>(x + r * a.x_row + k0 + j * step);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (k0 + j * step < whole) {
#pragma unroll
        for (int r = 0; r < M; ++r) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[r] = fmaf(up(y[r][j].v[i]), up(b[j].v[i]), v[r]);
            if (kGate) z[r] = fmaf(up(y[r][j].v[i]), up(c[j].v[i]), z[r]);
          }
        }
      }
  }
  if (whole + lane < a.k && (kWarps == 1 || warp == 0)) {
#pragma unroll
    for (int r = 0; r < M; ++r) {
      const float y = up(x[r * a.x_row + whole + lane]);
      v[r] = fmaf(y, up(w[whole + lane]), v[r]);
      if (kGate) z[r] = fmaf(y, up(g[whole + lane]), z[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < M; ++r)
#pragma unroll
    for (int d = 16; d; d /= 2) {
      v[r] += __shfl_xor_sync(0xffffffffu, v[r], d);
      if (kGate) z[r] += __shfl_xor_sync(0xffffffffu, z[r], d);
    }
  if (kWarps > 1) {
    if (lane == 0)
#pragma unroll
      for (int r = 0; r < M; ++r) sums[warp][r] = v[r], sums[warp][M + r] = z[r];
    __syncthreads();
    if (warp > 0) return;
#pragma unroll
    for (int r = 0; r < M; ++r) {
      v[r] = (sums[0][r] + sums[1][r]) + (sums[2][r] + sums[3][r]);
      if (kGate) z[r] = (sums[0][M + r] + sums[1][M + r]) + (sums[2][M + r] + sums[3][M + r]);
    }
  }
#pragma unroll
  for (int r = 0; r < M; ++r)
    if (lane == r) {
      float y = v[r];
      if (a.bias) y += up(b0);
      if (kGate) y *= act(a.gate_bias ? z[r] + up(b1) : z[r], a.act);
      else y = act(y, a.act);
      if (a.residual) y += up(old);
      down(y, static_cast<T*>(a.y) + r * a.y_row + col);
    }
}

template <class T, int M, bool kGate>
cudaError_t launch_few_rows(const op_linear_t& a, int sms, cudaStream_t st) {
  // four warps a row of the weight while one each leaves an SM fewer than eight, and rows that give
  // each several loads (us, one / four, rows x columns: 512 x 4,096 4.4 / 2.6, 1,024 x 12,288
  // 10.9 / 8.6, 2,048 x 4,096 6.1 / 6.9, 2,048 x 1,024 2.9 / 4.8)
  if (a.n < (int64_t)sms * 8 && a.k >= 2048) linear_few_kernel<T, M, kGate, 4><<<(unsigned)a.n, 128, 0, st>>>(a);
  else linear_few_kernel<T, M, kGate, 1><<<(unsigned)((a.n + 3) / 4), 128, 0, st>>>(a);
  return cudaGetLastError();
}

template <class T, bool kGate>
cudaError_t launch_few(const op_linear_t& a, int sms, cudaStream_t st) {
  switch (a.m) {
    case 1: return launch_few_rows<T, 1, kGate>(a, sms, st);
    default: return launch_few_rows<T, 2, kGate>(a, sms, st);
  }
}

// ---- aligned operands: tensor cores ---------------------------------------

// The weight is the operand whose 128 rows fill the tensor core's lanes, so that few rows of
// x cost few, and a step is 64 columns of both, brought by bulk copies into a ring of stages.
constexpr int kStep = 64;

constexpr int kWeightBytes = 128 * kStep * 2;

constexpr int kTailMax = 1 << 30;      // steps dealt out, at most

// ---- few tiles: a tile's columns split over a cluster

// A tile is 128 rows of the weight by up to 256 rows of x.  The blocks of a cluster take a share of
// its steps each, leave their sums in shared memory, and then each adds up and finishes a
// share of the rows, in the order of the blocks.  Bound by reading the weight: two blocks an
// SM keep 200 KB of it on the way (gated products of 17 to 32 rows 144, two stages of 36 a block).  (A second launch that adds partial results from memory took
// 2 to 3 us more, the last block adding them alone 40.)
template <int NT, bool kGate>
struct SplitShape {
  static constexpr int kXBytes = NT * kStep * 2;
  static constexpr int kStage = kWeightBytes * (kGate ? 2 : 1) + kXBytes;
  static constexpr int kStages = (NT <= 32 ? 106 : 212) * 1024 / kStage < 8 ? (NT <= 32 ? 106 : 212) * 1024 / kStage : 8;
  static constexpr int kSmem = kStages * kStage + 1024;
  static constexpr int kColumns = NT * (kGate ? 2 : 1);
  static constexpr int kAlloc = kColumns < 32 ? 32 : kColumns;
  static_assert(kColumns * 512 <= kStages * kStage, "the sums take the ring's place");
};

struct SplitArgs {
  op_linear_t a;
  int32_t split, steps, tiles_n;
  int32_t* status;
};

__device__ __forceinline__ float4 load_peer(uint32_t addr, uint32_t rank) {
  float4 v;
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}

template <class T>
struct alignas(8) Four {
  T v[4];
};

// Adds up and finishes rows first, first + 8 split, ... of the tile: four columns a lane, four rows
// at a time so that their loads overlap, then one by one.
template <int kAct, class T, int NT, bool kGate>
__device__ __forceinline__ void split_rows(const op_linear_t& a, uint32_t smem, int first, int split, int64_t row0, int rows,
                                           int64_t col) {
  const int n = a.n - col < 4 ? int(a.n - col) : 4;
  if (n <= 0) return;
  float bias[4] = {}, gate_bias[4] = {};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) {
      if (a.bias) bias[e] = up(static_cast<const T*>(a.bias)[col + e]);
      if (kGate && a.gate_bias) gate_bias[e] = up(static_cast<const T*>(a.gate_bias)[col + e]);
    }
  T* y = static_cast<T*>(a.y) + row0 * a.y_row + col;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + row0 * a.residual_row + col : nullptr;
  const bool wide_y = n == 4 && ((reinterpret_cast<uintptr_t>(y) | uintptr_t(a.y_row * 2)) & 7) == 0;
  const bool wide_res = n == 4 && ((reinterpret_cast<uintptr_t>(res) | uintptr_t(a.residual_row * 2)) & 7) == 0;
  const int step = 8 * split;
  auto take = [&](int r0, auto count) {
    constexpr int R = decltype(count)::value;
    float v[R][4] = {}, g[kGate ? R : 1][4] = {};
    Four<T> old[R];
    if (res) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const T* from = res + (r0 + i * step) * a.residual_row;
        if (wide_res) {
          old[i] = *reinterpret_cast<const Four<T>*>(from);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n) old[i].v[e] = from[e];
        }
      }
    }
#pragma unroll 2
    for (int32_t w = 0; w < split; ++w) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const uint32_t at = smem + ((r0 + i * step) * 128 + (threadIdx.x & 31) * 4) * 4;
        const float4 x = load_peer(at, w);
        v[i][0] += x.x, v[i][1] += x.y, v[i][2] += x.z, v[i][3] += x.w;
        if (kGate) {
          const float4 z = load_peer(at + NT * 512, w);
          float* to = g[kGate ? i : 0];
          to[0] += z.x, to[1] += z.y, to[2] += z.z, to[3] += z.w;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      T* to = y + (r0 + i * step) * a.y_row;
      Four<T> out;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float f = v[i][e] + bias[e];
        if (kGate) f *= act_of<kAct>(g[kGate ? i : 0][e] + gate_bias[e]);
        else f = act_of<kAct>(f);
        if (res) f += up(old[i].v[e]);
        down(f, &out.v[e]);
      }
      if (wide_y) {
        *reinterpret_cast<Four<T>*>(to) = out;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < n) to[e] = out.v[e];
      }
    }
  };
  int r = first;
#pragma unroll 1
  for (; r + 3 * step < rows; r += 4 * step) take(r, std::integral_constant<int, 4>{});
#pragma unroll 1
  for (; r < rows; r += step) take(r, std::integral_constant<int, 1>{});
}

template <class T, int NT, bool kGate>
__global__ void __launch_bounds__(256) linear_split_kernel(const __grid_constant__ CUtensorMap map_w,
                                                           const __grid_constant__ CUtensorMap map_g,
                                                           const __grid_constant__ CUtensorMap map_x,
                                                           const __grid_constant__ SplitArgs L) {
  using S = SplitShape<NT, kGate>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t bars[2 * S::kStages + 1];
  __shared__ uint32_t tmem_at, failed_word;
  volatile uint32_t* failed = &failed_word;
  const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
  float* sums = reinterpret_cast<float*>(raw + (smem - smem_addr(raw)));   // [columns][128], after the products
  const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  const op_linear_t& a = L.a;
  const int32_t all = blockIdx.x / L.split, rank = blockIdx.x - all * L.split;
  const int32_t tile_m = all / L.tiles_n, tile = all - tile_m * L.tiles_n;
  const int64_t row0 = (int64_t)tile_m * NT;
  const int rows = a.m - row0 < NT ? int(a.m - row0) : NT;
  const int32_t share = L.steps / L.split, more = L.steps - share * L.split;
  const int32_t k0 = rank * share + (rank < more ? rank : more), k1 = k0 + share + (rank < more);

  if (warp == 0 && lane == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    if (kGate) prefetch_map(&map_g);
    for (int i = 0; i < S::kStages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    bar_init(done, 1);
    failed_word = 0;
    fence_bar_init();
  }
  if (warp == 2) tmem_alloc<1>(smem_addr(&tmem_at), S::kAlloc);
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);

  // a whole warp goes along with one lane that issues, so that what the instructions take is known
  // to be the same in all lanes
  if (warp == 0) {
    uint32_t stage = 0, phase = 0, issued = 0;
    for (int32_t k = k0; k < k1; ++k) {
      if (!bar_wait(empty + 8 * stage, phase ^ 1, failed)) break;
      const uint32_t at = smem + stage * S::kStage, bar = full + 8 * stage;
      if (elect_one()) {
        bar_expect(bar, S::kStage);
        load_2d(at, &map_w, k * kStep, tile * 128, bar);
        if (kGate) load_2d(at + kWeightBytes, &map_g, k * kStep, tile * 128, bar);
        load_2d(at + S::kStage - S::kXBytes, &map_x, k * kStep, tile_m * NT, bar);
      }
      ++issued;
      if (++stage == S::kStages) stage = 0, phase ^= 1;
    }
    // every stage comes back before the block ends; after a failure the copies in flight get a
    // bounded wait each
    uint32_t quiet = 0;
    if (!gave_up(failed)) {
      for (int i = 0; i < S::kStages; ++i) {
        if (!bar_wait(empty + 8 * stage, phase ^ 1, failed)) break;
        if (++stage == S::kStages) stage = 0, phase ^= 1;
      }
    } else {
      for (uint32_t i = 0; i < S::kStages && i < issued; ++i) {
        if (stage == 0) phase ^= 1;
        stage = stage == 0 ? S::kStages - 1 : stage - 1;
        bar_pass(full + 8 * stage, phase, &quiet);
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc = mma_desc(std::is_same<T, __nv_bfloat16>::value, 128, NT, false);
    const uint64_t ring = tile_k(smem);
    uint32_t stage = 0, phase = 0;
    for (int32_t k = k0; k < k1; ++k) {
      if (!bar_wait(full + 8 * stage, phase, failed)) break;
      tc_after_sync();
      const uint64_t w = ring + stage * (S::kStage / 16), g = w + kWeightBytes / 16, x = w + (S::kStage - S::kXBytes) / 16;
      const bool add = k > k0;
      if (elect_one()) {
#pragma unroll
        for (int j = 0; j < kStep / 16; ++j) {
          mma_ss<1>(tmem, w + 2 * j, x + 2 * j, idesc, add || j > 0);
          if (kGate) mma_ss<1>(tmem + NT, g + 2 * j, x + 2 * j, idesc, add || j > 0);
        }
        mma_commit(empty + 8 * stage);
      }
      __syncwarp();
      if (++stage == S::kStages) stage = 0, phase ^= 1;
    }
    if (elect_one()) mma_commit(done);
  }
  __syncwarp();
  bar_pass(done, 0, failed);   // every copy has landed and been read
  tc_after_sync();
  {
    // the sums, [row of x][row of the weight]; warps of one half of the block take every other 16 rows
    const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    float* to = sums + (warp & 3) * 32 + lane;
#pragma unroll 1
    for (int c0 = (warp >> 2) * 16; c0 < rows; c0 += 32) {
      uint32_t v[16], g[kGate ? 16 : 1];
      tmem_load16(from + c0, v);
      if (kGate) tmem_load16(from + NT + c0, *reinterpret_cast<uint32_t(*)[kGate ? 16 : 1]>(g));
      tmem_wait_load();
      tmem_loaded(v);
      if (kGate) tmem_loaded(g);
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        to[(c0 + c) * 128] = __uint_as_float(v[c]);
        if (kGate) to[(NT + c0 + c) * 128] = __uint_as_float(g[kGate ? c : 0]);
      }
    }
  }
  tc_before_sync();
  __syncthreads();
  if (warp == 2) tmem_free<1>(tmem, S::kAlloc);
  if (L.split > 1) cluster_sync();
  const int64_t col = (int64_t)tile * 128 + lane * 4;
  switch (a.act) {
    case GMG_OP_RELU: split_rows<GMG_OP_RELU, T, NT, kGate>(a, smem, rank + warp * L.split, L.split, row0, rows, col); break;
    case GMG_OP_SILU: split_rows<GMG_OP_SILU, T, NT, kGate>(a, smem, rank + warp * L.split, L.split, row0, rows, col); break;
    case GMG_OP_GELU: split_rows<GMG_OP_GELU, T, NT, kGate>(a, smem, rank + warp * L.split, L.split, row0, rows, col); break;
    default: split_rows<GMG_OP_NONE, T, NT, kGate>(a, smem, rank + warp * L.split, L.split, row0, rows, col);
  }
  if (L.split > 1) cluster_sync();   // the others have read this block's sums
  if (threadIdx.x == 0 && *failed) atomicAdd(L.status, 1);
}

// ---- more rows of x: tiles over pairs of blocks

// A tile is 256 rows of the weight, 128 in each block of a pair, by 256 rows of x, half of
// them copied by each block.  A thread of the epilogue holds one weight row, i.e. one output
// column, and goes through the tile's rows of x; a warp writes 64 contiguous bytes of each.
//
// Tiles go to the workers (pairs, one for two SMs) in turn while they fill whole rounds.
// The steps of the tiles left over are dealt out evenly: a worker takes an equal run of
// them, which may end one tile and begin another.  A second launch adds the pieces of a tile
// in the order of their workers, so results do not depend on timing.
struct Sched {
  int32_t tiles_n, tiles_m, steps;     // weight-row tiles, x-row tiles, steps a tile
  int32_t workers, full;               // tiles taken whole
  int32_t tail, tail_workers;          // tiles dealt out by steps, to how many workers
  int32_t share, more;                 // steps of a tail worker; the first `more` take one more
  __host__ __device__ int32_t begin(int32_t w) const { return w * share + (w < more ? w : more); }
  __host__ __device__ int32_t owner(int32_t step) const {
    const int32_t longer = more * (share + 1);
    return step < longer ? step / (share + 1) : more + (step - longer) / share;
  }
};

struct Piece {
  int32_t tile_n, tile_m, k0, k1;
  int32_t tail_tile;                   // -1: a whole tile
  int32_t slot;                        // where a partial result goes
};

struct Pieces {
  const Sched& s;
  int32_t worker, tile, at, end;
  __device__ Pieces(const Sched& s, int32_t worker) : s(s), worker(worker), tile(worker), at(0), end(0) {
    if (worker < s.tail_workers) at = s.begin(worker), end = s.begin(worker + 1);
  }
  __device__ void place(int32_t t, Piece* p) const {
    // bands of eight x-row tiles, so that the workers of one time share rows of both operands
    const int32_t band = t / (8 * s.tiles_n), in = t - band * 8 * s.tiles_n;
    const int32_t wide = s.tiles_m - band * 8 < 8 ? s.tiles_m - band * 8 : 8;
    p->tile_n = in / wide;
    p->tile_m = band * 8 + in - p->tile_n * wide;
  }
  __device__ bool next(Piece* p) {
    if (tile < s.full) {
      place(tile, p);
      p->k0 = 0, p->k1 = s.steps, p->tail_tile = -1, p->slot = 0;
      tile += s.workers;
      return true;
    }
    if (at >= end) return false;
    const int32_t t = at / s.steps;
    place(s.full + t, p);
    p->k0 = at - t * s.steps;
    p->k1 = end - at < s.steps - p->k0 ? p->k0 + end - at : s.steps;
    p->tail_tile = p->k0 == 0 && p->k1 == s.steps ? -1 : t;
    p->slot = 2 * worker + (s.begin(worker) < t * s.steps);
    at += p->k1 - p->k0;
    return true;
  }
};

// The workers with a piece of tail tile t: from *first on, how many.  Only the first can have
// begun before the tile; its piece is then its second, in its second slot.
__device__ __forceinline__ int32_t pieces_of(const Sched& s, int32_t t, int32_t* first, int32_t* first_slot) {
  *first = s.owner(t * s.steps);
  *first_slot = 2 * *first + (s.begin(*first) < t * s.steps);
  return s.owner((t + 1) * s.steps - 1) - *first + 1;
}

constexpr int kHeadBytes = 4096;       // of the workspace: its first word counts waits that gave up

constexpr int kPair = 2, NT = 256;

template <bool kGate>
struct Shape {
  static constexpr int kXBytes = NT / kPair * kStep * 2;
  static constexpr int kStage = kWeightBytes * (kGate ? 2 : 1) + kXBytes;
  static constexpr int kStages = 212 * 1024 / kStage < 12 ? 212 * 1024 / kStage : 12;
  static constexpr int kSmem = kStages * kStage + 1024;
  static constexpr int kColumns = NT * (kGate ? 2 : 1);   // of TMEM, for one tile
  static constexpr int kBuffers = 2 * kColumns <= 512 ? 2 : 1;
  static constexpr int kAlloc = kColumns * kBuffers;
  static constexpr size_t kSlot = size_t(kColumns) * 128 * kPair;   // floats of a partial result
};

struct LinearArgs {
  op_linear_t a;
  Sched s;
  float* part;
  int32_t* status;
};

constexpr int kRoles = 384;            // warp 0 copies, 1 multiplies, 2 holds TMEM, 4 to 11 finish

// Finishes C rows of x of one output column from its sums.
template <int kAct, class T, bool kGate, int C>
__device__ __forceinline__ void finish_rows(const op_linear_t& a, const uint32_t (&v)[C], const uint32_t (&g)[kGate ? C : 1],
                                            float bias, float gate_bias, const T (&old)[C], bool add, T* y, int rows) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (c >= rows) break;
    float r = __uint_as_float(v[c]) + bias;
    if (kGate) r *= act_of<kAct>(__uint_as_float(g[kGate ? c : 0]) + gate_bias);
    else r = act_of<kAct>(r);
    if (add) r += up(old[c]);
    down(r, y + c * a.y_row);
  }
}

template <class T, bool kGate>
__global__ void __cluster_dims__(kPair, 1, 1) __launch_bounds__(kRoles) linear_kernel(const __grid_constant__ CUtensorMap map_w,
                                                        const __grid_constant__ CUtensorMap map_g,
                                                        const __grid_constant__ CUtensorMap map_x,
                                                        const __grid_constant__ LinearArgs L) {
  using S = Shape<kGate>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t bars[2 * S::kStages + 2 * S::kBuffers];
  __shared__ uint32_t tmem_at, failed_word;
  volatile uint32_t* failed = &failed_word;
  const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
  const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages,
                 drained = done + 8 * S::kBuffers;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int32_t worker = blockIdx.x / kPair;
  const Sched& s = L.s;

  if (warp == 0 && lane == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    if (kGate) prefetch_map(&map_g);
    for (int i = 0; i < S::kStages; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    for (int i = 0; i < S::kBuffers; ++i) bar_init(done + 8 * i, 1), bar_init(drained + 8 * i, 8 * kPair);
    failed_word = 0;
    fence_bar_init();
  }
  if (warp == 2) tmem_alloc<kPair>(smem_addr(&tmem_at), S::kAlloc);
  tc_before_sync();
  __syncthreads();
  cluster_sync();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);

  if (warp == 0) {
    // copies: a ring of stages, refilled as the products that read them complete
    uint32_t stage = 0, phase = 0, issued = 0;
    bool go = true;
    Pieces it(s, worker);
    Piece p;
    while (go && it.next(&p)) {
      const int32_t row_w = p.tile_n * (128 * kPair) + rank * 128, row_x = p.tile_m * NT + rank * (NT / kPair);
      for (int32_t k = p.k0; k < p.k1; ++k) {
        if (!(go = bar_wait(empty + 8 * stage, phase ^ 1, failed))) break;
        const uint32_t at = smem + stage * S::kStage;
        if (elect_one()) {
          // both blocks' copies count on the first block's barrier
          if (rank == 0) bar_expect(full + 8 * stage, 2 * S::kStage);
          const uint32_t bar = bar_of(full + 8 * stage, 0);
          load_2d_pair(at, &map_w, k * kStep, row_w, bar);
          if (kGate) load_2d_pair(at + kWeightBytes, &map_g, k * kStep, row_w, bar);
          load_2d_pair(at + S::kStage - S::kXBytes, &map_x, k * kStep, row_x, bar);
        }
        ++issued;
        if (++stage == S::kStages) stage = 0, phase ^= 1;
      }
    }
    // every stage comes back before the block ends: its copies have landed, and the products
    // have sent their arrivals; after a failure the copies in flight get a bounded wait each
    uint32_t quiet = 0;
    if (!gave_up(failed)) {
      for (int i = 0; i < S::kStages; ++i) {
        if (!bar_wait(empty + 8 * stage, phase ^ 1, failed)) break;
        if (++stage == S::kStages) stage = 0, phase ^= 1;
      }
    } else if (rank == 0) {
      for (uint32_t i = 0; i < S::kStages && i < issued; ++i) {
        if (stage == 0) phase ^= 1;
        stage = stage == 0 ? S::kStages - 1 : stage - 1;
        bar_pass(full + 8 * stage, phase, &quiet);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      constexpr uint32_t idesc = mma_desc(std::is_same<T, __nv_bfloat16>::value, 128 * kPair, NT, false);
      const uint64_t ring = tile_k(smem);
      uint32_t stage = 0, phase = 0;
      bool go = true;
      Pieces it(s, worker);
      Piece p;
      for (uint32_t n = 0; go && it.next(&p); ++n) {
        const uint32_t buf = n % S::kBuffers, d = tmem + buf * S::kColumns;
        if (!bar_wait(drained + 8 * buf, ((n / S::kBuffers) & 1) ^ 1, failed)) break;
        tc_after_sync();
        for (int32_t k = p.k0; k < p.k1; ++k) {
          if (!(go = bar_wait(full + 8 * stage, phase, failed))) break;
          tc_after_sync();
          const uint64_t w = ring + stage * (S::kStage / 16), g = w + kWeightBytes / 16, x = w + (S::kStage - S::kXBytes) / 16;
          const bool add = k > p.k0;
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < kStep / 16; ++j) {
              mma_ss<kPair>(d, w + 2 * j, x + 2 * j, idesc, add || j > 0);
              if (kGate) mma_ss<kPair>(d + NT, g + 2 * j, x + 2 * j, idesc, add || j > 0);
            }
            mma_commit_pair(empty + 8 * stage);
          }
          __syncwarp();
          if (++stage == S::kStages) stage = 0, phase ^= 1;
        }
        if (elect_one()) mma_commit_pair(done + 8 * buf);
        __syncwarp();
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    constexpr int C = 32;                  // rows of x at a time; two warps share a set of lanes
    const int part = warp & 3, odd = (warp - 4) >> 2;
    const op_linear_t& a = L.a;
    const uint32_t lanes = (uint32_t)(part * 32) << 16;
    const int feature = rank * 128 + part * 32 + lane;
    Pieces it(s, worker);
    Piece p;
    for (uint32_t n = 0; it.next(&p); ++n) {
      const uint32_t buf = n % S::kBuffers;
      const uint32_t d = tmem + lanes + buf * S::kColumns;
      const int64_t col = (int64_t)p.tile_n * (128 * kPair) + feature;
      const int64_t row0 = (int64_t)p.tile_m * NT;
      const int rows = a.m - row0 < NT ? int(a.m - row0) : NT;
      const bool in = col < a.n;
      float bias = 0.f, gate_bias = 0.f;
      if (in && a.bias) bias = up(static_cast<const T*>(a.bias)[col]);
      if (in && kGate && a.gate_bias) gate_bias = up(static_cast<const T*>(a.gate_bias)[col]);
      // a wait that gives up goes on with what it finds; the status says so
      bar_pass(done + 8 * buf, (n / S::kBuffers) & 1, failed);
      tc_after_sync();
      const T* res = a.residual ? static_cast<const T*>(a.residual) + row0 * a.residual_row + col : nullptr;
      T* y = static_cast<T*>(a.y) + row0 * a.y_row + col;
      float* mine = L.part + p.slot * S::kSlot + feature;
#pragma unroll 1
      for (int c0 = odd * C; c0 < rows; c0 += 2 * C) {
        uint32_t v[C], g[kGate ? C : 1];
        tmem_load32(d + c0, v);
        if (kGate) tmem_load32(d + NT + c0, g);
        const int here = rows - c0;
        T old[C];
        if (res && in && p.tail_tile < 0) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (c < here) old[c] = res[(c0 + c) * a.residual_row];
        }
        tmem_wait_load();
        tmem_loaded(v);
        if (kGate) tmem_loaded(g);
        if (p.tail_tile >= 0) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (c < here) {
              __stcg(mine + (c0 + c) * (128 * kPair), __uint_as_float(v[c]));
              if (kGate) __stcg(mine + (NT + c0 + c) * (128 * kPair), __uint_as_float(g[kGate ? c : 0]));
            }
        } else if (in) {
          T* to = y + c0 * a.y_row;
          switch (a.act) {
            case GMG_OP_RELU: finish_rows<GMG_OP_RELU, T, kGate, C>(a, v, g, bias, gate_bias, old, res, to, here); break;
            case GMG_OP_SILU: finish_rows<GMG_OP_SILU, T, kGate, C>(a, v, g, bias, gate_bias, old, res, to, here); break;
            case GMG_OP_GELU: finish_rows<GMG_OP_GELU, T, kGate, C>(a, v, g, bias, gate_bias, old, res, to, here); break;
            default: finish_rows<GMG_OP_NONE, T, kGate, C>(a, v, g, bias, gate_bias, old, res, to, here);
          }
        }
      }
      // TMEM may be written again
      tc_before_sync();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(bar_of(drained + 8 * buf, 0));
    }
    __syncwarp();
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  cluster_sync();   // the other block may still signal this one's barriers
  if (warp == 2) tmem_free<kPair>(tmem, S::kAlloc);
  if (threadIdx.x == 0 && *failed) atomicAdd(L.status, 1);
}

// Adds the pieces of the tail tiles: a warp takes a row of x and 128 output columns, four a
// lane, in the order of the pieces.
template <class T, bool kGate>
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearArgs L) {
  using S = Shape<kGate>;
  const Sched& s = L.s;
  const op_linear_t& a = L.a;
  const int32_t t = blockIdx.x / kPair, rank = blockIdx.x % kPair, lane = threadIdx.x & 31;
  int32_t first, slot;
  const int32_t all = pieces_of(s, t, &first, &slot);
  if (all == 1) return;      // written by the worker that had all of it
  Piece p;
  Pieces(s, 0).place(s.full + t, &p);
  const int32_t r = blockIdx.y * 8 + threadIdx.x / 32;
  const int64_t row = (int64_t)p.tile_m * NT + r;
  const int64_t col = (int64_t)p.tile_n * (128 * kPair) + rank * 128 + lane * 4;
  if (row >= a.m || col >= a.n) return;
  const float* from = L.part + r * (128 * kPair) + rank * 128 + lane * 4;
  float4 v = {}, g = {};
#pragma unroll 4
  for (int32_t w = 0; w < all; ++w) {
    const float* q = from + (w == 0 ? slot : 2 * (first + w)) * S::kSlot;
    const float4 x = __ldcg(reinterpret_cast<const float4*>(q));
    v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
    if (kGate) {
      const float4 y = __ldcg(reinterpret_cast<const float4*>(q + NT * (128 * kPair)));
      g.x += y.x, g.y += y.y, g.z += y.z, g.w += y.w;
    }
  }
  const float vs[4] = {v.x, v.y, v.z, v.w}, gs[4] = {g.x, g.y, g.z, g.w};
  finish4<T, kGate>(a, row, col, vs, gs);
}

int n_sm() {
  static std::atomic<int> count[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if ((n = count[dev].load(std::memory_order_relaxed)) == 0 &&
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
    count[dev].store(n, std::memory_order_relaxed);
  return n;
}

// How the tiles of pairs are dealt out, and the workspace.
Sched sched_for(const op_linear_t& a, int sms, size_t* work) {
  Sched s{};
  s.tiles_n = int32_t((a.n + 128 * kPair - 1) / (128 * kPair));
  s.tiles_m = int32_t((a.m + NT - 1) / NT);
  s.steps = int32_t((a.k + kStep - 1) / kStep);
  s.workers = sms / kPair;
  const int64_t tiles = (int64_t)s.tiles_n * s.tiles_m;
  s.full = int32_t(tiles / s.workers * s.workers);
  s.tail = int32_t(tiles - s.full);
  // Pieces a tile: each copies its share of the steps (a block takes in about 100 bytes a ns),
  // and pieces have to be written, read and added (a launch, and about 4,000 bytes a ns).
  const double step_ns = 0.01 * (a.gated ? Shape<true>::kStage : Shape<false>::kStage);
  const double slot = 4.0 * (a.gated ? Shape<true>::kSlot : Shape<false>::kSlot);
  const int64_t all = (int64_t)s.tail * s.steps;
  int64_t tw = s.tail;
  double best = s.steps * step_ns;
  for (int64_t n = 2; n <= 16 && all < kTailMax; ++n) {
    const int64_t w = s.tail * n < s.workers ? s.tail * n : s.workers;
    if (w <= tw || w > all) continue;
    const double ns = double(all) / w * step_ns + 2500.0 + 2 * slot * (w + s.tail) / 4000.0;
    if (ns < best) best = ns, tw = w;
  }
  s.tail_workers = int32_t(tw);
  if (tw > s.tail) {
    s.share = int32_t(all / tw);
    s.more = int32_t(all % tw);
  } else {
    s.share = s.steps;   // whole tiles only
  }
  *work = kHeadBytes + (tw > s.tail ? 2 * size_t(tw) * size_t(slot) : 0);
  return s;
}

struct Maps {
  CUtensorMap w, g, x;
};

bool make_maps(const op_linear_t& a, int32_t x_rows, Maps* m) {
  const int64_t size_w[2] = {a.k, a.n}, size_x[2] = {a.k, a.m};
  const int32_t box_w[2] = {kStep, 128}, box_x[2] = {kStep, x_rows};
  // a single row's stride is not used, but has to be a legal one
  const int64_t any = (a.k + 7) / 8 * 8;
  const int64_t sw = a.n == 1 ? any : a.w_row, sg = a.n == 1 ? any : a.gate_row, sx = a.m == 1 ? any : a.x_row;
  if (!make_map(&m->w, a.dtype, 2, a.w, size_w, &sw, box_w) || !make_map(&m->x, a.dtype, 2, a.x, size_x, &sx, box_x))
    return false;
  if (a.gated) return make_map(&m->g, a.dtype, 2, a.gate, size_w, &sg, box_w);
  m->g = m->w;
  return true;
}

template <class T, bool kGate>
cudaError_t launch_pairs(const op_linear_t& a, int sms, void* work, cudaStream_t st) {
  using S = Shape<kGate>;
  static gsim::OncePerDevice once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  auto kernel = linear_kernel<T, kGate>;
  if (!once.done(dev, [&] { return allow_smem(kernel, S::kSmem); }))
    return cudaErrorInvalidValue;
  Maps m;
  if (!make_maps(a, NT / kPair, &m)) return cudaErrorInvalidValue;
  LinearArgs L;
  size_t bytes;
  L.a = a;
  L.s = sched_for(a, sms, &bytes);
  L.status = static_cast<int32_t*>(work);
  L.part = reinterpret_cast<float*>(static_cast<char*>(work) + kHeadBytes);
  const int32_t busy = L.s.full > 0 ? L.s.workers : L.s.tail_workers;
  kernel<<<busy * kPair, kRoles, S::kSmem, st>>>(m.w, m.g, m.x, L);
  if (L.s.tail_workers > L.s.tail) {
    const int64_t rows = a.m < NT ? a.m : NT;
    linear_join_kernel<T, kGate><<<dim3((unsigned)(L.s.tail * kPair), (unsigned)((rows + 7) / 8)), 256, 0, st>>>(L);
  }
  return cudaGetLastError();
}

template <class T, int NT_, bool kGate>
cudaError_t launch_split(const op_linear_t& a, int sms, void* work, cudaStream_t st) {
  using S = SplitShape<NT_, kGate>;
  static gsim::OncePerDevice once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  auto kernel = linear_split_kernel<T, NT_, kGate>;
  if (!once.done(dev, [&] { return allow_smem(kernel, S::kSmem); }))
    return cudaErrorInvalidValue;
  Maps m;
  if (!make_maps(a, NT_, &m)) return cudaErrorInvalidValue;
  SplitArgs L;
  L.a = a;
  L.steps = int32_t((a.k + kStep - 1) / kStep);
  L.status = static_cast<int32_t*>(work);
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  // the widest clusters of which one a tile fits on the GPU at once: a second round costs as
  // much as the first (6,144 x 1,024, 16 rows, clusters of 6: 12 us, of 3: 7)
  L.tiles_n = int32_t((a.n + 127) / 128);
  const int64_t tiles = L.tiles_n * ((a.m + NT_ - 1) / NT_);
  static std::atomic<int> fits[64][9];   // clusters at once, by size; asked once per device
  for (L.split = L.steps < 8 ? L.steps : 8; L.split > 1; --L.split) {
    at[0].val.clusterDim.x = (unsigned)L.split;
    cfg.gridDim = dim3((unsigned)(sms / L.split * L.split));
    int n = dev < 64 ? fits[dev][L.split].load(std::memory_order_relaxed) : 0;
    if (n == 0 && cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) n = 0;
    if (dev < 64) fits[dev][L.split].store(n, std::memory_order_relaxed);
    if (n >= tiles) break;
  }
  at[0].val.clusterDim.x = (unsigned)L.split;
  cfg.gridDim = dim3((unsigned)(tiles * L.split));
  return cudaLaunchKernelEx(&cfg, kernel, m.w, m.g, m.x, L);
}

// Whether a call is one of few tiles: those of pairs would leave more than half of the SMs idle
// (us, over a cluster / over pairs: 4,096 x 4,096 with 256 rows 16.3 / 24.1, 512 rows 18.9 / 24.9,
// 1,024 rows, 64 tiles of pairs, 26.6 / 26.2; 12,288 x 4,096 with 256 rows, 48 tiles, 35.5 / 29.0).
bool few_tiles(const op_linear_t& a, int sms) {
  return a.m <= 128 || 2 * ((a.n + 255) / 256) * ((a.m + 255) / 256) <= sms / kPair;
}

template <class T, bool kGate>
cudaError_t launch_tiles(const op_linear_t& a, int sms, void* work, cudaStream_t st) {
  if (!few_tiles(a, sms)) return launch_pairs<T, kGate>(a, sms, work, st);
  if (a.m <= 16) return launch_split<T, 16, kGate>(a, sms, work, st);
  if (a.m <= 32) return launch_split<T, 32, kGate>(a, sms, work, st);
  if (a.m <= 64) return launch_split<T, 64, kGate>(a, sms, work, st);
  if (a.m <= 128 || kGate) return launch_split<T, 128, kGate>(a, sms, work, st);
  return launch_split<T, 256, false>(a, sms, work, st);
}

// Whether bulk copies can read the operands: rows on 16 bytes.
bool copyable(const op_linear_t& a) {
  auto ok = [](const void* p, int64_t row, int64_t rows) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows == 1 || row % 8 == 0);
  };
  return a.k > 0 && ok(a.x, a.x_row, a.m) && ok(a.w, a.w_row, a.n) && (!a.gated || ok(a.gate, a.gate_row, a.n)) &&
         a.x_row < (int64_t(1) << 38) && a.w_row < (int64_t(1) << 38) && a.gate_row < (int64_t(1) << 38);
}

template <class T>
cudaError_t launch(const op_linear_t& a, int sms, void* work, cudaStream_t st) {
  if (!copyable(a)) return launch_any<T>(a, st);
  if (a.m == 1 || (a.m <= kFewRows && a.n <= kFewTwo)) return a.gated ? launch_few<T, true>(a, sms, st) : launch_few<T, false>(a, sms, st);
  return a.gated ? launch_tiles<T, true>(a, sms, work, st) : launch_tiles<T, false>(a, sms, work, st);
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

size_t op_linear_work_bytes(const op_linear_t* args) {
  if (!args_ok(args)) return 0;
  const int sms = n_sm() > 1 ? n_sm() : 152;
  if (few_tiles(*args, sms) || args->n == 0 || !copyable(*args)) return kHeadBytes;
  size_t bytes;
  sched_for(*args, sms, &bytes);
  return bytes;
}

int op_linear(const op_linear_t* args, void* work, size_t work_bytes, gmg_stream_t stream) {
  if (!args_ok(args)) return GMG_EINVAL;
  if (!work || (reinterpret_cast<uintptr_t>(work) & 255) || work_bytes < op_linear_work_bytes(args)) return GMG_EWS;
  if (args->m == 0 || args->n == 0) return GMG_OK;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int sms = n_sm();
  if (sms < 2) return GMG_ECUDA;
  const cudaError_t e =
      args->dtype == GMG_OP_BF16 ? launch<__nv_bfloat16>(*args, sms, work, st) : launch<__half>(*args, sms, work, st);
  return e == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // extern "C"
