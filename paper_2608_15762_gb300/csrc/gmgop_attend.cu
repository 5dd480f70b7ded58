// Attention over a paged cache, with shared prefixes read once.  The C ABI is declared in
// include/gmgop.h.
//
// A work item is up to 128 rows (queries of consecutive tokens, all query heads of one
// key/value head: row = token * heads + head) against a run of keys, 64 a step.  One block
// takes one item:
//   warps 4 to 6   copies: page by page into a ring of 64-key slots, K_0 K_1 V_0 K_2 V_1 ...,
//            a warp every third slot (one warp takes 600 to 1,000 clocks to issue a slot's boxes)
//   warp 7   products: S_j = Q K_j^T into one of two TMEM buffers, O += P_j V_j into TMEM
//   warps 0 to 3   softmax: a thread holds one row.  It reads S_j, takes p = exp2(s c - m),
//            adds the sum, and puts P_j, rounded to the values' type, in S_j's place.
// S_{j+1} is computed while the softmax works on S_j.  The reference m need not be the exact
// running maximum, as it cancels: O is rescaled only where a score exceeds m by more than
// 2^8, so p stays below 2^8 (times 2^7 for fp16, whose small p would lose bits below 2^-14).
// P is rounded to the values' type because the tensor cores take it so (their sum l is of the
// unrounded ones): the error against 64 bits is 1.4 times that of probabilities in 32 bits.
//
// Queries that share a prefix lie next to each other, so a tile of rows reaches over their
// requests and every page of the prefix is read once a tile.  Long runs of keys are cut into
// several items; partial results (rows in fp32 with their log-sum-exp) are joined by a second
// kernel, in a fixed order.
//
// What bounds it, and what it measured (us a call, replayed; floor: bytes at 6.67 TB/s or products
// at 1,946 TFLOP/s):
//   32 requests of 6,000 tokens, one query each    125, floor 118: reading the cache
//   96 requests behind 32,768 shared tokens         74, floor 40: three tiles read the prefix from
//       the L2 cache (514 MB, 7.5 TB/s), then the start and end of 768 short items
//   chunks of prompts, 8,691 queries behind 4,000   242, floor 107: the softmax warps' instructions and
//       each step's waits (54% of the issue slots, two blocks an SM; the tensor cores are 41% busy)
//   8 requests behind 500 shared tokens             9.9: a launch and a chain of eight steps
// Two blocks an SM hide each other's waits; TMEM holds no third (O 128 columns, S and P 128).

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

#include "../../include/gmgop.h"
#include "gmg_once.h"
#include "gmgop_host.h"
#include "gmgop_ptx.cuh"

namespace gop {
namespace {

constexpr int kKeys = 64;              // a step
constexpr int kRows = 128;             // of a tile
constexpr int kThreads = 256, kCopiers = 3;
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

__device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
__device__ __forceinline__ uint32_t pack(__nv_bfloat16, float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack(__half, float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float unpack(__nv_bfloat16, uint32_t v, int i) { return __uint_as_float(i ? v & 0xffff0000u : v << 16); }
__device__ __forceinline__ float unpack(__half, uint32_t v, int i) {
  return __half2float(__ushort_as_half((unsigned short)(i ? v >> 16 : v & 0xffff)));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 in one 64-bit register pair: one instruction for both.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ void halves(uint64_t v, float* a, float* b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float v;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return v;
}

template <int DP>
struct Shape {
  static constexpr int kHalves = DP / 64;
  static constexpr int kQ = kRows * DP * 2;
  static constexpr int kSlot = kKeys * DP * 2;
  static constexpr int kSlots = 65536 / kSlot;
  static constexpr int kSmem = kQ + kSlots * kSlot + 1024;
  static constexpr int kColumns = 256;                    // of TMEM: O, then two buffers of S
};

// Place of V_j (and of K_j) in the order of copies, of n steps.
__device__ __forceinline__ int order_k(int j) { return j == 0 ? 0 : 2 * j - 1; }
__device__ __forceinline__ int order_v(int j, int n) { return j == n - 1 ? 2 * n - 1 : 2 * j + 2; }

template <class T, int DP>
__global__ void __launch_bounds__(kThreads, 2) attend_kernel(const __grid_constant__ CUtensorMap map_q,
                                                             const __grid_constant__ CUtensorMap map_kv,
                                                             const __grid_constant__ AttendArgs a) {
  using S = Shape<DP>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t bars[2 * S::kSlots + 8];
  __shared__ uint32_t tmem_at, failed_word, keep_o, bad[2][2];   // bad: keys of even and of odd steps
  volatile uint32_t* failed = &failed_word;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  // all heads of an item, then the next item: the long ones start first
  const int32_t item = blockIdx.x / a.n_kv, hk = blockIdx.x - item * a.n_kv;
  const Item it = a.items[item];
  const int32_t rows = it.n_tok * a.group;
  const int32_t first = it.lo / kKeys, n = it.hi > it.lo ? (it.hi + kKeys - 1) / kKeys - first : 0;

  if (n == 0) {   // queries that see nothing
    for (int r = threadIdx.x; r < rows; r += kThreads) {
      const int64_t t = it.tok0 + r / a.group;
      const int32_t h = hk * a.group + r % a.group;
      T* o = static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head;
      for (int d = 0; d < a.dim; d += 8) *reinterpret_cast<uint4*>(o + d) = uint4{};
      if (a.lse) a.lse[t * a.n_heads + h] = -INFINITY;
    }
    return;
  }

  const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
  unsigned char* base = raw + (smem - smem_addr(raw));
  const uint32_t slots = smem + S::kQ;
  const uint32_t full = smem_addr(bars), empty = full + 8 * S::kSlots, q_full = empty + 8 * S::kSlots,
                 s_full = q_full + 8, p_ready = s_full + 16, o_done = p_ready + 16, met = o_done + 16;
  // s_full, p_ready and o_done are two barriers each, for even and odd steps.  A wait tells a phase
  // from the one before it only, and every wait here has that one behind it: S_j is computed
  // after the product of step j - 2 is done.
  if (warp == 4 && lane == 0) {
    prefetch_map(&map_q);
    prefetch_map(&map_kv);
    for (int i = 0; i < S::kSlots; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
    bar_init(q_full, 1);
    bar_init(s_full, 1), bar_init(s_full + 8, 1);
    bar_init(p_ready, 4), bar_init(p_ready + 8, 4);
    bar_init(o_done, 1), bar_init(o_done + 8, 1);
    bar_init(met, 4);
    failed_word = keep_o = bad[0][0] = bad[0][1] = bad[1][0] = bad[1][1] = 0;
    fence_bar_init();
  }
  if (warp == 7) tmem_alloc<1>(smem_addr(&tmem_at), S::kColumns);
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0), tmem_s = tmem + 128;

  if (warp >= 4 && warp < 4 + kCopiers) {
    const int32_t box = a.page_tokens < kKeys ? a.page_tokens : kKeys;   // keys a copy
    if (warp == 4 && elect_one()) {
      const int32_t tile_rows = kRows / a.group * a.group;
      bar_expect(q_full, tile_rows * 128 * S::kHalves);
      for (int h = 0; h < S::kHalves; ++h) load_3d(smem + h * (kRows * 128), &map_q, h * 64, hk * a.group, it.tok0, q_full);
    }
    // the page numbers come 32 at a time, the next 32 on their way: a look-up for each slot took
    // about 1,000 clocks, twice what its products take
    const int shift = __ffs(a.page_tokens) - 1;
    const int32_t last = (it.hi - 1) >> shift;
    int32_t at0 = first * kKeys >> shift;
    auto look_up = [&](int32_t i) {
      const int32_t page = i <= last ? a.table[int64_t(it.row) * a.max_pages + i] : -1;
      return page >= 0 && page < a.n_pages ? page : a.n_pages;   // no such page: read as zeros
    };
    int32_t now = look_up(at0 + lane), next = look_up(at0 + 32 + lane);
    int e = warp - 4;
    for (; e < 2 * n; e += kCopiers) {
      // the e-th copy: K of step (e + 1) / 2 if e is 0 or odd (and not the last), else V
      const bool is_v = e == 2 * n - 1 || (e > 0 && e % 2 == 0);
      const int j = e == 2 * n - 1 ? n - 1 : is_v ? e / 2 - 1 : (e + 1) / 2;
      const int slot = e % S::kSlots;
      const int32_t k0 = (first + j) * kKeys;
      const int32_t from = it.lo > k0 ? (it.lo - k0) / box * box : 0, to = it.hi - k0 < kKeys ? it.hi - k0 : kKeys;
      if (is_v && (k0 >> shift) - at0 >= 32) {   // K is at most three steps ahead of V, 24 pages
        at0 += 32;
        now = next;
        next = look_up(at0 + 32 + lane);
      }
      // (this warp's copy before, three back, had all copies up to seven back consumed: the phase
      // before the one awaited is over, so the parity is not mistaken)
      if (!bar_wait(empty + 8 * slot, ((e / S::kSlots) & 1) ^ 1, failed)) break;
      const uint32_t bar = full + 8 * slot, dst = slots + slot * S::kSlot;
      if (elect_one()) bar_expect(bar, (to - from + box - 1) / box * box * 128 * S::kHalves);
      for (int32_t k = from; k < to; k += box) {
        const int32_t rel = ((k0 + k) >> shift) - at0;
        const int32_t page = rel < 32 ? __shfl_sync(0xffffffffu, now, rel) : __shfl_sync(0xffffffffu, next, rel - 32);
        const int32_t y = hk * a.page_tokens + ((k0 + k) & (a.page_tokens - 1)), z = page * a.planes + a.plane + is_v;
        if (elect_one())
#pragma unroll
          for (int h = 0; h < S::kHalves; ++h) load_3d(dst + h * (kKeys * 128) + k * 128, &map_kv, h * 64, y, z, bar);
      }
    }
    if (gave_up(failed)) {   // the copies in flight still have to land: a bounded wait for each
      uint32_t quiet = 0;
      for (int b = e - kCopiers; b >= 0 && b > e - kCopiers - S::kSlots; b -= kCopiers)
        bar_pass(full + 8 * (b % S::kSlots), (b / S::kSlots) & 1, &quiet);
      bar_pass(q_full, 0, &quiet);
    }
    __syncwarp();
  } else if (warp == 7) {
    // the whole warp goes along, so that what the instructions take is known to be the same in
    // all lanes; one lane issues
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t desc_s = mma_desc(kBf16, kRows, kKeys, false), desc_o = mma_desc(kBf16, kRows, DP, true);
    const uint32_t with = desc_s | (a.negative ? kMinusA : 0u);
    const uint64_t q = tile_k(smem), k_ring = tile_k(slots), v_ring = tile_n(slots, kKeys * 128);
    auto scores = [&](int j, uint32_t behind, uint32_t parity) {   // behind: what S_j waits for besides K_j
      const int e = order_k(j), slot = e % S::kSlots;
      if (!bar_wait_both(behind, parity, full + 8 * slot, (e / S::kSlots) & 1, failed)) return false;
      tc_after_sync();
      const uint64_t k = k_ring + slot * (S::kSlot / 16);
      const uint32_t d = tmem_s + (j & 1) * kKeys;
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
          mma_ss<1>(d, q + (i / 4) * (kRows * 128 / 16) + 2 * (i % 4), k + (i / 4) * (kKeys * 128 / 16) + 2 * (i % 4), with,
                    i > 0);
        mma_commit(empty + 8 * slot);
        mma_commit(s_full + 8 * (j & 1));
      }
      __syncwarp();
      return true;
    };
    bool go = scores(0, q_full, 0) && (n < 2 || scores(1, q_full, 0));
    for (int j = 0; go && j < n; ++j) {
      const int e = order_v(j, n), slot = e % S::kSlots;
      if (!bar_wait_both(p_ready + 8 * (j & 1), (j >> 1) & 1, full + 8 * slot, (e / S::kSlots) & 1, failed)) break;
      tc_after_sync();
      const uint64_t v = v_ring + slot * (S::kSlot / 16);
      const uint32_t p = tmem_s + (j & 1) * kKeys;
      const bool add = j > 0 || *reinterpret_cast<volatile uint32_t*>(&keep_o);
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < kKeys / 16; ++i) mma_ts(tmem, p + i * 8, v + i * (16 * 128 / 16), desc_o, add || i > 0);
        mma_commit(empty + 8 * slot);
        mma_commit(o_done + 8 * (j & 1));
      }
      __syncwarp();
      // S_{j+2} takes the place of P_j: once its product is done
      if (j + 2 < n) go = scores(j + 2, o_done + 8 * (j & 1), (j >> 1) & 1);
    }
    // the last arrival that nothing else waits for
    bar_pass(empty + 8 * ((2 * n - 1) % S::kSlots), ((2 * n - 1) / S::kSlots) & 1, failed);
  } else {
    const int r = threadIdx.x;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const int32_t tok = r / a.group;
    const float c = a.scale2;
    constexpr float kBias = std::is_same<T, __half>::value ? 7.f : 0.f;   // p is at most 2^(8 + kBias)
    // the keys that this row sees end here; rows beyond the tile's see what the last one does
    const int32_t own = tok < it.n_tok ? tok : it.n_tok - 1;
    const int32_t end = it.pos0 + own + 1 < it.hi ? it.pos0 + own + 1 : it.hi;
    const int32_t all_see = it.pos0 + 1 < it.hi ? it.pos0 + 1 : it.hi;    // keys that the first row sees
    float m = -INFINITY, l = 0.f;
    uint32_t meetings = 0;                // of the four warps: waits that are bounded, as all are
    for (int j = 0; j < n; ++j) {
      const int32_t k0 = (first + j) * kKeys;
      bar_pass(s_full + 8 * (j & 1), (j >> 1) & 1, failed);
      tc_after_sync();
      const uint32_t s_at = tmem_s + lanes + (j & 1) * kKeys;
      uint32_t lo[32], hi[32];
      tmem_load32(s_at, lo);
      tmem_load32(s_at + 32, hi);
      tmem_wait_load();
      tmem_loaded(lo);
      tmem_loaded(hi);
      const bool masked = k0 < it.lo || k0 + kKeys > all_see;
      // scores that this row does not see become -inf, and their p 0 (c > 0)
      uint64_t sees = ~0ull;
      if (masked) {
        const int below = it.lo > k0 ? it.lo - k0 : 0, upto = end - k0 < 0 ? 0 : end - k0 < kKeys ? end - k0 : kKeys;
        sees = upto <= below ? 0 : (upto == 64 ? ~0ull : (1ull << upto) - 1) & ~((1ull << below) - 1);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (!(sees >> i & 1)) lo[i] = 0xff800000u;
          if (!(sees >> (i + 32) & 1)) hi[i] = 0xff800000u;
        }
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        mx[0] = max3(mx[0], lo[i], lo[i + 1]);
        mx[1] = max3(mx[1], lo[i + 2], lo[i + 3]);
        mx[2] = max3(mx[2], hi[i], hi[i + 1]);
        mx[3] = max3(mx[3], hi[i + 2], hi[i + 3]);
      }
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      const float here = top * c;
      const bool raise = here > m + 8.f || (m == -INFINITY && here > -INFINITY);
      if (__any_sync(0xffffffffu, raise)) {
        const float f = raise ? (m == -INFINITY ? 0.f : exp2_fast(m - here)) : 1.f;
        if (raise) m = here;
        l *= f;
        if (j > 0) {
          bar_pass(o_done + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, failed);
          tc_after_sync();
#pragma unroll 1
          for (int d = 0; d < DP; d += 32) {
            uint32_t o[32];
            tmem_load32(tmem + lanes + d, o);
            tmem_wait_load();
            tmem_loaded(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_store32(tmem + lanes + d, o);
          }
          tmem_wait_store();
        }
      }
      // p, packed over the first half of the scores' registers
      const float shift = m == -INFINITY ? 0.f : kBias - m;
      const uint64_t c2 = two(c, c), shift2 = two(shift, shift);
      uint64_t sum[4] = {};
      uint32_t p[32];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x, y, z, w;
        halves(fma2(two(__uint_as_float(lo[2 * i]), __uint_as_float(lo[2 * i + 1])), c2, shift2), &x, &y);
        halves(fma2(two(__uint_as_float(hi[2 * i]), __uint_as_float(hi[2 * i + 1])), c2, shift2), &z, &w);
        x = exp2_fast(x), y = exp2_fast(y), z = exp2_fast(z), w = exp2_fast(w);
        sum[i & 1] = add2(sum[i & 1], two(x, y));
        sum[2 + (i & 1)] = add2(sum[2 + (i & 1)], two(z, w));
        p[i] = pack(T(), x, y);
        p[16 + i] = pack(T(), z, w);
      }
      {
        float x, y;
        halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), &x, &y);
        l += x + y;
      }
      tmem_store32(s_at, p);
      tmem_wait_store();
      if (masked) {
        // Keys outside the item: whatever lies there must not meet the zeros of P.  So must
        // no value that is not finite and that some row does not see.
        const int e = order_v(j, n), slot = e % S::kSlots;
        bar_pass(full + 8 * slot, (e / S::kSlots) & 1, failed);
        unsigned char* v = base + S::kQ + slot * S::kSlot;
        const int below = it.lo > k0 ? it.lo - k0 : 0, upto = it.hi - k0 < kKeys ? it.hi - k0 : kKeys;
        for (int i = r; i < kKeys * S::kHalves; i += 128) {
          const int key = i % kKeys;
          if (key >= below && key < upto) continue;
          uint4* at = reinterpret_cast<uint4*>(v + (i / kKeys) * (kKeys * 128) + key * 128);
#pragma unroll
          for (int q = 0; q < 8; ++q) at[q] = uint4{};
        }
        if (k0 + kKeys > all_see && all_see < it.hi) {
          // Words by step parity: a warp may be in the next step while another has yet to read this
          // one's, but no further (S_{j+2} waits for every warp's P_j).
          uint32_t* mine = bad[j & 1];
          constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
          for (int i = r; i < kKeys * S::kHalves; i += 128) {
            const int key = i % kKeys;
            if (key < below || key >= upto) continue;
            const uint4* at = reinterpret_cast<const uint4*>(v + (i / kKeys) * (kKeys * 128) + key * 128);
            bool odd = false;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint4 x = at[q];
              const uint32_t w[4] = {x.x & kExp, x.y & kExp, x.z & kExp, x.w & kExp};
#pragma unroll
              for (int b = 0; b < 4; ++b) odd |= (w[b] & 0xffff) == (kExp & 0xffff) || w[b] >> 16 == kExp >> 16;
            }
            if (odd) atomicOr(&mine[key >> 5], 1u << (key & 31));
          }
          bar_meet(met, &meetings, failed);
          // one answer for the warp (after a wait gave up, others may find otherwise)
          const uint64_t found = __shfl_sync(0xffffffffu, (uint64_t)*reinterpret_cast<volatile uint32_t*>(&mine[1]) << 32 |
                                                              *reinterpret_cast<volatile uint32_t*>(&mine[0]), 0);
          if (found) {
            // Their share of O is added here, to the rows that see them; the products get zeros.
            if (j > 0) {
              bar_pass(o_done + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, failed);
              tc_after_sync();
            }
#pragma unroll 1
            for (int d = 0; d < DP; d += 32) {
              uint32_t o[32];
              tmem_load32(tmem + lanes + d, o);
              tmem_wait_load();
              tmem_loaded(o);
              if (j == 0) {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0;
              }
#pragma unroll 1
              for (uint64_t rest = found; rest; rest &= rest - 1) {
                const int key = __ffsll((long long)rest) - 1;
                uint32_t pair;
                tmem_load1(s_at + key / 2, &pair);
                tmem_wait_load();
                asm volatile("" : "+r"(pair));
                if (sees >> key & 1) {
                  const float weight = unpack(T(), pair, key & 1);
                  const T* row = reinterpret_cast<const T*>(v + (d / 64) * (kKeys * 128) + key * 128);
#pragma unroll
                  for (int i = 0; i < 32; ++i) {
                    const int x = (d & 32) + i;
                    o[i] = __float_as_uint(fmaf(weight, up(row[(((x / 8) ^ (key & 7)) * 8) + x % 8]), __uint_as_float(o[i])));
                  }
                }
                __syncwarp();
              }
              tmem_store32(tmem + lanes + d, o);
            }
            tmem_wait_store();
            bar_meet(met, &meetings, failed);
            for (int i = r; i < kKeys * S::kHalves; i += 128)
              if (found >> (i % kKeys) & 1) {
                uint4* at = reinterpret_cast<uint4*>(v + (i / kKeys) * (kKeys * 128) + (i % kKeys) * 128);
#pragma unroll
                for (int q = 0; q < 8; ++q) at[q] = uint4{};
              }
            if (r == 0) {
              mine[0] = mine[1] = 0;
              if (j == 0) keep_o = 1;
            }
            bar_meet(met, &meetings, failed);
          }
        }
        fence_async();
      }
      tc_before_sync();
      __syncwarp();
      if (lane == 0) bar_arrive(p_ready + 8 * (j & 1));
    }
    bar_pass(o_done + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, failed);
    tc_after_sync();
    const bool in = tok < it.n_tok;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float lse2 = l == 0.f ? -INFINITY : m - kBias + log2f(l);
    const int32_t h = hk * a.group + r - tok * a.group;
    const int64_t t = it.tok0 + tok;
    const int64_t part = hk * a.part_rows + it.part + r;
    T* out = static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head;
    float* part_o = a.part_o + part * a.dim;
    if (in) {
      if (it.part >= 0) a.part_lse[part] = lse2;
      else if (a.lse) a.lse[t * a.n_heads + h] = lse2 * 0.69314718055994531f;
    }
#pragma unroll 1
    for (int d = 0; d < a.dim; d += 32) {
      uint32_t o[32];
      tmem_load32(tmem + lanes + d, o);
      tmem_wait_load();
      tmem_loaded(o);
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(l == 0.f ? 0.f : __uint_as_float(o[i]) * inv);
      if (in && it.part >= 0) {
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          if (d + i < a.dim) __stcg(reinterpret_cast<uint4*>(part_o + d + i), uint4{o[i], o[i + 1], o[i + 2], o[i + 3]});
      } else if (in) {
#pragma unroll
        for (int i = 0; i < 32; i += 8)
          if (d + i < a.dim) {
            uint4 v;
            v.x = pack(T(), __uint_as_float(o[i]), __uint_as_float(o[i + 1]));
            v.y = pack(T(), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
            v.z = pack(T(), __uint_as_float(o[i + 4]), __uint_as_float(o[i + 5]));
            v.w = pack(T(), __uint_as_float(o[i + 6]), __uint_as_float(o[i + 7]));
            *reinterpret_cast<uint4*>(out + d + i) = v;
          }
      }
      __syncwarp();
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (warp == 7) tmem_free<1>(tmem, S::kColumns);
  if (threadIdx.x == 0 && *failed) atomicAdd(&a.status[5], 1);
}

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
  int32_t steps() const { return hi > lo ? (hi + kKeys - 1) / kKeys - lo / kKeys : 0; }
};

constexpr int64_t kMinSteps = 6;   // of an item that is cut (16 requests behind 8,000 tokens: 2 25 us, 6 15, 8 15; 8 short ones: 6 11, 8 13)
// Up to so many steps a block takes alone, where one round of blocks is enough (us on the GPU / a call
// from the host, joined and alone: 8 requests behind 500 tokens 11.4 / 16.5 and 9.7 / 12.8, 32 of up to
// 616 tokens 13.9 / 17.0 and 11.8 / 13.1; with 16 steps one request of 1,000 tokens 11.8 and 14.0).
constexpr int64_t kAloneSteps = 12;
constexpr int64_t kItemSteps = 4;  // what an item costs beyond its steps (0: 96 requests behind 32,768 tokens 81 us, 4: 73)
constexpr int64_t kJoinSteps = 8;  // what writing and joining a tile's partial results costs, in steps

void plan_items(const op_attend_desc_t& d, int32_t n_sm, Work* w) {
  const int32_t group = d.n_heads / d.n_kv_heads, tile = kRows / group;
  // a small step, which one round of blocks takes with a few steps each: apart and uncut, so that
  // nothing is left to join
  int64_t alone = 0, longest = 0;
  for (int32_t b = 0; b < d.n_batch; ++b) {
    alone += (d.q_len[b] + tile - 1) / tile;
    if (d.q_len[b] > 0) longest = std::max<int64_t>(longest, (d.kv_len[b] + kKeys - 1) / kKeys);
  }
  const bool small = alone * d.n_kv_heads <= 2 * n_sm && longest <= kAloneSteps;
  std::vector<Run> runs;
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
    const bool pool = !small && (apart - together) * (prefix / kKeys) > kJoinSteps * together + apart;
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
  for (const Run& r : runs) steps += r.steps() + kItemSteps;
  const int64_t most = std::max(small ? kAloneSteps : kMinSteps, (steps * d.n_kv_heads + 2 * n_sm - 1) / (2 * n_sm));
  // cut; then longest first, so that short items fill the end (equal ones keep their order:
  // tiles that read the same keys stay together)
  struct Cut {
    int32_t run, part, parts;
  };
  std::vector<int32_t> parts(runs.size()), base(runs.size(), -1), joined(runs.size(), 0);
  for (size_t i = 0; i < runs.size(); ++i) parts[i] = int32_t(std::max<int64_t>(1, (runs[i].steps() + most - 1) / most));
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
    return runs[x.run].steps() / x.parts > runs[y.run].steps() / y.parts;
  });
  for (const Cut& cut : cuts) {
    const Run& r = runs[cut.run];
    const int64_t s0 = r.lo / kKeys, n = r.steps();
    const int64_t a = s0 + n * cut.part / cut.parts, b = s0 + n * (cut.part + 1) / cut.parts;
    Item it{};
    it.tok0 = r.tok0, it.n_tok = r.n_tok, it.row = r.row, it.pos0 = r.pos0;
    it.lo = std::max(r.lo, int32_t(a * kKeys));
    it.hi = int32_t(std::min<int64_t>(r.hi, b * kKeys));
    if (n == 0) it.lo = it.hi = 0;
    it.part = base[cut.run] < 0 ? -1 : base[cut.run] + cut.part * r.n_tok * group;
    w->items.push_back(it);
  }
}

template <class T, int DP>
cudaError_t launch(const op_attend_plan_t& p, const CUtensorMap& q, const CUtensorMap& kv, const AttendArgs& a, cudaStream_t st) {
  static gsim::OncePerDevice once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  auto kernel = attend_kernel<T, DP>;
  if (!once.done(dev, [&] { return allow_smem(kernel, Shape<DP>::kSmem); }))
    return cudaErrorInvalidValue;
  kernel<<<(unsigned)(p.n_items * (int64_t)p.n_kv_heads), kThreads, Shape<DP>::kSmem, st>>>(q, kv, a);
  if (p.n_joins > 0) {
    const int64_t heads = (int64_t)p.join_tokens * p.n_heads;
    attend_join_kernel<T><<<dim3((unsigned)p.n_joins, (unsigned)std::min<int64_t>(heads, 1024)), 128, 0, st>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

int op_attend_plan(const op_attend_desc_t* d, int32_t n_sm, op_attend_plan_t* plan, int32_t* items,
                   size_t item_bytes) try {
  if (!desc_ok(d) || !plan || n_sm < 1) return GMG_EINVAL;
  Work w;
  plan_items(*d, n_sm, &w);
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
  if (items) {
    if (item_bytes < p.plan_bytes) return GMG_EWS;
    Item* to = reinterpret_cast<Item*>(items);
    std::copy(w.items.begin(), w.items.end(), to);
    std::copy(w.joins.begin(), w.joins.end(), reinterpret_cast<Join*>(to + w.items.size()));
  }
  *plan = p;
  return GMG_OK;
} catch (const std::bad_alloc&) {
  return GMG_ENOMEM;
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
  if (!d_items || (reinterpret_cast<uintptr_t>(d_items) & 15) || !q || !out || !aligned(q, q_tok, q_head, 2) ||
      !aligned(out, out_tok, out_head, 2) || !(scale == scale))
    return GMG_EINVAL;
  if (!work || (reinterpret_cast<uintptr_t>(work) & 255) || work_bytes < plan->work_bytes) return GMG_EWS;
  const int64_t plane = int64_t(cache->n_kv_heads) * cache->page_tokens;   // rows of a page's K or V
  const int64_t planes = int64_t(cache->n_pages) * cache->n_layers * 2;
  if (planes + 2 * cache->n_layers > 0x7fffffff || plane > 0x7fffffff) return GMG_ERANGE;
  AttendArgs a{};
  a.items = reinterpret_cast<const Item*>(d_items);
  a.joins = reinterpret_cast<const Join*>(a.items + plan->n_items);
  a.table = cache->table;
  a.status = cache->status;
  a.max_pages = cache->max_pages;
  a.page_tokens = cache->page_tokens;
  a.n_pages = cache->n_pages;
  a.planes = cache->n_layers * 2;
  a.plane = layer * 2;
  a.n_heads = plan->n_heads;
  a.n_kv = plan->n_kv_heads;
  a.group = plan->n_heads / plan->n_kv_heads;
  a.dim = plan->head_dim;
  // a scale of 0 gives every key one weight, as a tiny one does, whose product with -inf is -inf
  a.scale2 = fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-30f);
  a.negative = scale < 0.f;
  a.out = out, a.o_tok = out_tok, a.o_head = out_head;
  a.lse = lse;
  a.part_rows = plan->part_rows;
  a.part_o = reinterpret_cast<float*>(work);
  a.part_lse = a.part_o + plan->part_rows * plan->n_kv_heads * plan->head_dim;
  CUtensorMap map_q, map_kv;
  const int32_t box = cache->page_tokens < kKeys ? cache->page_tokens : kKeys;
  const int64_t size_q[3] = {plan->head_dim, plan->n_heads, plan->n_tokens};
  // strides of a single head or token are not used, but have to be legal ones
  const int64_t stride_q[2] = {plan->n_heads > 1 ? q_head : plan->head_dim, plan->n_tokens > 1 ? q_tok : plan->head_dim};
  const int32_t box_q[3] = {64, a.group, kRows / a.group};
  const int64_t size_kv[3] = {plan->head_dim, plane, planes}, stride_kv[2] = {plan->head_dim, plane * plan->head_dim};
  const int32_t box_kv[3] = {64, box, 1};
  if (!make_map(&map_q, cache->dtype, 3, q, size_q, stride_q, box_q) ||
      !make_map(&map_kv, cache->dtype, 3, cache->pool, size_kv, stride_kv, box_kv))
    return GMG_ECUDA;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (cache->dtype == GMG_OP_BF16)
    e = plan->head_dim <= 64 ? launch<__nv_bfloat16, 64>(*plan, map_q, map_kv, a, st)
                             : launch<__nv_bfloat16, 128>(*plan, map_q, map_kv, a, st);
  else
    e = plan->head_dim <= 64 ? launch<__half, 64>(*plan, map_q, map_kv, a, st)
                             : launch<__half, 128>(*plan, map_q, map_kv, a, st);
  return e == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // extern "C"
