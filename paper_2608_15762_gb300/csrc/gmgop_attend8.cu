// Attention over a paged cache in 8 bits, with a scale for each block of 16 tokens and head.  The C
// ABI is declared in include/gmgop.h.
//
// With value scales v_j, P holds w = exp2(s + log2 v - m) and a row's sum takes w / v: one exponent
// for both, so that P uses its type's range whatever the scales, and O has them right.  The reference
// m is of the w and need not be the exact running maximum: it is raised where a w would exceed
// a power of two times it.
//
// Tiles of up to 16 rows (queries of consecutive tokens, all query heads of one key/value head:
// row = token * heads + head), a decode step's, turn the products round:
//   S^T [128 keys][rows] = K Q^T,   O^T [128 dims][rows] += V^T P^T.
// Keys fill the tensor core's 128 lanes and rows are columns, so that a step of few rows costs few columns,
// exponentials and registers, and K and V are read once, as the codes that they are, by fp8 products.
// What the codes meet is split into several of them: Q as bf16 and fp16 have it, P to 12 bits, small weights too.
// Memory bounds it where there is enough to read (the decode step below: 167 us, 6.5 TB/s); a small step is a
// launch and the chain of its few steps (8 requests behind 500 tokens 9.9 us).
//
// Tiles of more rows, up to 128, lie with their rows on the lanes, against 64 keys a step.  K is taken as the
// codes that it is here too, by Q's.  V becomes fp16, which holds e4m3 exactly, on its way through shared
// memory, which costs fewer instructions than splitting P would; P is fp16: its rounding, 2^-11, is what the
// tensor cores take.  The softmax warps' instructions and the latency of a step's chain bound it: chunks of prompts
// take 335 us at 57% of the issue slots and 25% of the tensor cores' cycles, and 96 requests behind 32,768 shared tokens
// 83 us at 50% and 38%.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "../../include/gmgop.h"
#include "gmg_once.h"
#include "gmgop_attend.cuh"
#include "gmgop_host.h"
#include "gmgop_ptx.cuh"

namespace gop {
namespace {

constexpr int kCopiers = 3;
constexpr float kNone = -3e38f;        // the reference of a row that has seen nothing: below any score

struct Args8 {
  AttendArgs a;
  const void* q;
  int64_t q_tok, q_head;
  const unsigned char* pool;
  int64_t page_bytes, scale_at;        // of a page; of the layer's scales in it
};

__device__ __forceinline__ void wide16(uint4 v, uint32_t* o) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = wide2((uint16_t)w[i]);
    o[2 * i + 1] = wide2((uint16_t)(w[i] >> 16));
  }
}

// 16 codes of a row of a slot, where the copy has put them.
template <int DP>
__device__ __forceinline__ uint4* codes_at(unsigned char* slot, int row, int c) {
  const int x = DP == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3);
  return reinterpret_cast<uint4*>(slot + row * DP + x * 16);
}

__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

__device__ __forceinline__ void tmem_load4(uint32_t addr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(addr));
}
// Registers of a warp group's threads: what the copies and products leave, the softmax has.
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// Queries that see nothing.
template <class T>
__device__ void sees_nothing(const AttendArgs& a, const Item& it, int32_t hk, int32_t rows) {
  for (int r = threadIdx.x; r < rows; r += blockDim.x) {
    const int64_t t = it.tok0 + r / a.group;
    const int32_t h = hk * a.group + r % a.group;
    T* o = static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head;
    for (int d = 0; d < a.dim; d += 8) *reinterpret_cast<uint4*>(o + d) = uint4{};
    if (a.lse) a.lse[t * a.n_heads + h] = -INFINITY;
  }
}

// Scales of eight steps, as the copying warps bring them: a step's blocks of 16 keys, K's and then V's.  With the
// slots that there are a step's place is read before the copies are eight steps further.
constexpr int kScaleSteps = 8;
template <int kKeys>
struct ScaleRing {
  float s[kScaleSteps][2][kKeys / 16];
};
__device__ __forceinline__ void copy_word(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// An arrival on `bar` when this thread's copies so far are done.
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
constexpr int kFullCount = 33;        // arrivals at a slot's barrier: of its bytes, and of each lane's scales

// A copying warp: every kCopiers-th slot of K_0 K_1 V_0 K_2 V_1 ..., page by page, rows of kRow bytes;
// with K_j the scales of step j.
template <int kKeys, int kRow, int kSlots>
__device__ __forceinline__ void copy_pages(const CUtensorMap& map, const Args8& g, const Item& it, int32_t hk, int32_t first,
                                           int32_t n, int e, int lane, uint32_t slots, uint32_t full, uint32_t empty,
                                           ScaleRing<kKeys>& scales, volatile uint32_t* failed) {
  const AttendArgs& a = g.a;
  const int32_t box = a.page_tokens < kKeys ? a.page_tokens : kKeys;   // keys a copy
  // the page numbers come 32 at a time, the next 32 on their way
  const int shift = __ffs(a.page_tokens) - 1;
  const int32_t last = (it.hi - 1) >> shift;
  int32_t at0 = first * kKeys >> shift;
  auto look_up = [&](int32_t i) {
    const int32_t page = i <= last ? a.table[int64_t(it.row) * a.max_pages + i] : -1;
    return page >= 0 && page < a.n_pages ? page : a.n_pages;   // no such page: read as zeros
  };
  int32_t now = look_up(at0 + lane), next = look_up(at0 + 32 + lane);
  auto page_at = [&](int32_t rel) {
    const int32_t x = __shfl_sync(0xffffffffu, now, rel & 31), y = __shfl_sync(0xffffffffu, next, rel & 31);
    return rel < 32 ? x : y;
  };
  for (; e < 2 * n; e += kCopiers) {
    // the e-th copy: K of step (e + 1) / 2 if e is 0 or odd (and not the last), else V
    const bool is_v = e == 2 * n - 1 || (e > 0 && e % 2 == 0);
    const int j = e == 2 * n - 1 ? n - 1 : is_v ? e / 2 - 1 : (e + 1) / 2;
    const int slot = e % kSlots;
    const int32_t k0 = (first + j) * kKeys;
    const int32_t from = it.lo > k0 ? (it.lo - k0) / box * box : 0, to = it.hi - k0 < kKeys ? it.hi - k0 : kKeys;
    if (is_v && (k0 >> shift) - at0 >= 32) {   // K is at most three steps ahead of V, 24 pages
      at0 += 32;
      now = next;
      next = look_up(at0 + 32 + lane);
    }
    if (!bar_wait(empty + 8 * slot, ((e / kSlots) & 1) ^ 1, failed)) break;
    const uint32_t bar = full + 8 * slot, dst = slots + slot * (kKeys * kRow);
    if (elect_one()) bar_expect(bar, (to - from + box - 1) / box * box * kRow);
    for (int32_t k = from; k < to; k += box) {
      const int32_t page = page_at(((k0 + k) >> shift) - at0);
      const int32_t y = ((a.plane + is_v) * a.n_kv + hk) * a.page_tokens + ((k0 + k) & (a.page_tokens - 1));
      if (elect_one()) load_3d(dst + k * kRow, &map, 0, y, page, bar);
    }
    if (!is_v) {
      constexpr int kBlocks = kKeys / 16;
      const int32_t k = k0 + lane % kBlocks * 16, v = lane / kBlocks & 1;
      const int32_t page = page_at((k >> shift) - at0);
      float* at = &scales.s[j & (kScaleSteps - 1)][v][lane % kBlocks];
      if (lane < 2 * kBlocks) {
        if (page < a.n_pages && k < it.hi) {
          const int32_t blocks = a.page_tokens / 16;
          copy_word(smem_addr(at), g.pool + page * g.page_bytes + g.scale_at +
                                       4 * (int64_t(v * a.n_kv + hk) * blocks + (k & (a.page_tokens - 1)) / 16));
        } else {
          *at = 1.f;
        }
      }
    }
    copies_arrive(bar);
  }
  if (gave_up(failed)) {   // the copies in flight still have to land: a bounded wait for each
    uint32_t quiet = 0;
    for (int b = e - kCopiers; b >= 0 && b > e - kCopiers - kSlots; b -= kCopiers)
      bar_pass(full + 8 * (b % kSlots), (b / kSlots) & 1, &quiet);
  }
  __syncwarp();
}

__device__ __forceinline__ bool has_nan(uint4 v) {
  const uint32_t any = ((v.x & 0x7f7f7f7fu) + 0x01010101u) | ((v.y & 0x7f7f7f7fu) + 0x01010101u) |
                       ((v.z & 0x7f7f7f7fu) + 0x01010101u) | ((v.w & 0x7f7f7f7fu) + 0x01010101u);
  return any & 0x80808080u;
}
// Codes that are NaN become zeros; first_nan, a byte a dimension, falls to the first query that sees one.  (Apart from the
// loops that need it so rarely: its instructions would lie between theirs.)
__device__ __noinline__ uint4 without_nan(uint4 v, uint32_t* first_nan, uint32_t query) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll 1
    for (int b = 0; b < 4; ++b)
      if ((w[i] >> (8 * b) & 0x7f) == 0x7f) {
        uint32_t was = *reinterpret_cast<volatile uint32_t*>(first_nan + i);
        while ((was >> (8 * b) & 0xff) > query) {   // (ends: the byte only falls)
          const uint32_t found = atomicCAS(first_nan + i, was, (was & ~(0xffu << (8 * b))) | query << (8 * b));
          if (found == was) break;
          was = found;
        }
        w[i] &= ~(0xffu << (8 * b));
      }
  return uint4{w[0], w[1], w[2], w[3]};
}

// 16 columns over the warp's lanes (two a register pair), summed or their largest: lane 2 i has column i's in the end.
template <class F>
__device__ __forceinline__ void over_lanes(const uint64_t* pairs, float* out, int lane, F join) {
  float x[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) halves(pairs[i], &x[2 * i], &x[2 * i + 1]);
  // each step keeps half of the columns
#pragma unroll
  for (int d = 16, k = 8; k; d /= 2, k /= 2) {
    const bool upper = lane & d;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < k) {
        const float give = upper ? x[i] : x[i + k];
        const float keep = upper ? x[i + k] : x[i];
        x[i] = join(keep, __shfl_xor_sync(0xffffffffu, give, d));
      }
  }
  x[0] = join(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
  if (!(lane & 1)) out[lane / 2] = x[0];
}
__device__ __forceinline__ void column_sums(const uint64_t* l2, float* out, int lane) {
  over_lanes(l2, out, lane, [](float a, float b) { return a + b; });
}

// A row's sum l of the weights against reference m (log2): 1 / l to inv[row], its log-sum-exp where it goes.
template <class T>
__device__ __forceinline__ void finish_row(const AttendArgs& a, const Item& it, int32_t hk, int32_t row, float l, float m, float* inv) {
  const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
  inv[row] = l == 0.f ? 0.f : 1.f / l;
  if (it.part >= 0) {
    a.part_lse[hk * a.part_rows + it.part + row] = lse2;
  } else if (a.lse) {
    const int32_t tok = row / a.group;
    a.lse[(int64_t)(it.tok0 + tok) * a.n_heads + hk * a.group + row - tok * a.group] = lse2 * 0.69314718055994531f;
  }
}

// Where a thread's dimension of one row after the other goes.
template <class T>
struct Rows {
  float* part;
  T* out;
  int64_t next_tok;
  int32_t tok, h;
  __device__ Rows(const AttendArgs& a, const Item& it, int32_t hk, int32_t row, int32_t dim) {
    tok = row / a.group, h = row - tok * a.group;
    part = a.part_o + (hk * a.part_rows + it.part + row) * a.dim + dim;
    out = static_cast<T*>(a.out) + (it.tok0 + tok) * a.o_tok + (hk * a.group + h) * a.o_head + dim;
    next_tok = a.o_tok - (a.group - 1) * a.o_head;
  }
  __device__ void put(const AttendArgs&, const Item& it, float v, float inv, int nan_at) {
    v = inv == 0.f ? 0.f : v * inv;
    if (nan_at <= tok) v = NAN;
    if (it.part >= 0) __stcg(part, v);
    else *reinterpret_cast<unsigned short*>(out) = (unsigned short)pack(T(), v, v);
  }
  __device__ void next(const AttendArgs& a) {
    part += a.dim;
    if (++h == a.group) h = 0, ++tok, out += next_tok;
    else out += a.o_head;
  }
};

template <class T>
__device__ __forceinline__ T from_bits(uint32_t v) {
  const unsigned short s = (unsigned short)v;
  return *reinterpret_cast<const T*>(&s);
}

// Eight elements of a row of Q, from an address that there is (what is none is the caller's to drop): the loads of a
// thread stay free of branches, so that none waits for another.
template <class T>
__device__ __forceinline__ uint4 q_piece(const Args8& g, const Item& it, int32_t hk, int32_t rows, int32_t row, int32_t piece,
                                         uint32_t per_group) {
  row = min(row, rows - 1);
  const int32_t tok = row * per_group >> 16;
  return *reinterpret_cast<const uint4*>(static_cast<const T*>(g.q) + (it.tok0 + tok) * g.q_tok +
                                         (hk * g.a.group + row - tok * g.a.group) * g.q_head + min(piece * 8, g.a.dim - 8));
}

// ---------------------------------------------------------------------------
// Few rows: codes straight into the products
// ---------------------------------------------------------------------------

// Numbers of more bits than a code has, as a sum of codes.  Q's are of K's type (e4m3, 4 bits): x = t_0 + t_1 / 16 + t_2 / 256,
// each the nearest to 16 times what the ones before it leave.  Two terms hold bf16 exactly (as far as 2^-14, of 2^8 at
// most), three fp16 (as far as 2^-18).
//
// P's are e5m2 (3 bits, from 2^-16 to 57,344): x = t_0 + t_1 / 8 + t_2 / 64 + t_3 / 512, off by at most 2^-12 of itself or 2^-26.
// A row's largest weight is at least 2^kBiasFew: weights have their 12 bits down to 2^-25 of it, and
// what is below 2^-37 of it is lost.  That range is for rows where one key has most of the weight and a small value: the result is then
// the sum of very many small weights, of which e4m3, with 2^-26, loses too much (131,072 keys of one weight, e^-17 of the largest, whose
// value is a fiftieth of theirs: 3.2e-2 of the result, in three terms of e4m3 1.1e-1, in these 2e-6).
constexpr int kFewKeys = 128, kFewRows = 16;   // of a step, of a tile
constexpr float kBiasFew = 11.f, kMostFew = 4.75f;   // a weight is at most 2^15.75 < 57,344

template <class T>
struct TermsQ {
  static constexpr int kN = std::is_same<T, __nv_bfloat16>::value ? 2 : 3;
};
constexpr int kTermsP = 4;

template <class T>
struct FewShape {
  static constexpr int kTerms = TermsQ<T>::kN;
  static constexpr int kQ = 6144, kP = kTermsP * kFewKeys * 16;   // Q: terms of 16 rows of 128 bytes
  static constexpr int kSlot = kFewKeys * 128, kSlots = 6;
  static constexpr int kRingAt = (kQ + kP + 1023) / 1024 * 1024;
  static constexpr int kMiscAt = kRingAt + kSlots * kSlot;
  static constexpr int kSmem = kMiscAt + 2048;
  static constexpr int kThreads = 256;
  static constexpr int kColumns = 256, kS = 64, kSTwo = 64;    // of TMEM: O^T, then S^T twice
  static_assert(kSmem <= 115712, "two blocks an SM");
};

struct FewMisc {
  ScaleRing<kFewKeys> scales;
  float top[4][kFewRows];              // the warps' largest weights where references are raised
  float unit[kFewRows];                // of a row's Q: the power of two that its terms are multiples of
  uint32_t first_nan[32];
  uint64_t bars[2 * 6 + 8];
  uint32_t tmem_at, failed, flag[2];
};
static_assert(sizeof(FewMisc) <= 2048, "fits behind the ring");

// D (+)= A B^T for 32 codes of A and B.
__device__ __forceinline__ void mma8_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
// A of e4m3 (type 0), B of e4m3 or of e5m2 (1), fp32 sums.
__host__ __device__ constexpr uint32_t mma8_desc(int m, int n, bool a_rows, bool b_rows, bool b_e5m2) {
  return (1u << 4) | ((b_e5m2 ? 1u : 0u) << 10) | ((a_rows ? 1u : 0u) << 15) | ((b_rows ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
// No swizzle, rows (N) contiguous, 16 of a column in 16 bytes: eight columns after each other; the next eight are
// `deeper` bytes on, the next 16 rows `further`.
__device__ __forceinline__ uint64_t tile_n16(uint32_t addr, uint32_t deeper, uint32_t further) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(deeper >> 4) << 16) | ((uint64_t)(further >> 4) << 32) | (1ull << 46);
}

// The next term of Q's x and y: its codes; x and y become 16 times what it leaves.
__device__ __forceinline__ uint16_t next_term(uint64_t* xy) {
  float x, y;
  halves(*xy, &x, &y);
  const uint16_t c = codes2(x, y);
  const uint32_t h = wide2(c);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  *xy = fma2(two(f.x, f.y), two(-16.f, -16.f), fma2(*xy, two(16.f, 16.f), 0ull));
  return c;
}

// The same of P's, with 8 times what is left (the codes are the upper bytes of fp16).
__device__ __forceinline__ uint16_t next_weight(uint64_t* xy) {
  float x, y;
  halves(*xy, &x, &y);
  uint16_t c;
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(c) : "f"(y), "f"(x));
  const uint32_t h = __byte_perm(c, 0, 0x1404);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  *xy = fma2(two(f.x, f.y), two(-8.f, -8.f), fma2(*xy, two(8.f, 8.f), 0ull));
  return c;
}

template <class T>
__global__ void __launch_bounds__(FewShape<T>::kThreads, 2) attend8_few_kernel(const __grid_constant__ CUtensorMap map_kv,
                                                                             const __grid_constant__ Args8 g) {
  using S = FewShape<T>;
  extern __shared__ __align__(1024) unsigned char base[];
  const AttendArgs& a = g.a;
  unsigned char* const p_mem = base + S::kQ;
  FewMisc& misc = *reinterpret_cast<FewMisc*>(base + S::kMiscAt);
  volatile uint32_t* failed = &misc.failed;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  const int32_t item = blockIdx.x / a.n_kv, hk = blockIdx.x - item * a.n_kv;
  const Item it = a.items[item];
  const int32_t rows = it.n_tok * a.group;
  const int32_t first = it.lo / kFewKeys, n = it.hi > it.lo ? (it.hi + kFewKeys - 1) / kFewKeys - first : 0;

  if (n == 0) {   // queries that see nothing
    sees_nothing<T>(a, it, hk, rows);
    return;
  }

  const uint32_t full = smem_addr(misc.bars), empty = full + 8 * S::kSlots, q_ready = empty + 8 * S::kSlots,
                 s_full = q_ready + 8, p_ready = s_full + 8, o_done = p_ready + 8, met = o_done + 8;
  // S_{j+1} is computed when P_{j-1} is there, after all have waited for S_{j-1}: two phases may be complete that
  // nobody has waited for, so s_full is two barriers (the second behind the others).
  const uint32_t s_full_odd = met + 8;
  if (warp == 4 && lane == 0) {
    prefetch_map(&map_kv);
    for (int i = 0; i < S::kSlots; ++i) bar_init(full + 8 * i, kFullCount), bar_init(empty + 8 * i, 1);
    bar_init(q_ready, 4), bar_init(s_full, 1), bar_init(s_full_odd, 1), bar_init(p_ready, 4), bar_init(o_done, 1), bar_init(met, 4);
    misc.failed = misc.flag[0] = misc.flag[1] = 0;
    fence_bar_init();
  }
  if (threadIdx.x < 32) misc.first_nan[threadIdx.x] = 0xffffffffu;
  if (warp == 7) tmem_alloc<1>(smem_addr(&misc.tmem_at), S::kColumns);
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, misc.tmem_at, 0), tmem_s = tmem + S::kS;

  if (warp >= 4 && warp < 4 + kCopiers) {
    copy_pages<kFewKeys, 128, S::kSlots>(map_kv, g, it, hk, first, n, warp - 4, lane, smem_addr(base + S::kRingAt), full, empty, misc.scales,
                               failed);
  } else if (warp == 7) {
    constexpr uint32_t desc_s = mma8_desc(kFewKeys, kFewRows * S::kTerms, false, false, false),
                       desc_o = mma8_desc(128, kFewRows * kTermsP, true, true, true);
    const uint64_t q = tile_k(smem_addr(base)), p = tile_n16(smem_addr(p_mem), 128, kFewKeys * 16);
    const uint64_t k_ring = tile_k(smem_addr(base + S::kRingAt)), v_ring = tile_n(smem_addr(base + S::kRingAt), kFewKeys * 128);
    const int k_steps = (a.dim + 31) / 32;
    auto scores = [&](int j) {
      const int e = j == 0 ? 0 : 2 * j - 1, slot = e % S::kSlots;
      if (!bar_wait(full + 8 * slot, (e / S::kSlots) & 1, failed)) return false;
      tc_after_sync();
      const uint64_t k = k_ring + slot * (S::kSlot / 16);
      const uint32_t d = tmem_s + (j & 1) * S::kSTwo;
      if (elect_one()) {
        for (int i = 0; i < k_steps; ++i) mma8_ss(d, k + 2 * i, q + 2 * i, desc_s, i > 0);
        mma_commit(empty + 8 * slot);
        mma_commit(j & 1 ? s_full_odd : s_full);
      }
      __syncwarp();
      return true;
    };
    int asked = 0, done = 0;
    bool go = bar_wait(q_ready, 0, failed) && scores(0);
    asked += go;
    for (int j = 0; go && j < n; ++j) {
      if (j + 1 < n) {
        if (!scores(j + 1)) break;
        ++asked;
      }
      const int e = j == n - 1 ? 2 * n - 1 : 2 * j + 2, slot = e % S::kSlots;
      if (!bar_wait_both(p_ready, j & 1, full + 8 * slot, (e / S::kSlots) & 1, failed)) break;
      tc_after_sync();
      const uint64_t v = v_ring + slot * (S::kSlot / 16);
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < kFewKeys / 32; ++i) mma8_ss(tmem, v + i * (32 * 128 / 16), p + i * (32 * 16 / 16), desc_o, j > 0 || i > 0);
        mma_commit(empty + 8 * slot);
        mma_commit(o_done);
      }
      __syncwarp();
      ++done;
    }
    uint32_t quiet = 0;
    if (asked > 0) bar_pass((asked - 1) & 1 ? s_full_odd : s_full, ((asked - 1) >> 1) & 1, &quiet);
    if (done > 0) bar_pass(o_done, (done - 1) & 1, &quiet);
  } else {
    const int r = threadIdx.x;           // the key of a step, and the dimension of O^T
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    uint32_t meetings = 0;
    int32_t key = first * kFewKeys + r;
    {
      // a row's 8 elements a step, to its terms: codes of row `term * 16 + row`.  Each row is first multiplied by the power of
      // two that brings its largest to between 2^7 and 2^8: a tile's rows may be of several requests.
      constexpr int kEach = kFewRows * 16 / 128;
      const uint32_t per_group = 65536 / a.group + 1;   // row * per_group >> 16 is row / group
      uint4 v[kEach];
      constexpr uint32_t kInf = std::is_same<T, __nv_bfloat16>::value ? 0x7f80 : 0x7c00;
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[i] = q_piece<T>(g, it, hk, rows, (r + 128 * i) / 16, (r + 128 * i) % 16, per_group);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (r / 16 + 8 * i >= rows || r % 16 * 8 >= a.dim) v[i] = uint4{};
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int x = r + 128 * i, row = x / 16, c = x % 16;
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        uint32_t top = 0;                // of the row's finite |q|
        for (const uint32_t y : w)
          for (const uint32_t z : {y & 0x7fff, y >> 16 & 0x7fff})
            if (z < kInf && z > top) top = z;
#pragma unroll
        for (int d = 8; d; d /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const int e = max(min(134 - (int)(__float_as_uint(up(from_bits<T>(top))) >> 23), 126), -120);
        float by = __int_as_float((e + 127) << 23);
        if (c == 0) misc.unit[row] = __int_as_float((127 - e) << 23);
        if (a.negative) by = -by;
        uint64_t xy[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x0 = unpack(T(), w[k], 0) * by, x1 = unpack(T(), w[k], 1) * by;
          xy[k] = two(fmaf(x0, 0.f, x0), fmaf(x1, 0.f, x1));   // (infinities to NaN: there is no code for them)
        }
#pragma unroll
        for (int t = 0; t < S::kTerms; ++t) {
          uint32_t o[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t lo = next_term(&xy[2 * k]), hi = next_term(&xy[2 * k + 1]);
            o[k] = lo | hi << 16;
          }
          const int at = t * kFewRows + row;
          *reinterpret_cast<uint2*>(base + at * 128 + ((c / 2) ^ (at & 7)) * 16 + (c & 1) * 8) = uint2{o[0], o[1]};
        }
      }
      fence_async();
      __syncwarp();
      if (lane == 0) bar_arrive(q_ready);
    }
    const int32_t all_see = it.pos0 + 1 < it.hi ? it.pos0 + 1 : it.hi;    // keys that the first row sees
    uint64_t l2[8];                      // of this key's share of the rows' sums
#pragma unroll
    for (int i = 0; i < 8; ++i) l2[i] = 0;
    uint64_t neg_m[8];                   // minus the rows' references; all threads have the same
#pragma unroll
    for (int i = 0; i < 8; ++i) neg_m[i] = two(-kNone, -kNone);
    for (int j = 0; j < n; ++j, key += kFewKeys) {
      const int32_t k0 = (first + j) * kFewKeys;
      const bool in = key >= it.lo && key < it.hi, masked = k0 < it.lo || k0 + kFewKeys > all_see;
      uint32_t sees = 0xffffu;           // rows that see this key: those of its token and later ones
      if (masked) {
        const int64_t before = key <= it.pos0 ? 0 : int64_t(key - it.pos0) * a.group;
        sees = !in || before >= 16 ? 0 : 0xffffu << before;
      }
      bar_pass(j & 1 ? s_full_odd : s_full, (j >> 1) & 1, failed);
      tc_after_sync();
      const uint32_t s_at = tmem_s + lanes + (j & 1) * S::kSTwo;
      const float ks = misc.scales.s[j & (kScaleSteps - 1)][0][r / 16], vs = misc.scales.s[j & (kScaleSteps - 1)][1][r / 16];
      const float c = a.scale2 * fminf(fmaxf(ks, 8.6736174e-19f), 1.1529215e18f);   // 2^-60 .. 2^60
      const float lv0 = __log2f(fminf(fmaxf(vs, 8.6736174e-19f), 1.1529215e18f)), lv = lv0 + kBiasFew;
      uint64_t x[8];                     // scores, then exponents, of two rows each
      auto scale_of = [&](int i) {       // of rows 2 i and 2 i + 1
        const float4 u = reinterpret_cast<const float4*>(misc.unit)[i / 2];
        return fma2(i & 1 ? two(u.z, u.w) : two(u.x, u.y), two(c, c), 0ull);
      };
      auto sums = [&]() {
        uint32_t t[S::kTerms][16];
#pragma unroll
        for (int k = 0; k < S::kTerms; ++k) tmem_load16(s_at + 16 * k, t[k]);
        tmem_wait_load();
#pragma unroll
        for (int k = 0; k < S::kTerms; ++k) tmem_loaded(t[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = two(__uint_as_float(t[S::kTerms - 1][2 * i]), __uint_as_float(t[S::kTerms - 1][2 * i + 1]));
#pragma unroll
          for (int k = S::kTerms - 2; k >= 0; --k)
            x[i] = fma2(x[i], two(0.0625f, 0.0625f), two(__uint_as_float(t[k][2 * i]), __uint_as_float(t[k][2 * i + 1])));
        }
      };
      auto exponents = [&]() {
        sums();
        float most = -INFINITY;
        const uint64_t lv2 = two(lv, lv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = fma2(x[i], scale_of(i), add2(neg_m[i], lv2));
          float u, w;
          halves(x[i], &u, &w);
          if (masked) {
            if (!(sees >> (2 * i) & 1)) u = -INFINITY;
            if (!(sees >> (2 * i + 1) & 1)) w = -INFINITY;
            x[i] = two(u, w);
          }
          most = max3(most, __float_as_uint(u), __float_as_uint(w));
        }
        return most;
      };
      bool raise = j == 0;
      if (j > 0) {
        if (__any_sync(0xffffffffu, exponents() > kMostFew + kBiasFew) && lane == 0) misc.flag[j & 1] = j + 1;
        bar_meet(met, &meetings, failed);
        raise = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(&misc.flag[j & 1]), 0) == j + 1u;
      }
      if (raise) {
        // references are raised, or set: the columns' maxima over the keys
        sums();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float u, w;
          halves(fma2(x[i], scale_of(i), two(lv, lv)), &u, &w);
          if (!(u == u) || !(sees >> (2 * i) & 1)) u = -INFINITY;
          if (!(w == w) || !(sees >> (2 * i + 1) & 1)) w = -INFINITY;
          x[i] = two(u, w);
        }
        over_lanes(x, misc.top[warp], lane, [](float u, float w) { return fmaxf(u, w); });
        bar_meet(met, &meetings, failed);
        uint64_t f[8];                   // what they take from the sums and from O's terms
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float u, w;
          halves(neg_m[i], &u, &w);
          float tops[2] = {-u, -w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 t = *reinterpret_cast<const float2*>(&misc.top[k][2 * i]);
            tops[0] = fmaxf(tops[0], t.x - kBiasFew), tops[1] = fmaxf(tops[1], t.y - kBiasFew);
          }
          neg_m[i] = two(-tops[0], -tops[1]);
          f[i] = two(-u == tops[0] ? 1.f : exp2_fast(-u - tops[0]), -w == tops[1] ? 1.f : exp2_fast(-w - tops[1]));
          l2[i] = fma2(l2[i], f[i], 0ull);
        }
        if (j > 0) {
          bar_pass(o_done, (j - 1) & 1, failed);
          tc_after_sync();
#pragma unroll 1
          for (int k = 0; k < kTermsP; ++k) {
            uint32_t o[16];
            tmem_load16(tmem + lanes + 16 * k, o);
            tmem_wait_load();
            tmem_loaded(o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float u, w;
              halves(fma2(two(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1])), f[i], 0ull), &u, &w);
              o[2 * i] = __float_as_uint(u), o[2 * i + 1] = __float_as_uint(w);
            }
            tmem_store16(tmem + lanes + 16 * k, o);
          }
          tmem_wait_store();
        }
        exponents();
      }
      const float inv = exp2_fast(-lv0);
      uint32_t p[kTermsP][4];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float u, w;
        halves(x[i], &u, &w);
        uint64_t left = two(exp2_fast(u), exp2_fast(w));
        l2[i] = fma2(left, two(inv, inv), l2[i]);
#pragma unroll
        for (int k = 0; k < kTermsP; ++k) {
          const uint32_t both = next_weight(&left);
          p[k][i / 2] = i & 1 ? p[k][i / 2] | both << 16 : both;
        }
      }
      if (j > 0) bar_pass(o_done, (j - 1) & 1, failed);   // P is read
#pragma unroll
      for (int k = 0; k < kTermsP; ++k)
        *reinterpret_cast<uint4*>(p_mem + k * (kFewKeys * 16) + r * 16) = uint4{p[k][0], p[k][1], p[k][2], p[k][3]};
      if (masked) {
        // Keys outside the item: whatever lies there must not meet the zeros of P.  Nor must a NaN that some row
        // does not see; those that see it get theirs at the end.
        const int e = j == n - 1 ? 2 * n - 1 : 2 * j + 2, slot = e % S::kSlots;
        bar_pass(full + 8 * slot, (e / S::kSlots) & 1, failed);
        const uint32_t query = key <= it.pos0 ? 0 : min(key - it.pos0, 254);
#pragma unroll 1
        for (int c16 = 0; c16 < 8; ++c16) {
          uint4* at = codes_at<128>(base + S::kRingAt + slot * S::kSlot, r, c16);
          uint4 v = in ? *at : uint4{};
          if (has_nan(v)) v = without_nan(v, misc.first_nan + 4 * c16, query);
          *at = v;
        }
      }
      fence_async();
      tc_before_sync();
      __syncwarp();
      if (lane == 0) bar_arrive(p_ready);
    }
    bar_pass(o_done, (n - 1) & 1, failed);
    tc_after_sync();
    // the rows' sums over the keys, in P's place: [4][16], then 1 / sum
    float* total = reinterpret_cast<float*>(p_mem);
    column_sums(l2, total + warp * kFewRows, lane);
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (lane == i) {
          float u, w;
          halves(neg_m[i], &u, &w);
          misc.top[0][2 * i] = -u, misc.top[0][2 * i + 1] = -w;
        }
    }
    bar_meet(met, &meetings, failed);
    if (r < rows)
      finish_row<T>(a, it, hk, r, (total[r] + total[kFewRows + r]) + (total[2 * kFewRows + r] + total[3 * kFewRows + r]),
                    misc.top[0][r] - kBiasFew, total + 4 * kFewRows);
    bar_meet(met, &meetings, failed);
    // a row after the other, a dimension a thread
    Rows<T> at(a, it, hk, 0, r);
    const int nan_at = misc.first_nan[r / 4] >> (8 * (r % 4)) & 0xff;
#pragma unroll 1
    for (int row = 0; row < rows; row += 4) {
      uint32_t o[kTermsP][4];
#pragma unroll
      for (int k = 0; k < kTermsP; ++k) tmem_load4(tmem + lanes + 16 * k + row, o[k]);
      tmem_wait_load();
#pragma unroll
      for (int k = 0; k < kTermsP; ++k) tmem_loaded(o[k]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = __uint_as_float(o[kTermsP - 1][i]);
#pragma unroll
        for (int k = kTermsP - 2; k >= 0; --k) v = fmaf(v, 0.125f, __uint_as_float(o[k][i]));
        if (row + i < rows && r < a.dim) at.put(a, it, v, total[4 * kFewRows + row + i], nan_at);
        at.next(a);
      }
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (warp == 7) tmem_free<1>(tmem, S::kColumns);
  if (threadIdx.x == 0 && *failed) atomicAdd(&a.status[5], 1);
}


// ---------------------------------------------------------------------------
// Many rows: codes to fp16 on the way
// ---------------------------------------------------------------------------

//   warps 0 to 3    the softmax: a thread holds one row
//   warps 4, 5      keys from slots of codes to slots of fp16; warps 6, 7 values
//   warps 8, 9      copies: the pages of 64 keys, or values, a slot
//   warp 11         products: S_j = Q K_j^T into one of two TMEM buffers, O += P_j V_j into TMEM
constexpr int kKeys = 64, kRows = 128;   // of a step, of a tile
constexpr int kThreads = 384;
// A weight is at most 2^(kMost + kBias), in fp16's range, and the largest at least 2^kBias: weights have fp16's 11 bits down to
// 2^-22 of it, and what is below 2^-33 of it is lost.  (With 4 and 11, 2^-29: 131,072 keys of one weight, e^-20 of the largest, whose
// value is a fiftieth of theirs, were 1% off.)  A raised reference takes the whole warp through O, so all of its rows are
// raised then: a call on chunks of prompts 337 us, with 4 and 11 335, with 10 and 5 342; each row by itself with 7 and 8 345.
constexpr float kBias = 8.f, kMost = 7.f;

template <class T, int DP>
struct Shape {
  static constexpr int kTerms = TermsQ<T>::kN;
  static constexpr int kTerm = kRows * DP, kQ = kTerms * kTerm;
  static constexpr int kWide = kKeys * DP * 2, kWideSlots = 2;                       // V in fp16
  static constexpr int kCodes = kKeys * DP, kCodeSlots = DP == 64 ? 4 : kTerms == 2 ? 3 : 2;   // of K, and of V
  static constexpr int kWideAt = kQ, kCodesAt = kWideAt + kWideSlots * kWide;
  static constexpr int kMiscAt = kCodesAt + 2 * kCodeSlots * kCodes;
  static constexpr int kSmem = kMiscAt + 1024;
  static constexpr int kColumns = 256;                    // of TMEM: O, then two buffers of S
  static_assert(kSmem <= 115712, "two blocks an SM");
};

// Full and empty, by slot.
template <int N>
struct Ring {
  uint64_t full[N], empty[N];
};

template <class T, int DP>
struct Misc {
  ScaleRing<kKeys> scales;
  uint32_t first_nan[32];              // by dimension, a byte: the first query that sees a NaN where rows see different keys
  signed char q_scale[kRows];          // the power of two that a row of Q is multiplied by
  Ring<Shape<T, DP>::kCodeSlots> codes_k, codes_v;
  Ring<Shape<T, DP>::kWideSlots> wide;
  uint64_t q_ready, s_full[2], p_ready[2], o_done[2];
  uint32_t tmem_at, failed, any_nan;
};
static_assert(sizeof(Misc<__half, 128>) <= 1024 && sizeof(Misc<__half, 64>) <= 1024, "fits behind the slots");

// As tile_k, in rows of 64 bytes and the 64-byte swizzle.
__device__ __forceinline__ uint64_t tile_k64(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (1ull << 16) | ((uint64_t)(512 >> 4) << 32) | (1ull << 46) | (4ull << 61);
}
// The next term of x and y, itself: its codes; x and y become what it leaves.
__device__ __forceinline__ uint16_t next_code(uint64_t* xy) {
  float x, y;
  halves(*xy, &x, &y);
  const uint16_t c = codes2(x, y);
  const uint32_t h = wide2(c);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  *xy = two(x - f.x, y - f.y);
  return c;
}

// The slots of a ring in order: a wait tells its phase from the one before it, which the same wait has had before.
template <int N>
struct Turn {
  uint32_t full, empty;
  int slot = 0;
  uint32_t parity = 0;                 // of the full one; an empty one is awaited with the other
  __device__ explicit Turn(Ring<N>& r) : full(smem_addr(r.full)), empty(smem_addr(r.empty)) {}
  __device__ uint32_t full_bar() const { return full + 8 * slot; }
  __device__ uint32_t empty_bar() const { return empty + 8 * slot; }
  __device__ void next() {
    if (++slot == N) slot = 0, parity ^= 1;
  }
};

__device__ __forceinline__ float in_range(float scale) { return fminf(fmaxf(scale, 8.6736174e-19f), 1.1529215e18f); }   // 2^-60 .. 2^60

// A copying warp: K (with the scales), or V, page by page.
template <int DP, int kSlots, bool kKeysToo>
__device__ __forceinline__ void copy_tiles(const CUtensorMap& map, const Args8& g, const Item& it, int32_t hk, int32_t first,
                                           int32_t n, int lane, uint32_t slots, Ring<kSlots>& ring, ScaleRing<kKeys>& scales,
                                           volatile uint32_t* failed) {
  const AttendArgs& a = g.a;
  const int32_t box = a.page_tokens < kKeys ? a.page_tokens : kKeys;   // keys a copy
  // the page numbers come 32 at a time, the next 32 on their way
  const int shift = __ffs(a.page_tokens) - 1;
  const int32_t last = (it.hi - 1) >> shift;
  int32_t at0 = first * kKeys >> shift;
  auto look_up = [&](int32_t i) {
    const int32_t page = i <= last ? a.table[int64_t(it.row) * a.max_pages + i] : -1;
    return page >= 0 && page < a.n_pages ? page : a.n_pages;   // no such page: read as zeros
  };
  int32_t now = look_up(at0 + lane), next = look_up(at0 + 32 + lane);
  Turn<kSlots> turn(ring);
  int j = 0;
  for (; j < n; ++j) {
    const int32_t k0 = (first + j) * kKeys;
    const int32_t from = it.lo > k0 ? (it.lo - k0) / box * box : 0, to = it.hi - k0 < kKeys ? it.hi - k0 : kKeys;
    if ((k0 >> shift) - at0 >= 32) {
      at0 += 32;
      now = next;
      next = look_up(at0 + 32 + lane);
    }
    if (!bar_wait(turn.empty_bar(), turn.parity ^ 1, failed)) break;
    const uint32_t bar = turn.full_bar(), dst = slots + turn.slot * (kKeys * DP);
    if (elect_one()) bar_expect(bar, (to - from + box - 1) / box * box * DP);
    for (int32_t k = from; k < to; k += box) {
      // (a step has at most four pages, so it does not reach beyond the 32 before the next ones move up)
      const int32_t page = __shfl_sync(0xffffffffu, now, ((k0 + k) >> shift) - at0);
      const int32_t y = ((a.plane + !kKeysToo) * a.n_kv + hk) * a.page_tokens + ((k0 + k) & (a.page_tokens - 1));
      if (elect_one()) load_3d(dst + k * DP, &map, 0, y, page, bar);
    }
    if (kKeysToo) {
      const int32_t k = k0 + (lane & 3) * 16, v = lane >> 2 & 1;
      const int32_t page = __shfl_sync(0xffffffffu, now, ((k >> shift) - at0) & 31);
      float* at = &scales.s[j & (kScaleSteps - 1)][v][lane & 3];
      if (lane < 8) {
        if (page < a.n_pages && k < it.hi) {
          const int32_t blocks = a.page_tokens / 16;
          copy_word(smem_addr(at), g.pool + page * g.page_bytes + g.scale_at +
                                       4 * (int64_t(v * a.n_kv + hk) * blocks + (k & (a.page_tokens - 1)) / 16));
        } else {
          *at = 1.f;
        }
      }
      copies_arrive(bar);
    }
    turn.next();
  }
  if (gave_up(failed)) {   // the copies in flight still have to land: a bounded wait for each
    uint32_t quiet = 0;
    for (int b = j - 1; b >= 0 && b >= j - kSlots; --b) bar_pass(smem_addr(&ring.full[b % kSlots]), (b / kSlots) & 1, &quiet);
  }
  __syncwarp();
}

// Four warps: V's codes to fp16, a thread half of a key's.
template <class T, int DP>
__device__ __forceinline__ void widen(unsigned char* codes, unsigned char* wide, Misc<T, DP>& misc, const Item& it, int32_t first,
                                      int32_t n, int32_t all_see) {
  volatile uint32_t* failed = &misc.failed;
  const int r = threadIdx.x & 63, part = threadIdx.x >> 6 & 1;
  Turn<Shape<T, DP>::kCodeSlots> from(misc.codes_v);
  Turn<Shape<T, DP>::kWideSlots> to(misc.wide);
  for (int j = 0; j < n; ++j) {
    const int32_t k0 = (first + j) * kKeys, key = k0 + r;
    bar_pass(from.full_bar(), from.parity, failed);
    bar_pass(to.empty_bar(), to.parity ^ 1, failed);
    unsigned char *x = codes + from.slot * (kKeys * DP), *y = wide + to.slot * (kKeys * DP * 2);
    const bool masked = k0 < it.lo || k0 + kKeys > all_see;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
      const int c16 = part * (DP / 32) + i;
      uint4 v = *codes_at<DP>(x, r, c16);
      if (masked) {
        // Keys outside the item: whatever lies there must not meet the zeros of P.  Nor must a NaN that
        // some row does not see; those that see it get theirs at the end.
        if (key < it.lo || key >= it.hi) v = uint4{};
        if (has_nan(v)) {
          v = without_nan(v, misc.first_nan + 4 * c16, key <= it.pos0 ? 0 : min(key - it.pos0, 254));
          misc.any_nan = 1;
        }
      }
      uint32_t o[8];
      wide16(v, o);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        *reinterpret_cast<uint4*>(y + (c16 / 4) * (kKeys * 128) + r * 128 + (((2 * c16 + k) % 8) ^ (r & 7)) * 16) =
            uint4{o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]};
    }
    fence_async();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(from.empty_bar()), bar_arrive(to.full_bar());
    from.next();
    to.next();
  }
}

template <class T, int DP>
__global__ void __launch_bounds__(kThreads, 2) attend8_kernel(const __grid_constant__ CUtensorMap map_kv,
                                                              const __grid_constant__ Args8 g) {
  using S = Shape<T, DP>;
  extern __shared__ __align__(1024) unsigned char base[];
  const AttendArgs& a = g.a;
  Misc<T, DP>& misc = *reinterpret_cast<Misc<T, DP>*>(base + S::kMiscAt);
  volatile uint32_t* failed = &misc.failed;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  // all heads of an item, then the next item: the long ones start first
  const int32_t item = blockIdx.x / a.n_kv, hk = blockIdx.x - item * a.n_kv;
  const Item it = a.items[item];
  const int32_t rows = it.n_tok * a.group;
  const int32_t first = it.lo / kKeys, n = it.hi > it.lo ? (it.hi + kKeys - 1) / kKeys - first : 0;

  if (n == 0) {
    sees_nothing<T>(a, it, hk, rows);
    return;
  }

  const uint32_t q_ready = smem_addr(&misc.q_ready), s_full = smem_addr(misc.s_full), p_ready = smem_addr(misc.p_ready),
                 o_done = smem_addr(misc.o_done);
  // s_full, p_ready and o_done are two barriers each, for even and odd steps.  A wait tells a phase
  // from the one before it only, and every wait here has that one behind it: S_j is computed
  // after the product of step j - 2 is done.
  if (warp == 8 && lane == 0) {
    prefetch_map(&map_kv);
    for (int i = 0; i < S::kCodeSlots; ++i) {
      bar_init(smem_addr(&misc.codes_k.full[i]), kFullCount), bar_init(smem_addr(&misc.codes_k.empty[i]), 1);
      bar_init(smem_addr(&misc.codes_v.full[i]), 1), bar_init(smem_addr(&misc.codes_v.empty[i]), 4);
    }
    for (int i = 0; i < S::kWideSlots; ++i) bar_init(smem_addr(&misc.wide.full[i]), 4), bar_init(smem_addr(&misc.wide.empty[i]), 1);
    bar_init(q_ready, 8);
    for (int i = 0; i < 2; ++i) bar_init(s_full + 8 * i, 1), bar_init(p_ready + 8 * i, 4), bar_init(o_done + 8 * i, 1);
    misc.failed = misc.any_nan = 0;
    fence_bar_init();
  }
  if (threadIdx.x < 32) misc.first_nan[threadIdx.x] = 0xffffffffu;
  if (warp == 11) tmem_alloc<1>(smem_addr(&misc.tmem_at), S::kColumns);
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, misc.tmem_at, 0), tmem_s = tmem + 128;
  const int32_t all_see = it.pos0 + 1 < it.hi ? it.pos0 + 1 : it.hi;    // keys that the first row sees

  if (warp >= 8) {
    fewer_registers<40>();
    if (warp < 10) {
      if (warp == 8)
        copy_tiles<DP, S::kCodeSlots, true>(map_kv, g, it, hk, first, n, lane, smem_addr(base + S::kCodesAt), misc.codes_k,
                                            misc.scales, failed);
      else
        copy_tiles<DP, S::kCodeSlots, false>(map_kv, g, it, hk, first, n, lane,
                                             smem_addr(base + S::kCodesAt + S::kCodeSlots * S::kCodes), misc.codes_v, misc.scales,
                                             failed);
    } else if (warp == 11) {
      // the whole warp goes along; one lane issues
      constexpr uint32_t desc_s = mma8_desc(kRows, kKeys, false, false, false), desc_o = mma_desc(false, kRows, DP, true);
      const uint32_t k_at = smem_addr(base + S::kCodesAt);
      const uint64_t q = DP == 64 ? tile_k64(smem_addr(base)) : tile_k(smem_addr(base)),
                     k_ring = DP == 64 ? tile_k64(k_at) : tile_k(k_at), v_ring = tile_n(smem_addr(base + S::kWideAt), kKeys * 128);
      Turn<S::kCodeSlots> kt(misc.codes_k);
      Turn<S::kWideSlots> vt(misc.wide);
      auto scores = [&](int j, uint32_t behind, uint32_t parity) {   // behind: what S_j waits for besides K_j
        if (!bar_wait_both(behind, parity, kt.full_bar(), kt.parity, failed)) return false;
        tc_after_sync();
        const uint64_t k = k_ring + kt.slot * (S::kCodes / 16);
        const uint32_t d = tmem_s + (j & 1) * kKeys;
        if (elect_one()) {
#pragma unroll
          for (int t = 0; t < S::kTerms; ++t)
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) mma8_ss(d, q + t * (S::kTerm / 16) + 2 * i, k + 2 * i, desc_s, t > 0 || i > 0);
          mma_commit(kt.empty_bar());
          mma_commit(s_full + 8 * (j & 1));
        }
        __syncwarp();
        kt.next();
        return true;
      };
      int asked = 0, done = 0;            // S and O that are on their way
      bool go = scores(0, q_ready, 0);
      asked += go;
      if (go && n > 1) go = scores(1, q_ready, 0), asked += go;
      for (int j = 0; go && j < n; ++j) {
        if (!bar_wait_both(p_ready + 8 * (j & 1), (j >> 1) & 1, vt.full_bar(), vt.parity, failed)) break;
        tc_after_sync();
        const uint64_t v = v_ring + vt.slot * (S::kWide / 16);
        const uint32_t p = tmem_s + (j & 1) * kKeys;
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < kKeys / 16; ++i) mma_ts(tmem, p + i * 8, v + i * (16 * 128 / 16), desc_o, j > 0 || i > 0);
          mma_commit(vt.empty_bar());
          mma_commit(o_done + 8 * (j & 1));
        }
        __syncwarp();
        vt.next();
        ++done;
        // S_{j+2} takes the place of P_j: once its product is done
        if (j + 2 < n) go = scores(j + 2, o_done + 8 * (j & 1), (j >> 1) & 1), asked += go;
      }
      uint32_t quiet = 0;
      if (asked > 0) bar_pass(s_full + 8 * ((asked - 1) & 1), ((asked - 1) >> 1) & 1, &quiet);
      if (done > 0) bar_pass(o_done + 8 * ((done - 1) & 1), ((done - 1) >> 1) & 1, &quiet);
    }
  } else {
    {
      // Q's terms to shared memory, 8 elements a step: consecutive threads along a row, which is first multiplied by the
      // power of two that brings its largest to between 2^7 and 2^8
      // (one at a time, the next on its way: a block goes through this code a few times, and more of it would be
      // fetched for longer than it runs; four at a time chunks of prompts took 355 us, one 345)
      constexpr int kLanes = DP / 8, kEach = kRows * kLanes / 256, kApart = 256 / kLanes;
      const int c = threadIdx.x % kLanes, row0 = threadIdx.x / kLanes;
      const uint32_t per_group = 65536 / a.group + 1;   // row * per_group >> 16 is row / group, for rows below 128
      auto piece = [&](int i) { return q_piece<T>(g, it, hk, rows, row0 + i * kApart, c, per_group); };
      uint4 ahead = piece(0);
#pragma unroll 1
      for (int i = 0; i < kEach && i * kApart < rows; ++i) {
        uint4 v = ahead;
        ahead = piece(i + 1);
        const int row = row0 + i * kApart;
        if (row >= rows || c * 8 >= a.dim) v = uint4{};
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        // of |q| (a row that holds an infinity is NaN in the end, whatever its scale)
        uint32_t both = most_of(T(), most_of(T(), w[0] & 0x7fff7fff, w[1] & 0x7fff7fff), most_of(T(), w[2] & 0x7fff7fff, w[3] & 0x7fff7fff));
#pragma unroll
        for (int d = kLanes / 2; d; d /= 2) both = most_of(T(), both, __shfl_xor_sync(0xffffffffu, both, d));
        const float most = fmaxf(unpack(T(), both, 0), unpack(T(), both, 1));
        const int e = max(min(134 - (int)(__float_as_uint(most) >> 23), 126), -120);
        if (c == 0) misc.q_scale[row] = (signed char)e;
        float by = __int_as_float((e + 127) << 23);
        if (a.negative) by = -by;
        uint64_t xy[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x0 = unpack(T(), w[k], 0) * by, x1 = unpack(T(), w[k], 1) * by;
          xy[k] = two(fmaf(x0, 0.f, x0), fmaf(x1, 0.f, x1));   // (infinities to NaN: there is no code for them)
        }
        // 16 bytes of a row, where the products look for them: the swizzle of rows of DP bytes
        unsigned char* at = base + row * DP + ((c / 2) ^ (DP == 64 ? row >> 1 & 3 : row & 7)) * 16 + (c & 1) * 8;
#pragma unroll
        for (int t = 0; t < S::kTerms; ++t) {
          uint32_t o[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t lo = next_code(&xy[2 * k]), hi = next_code(&xy[2 * k + 1]);
            o[k] = lo | hi << 16;
          }
          *reinterpret_cast<uint2*>(at + t * S::kTerm) = uint2{o[0], o[1]};
        }
      }
      fence_async();
      __syncwarp();
      if (lane == 0) bar_arrive(q_ready);
    }
    if (warp >= 4) {
      fewer_registers<72>();
      widen<T, DP>(base + S::kCodesAt + S::kCodeSlots * S::kCodes, base + S::kWideAt, misc, it, first, n, all_see);
    } else {
      more_registers<128>();
      const int r = threadIdx.x;
      bar_pass(q_ready, 0, failed);      // (the rows' scales are others' work)
      // (rows beyond the tile's hold whatever was there: their scores count as nothing)
      const float c_all = r < rows ? a.scale2 * __int_as_float((127 - misc.q_scale[r]) << 23) : 0.f;
      const uint32_t lanes = (uint32_t)(warp * 32) << 16;
      const int32_t tok = r / a.group;
      // the keys that this row sees end here; rows beyond the tile's see what the last one does
      const int32_t own = tok < it.n_tok ? tok : it.n_tok - 1;
      const int32_t end = it.pos0 + own + 1 < it.hi ? it.pos0 + own + 1 : it.hi;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n; ++j) {
        const int32_t k0 = (first + j) * kKeys;
        bar_pass(s_full + 8 * (j & 1), (j >> 1) & 1, failed);
        tc_after_sync();
        const uint32_t s_at = tmem_s + lanes + (j & 1) * kKeys;
        uint32_t s[64];
        tmem_load32(s_at, s);
        tmem_load32(s_at + 32, s + 32);
        // of a block of 16 keys: what a score is multiplied by, log2 v; each of eight lanes has one of them
        const float mine = in_range(misc.scales.s[j & (kScaleSteps - 1)][lane >> 2 & 1][lane & 3]);
        const float either = lane & 4 ? __log2f(mine) : mine;
        float2 block[4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
          block[b] = float2{fmaxf(c_all * __shfl_sync(0xffffffffu, either, b), 1e-37f), __shfl_sync(0xffffffffu, either, 4 + b)};
        tmem_wait_load();
        tmem_loaded(s);
        // -inf for what this row does not see (its multipliers are > 0)
        if (k0 < it.lo || k0 + kKeys > all_see) {
          const int below = it.lo > k0 ? it.lo - k0 : 0, upto = end - k0 < 0 ? 0 : end - k0 < kKeys ? end - k0 : kKeys;
          const uint64_t sees = upto <= below ? 0 : (upto == 64 ? ~0ull : (1ull << upto) - 1) & ~((1ull << below) - 1);
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (!(sees >> i & 1)) s[i] = 0xff800000u;
        }
        float top = -INFINITY;           // of s c + log2 v
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int i = 8 * b; i < 8 * b + 8; ++i) mx[i & 1] = max3(mx[i & 1], s[2 * i], s[2 * i + 1]);
          top = fmaxf(top, fmaf(fmaxf(mx[0], mx[1]), block[b].x, block[b].y));
        }
        const bool raise = top > m + kMost || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, raise)) {
          const float f = top > m ? (m == -INFINITY ? 0.f : exp2_fast(m - top)) : 1.f;
          m = fmaxf(m, top);
          l *= f;
          if (j > 0) {
            bar_pass(o_done + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, failed);
            tc_after_sync();
#pragma unroll 1
            for (int d = 0; d < DP; d += 16) {
              uint32_t o[16];
              tmem_load16(tmem + lanes + d, o);
              tmem_wait_load();
              tmem_loaded(o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_store16(tmem + lanes + d, o);
            }
            tmem_wait_store();
          }
        }
        const float shift = m == -INFINITY ? 0.f : kBias - m;
        uint32_t p[32];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const uint64_t c2 = two(block[b].x, block[b].x), shift2 = two(block[b].y + shift, block[b].y + shift);
          uint64_t sum[2] = {};
#pragma unroll
          for (int i = 8 * b; i < 8 * b + 8; ++i) {
            float x, y;
            halves(fma2(two(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, shift2), &x, &y);
            x = exp2_fast(x), y = exp2_fast(y);
            sum[i & 1] = add2(sum[i & 1], two(x, y));
            p[i] = pack(__half(), x, y);
          }
          float x, y;
          halves(add2(sum[0], sum[1]), &x, &y);
          l = fmaf(x + y, exp2_fast(-block[b].y), l);
        }
        tmem_store32(s_at, p);
        tmem_wait_store();
        tc_before_sync();
        __syncwarp();
        if (lane == 0) bar_arrive(p_ready + 8 * (j & 1));
      }
      bar_pass(o_done + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, failed);
      tc_after_sync();
      const bool in = tok < it.n_tok, any_nan = *reinterpret_cast<volatile uint32_t*>(&misc.any_nan);
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
      for (int d = 0; d < a.dim && warp * 32 < rows; d += 16) {
        uint32_t o[16];
        tmem_load16(tmem + lanes + d, o);
        tmem_wait_load();
        tmem_loaded(o);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(l == 0.f ? 0.f : __uint_as_float(o[i]) * inv);
        if (any_nan)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((int)(misc.first_nan[(d + i) / 4] >> (8 * (i % 4)) & 0xff) <= tok) o[i] = 0x7fc00000u;
        if (in && it.part >= 0) {
#pragma unroll
          for (int i = 0; i < 16; i += 4) __stcg(reinterpret_cast<uint4*>(part_o + d + i), uint4{o[i], o[i + 1], o[i + 2], o[i + 3]});
        } else if (in) {
#pragma unroll
          for (int i = 0; i < 16; i += 8) {
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
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (warp == 11) tmem_free<1>(tmem, S::kColumns);
  if (threadIdx.x == 0 && *failed) atomicAdd(&a.status[5], 1);
}

// A plan is for one of the kernels: the one whose steps and items take less time (in clocks, as measured; the many rows'
// steps are of 64 keys).  Few rows and many: a decode step of 64 requests of 8,000 tokens or so, 32 + 8 heads of 128, 167 us and
// 243; one request of 131,072 tokens (fp16, 4 tokens of 5 heads each) 48 and 60; 96 requests behind 32,768 shared tokens
// 195 and 83; chunks of prompts behind 4,000 tokens, 24 + 8 heads of 64, 1,846 and 335.
// A tile's start and end count as so many steps where the keys are cut: 4 for few rows (with 3, three short decode steps
// of 6.4, 7.5 and 121 us became 7.3, 8.9 and 129).
constexpr Cutting kCuttingFew = {kFewKeys, kFewRows, 4, 8, 4, 5, true}, kCuttingMany = {kKeys, kRows, 6, 12, 4, 8, true};
constexpr int64_t kFewClocks = 1900, kManyClocks = 1300;

template <class T, int DP>
cudaError_t launch_many(const op_attend_plan_t& p, const CUtensorMap& kv, const Args8& g, cudaStream_t st) {
  static gsim::OncePerDevice once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  auto kernel = attend8_kernel<T, DP>;
  if (!once.done(dev, [&] { return allow_smem(kernel, Shape<T, DP>::kSmem); })) return cudaErrorInvalidValue;
  kernel<<<(unsigned)(p.n_items * (int64_t)p.n_kv_heads), kThreads, Shape<T, DP>::kSmem, st>>>(kv, g);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_few(const op_attend_plan_t& p, const CUtensorMap& kv, const Args8& g, cudaStream_t st) {
  static gsim::OncePerDevice once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  auto kernel = attend8_few_kernel<T>;
  if (!once.done(dev, [&] { return allow_smem(kernel, FewShape<T>::kSmem); })) return cudaErrorInvalidValue;
  kernel<<<(unsigned)(p.n_items * (int64_t)p.n_kv_heads), FewShape<T>::kThreads, FewShape<T>::kSmem, st>>>(kv, g);
  return cudaGetLastError();
}

template <class T, int DP>
cudaError_t launch(const op_attend_plan_t& p, bool few, const CUtensorMap& kv, const Args8& g, cudaStream_t st) {
  const cudaError_t e = few ? launch_few<T>(p, kv, g, st) : launch_many<T, DP>(p, kv, g, st);
  if (e != cudaSuccess || p.n_joins == 0) return e;
  const int64_t heads = (int64_t)p.join_tokens * p.n_heads;
  attend_join_kernel<T><<<dim3((unsigned)p.n_joins, (unsigned)std::min<int64_t>(heads, 1024)), 128, 0, st>>>(g.a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

int op_attend8_plan(const op_attend_desc_t* d, int32_t n_sm, op_attend8_plan_t* plan, int32_t* items,
                    size_t item_bytes) try {
  if (!desc_ok(d, kRows) || d->head_dim % 16 || d->page_tokens < 16 || !plan || n_sm < 1) return GMG_EINVAL;
  Runs few, many;
  list_runs(*d, n_sm, kCuttingMany, &many);
  bool is_few = d->n_heads / d->n_kv_heads <= kFewRows;
  if (is_few) {
    list_runs(*d, n_sm, kCuttingFew, &few);
    is_few = all_steps(few, kCuttingFew) * kFewClocks <= all_steps(many, kCuttingMany) * kManyClocks;
  }
  Work w;
  cut_runs(*d, is_few ? few : many, is_few ? kCuttingFew : kCuttingMany, &w);
  const int rc = fill_plan(d, w, &plan->p, items, item_bytes);
  if (rc == GMG_OK || rc == GMG_EWS) plan->few = is_few, plan->reserved = 0;
  return rc;
} catch (const std::bad_alloc&) {
  return GMG_ENOMEM;
}

int op_attend8(const op_attend8_plan_t* plan8, const int32_t* d_items, const op_cache_t* cache, int32_t layer,
               int32_t dtype, const void* q, int64_t q_tok, int64_t q_head, float scale, void* out, int64_t out_tok,
               int64_t out_head, float* lse, void* work, size_t work_bytes, gmg_stream_t stream) {
  if (!plan8 || !cache8_ok(cache) || layer < 0 || layer >= cache->n_layers) return GMG_EINVAL;
  const op_attend_plan_t* plan = &plan8->p;
  if (plan->head_dim != cache->head_dim || plan->n_kv_heads != cache->n_kv_heads ||
      plan->page_tokens != cache->page_tokens || plan->max_seq >= cache->n_seq ||
      plan->max_kv > int64_t(cache->max_pages) * cache->page_tokens)
    return GMG_EINVAL;
  if (dtype != GMG_OP_BF16 && dtype != GMG_OP_F16) return GMG_EINVAL;
  if (plan->n_tokens == 0) return GMG_OK;
  if (!d_items || (reinterpret_cast<uintptr_t>(d_items) & 15) || !q || !out || !aligned(q, q_tok, q_head, 2) ||
      !aligned(out, out_tok, out_head, 2) || !(scale == scale))
    return GMG_EINVAL;
  if (!work || (reinterpret_cast<uintptr_t>(work) & 255) || work_bytes < plan->work_bytes) return GMG_EWS;
  const int64_t rows = int64_t(cache->n_layers) * 2 * cache->n_kv_heads * cache->page_tokens;   // of a page
  if (rows > 0x7fffffff) return GMG_ERANGE;
  Args8 g{};
  AttendArgs& a = g.a;
  a.items = reinterpret_cast<const Item*>(d_items);
  a.joins = reinterpret_cast<const Join*>(a.items + plan->n_items);
  a.table = cache->table;
  a.status = cache->status;
  a.max_pages = cache->max_pages;
  a.page_tokens = cache->page_tokens;
  a.n_pages = cache->n_pages;
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
  g.q = q, g.q_tok = q_tok, g.q_head = q_head;
  g.pool = static_cast<const unsigned char*>(cache->pool);
  g.page_bytes = page8_bytes(*cache);
  g.scale_at = page8_scales(*cache) + int64_t(layer) * 2 * cache->n_kv_heads * (cache->page_tokens / 16) * 4;
  CUtensorMap map_kv;
  const int64_t size[3] = {cache->head_dim, rows, cache->n_pages}, stride[2] = {cache->head_dim, g.page_bytes};
  const int32_t dp = plan8->few || cache->head_dim > 64 ? 128 : 64;
  const int32_t box[3] = {dp, std::min(cache->page_tokens, plan8->few ? kFewKeys : kKeys), 1};
  if (!make_map8(&map_kv, 3, cache->pool, size, stride, box)) return GMG_ECUDA;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == GMG_OP_BF16)
    e = dp == 64 ? launch<__nv_bfloat16, 64>(*plan, plan8->few, map_kv, g, st) : launch<__nv_bfloat16, 128>(*plan, plan8->few, map_kv, g, st);
  else
    e = dp == 64 ? launch<__half, 64>(*plan, plan8->few, map_kv, g, st) : launch<__half, 128>(*plan, plan8->few, map_kv, g, st);
  return e == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // extern "C"
