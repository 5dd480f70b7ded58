// Pages of a cache: free, fork, grow (copy on write), compact.  The C ABI is
// declared in include/gmgop.h.
//
// A free page is one without references; nothing else records it.  Pages are
// handed out in increasing order, so the result of a call does not depend on how
// its threads run: the r-th page that a call needs is the free page of rank r,
// found by counting free pages per block of kBlockPages pages, a prefix over the
// blocks, and a prefix within each block.  The plan is made by the block that counts
// last, which alone sees all counts.  Launches: count and plan / rank / apply and copy
// for grow and compact, check / apply for free and fork; the first two are one where
// one block holds all pages, and free and fork are one launch of one block while it has
// at most kFewCells table entries to go through (a step that frees 12 requests, forks 24 and
// grows 84, 4,096 pages: 4 launches instead of 7, 27 -> 24 us on the GPU, 48 -> 33 for the host).
//
// Copies are bound by memory: 1,207 pages of 128 KB compacted in 43 us (7.4 TB/s, part of it
// in the L2 cache), 53 with the plan; the small calls by their launches and a chain of
// about ten dependent loads each.

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gmgop.h"
#include "gmgop_host.h"

namespace gop {
namespace {

constexpr int kThreads = 256;         // of the blocks that apply and copy
constexpr int kPlanThreads = 1024;    // of those that check, count and plan
constexpr int kPerThread = 16;
constexpr int kBlockPages = kPlanThreads * kPerThread;
constexpr int64_t kFewCells = 16384;
constexpr int kCopyBytes = 32768;   // bytes of a page that one block copies at a time

struct Entry {      // what grow needs of a list entry after its plan
  int32_t seq, old_len, off, tail;  // tail: the page to copy first, or -1
};

struct Scratch {
  int32_t* ticket;   // blocks that have counted (back to 0 at the end of each call)
  int32_t* plan;     // [0] pages to hand out / to move, [1] L (compact)
  int32_t* mark;     // [n_seq] the entry that lists a row
  Entry* entry;      // [n_seq]
  int32_t* block;    // [blocks + 1] free pages in the blocks before
  int32_t* list;     // [n_pages] free pages by rank
  int32_t* from;     // [n_pages] pages to move, by rank
  int32_t* rank;     // [n_pages] rank of a page to move
};

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }
int32_t blocks_of(const op_cache_t& c) { return (c.n_pages + kBlockPages - 1) / kBlockPages; }

size_t layout(const op_cache_t& c, char* base, Scratch* s) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char* p = base + o;
    o = up256(o + bytes);
    return p;
  };
  char* head = take(256);
  char* mark = take(4 * size_t(c.n_seq));
  char* entry = take(sizeof(Entry) * size_t(c.n_seq));
  char* block = take(4 * (size_t(blocks_of(c)) + 1));
  char* list = take(4 * size_t(c.n_pages));
  char* from = take(4 * size_t(c.n_pages));
  char* rank = take(4 * size_t(c.n_pages));
  if (s) {
    s->ticket = reinterpret_cast<int32_t*>(head);
    s->plan = s->ticket + 8;
    s->mark = reinterpret_cast<int32_t*>(mark);
    s->entry = reinterpret_cast<Entry*>(entry);
    s->block = reinterpret_cast<int32_t*>(block);
    s->list = reinterpret_cast<int32_t*>(list);
    s->from = reinterpret_cast<int32_t*>(from);
    s->rank = reinterpret_cast<int32_t*>(rank);
  }
  return o;
}

size_t page_bytes(const op_cache_t& c) {
  return size_t(c.n_layers) * 2 * c.n_kv_heads * c.page_tokens * c.head_dim * 2;
}

// Pages for len tokens.
__device__ __forceinline__ int64_t pages_for(int64_t len, int32_t page) { return (len + page - 1) / page; }

// The smallest entry with a fault, and its code: faults are kept as entry * 8 + code.
struct Faults {
  unsigned long long* worst;
  __device__ void add(int32_t i, int32_t code) const {
    atomicMin(worst, (unsigned long long)i * 8 + (unsigned)code);
  }
};
constexpr unsigned long long kNoFault = ~0ull;

// Exclusive prefix over the kPlanThreads threads of the block, and the total.
__device__ int32_t block_prefix(int32_t v, int32_t* total) {
  __shared__ int32_t warp_sum[32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int32_t s = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int32_t t = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += t;
  }
  __syncthreads();
  if (lane == 31) warp_sum[w] = s;
  __syncthreads();
  int32_t sums = warp_sum[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int32_t t = __shfl_up_sync(0xffffffffu, sums, d);
    if (lane >= d) sums += t;
  }
  *total = __shfl_sync(0xffffffffu, sums, 31);
  const int32_t before = __shfl_sync(0xffffffffu, sums, w > 0 ? w - 1 : 0);
  return (w > 0 ? before : 0) + s - v;
}

// Free pages among this thread's kPerThread, as bits; pages beyond the end count as used.
__device__ uint32_t free_bits(const op_cache_t& c, int64_t first) {
  uint32_t bits = 0;
  if (first + kPerThread <= c.n_pages && (reinterpret_cast<uintptr_t>(c.refs) & 15) == 0) {
    int4 v[kPerThread / 4];
#pragma unroll
    for (int j = 0; j < kPerThread / 4; ++j) v[j] = reinterpret_cast<const int4*>(c.refs + first)[j];
#pragma unroll
    for (int j = 0; j < kPerThread / 4; ++j)
      bits |= ((v[j].x == 0) | (v[j].y == 0) << 1 | (v[j].z == 0) << 2 | (v[j].w == 0) << 3) << (4 * j);
    return bits;
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (first + j < c.n_pages && c.refs[first + j] == 0) bits |= 1u << j;
  return bits;
}

// Marks every listed row with its first entry and reports rows that are out of range or
// listed twice (the later entries find another's mark).  All threads of one block.
__device__ void check_rows(const op_cache_t& c, const int32_t* rows, int32_t n, int32_t* mark, Faults f) {
  for (int32_t i = threadIdx.x; i < n; i += kPlanThreads) {
    const int32_t r = rows[i];
    if (r < 0 || r >= c.n_seq) f.add(i, GMG_PAGE_SEQ);
    else mark[r] = i;
  }
  __syncthreads();
  // of the entries of a row any may have left its mark: the others then take it down to the first
  bool other = false;
  for (int32_t i = threadIdx.x; i < n; i += kPlanThreads) {
    const int32_t r = rows[i];
    if (r >= 0 && r < c.n_seq && mark[r] != i) {
      atomicMin(&mark[r], i);
      other = true;
    }
  }
  if (!__syncthreads_or(other)) return;
  for (int32_t i = threadIdx.x; i < n; i += kPlanThreads) {
    const int32_t r = rows[i];
    if (r >= 0 && r < c.n_seq && mark[r] != i) f.add(i, GMG_PAGE_TWICE);
  }
}

__device__ void write_status(const op_cache_t& c, unsigned long long worst) {
  c.status[0] = worst == kNoFault ? GMG_PAGE_OK : int32_t(worst & 7);
  c.status[1] = worst == kNoFault ? 0 : int32_t(worst >> 3);
}

// ---- free and fork -------------------------------------------------------

// Entries [i0, i1) of the list, all threads of the block over their table cells.
__device__ void free_rows(const op_cache_t& c, const int32_t* seq, int32_t i0, int32_t i1) {
  for (int64_t e = threadIdx.x; e < (int64_t)(i1 - i0) * c.max_pages; e += blockDim.x) {
    const int32_t i = int32_t(e / c.max_pages);
    int32_t* cell = c.table + int64_t(seq[i0 + i]) * c.max_pages + (e - (int64_t)i * c.max_pages);
    const int32_t p = *cell;
    if (p < 0) continue;
    if (p < c.n_pages) atomicSub(&c.refs[p], 1);
    *cell = -1;
  }
  for (int32_t i = i0 + threadIdx.x; i < i1; i += blockDim.x) c.lens[seq[i]] = 0;
}

template <bool kApply>
__global__ void __launch_bounds__(kPlanThreads) free_check_kernel(op_cache_t c, const int32_t* seq, int32_t n, Scratch s) {
  __shared__ unsigned long long worst;
  if (threadIdx.x == 0) worst = kNoFault;
  __syncthreads();
  check_rows(c, seq, n, s.mark, Faults{&worst});
  __syncthreads();
  if (threadIdx.x == 0) write_status(c, worst);
  if (kApply && worst == kNoFault) free_rows(c, seq, 0, n);
}

__global__ void __launch_bounds__(kThreads) free_apply_kernel(op_cache_t c, const int32_t* seq) {
  if (c.status[0] == GMG_PAGE_OK) free_rows(c, seq, blockIdx.x, blockIdx.x + 1);
}

// (A new row is never a source, so the lengths read are those of before the call.)
__device__ void fork_rows(const op_cache_t& c, const int32_t* src, const int32_t* dst, const int32_t* keep, int32_t i0,
                          int32_t i1) {
  for (int64_t e = threadIdx.x; e < (int64_t)(i1 - i0) * c.max_pages; e += blockDim.x) {
    const int32_t i = i0 + int32_t(e / c.max_pages), j = int32_t(e - (int64_t)(i - i0) * c.max_pages), a = src[i];
    if (j >= pages_for(keep ? keep[i] : c.lens[a], c.page_tokens)) continue;
    const int32_t p = c.table[int64_t(a) * c.max_pages + j];
    c.table[int64_t(dst[i]) * c.max_pages + j] = p;
    if (p >= 0 && p < c.n_pages) atomicAdd(&c.refs[p], 1);
  }
  for (int32_t i = i0 + threadIdx.x; i < i1; i += blockDim.x) c.lens[dst[i]] = keep ? keep[i] : c.lens[src[i]];
}

template <bool kApply>
__global__ void __launch_bounds__(kPlanThreads) fork_check_kernel(op_cache_t c, const int32_t* src, const int32_t* dst,
                                                                  const int32_t* keep, int32_t n, Scratch s) {
  __shared__ unsigned long long worst;
  if (threadIdx.x == 0) worst = kNoFault;
  __syncthreads();
  const Faults f{&worst};
  check_rows(c, dst, n, s.mark, f);
  __syncthreads();
  for (int32_t i = threadIdx.x; i < n; i += kPlanThreads) {
    const int32_t a = src[i], b = dst[i];
    if (a < 0 || a >= c.n_seq) {
      f.add(i, GMG_PAGE_SEQ);
      continue;
    }
    const int32_t m = s.mark[a];   // a's own entry if a is a new row too, else anything
    if (m >= 0 && m < n && dst[m] == a) f.add(i, GMG_PAGE_TWICE);
    const int32_t len = c.lens[a];
    if (len < 0 || pages_for(len, c.page_tokens) > c.max_pages || (keep && (keep[i] < 0 || keep[i] > len)))
      f.add(i, GMG_PAGE_LONG);
    if (b >= 0 && b < c.n_seq && (c.lens[b] != 0 || c.table[int64_t(b) * c.max_pages] >= 0)) f.add(i, GMG_PAGE_USED);
  }
  __syncthreads();
  if (threadIdx.x == 0) write_status(c, worst);
  if (kApply && worst == kNoFault) fork_rows(c, src, dst, keep, 0, n);
}

__global__ void __launch_bounds__(kThreads) fork_apply_kernel(op_cache_t c, const int32_t* src, const int32_t* dst,
                                                              const int32_t* keep) {
  if (c.status[0] == GMG_PAGE_OK) fork_rows(c, src, dst, keep, blockIdx.x, blockIdx.x + 1);
}

// ---- grow and compact: count, rank, apply --------------------------------

// True in the block that counts last; it then sees every block's count.
__device__ bool count_free(const op_cache_t& c, const Scratch& s) {
  __shared__ bool last;
  int32_t total;
  block_prefix(__popc(free_bits(c, (int64_t)blockIdx.x * kBlockPages + threadIdx.x * kPerThread)), &total);
  if (gridDim.x == 1) {
    if (threadIdx.x == 0) s.block[0] = total;
    return true;
  }
  if (threadIdx.x == 0) {
    s.block[blockIdx.x] = total;
    __threadfence();
    last = atomicAdd(s.ticket, 1) == (int32_t)gridDim.x - 1;
  }
  __syncthreads();
  if (last) __threadfence();
  return last;
}

// The counts become the free pages before each block; returns their sum.
__device__ int32_t prefix_blocks(const Scratch& s, int32_t blocks) {
  int32_t before = 0;
  for (int32_t b0 = 0; b0 < blocks; b0 += kPlanThreads) {
    const int32_t b = b0 + threadIdx.x;
    int32_t total;
    const int32_t v = b < blocks ? __ldcg(&s.block[b]) : 0;
    const int32_t p = block_prefix(v, &total);
    if (b < blocks) s.block[b] = before + p;
    before += total;
  }
  if (threadIdx.x == 0) {
    s.block[blocks] = before;
    *s.ticket = 0;
  }
  __syncthreads();
  return before;
}

// The free pages of the first ranks go to the list and get their reference.
__device__ void grow_take(const op_cache_t& c, const Scratch& s, int32_t want) {
  const int32_t before = s.block[blockIdx.x];
  if (before >= want) return;
  const int64_t first = (int64_t)blockIdx.x * kBlockPages + threadIdx.x * kPerThread;
  const uint32_t bits = free_bits(c, first);
  int32_t total;
  int32_t r = before + block_prefix(__popc(bits), &total);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (bits >> j & 1) {
      if (r < want) {
        s.list[r] = int32_t(first + j);
        c.refs[first + j] = 1;
      }
      ++r;
    }
}

__global__ void __launch_bounds__(kPlanThreads) grow_count_kernel(op_cache_t c, const int32_t* seq, const int32_t* add,
                                                              int32_t n, Scratch s) {
  if (!count_free(c, s)) return;
  const int32_t n_free = prefix_blocks(s, gridDim.x);
  __shared__ unsigned long long worst;
  if (threadIdx.x == 0) worst = kNoFault;
  __syncthreads();
  const Faults f{&worst};
  check_rows(c, seq, n, s.mark, f);
  int64_t need = 0;   // of the entries before, the same in all threads
  for (int32_t i0 = 0; i0 < n; i0 += 256) {
    const int32_t i = threadIdx.x < 256 ? i0 + threadIdx.x : n;
    int32_t mine = 0;
    Entry e{0, 0, 0, -1};
    if (i < n && seq[i] >= 0 && seq[i] < c.n_seq) {
      e.seq = seq[i];
      e.old_len = c.lens[e.seq];
      const int64_t len = (int64_t)e.old_len + add[i];
      if (e.old_len < 0 || add[i] < 0 || pages_for(len, c.page_tokens) > c.max_pages) {
        f.add(i, GMG_PAGE_LONG);
      } else {
        const int32_t have = int32_t(pages_for(e.old_len, c.page_tokens));
        mine = int32_t(pages_for(len, c.page_tokens)) - have;
        if (add[i] > 0 && e.old_len % c.page_tokens) {
          const int32_t p = c.table[int64_t(e.seq) * c.max_pages + have - 1];
          if (p >= 0 && p < c.n_pages && c.refs[p] > 1) {
            e.tail = p;
            ++mine;
          }
        }
      }
    }
    int32_t total;
    const int32_t p = block_prefix(mine, &total);
    if (i < n) {
      e.off = int32_t(need + p < c.n_pages ? need + p : c.n_pages);
      s.entry[i] = e;
    }
    need += total;   // a round's needs are below 2^31: 256 rows of at most max_pages <= 2^22
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    write_status(c, worst);
    if (worst == kNoFault && need > n_free) {
      c.status[0] = GMG_PAGE_FULL;
      const int64_t missing = need - n_free;
      c.status[1] = missing < 0x7fffffff ? int32_t(missing) : 0x7fffffff;
    }
    s.plan[0] = c.status[0] == GMG_PAGE_OK ? int32_t(need) : 0;
  }
  if (gridDim.x == 1) {
    __syncthreads();
    grow_take(c, s, s.plan[0]);
  }
}

__global__ void __launch_bounds__(kPlanThreads) grow_take_kernel(op_cache_t c, Scratch s) { grow_take(c, s, s.plan[0]); }

// Bytes [at, at + kCopyBytes) of a page, all threads, eight 16-byte loads in flight each.
__device__ void copy_part(const op_cache_t& c, size_t bytes, int32_t from, int32_t to, size_t at) {
  const char* a = static_cast<const char*>(c.pool) + size_t(from) * bytes;
  char* b = static_cast<char*>(c.pool) + size_t(to) * bytes;
  constexpr int kEach = kCopyBytes / 16 / kThreads;
  uint4 v[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const size_t o = at + size_t(j * kThreads + threadIdx.x) * 16;
    if (o < bytes) v[j] = __ldcs(reinterpret_cast<const uint4*>(a + o));
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const size_t o = at + size_t(j * kThreads + threadIdx.x) * 16;
    if (o < bytes) *reinterpret_cast<uint4*>(b + o) = v[j];
  }
}

__global__ void __launch_bounds__(kThreads) grow_apply_kernel(op_cache_t c, const int32_t* add, int32_t n, size_t bytes,
                                                              Scratch s) {
  if (c.status[0] != GMG_PAGE_OK) return;
  for (int32_t i = blockIdx.y; i < n; i += gridDim.y) {
    const Entry e = s.entry[i];
    if (blockIdx.x == 0) {
      int32_t* row = c.table + int64_t(e.seq) * c.max_pages;
      const int32_t have = int32_t(pages_for(e.old_len, c.page_tokens));
      const int32_t want = int32_t(pages_for((int64_t)e.old_len + add[i], c.page_tokens));
      const int32_t* fresh = s.list + e.off + (e.tail >= 0);
      for (int32_t j = threadIdx.x; j < want - have; j += kThreads) row[have + j] = fresh[j];
      if (threadIdx.x == 0) {
        c.lens[e.seq] = e.old_len + add[i];
        if (e.tail >= 0) {
          row[have - 1] = s.list[e.off];
          atomicSub(&c.refs[e.tail], 1);
        }
      }
    }
    if (e.tail >= 0)
      for (size_t at = size_t(blockIdx.x) * kCopyBytes; at < bytes; at += size_t(gridDim.x) * kCopyBytes)
        copy_part(c, bytes, e.tail, s.list[e.off], at);
  }
}

__device__ void compact_rank(const op_cache_t& c, const Scratch& s) {
  const int32_t moves = s.plan[0], used = s.plan[1];
  const int64_t first = (int64_t)blockIdx.x * kBlockPages + threadIdx.x * kPerThread;
  const uint32_t bits = free_bits(c, first);
  int32_t total;
  int32_t before = s.block[blockIdx.x] + block_prefix(__popc(bits), &total);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int64_t p = first + j;
    if (p >= c.n_pages) break;
    const bool is_free = bits >> j & 1;
    if (is_free && p < used) s.list[before] = int32_t(p);
    if (!is_free && p >= used) {
      const int32_t r = int32_t(p) - before - (used - moves);   // used pages before p, less those below `used`
      s.from[r] = int32_t(p);
      s.rank[p] = r;
    }
    before += is_free;
  }
}

__global__ void __launch_bounds__(kPlanThreads) compact_count_kernel(op_cache_t c, Scratch s) {
  if (!count_free(c, s)) return;
  const int32_t n_free = prefix_blocks(s, gridDim.x);
  const int32_t used = c.n_pages - n_free;
  // free pages below `used`: whole blocks, then the part of the block that it lies in
  const int32_t b = used / kBlockPages;
  int32_t total;
  const int64_t first = (int64_t)b * kBlockPages + threadIdx.x * kPerThread;
  uint32_t bits = free_bits(c, first);
  if (first + kPerThread > used) bits &= first >= used ? 0u : (1u << (used - first)) - 1;
  block_prefix(__popc(bits), &total);
  if (threadIdx.x == 0) {
    const int32_t moves = s.block[b] + total;
    s.plan[0] = moves;
    s.plan[1] = used;
    c.status[0] = GMG_PAGE_OK;
    c.status[1] = 0;
    c.status[2] = moves;
    c.status[3] = used;
  }
  if (gridDim.x == 1) {
    __syncthreads();
    compact_rank(c, s);
  }
}

__global__ void __launch_bounds__(kPlanThreads) compact_rank_kernel(op_cache_t c, Scratch s) { compact_rank(c, s); }

__global__ void __launch_bounds__(kThreads) compact_apply_kernel(op_cache_t c, size_t bytes, Scratch s) {
  const int32_t moves = s.plan[0], used = s.plan[1];
  const int64_t cells = (int64_t)c.n_seq * c.max_pages;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < cells; i += (int64_t)gridDim.x * kThreads) {
    const int32_t p = c.table[i];
    if (p < used || p >= c.n_pages) continue;
    const int32_t r = s.rank[p];
    if (r >= 0 && r < moves && s.from[r] == p) c.table[i] = s.list[r];
  }
  const int64_t parts = int64_t((bytes + kCopyBytes - 1) / kCopyBytes);
  for (int64_t w = blockIdx.x; w < moves * parts; w += gridDim.x) {
    const int32_t r = int32_t(w / parts);
    const int64_t part = w % parts;
    const int32_t from = s.from[r], to = s.list[r];
    copy_part(c, bytes, from, to, size_t(part) * kCopyBytes);
    if (part == 0 && threadIdx.x == 0) {
      c.refs[to] = c.refs[from];
      c.refs[from] = 0;
    }
  }
}

int check(const op_cache_t* c, int32_t n, void* scratch, size_t scratch_bytes, Scratch* s) {
  if (!cache_ok(c) || n < 0 || n > c->n_seq) return GMG_EINVAL;
  if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || scratch_bytes < layout(*c, nullptr, nullptr))
    return GMG_EWS;
  layout(*c, static_cast<char*>(scratch), s);
  return GMG_OK;
}

int done() { return cudaGetLastError() == cudaSuccess ? GMG_OK : GMG_ECUDA; }

int empty_list(const op_cache_t* c, cudaStream_t st) {
  return cudaMemsetAsync(c->status, 0, 8, st) == cudaSuccess ? GMG_OK : GMG_ECUDA;
}

}  // namespace
}  // namespace gop

using namespace gop;

extern "C" {

size_t op_page_scratch_bytes(const op_cache_t* cache) { return cache_ok(cache) ? layout(*cache, nullptr, nullptr) : 0; }

int op_free(const op_cache_t* cache, const int32_t* seq, int32_t n, void* scratch, size_t scratch_bytes,
            gmg_stream_t stream) {
  Scratch s;
  const int rc = check(cache, n, scratch, scratch_bytes, &s);
  if (rc != GMG_OK) return rc;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (n == 0) return empty_list(cache, st);
  if (!seq) return GMG_EINVAL;
  if ((int64_t)n * cache->max_pages <= kFewCells) {
    free_check_kernel<true><<<1, kPlanThreads, 0, st>>>(*cache, seq, n, s);
  } else {
    free_check_kernel<false><<<1, kPlanThreads, 0, st>>>(*cache, seq, n, s);
    free_apply_kernel<<<n, kThreads, 0, st>>>(*cache, seq);
  }
  return done();
}

int op_fork(const op_cache_t* cache, const int32_t* src, const int32_t* dst, const int32_t* keep, int32_t n,
            void* scratch, size_t scratch_bytes, gmg_stream_t stream) {
  Scratch s;
  const int rc = check(cache, n, scratch, scratch_bytes, &s);
  if (rc != GMG_OK) return rc;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (n == 0) return empty_list(cache, st);
  if (!src || !dst) return GMG_EINVAL;
  if ((int64_t)n * cache->max_pages <= kFewCells) {
    fork_check_kernel<true><<<1, kPlanThreads, 0, st>>>(*cache, src, dst, keep, n, s);
  } else {
    fork_check_kernel<false><<<1, kPlanThreads, 0, st>>>(*cache, src, dst, keep, n, s);
    fork_apply_kernel<<<n, kThreads, 0, st>>>(*cache, src, dst, keep);
  }
  return done();
}

int op_grow(const op_cache_t* cache, const int32_t* seq, const int32_t* add, int32_t n, void* scratch,
            size_t scratch_bytes, gmg_stream_t stream) {
  Scratch s;
  const int rc = check(cache, n, scratch, scratch_bytes, &s);
  if (rc != GMG_OK) return rc;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (n == 0) return empty_list(cache, st);
  if (!seq || !add) return GMG_EINVAL;
  const size_t bytes = page_bytes(*cache);
  const int32_t blocks = blocks_of(*cache);
  grow_count_kernel<<<blocks, kPlanThreads, 0, st>>>(*cache, seq, add, n, s);
  if (blocks > 1) grow_take_kernel<<<blocks, kPlanThreads, 0, st>>>(*cache, s);
  const size_t parts = (bytes + kCopyBytes - 1) / kCopyBytes;
  const dim3 grid(unsigned(parts < 64 ? parts : 64), unsigned(n < 65535 ? n : 65535));
  grow_apply_kernel<<<grid, kThreads, 0, st>>>(*cache, add, n, bytes, s);
  return done();
}

int op_compact(const op_cache_t* cache, void* scratch, size_t scratch_bytes, gmg_stream_t stream) {
  Scratch s;
  const int rc = check(cache, 0, scratch, scratch_bytes, &s);
  if (rc != GMG_OK) return rc;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int32_t blocks = blocks_of(*cache);
  compact_count_kernel<<<blocks, kPlanThreads, 0, st>>>(*cache, s);
  if (blocks > 1) compact_rank_kernel<<<blocks, kPlanThreads, 0, st>>>(*cache, s);
  // as many blocks as there can be parts to copy, up to 64 an SM: a part each keeps more loads
  // on the way than a few blocks that take them in turn
  const size_t bytes = page_bytes(*cache);
  const int64_t parts = (int64_t)((bytes + kCopyBytes - 1) / kCopyBytes) * ((cache->n_pages + 1) / 2);
  const int64_t cells = ((int64_t)cache->n_seq * cache->max_pages + kThreads - 1) / kThreads;
  int64_t grid = parts > cells ? parts : cells;
  if (grid > 152 * 64) grid = 152 * 64;
  compact_apply_kernel<<<(unsigned)grid, kThreads, 0, st>>>(*cache, bytes, s);
  return done();
}

}  // extern "C"
