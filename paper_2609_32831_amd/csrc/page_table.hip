// page_table.hip -- block tables and slot maps built on the device from the
// sequences' lengths, and the list of free pages they are served from.
//
// A sequence of n rows owns the pages named by the first ceil(n / P) entries
// of its table row; pages may be shared.  The free list is swept from the
// tables (every page that no entry names, ascending), so nothing counts
// references and the same tables always give the same list.  A step serves
// the sequences in order from the list's front: with need_s pages each, s
// takes entries [sum of need before s, + need_s) of the list.
//
// Both are bound by latency, not by bytes (a table of 1000 sequences of 64
// pages is 256 KB).
#include "page_common.h"

namespace uc {
namespace {

__device__ inline int blocks_of(int n, int lgP) { return (int)(((int64_t)n + (1 << lgP) - 1) >> lgP); }

__global__ void page_clear_kernel(uint32_t* __restrict__ mark, int words) {
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < words; i += gridDim.x * blockDim.x) mark[i] = 0;
}

// one thread per table entry; a byte per page, written with one value only
__global__ void page_mark_kernel(const int32_t* __restrict__ table, const int32_t* __restrict__ len,
                                 int S, int ld, int lgP, int n_pages, uint8_t* __restrict__ mark) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  for (int s = blockIdx.y; s < S; s += gridDim.y) {
    const int held = min(blocks_of(max(len[s], 0), lgP), ld);
    if (c >= held) continue;
    const int p = table[(int64_t)s * ld + c];
    if ((uint32_t)p < (uint32_t)n_pages) mark[p] = 1;
  }
}

constexpr int kListPages = 16 * 1024;  // pages of a workgroup's pass

// bit i: page first + i is free (first a multiple of 16; mark is padded to 16)
__device__ inline uint32_t open_pages(const uint8_t* __restrict__ mark, int first, int n_pages) {
  uint32_t open = 0;
  if (first < n_pages) {
    const uint4 v = *reinterpret_cast<const uint4*>(mark + first);
    const uint32_t m[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (first + i < n_pages && !((m[i >> 2] >> (8 * (i & 3))) & 0xFF)) open |= 1u << i;
  }
  return open;
}

__global__ __launch_bounds__(1024) void page_count_kernel(const uint8_t* __restrict__ mark, int n_pages,
                                                          int32_t* __restrict__ count) {
  __shared__ int part[16];
  int total;
  block_scan((int)__popc(open_pages(mark, blockIdx.x * kListPages + threadIdx.x * 16, n_pages)), part, total);
  if (threadIdx.x == 0) count[blockIdx.x] = total;
}

// Unmarked pages to the list: one workgroup for every kListPages, behind those
// of the ranges before it (count null: counted here, every workgroup for
// itself).
__global__ __launch_bounds__(1024) void page_list_kernel(const uint8_t* __restrict__ mark, int n_pages,
                                                         const int32_t* __restrict__ count,
                                                         int32_t* __restrict__ list, int32_t* __restrict__ pool) {
  __shared__ int part[16];
  int base, all, total, before = 0, sum = 0;
  const int p0 = blockIdx.x * kListPages, p1 = min(n_pages, p0 + kListPages);
  const int first = p0 + threadIdx.x * 16;
  const uint32_t open = open_pages(mark, first, n_pages);
  if (count) {
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 1024) {
      sum += count[i];
      if (i < (int)blockIdx.x) before += count[i];
    }
  } else {
#pragma unroll 4
    for (int b = 0; b < (int)gridDim.x; ++b) {
      const int at = b * kListPages + threadIdx.x * 16;
      if (at >= n_pages) break;
      const uint4 v = *reinterpret_cast<const uint4*>(mark + at);  // (bytes of 0 and 1, zeros behind the last)
      const int free = min(16, n_pages - at) - (__popc(v.x) + __popc(v.y) + __popc(v.z) + __popc(v.w));
      sum += free;
      if (b < (int)blockIdx.x) before += free;
    }
  }
  block_scan(before, part, base);
  block_scan(sum, part, all);
  const int upto = block_scan((int)__popc(open), part, total);
  int at = base + upto - __popc(open);
  for (uint32_t left = open; left; left &= left - 1) list[at++] = first + __ffs(left) - 1;
  // -1 behind the last: every workgroup the entries of its own range
  for (int i = max(all, p0) + threadIdx.x; i < p1; i += 1024) list[i] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    pool[0] = 0;
    pool[1] = all;
  }
}

// All of it in one workgroup, the marks as bits in LDS: for short tables.
constexpr int kSmallPages = 32768, kSmallEntries = 16384;
__global__ __launch_bounds__(1024) void page_free_small_kernel(const int32_t* __restrict__ table,
                                                               const int32_t* __restrict__ len, int S, int ld, int lgP,
                                                               int n_pages, int32_t* __restrict__ list,
                                                               int32_t* __restrict__ pool) {
  __shared__ uint32_t held[kSmallPages / 32];
  __shared__ int part[16];
  for (int i = threadIdx.x; i < kSmallPages / 32; i += 1024) held[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < S * ld; i += 1024) {
    const int s = i / ld, c = i - s * ld, p = table[i];
    if (c < blocks_of(max(len[s], 0), lgP) && (uint32_t)p < (uint32_t)n_pages) atomicOr(&held[p >> 5], 1u << (p & 31));
  }
  __syncthreads();
  const int first = threadIdx.x * 32;  // a word of pages per thread
  uint32_t open = first < n_pages ? ~held[threadIdx.x] : 0;
  if (n_pages - first < 32 && first < n_pages) open &= (1u << (n_pages - first)) - 1;
  int total;
  const int upto = block_scan((int)__popc(open), part, total);
  int at = upto - __popc(open);
  for (uint32_t left = open; left; left &= left - 1) list[at++] = first + __ffs(left) - 1;
  for (int i = total + threadIdx.x; i < n_pages; i += 1024) list[i] = -1;
  if (threadIdx.x == 0) {
    pool[0] = 0;
    pool[1] = total;
  }
}

struct StepArgs {
  const int32_t* len;
  const int32_t* more;
  int32_t* table;
  const int32_t* list;
  const int32_t* pool;
  int32_t* len_out;
  int32_t* q_start;
  int32_t* slots;
  int32_t* pool_out;
  uint8_t* refused;
  int S, ld, lgP, n_pages, n_slots;
};

// One workgroup: two scans over the sequences (pages taken, tokens before),
// then every sequence's new table entries and, unless a second kernel writes
// them, slots: a thread its own sequence's where they are few (a decode step),
// the wave one sequence after the other where they are many.
constexpr int kFew = 2;
__global__ __launch_bounds__(1024) void page_step_kernel(StepArgs a, bool with_slots) {
  __shared__ int64_t part[16];
  __shared__ int s_taken;
  const int lane = threadIdx.x & 63;
  const int head = max(a.pool[0], 0), list_end = a.pool[1];
  const int left = max(min(list_end, a.n_pages) - head, 0);  // entries the list still holds
  if (threadIdx.x == 0) s_taken = 0;
  int64_t pages = 0, tokens = 0;  // of the sequences before this pass
  const int P = 1 << a.lgP;
  auto slot = [&](const int32_t* trow, const int32_t* take, int held, int j) {
    const int c = j >> a.lgP, page = c >= held ? take[c - held] : trow[c];
    return (uint32_t)page < (uint32_t)a.n_pages ? page * P + (j & (P - 1)) : -1;
  };
  for (int s0 = 0; s0 < a.S; s0 += blockDim.x) {
    const int s = s0 + threadIdx.x;
    int n = 0, k = 0, held = 0, after = 0;
    if (s < a.S) {
      n = max(a.len[s], 0);
      k = min(max(a.more[s], 0), INT32_MAX - n);
      held = blocks_of(n, a.lgP);
      after = blocks_of(n + k, a.lgP);
    }
    const int need = after - held;
    int64_t total;
    const int64_t upto = pages + block_scan((int64_t)need, part, total);
    pages += total;
    const int64_t to = tokens + block_scan((int64_t)k, part, total);
    tokens += total;
    const int first = (int)min(to - k, (int64_t)a.n_slots), end = (int)min(to, (int64_t)a.n_slots);
    const bool ok = s < a.S && (need == 0 || upto <= left) && after <= a.ld && to <= a.n_slots;
    const int take_at = ok ? (int)(head + upto - need) : 0;
    if (s < a.S) {
      a.q_start[s] = first;
      if (s == a.S - 1) a.q_start[a.S] = end;
      a.len_out[s] = ok ? n + k : n;
      a.refused[s] = !ok;
      if (ok && need) atomicMax(&s_taken, (int)upto);
    }
    const bool few = need <= kFew && (!with_slots || k <= kFew);
    if (ok && few) {
      int32_t* trow = a.table + (int64_t)s * a.ld;
      const int32_t* take = a.list + take_at;
      if (with_slots)
        for (int i = 0; i < k; ++i) a.slots[first + i] = slot(trow, take, held, n + i);
      for (int c = 0; c < need; ++c) trow[held + c] = take[c];
    }
    for (uint64_t todo = __builtin_amdgcn_ballot_w64(s < a.S && (ok ? !few : with_slots && end > first)); todo;
         todo &= todo - 1) {
      const int from = __ffsll((unsigned long long)todo) - 1;
      const int sq = s - lane + from, n2 = __shfl(n, from, 64), h2 = __shfl(held, from, 64);
      const int f2 = __shfl(first, from, 64), e2 = __shfl(end, from, 64), need2 = __shfl(need, from, 64);
      const bool ok2 = __shfl((int)ok, from, 64);
      int32_t* trow = a.table + (int64_t)sq * a.ld;
      const int32_t* take = a.list + __shfl(take_at, from, 64);
      if (with_slots)
        for (int i = lane; i < e2 - f2; i += 64) a.slots[f2 + i] = ok2 ? slot(trow, take, h2, n2 + i) : -1;
      if (ok2)
        for (int c = lane; c < need2; c += 64) trow[h2 + c] = take[c];
    }
  }
  __syncthreads();
  if (with_slots)
    for (int64_t i = tokens + threadIdx.x; i < a.n_slots; i += blockDim.x) a.slots[i] = -1;
  if (threadIdx.x == 0) {
    a.pool_out[0] = head + s_taken;
    a.pool_out[1] = list_end;
  }
}

// a thread per token, after page_step_kernel: its sequence by search
__global__ __launch_bounds__(256) void page_slots_kernel(StepArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n_slots) return;
  int slot = -1;
  if (i < a.q_start[a.S]) {
    int s = 0;
    for (int hi = a.S; hi - s > 1;) {
      const int mid = (s + hi) >> 1;
      if (a.q_start[mid] <= i) s = mid;
      else hi = mid;
    }
    if (!a.refused[s]) {
      const int j = a.len_out[s] - (a.q_start[s + 1] - i);  // (a sequence that was served has all its tokens)
      const int page = a.table[(int64_t)s * a.ld + (j >> a.lgP)];
      if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.lgP) + (j & ((1 << a.lgP) - 1));
    }
  }
  a.slots[i] = slot;
}

}  // namespace

static int list_blocks(int n_pages) { return (n_pages + kListPages - 1) / kListPages; }
static size_t mark_bytes(int n_pages) { return ((size_t)n_pages + 15) & ~(size_t)15; }

size_t page_free_workspace(int n_pages) {
  return mark_bytes(n_pages) + (((size_t)list_blocks(n_pages) * sizeof(int32_t) + 255) & ~(size_t)255);
}

// Three launches, four where the pages are very many: up to kFewRanges ranges
// it is cheaper that every workgroup of the list counts the pages before its
// own than that a launch does (a table of 1000 sequences over 9 ranges, with the
// step behind it: 23.0 us, and 26.3 with the launch; 200000 pages alone 16.3 and
// 15.7, 400000 21.5 and 16.0).
constexpr int kFewRanges = 12;
hipError_t launch_page_free(const int32_t* table, const int32_t* len, int S, int ld, int lgP,
                            int n_pages, int32_t* list, int32_t* pool, void* ws, hipStream_t st) {
  if ((int64_t)S * ld <= kSmallEntries && n_pages <= kSmallPages) {
    hipLaunchKernelGGL(page_free_small_kernel, dim3(1), dim3(1024), 0, st, table, len, S, ld, lgP, n_pages, list, pool);
    return hipGetLastError();
  }
  uint8_t* mark = (uint8_t*)ws;
  const int words = (int)(mark_bytes(n_pages) / 4);
  hipLaunchKernelGGL(page_clear_kernel, dim3(min(256, (words + 255) / 256)), dim3(256), 0, st,
                     (uint32_t*)mark, words);
  hipLaunchKernelGGL(page_mark_kernel, dim3((ld + 255) / 256, min(S, 65535)), dim3(256), 0, st, table, len,
                     S, ld, lgP, n_pages, mark);
  const int blocks = list_blocks(n_pages);
  if (blocks <= kFewRanges) {
    hipLaunchKernelGGL(page_list_kernel, dim3(blocks), dim3(1024), 0, st, mark, n_pages, nullptr, list, pool);
  } else {
    int32_t* count = (int32_t*)(mark + mark_bytes(n_pages));
    hipLaunchKernelGGL(page_count_kernel, dim3(blocks), dim3(1024), 0, st, mark, n_pages, count);
    hipLaunchKernelGGL(page_list_kernel, dim3(blocks), dim3(1024), 0, st, mark, n_pages, count, list, pool);
  }
  return hipGetLastError();
}

// Slots in a launch of their own where they are many: one workgroup writes
// 50000 of them in some 30 microseconds, the second kernel in 4 and its launch.
hipError_t launch_page_step(int S, const int32_t* len, const int32_t* more, int32_t* table, int ld,
                            int lgP, int n_pages, const int32_t* list, const int32_t* pool,
                            int32_t* len_out, int32_t* q_start, int32_t* slots, int n_slots,
                            int32_t* pool_out, uint8_t* refused, hipStream_t st) {
  const StepArgs a{len, more, table, list, pool, len_out, q_start, slots, pool_out, refused,
                   S, ld, lgP, n_pages, n_slots};
  const bool with_slots = n_slots <= 4096;
  hipLaunchKernelGGL(page_step_kernel, dim3(1), dim3(S <= 256 ? 256 : 1024), 0, st, a, with_slots);
  if (!with_slots) hipLaunchKernelGGL(page_slots_kernel, dim3((n_slots + 255) / 256), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace uc
