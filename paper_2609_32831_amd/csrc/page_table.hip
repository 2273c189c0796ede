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

// one workgroup: 16 pages per thread and pass, unmarked ones to the list
__global__ __launch_bounds__(1024) void page_list_kernel(const uint8_t* __restrict__ mark, int n_pages,
                                                         int32_t* __restrict__ list,
                                                         int32_t* __restrict__ pool) {
  __shared__ int part[16];
  int base = 0;
  for (int p0 = 0; p0 < n_pages; p0 += 16 * 1024) {
    const int first = p0 + threadIdx.x * 16;
    uint32_t m[4] = {~0u, ~0u, ~0u, ~0u};
    if (first < n_pages) {  // mark is padded to 16 bytes
      const uint4 v = *reinterpret_cast<const uint4*>(mark + first);
      m[0] = v.x, m[1] = v.y, m[2] = v.z, m[3] = v.w;
    }
    uint32_t open = 0;  // bit i: page first + i is free
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (first + i < n_pages && !((m[i >> 2] >> (8 * (i & 3))) & 0xFF)) open |= 1u << i;
    int total;
    const int upto = block_scan((int)__popc(open), part, total);
    int at = base + upto - __popc(open);
    for (uint32_t left = open; left; left &= left - 1) list[at++] = first + __ffs(left) - 1;
    base += total;
  }
  for (int i = base + threadIdx.x; i < n_pages; i += blockDim.x) list[i] = -1;
  if (threadIdx.x == 0) {
    pool[0] = 0;
    pool[1] = base;
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
// then every sequence's new table entries and slots.
__global__ __launch_bounds__(1024) void page_step_kernel(StepArgs a) {
  __shared__ int64_t part[16];
  __shared__ int s_taken;
  const int head = max(a.pool[0], 0), list_end = a.pool[1];
  const int left = max(min(list_end, a.n_pages) - head, 0);  // entries the list still holds
  if (threadIdx.x == 0) s_taken = 0;
  int64_t pages = 0, tokens = 0;  // of the sequences before this pass
  const int P = 1 << a.lgP;
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
    if (s < a.S) {
      const int first = (int)min(to - k, (int64_t)a.n_slots), end = (int)min(to, (int64_t)a.n_slots);
      const bool ok = (need == 0 || upto <= left) && after <= a.ld && to <= a.n_slots;
      a.q_start[s] = first;
      if (s == a.S - 1) a.q_start[a.S] = end;
      if (ok) {
        int32_t* trow = a.table + (int64_t)s * a.ld;
        const int32_t* take = a.list + head + (upto - need);
        for (int c = 0; c < need; ++c) trow[held + c] = take[c];
        for (int i = 0; i < k; ++i) {
          const int j = n + i, c = j >> a.lgP;
          const int page = c >= held ? take[c - held] : trow[c];
          a.slots[first + i] = (uint32_t)page < (uint32_t)a.n_pages ? page * P + (j & (P - 1)) : -1;
        }
        if (need) atomicMax(&s_taken, (int)upto);
      } else {
        for (int i = first; i < end; ++i) a.slots[i] = -1;
      }
      a.len_out[s] = ok ? n + k : n;
      a.refused[s] = !ok;
    }
  }
  __syncthreads();
  for (int64_t i = tokens + threadIdx.x; i < a.n_slots; i += blockDim.x) a.slots[i] = -1;
  if (threadIdx.x == 0) {
    a.pool_out[0] = head + s_taken;
    a.pool_out[1] = list_end;
  }
}

}  // namespace

size_t page_free_workspace(int n_pages) { return (((size_t)n_pages + 15) & ~(size_t)15) + 256; }

hipError_t launch_page_free(const int32_t* table, const int32_t* len, int S, int ld, int lgP,
                            int n_pages, int32_t* list, int32_t* pool, void* ws, hipStream_t st) {
  uint8_t* mark = (uint8_t*)ws;
  const int words = (n_pages + 15) / 16 * 4;
  hipLaunchKernelGGL(page_clear_kernel, dim3(min(256, (words + 255) / 256)), dim3(256), 0, st,
                     (uint32_t*)mark, words);
  if (S > 0 && ld > 0)
    hipLaunchKernelGGL(page_mark_kernel, dim3((ld + 255) / 256, min(S, 65535)), dim3(256), 0, st, table, len,
                       S, ld, lgP, n_pages, mark);
  hipLaunchKernelGGL(page_list_kernel, dim3(1), dim3(1024), 0, st, mark, n_pages, list, pool);
  return hipGetLastError();
}

hipError_t launch_page_step(int S, const int32_t* len, const int32_t* more, int32_t* table, int ld,
                            int lgP, int n_pages, const int32_t* list, const int32_t* pool,
                            int32_t* len_out, int32_t* q_start, int32_t* slots, int n_slots,
                            int32_t* pool_out, uint8_t* refused, hipStream_t st) {
  const StepArgs a{len, more, table, list, pool, len_out, q_start, slots, pool_out, refused,
                   S, ld, lgP, n_pages, n_slots};
  hipLaunchKernelGGL(page_step_kernel, dim3(1), dim3(S <= 256 ? 256 : 1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace uc
