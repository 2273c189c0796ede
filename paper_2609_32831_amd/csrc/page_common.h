// page_common.h -- what the kernels of the paged 4-bit cache share: where a
// row lies, how it is held, and how a call's sequences are cut into work.
//
// A row (one KV head of one token, D channels) is D/2 bytes of 4-bit codes and
// NG = D / group scale words.  A word holds the group's step s (low half, a
// bf16 with 4 significant bits) and minimum m (high half, a bf16); a code c
// stands for c * s + m.  c has 4 significant bits and s has 4, so c * s has 8: the
// prompt kernel's matrix products take it in one plane, in fp16 with a power of
// two of 16 rows taken out; the single-token kernel's take c.
// Keys' codes lie in the order of the matrix operand (16 keys x 32 channels,
// lane (key, g) holding 8 channels of every 32): the 32-bit word (D/32) g + t
// of a row holds channels 32 t + 8 g .. 32 t + 8 g + 7, so that a lane's codes
// of a whole row are one load.  Values' codes lie in channel order.
#pragma once

#include "mfma_util.h"
#include "uc_common.h"

namespace uc {

struct PageCache {
  const uint8_t* codes_k;
  const uint8_t* codes_v;
  const uint32_t* scale_k;
  const uint32_t* scale_v;
  int n_pages, lgP, Hkv, D, ng;
};

// one attention call over the cache
struct PageAttendArgs {
  PageCache pc;
  const int32_t* q_start;
  const int32_t* len;
  const int32_t* table;
  const void* q;
  void* o;
  float* lse;
  int64_t q_ld;  // elements between tokens of q; o is [T, Hq, D]
  int S, T, ld, G;
  float scale_log2;
};

// blocks of 16 query rows of a KV head up to which a sequence counts as single
// tokens, and units of work of such a block beside its tiles of 64 rows (5, 8,
// 12 and 16: 64.9, 56.8, 59.1 and 59.6 us for 61 sequences of 1 to 40000 rows)
constexpr int kFewBlocks = 4, kStart = 8;

// a bf16 in the low / high half of a word
__device__ inline float word_step(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float word_min(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// page of row r of a table row, or -1 where the entry names none
__device__ inline int page_of(const int32_t* __restrict__ trow, int r, int lgP, int n_pages) {
  const int p = trow[r >> lgP];
  return (uint32_t)p < (uint32_t)n_pages ? p : -1;
}

// index of (page, head, row of the page) among the cache's rows
__device__ inline int64_t page_row(int page, int Hkv, int h, int lgP, int r) {
  return ((((int64_t)page * Hkv + h) << lgP)) + (r & ((1 << lgP) - 1));
}

// inclusive scan over the workgroup (blockDim a multiple of 64, at most
// 1024); total: the sum.  part: 16 values of LDS.
template <class T>
__device__ inline T block_scan(T x, T* part, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // part may still be read from an earlier scan
  if (lane == 63) part[wave] = x;
  __syncthreads();
  T before = 0;
  total = 0;
  for (int w = 0; w < waves; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  return x + before;
}

}  // namespace uc
