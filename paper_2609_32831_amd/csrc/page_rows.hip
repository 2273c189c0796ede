// page_rows.hip -- rows into and out of the paged 4-bit cache.
//
// Append: a row's D channels are quantised by groups of G, in binary32:
//   m = bf16(min x), s = (max x - m) / 15 rounded up to 4 significant bits,
//   code = s > 0 ? clamp(rint((x - m) / s), 0, 15) : 0
// with every x held to +-2^126 and a NaN read as 0, so that what is stored is
// finite and a row that a mask hides cannot reach another row's result.  For
// bf16 rows m is exact; the step is rounded up so that 15 of them still span
// the group (it grows by an eighth at most, 6 % on average).
// Each row stands for itself, so a slot is written without reading its page.
//
// Bound by bytes: 2 D elements in and D + 8 NG bytes out per row and head.
// 16 lanes (D = 128) or 8 (D = 64) take a row's keys and values, 8 channels of
// each: one 16-byte load of 16-bit rows, one 4-byte store of codes.  16001 rows
// of 4 heads of 128 bf16 (42 MB): append 14 us, read 9 us.  The append is held up
// by its arithmetic, 25 vector instructions an element (406 a wave for 16 elements
// a lane: two divisions, a reciprocal, the bounds and the steps between lanes
// among them; with a division for every element 18.6 us; keys and values by
// different threads 16.4; every element held to its bounds 15.6).
#include "page_common.h"

namespace uc {
namespace {

constexpr float kMost = 8.507059173023462e+37f;  // 2^126

// 8 consecutive elements from element i on as floats (16-byte aligned)
template <int DT>
__device__ inline void load8(const void* p, int64_t i, float (&x)[8]) {
  if constexpr (DT == UC_F32) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = f[0], b = f[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const mf::u4 w = *reinterpret_cast<const mf::u4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = DT == UC_BF16 ? __uint_as_float(w[e] << 16) : f16_to_f32((uint16_t)w[e]);
      x[2 * e + 1] = DT == UC_BF16 ? __uint_as_float(w[e] & 0xFFFF0000u) : f16_to_f32((uint16_t)(w[e] >> 16));
    }
  }
}

template <int DT>
__device__ inline void store8(void* p, int64_t i, const float (&x)[8]) {
  if constexpr (DT == UC_F32) {
    float4* f = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    f[0] = float4{x[0], x[1], x[2], x[3]};
    f[1] = float4{x[4], x[5], x[6], x[7]};
  } else {
    mf::u4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = DT == UC_BF16 ? mf::bf2(x[2 * e], x[2 * e + 1]) : mf::h2(x[2 * e], x[2 * e + 1]);
    *reinterpret_cast<mf::u4*>(static_cast<uint16_t*>(p) + i) = w;
  }
}

// where a lane's 8 channels (8 c .. 8 c + 7) of a row's codes lie, in words
template <int D, bool KEYS>
__device__ inline int code_word(int c) {
  return KEYS ? (D / 32) * (c & 3) + (c >> 2) : c;
}

struct RowArgs {
  PageCache cache;
  const void* k;
  const void* v;
  int64_t ld;  // elements between tokens
  int T;
  const int32_t* slots;
  const int32_t* copies;  // n_copies of (source page, destination page, rows)
  int n_copies;
};

// a quotient to its code, nearest even
__device__ inline uint32_t code_of(float q) { return (uint32_t)__builtin_amdgcn_fmed3f(rintf(q), 0.0f, 15.0f); }

// blocks [0, row_blocks): rows; then one block per copy.
template <int D, int DT>
__global__ __launch_bounds__(256) void page_append_kernel(RowArgs a, int row_blocks) {
  constexpr int LANES = D / 8;
  const PageCache& pc = a.cache;
  const int P = 1 << pc.lgP, ng = pc.ng;
  const int h = blockIdx.x % pc.Hkv, block = blockIdx.x / pc.Hkv;  // a token's heads lie together
  if (block >= row_blocks) {
    // rows 0 .. n-1 of every head of a page, to another page
    const int32_t* cp = a.copies + 3 * (block - row_blocks);
    const int src = cp[0], dst = cp[1], n = min(cp[2], P);
    if ((uint32_t)src >= (uint32_t)pc.n_pages || (uint32_t)dst >= (uint32_t)pc.n_pages || src == dst || n <= 0) return;
    const int64_t from = page_row(src, pc.Hkv, h, pc.lgP, 0), to = page_row(dst, pc.Hkv, h, pc.lgP, 0);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint32_t* codes = (uint32_t*)(kv ? pc.codes_v : pc.codes_k);
      uint32_t* scale = (uint32_t*)(kv ? pc.scale_v : pc.scale_k);
      for (int i = threadIdx.x; i < n * (D / 8); i += blockDim.x) codes[to * (D / 8) + i] = codes[from * (D / 8) + i];
      for (int i = threadIdx.x; i < n * ng; i += blockDim.x) scale[to * ng + i] = scale[from * ng + i];
    }
    return;
  }
  const int t = block * (256 / LANES) + threadIdx.x / LANES, c = threadIdx.x % LANES;
  // the row and its slot at a time, wherever it goes
  float x[2][8] = {};
  int slot = -1;
  if (t < a.T) {
    load8<DT>(a.k, (int64_t)t * a.ld + h * D + c * 8, x[0]);
    load8<DT>(a.v, (int64_t)t * a.ld + h * D + c * 8, x[1]);
    slot = a.slots[t];
  }
  const bool live = slot >= 0 && (slot >> pc.lgP) < pc.n_pages;
  const int64_t row = live ? page_row(slot >> pc.lgP, pc.Hkv, h, pc.lgP, slot) : 0;
  const int lg = __builtin_ctz(LANES) - __builtin_ctz(ng), per = 1 << lg;  // lanes of one group
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float(&y)[8] = x[kv];
    // a NaN or what passes the bound has larger bits than the bound
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(y[e]) & 0x7FFFFFFFu);
    if (__builtin_amdgcn_ballot_w64(most > __float_as_uint(kMost))) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] != y[e] ? 0.0f : fminf(fmaxf(y[e], -kMost), kMost);
    }
    float lo = y[0], hi = y[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = fminf(lo, y[e]);
      hi = fmaxf(hi, y[e]);
    }
    for (int o = 1; o < per; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o, 64));
      hi = fmaxf(hi, __shfl_xor(hi, o, 64));
    }
    const uint32_t mb = f32_to_bf16_bits(lo);
    const float m = bf16_to_f32(mb);
    const uint32_t sb = (__float_as_uint(fmaxf(hi - m, 0.0f) / 15.0f) + 0x000FFFFFu) & 0xFFF00000u;
    const float s = __uint_as_float(sb);
    // Quotients rounded as IEEE division does, by one reciprocal for all: with
    // r = 1 / s rounded to nearest and q within an ulp of d / s, q + (d - q s) r
    // is d / s rounded to nearest (Markstein 1990, for a divisor whose bits are
    // not all ones; s has four).  In this range of s nothing that counts passes
    // the type's range.
    uint32_t w = 0;
    if (s >= 0x1p-90f && s <= 0x1p100f) {
      const float r = 1.0f / s;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = y[e] - m, q = d * r;
        w |= code_of(fmaf(fmaf(-q, s, d), r, q)) << (4 * e);
      }
    } else if (s > 0.0f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w |= code_of((y[e] - m) / s) << (4 * e);
    }
    if (!live) continue;
    uint32_t* codes = (uint32_t*)(kv ? pc.codes_v : pc.codes_k);
    uint32_t* scale = (uint32_t*)(kv ? pc.scale_v : pc.scale_k);
    codes[row * (D / 8) + (kv ? code_word<D, false>(c) : code_word<D, true>(c))] = w;
    if ((c & (per - 1)) == 0) scale[row * ng + (c >> lg)] = (sb >> 16) | (mb << 16);
  }
}

template <int D, int DT>
__global__ __launch_bounds__(256) void page_read_kernel(PageCache pc, const int32_t* __restrict__ slots, int T,
                                                        void* kout, void* vout, int64_t ld) {
  constexpr int LANES = D / 8;
  const int h = blockIdx.x % pc.Hkv;
  const int t = blockIdx.x / pc.Hkv * (256 / LANES) + threadIdx.x / LANES, c = threadIdx.x % LANES;
  if (t >= T) return;
  const int slot = slots[t];
  const bool live = slot >= 0 && (slot >> pc.lgP) < pc.n_pages;
  const int64_t row = live ? page_row(slot >> pc.lgP, pc.Hkv, h, pc.lgP, slot) : 0;
  uint32_t w[2], sw[2];
  w[0] = ((const uint32_t*)pc.codes_k)[row * (D / 8) + code_word<D, true>(c)];
  w[1] = ((const uint32_t*)pc.codes_v)[row * (D / 8) + code_word<D, false>(c)];
  sw[0] = pc.scale_k[row * pc.ng + c * pc.ng / LANES];
  sw[1] = pc.scale_v[row * pc.ng + c * pc.ng / LANES];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      x[e] = live ? fmaf((float)((w[kv] >> (4 * e)) & 15u), word_step(sw[kv]), word_min(sw[kv])) : 0.0f;
    store8<DT>(kv ? vout : kout, (int64_t)t * ld + h * D + c * 8, x);
  }
}

}  // namespace

hipError_t launch_page_append(const PageCache& pc, const void* k, const void* v, int dt, int64_t ld, int T,
                              const int32_t* slots, const int32_t* copies, int n_copies, hipStream_t st) {
  const int per = 256 / (pc.D / 8), row_blocks = (T + per - 1) / per;
  if (row_blocks + n_copies == 0) return hipSuccess;
  const RowArgs a{pc, k, v, ld, T, slots, copies, n_copies};
  const dim3 grid((row_blocks + n_copies) * pc.Hkv);
#define UC_APPEND(DIM, TYPE) \
  hipLaunchKernelGGL((page_append_kernel<DIM, TYPE>), grid, dim3(256), 0, st, a, row_blocks)
  if (pc.D == 128) {
    if (dt == UC_BF16) UC_APPEND(128, UC_BF16);
    else if (dt == UC_F16) UC_APPEND(128, UC_F16);
    else UC_APPEND(128, UC_F32);
  } else {
    if (dt == UC_BF16) UC_APPEND(64, UC_BF16);
    else if (dt == UC_F16) UC_APPEND(64, UC_F16);
    else UC_APPEND(64, UC_F32);
  }
#undef UC_APPEND
  return hipGetLastError();
}

hipError_t launch_page_read(const PageCache& pc, const int32_t* slots, int T, void* kout, void* vout, int dt,
                            int64_t ld, hipStream_t st) {
  if (T == 0) return hipSuccess;
  const int per = 256 / (pc.D / 8);
  const dim3 grid((T + per - 1) / per * pc.Hkv);
#define UC_READ(DIM, TYPE) \
  hipLaunchKernelGGL((page_read_kernel<DIM, TYPE>), grid, dim3(256), 0, st, pc, slots, T, kout, vout, ld)
  if (pc.D == 128) {
    if (dt == UC_BF16) UC_READ(128, UC_BF16);
    else if (dt == UC_F16) UC_READ(128, UC_F16);
    else UC_READ(128, UC_F32);
  } else {
    if (dt == UC_BF16) UC_READ(64, UC_BF16);
    else if (dt == UC_F16) UC_READ(64, UC_F16);
    else UC_READ(64, UC_F32);
  }
#undef UC_READ
  return hipGetLastError();
}

}  // namespace uc
