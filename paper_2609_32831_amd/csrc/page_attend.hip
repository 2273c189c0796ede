// page_attend.hip -- attention over a paged cache held in 4 bits: single
// tokens (few query rows of a KV head), prompts (any number), and the
// vector-ALU form that stands for both.
//
// A sequence of len rows whose last n are this call's queries: query i sees
// rows j < len - n + i + 1.  The n * G query rows of a KV head (G query heads
// share it) are ordered r = i * G + g.
//
// Single tokens.  With code c, step s and minimum m of a group g of channels,
//   q . k = sum_g s_g (q_g . c_g) + m_g sum(q_g)
//   sum_j p_j v_jd = sum_j (p_j s_jg) c_jd + sum_j p_j m_jg
// so the products run on whole codes, which a bf16 holds exactly, and the
// steps are applied once per (key, group) instead of once per element.  The
// codes become bf16 by two bit operations per pair: code | 0x4300 is 128 +
// code; the 128s leave through the accumulators' start (keys: -128 sum(q_g))
// and through the minima (values: m - 128 s).  Keys lie in operand order and
// go from the load straight to the matrix instruction; values pass LDS still
// as codes and are transposed by ds_read_b64_tr_b4 (16 x 16 codes).
// Probabilities enter the second product as bf16 hi + lo parts (16 bits).
//
// Work is cut evenly without the host knowing any length: the tiles (64 keys)
// of all sequences form one line, and workgroup w of W takes the w-th of W
// equal pieces (or each of its waves one of 4 W, where sequences are many).  A
// sequence that lies within one piece is written from there; one cut into
// several leaves a record (m, l, o) per piece, merged by a second kernel in the
// order of the pieces.
#include <algorithm>

#include "page_common.h"

namespace uc {
namespace {

using namespace mf;

constexpr int WAVES = 4;
constexpr int KT = 64;         // keys per tile
constexpr float kLazy = 8.0f;  // base-2 headroom before the reference maximum is raised
constexpr float kNone = -3.0e38f;  // the reference maximum before any visible key
constexpr float kFar = 0x1p16f;    // references beyond it: their own rounding counts

struct Seq {
  int q0, n, len;
};

// a sequence's first token, tokens and rows, held to the call's arrays
__device__ inline Seq seq_of(const PageAttendArgs& a, int s) {
  Seq x;
  x.q0 = min(max(a.q_start[s], 0), a.T);
  x.n = min(max(a.q_start[s + 1], x.q0), a.T) - x.q0;
  x.len = (int)min((int64_t)max(a.len[s], 0), min((int64_t)a.ld << a.pc.lgP, (int64_t)INT32_MAX));
  return x;
}

// the same in scalar registers, for a sequence that the whole wave works on
__device__ inline Seq scalar(const Seq& x) {
  return Seq{__builtin_amdgcn_readfirstlane(x.q0), __builtin_amdgcn_readfirstlane(x.n),
             __builtin_amdgcn_readfirstlane(x.len)};
}

template <int QT>
__device__ inline float q_val(const void* q, int64_t i) {
  return load_elem(q, QT, i);
}

template <int QT>
__device__ inline void put(void* o, int64_t i, float x) {
  if constexpr (QT == UC_F32) static_cast<float*>(o)[i] = x;
  else static_cast<uint16_t*>(o)[i] = QT == UC_BF16 ? f32_to_bf16_bits(x) : f32_to_f16_bits(x);
}

// natural log-sum-exp of a row from its base-2 reference maximum and sum
__device__ inline float lse_of(float m, float l) { return l > 0.0f ? (m + log2f(l)) * kLn2 : l == 0.0f ? -INFINITY : l; }

// ---------------------------------------------------------------- vector ALU
// A query row by one workgroup of 256: keys in chunks of 256, one per thread
// for the logits, one channel per thread for the values.
template <int D>
struct RowLds {
  float sq[D], sp[256], red[WAVES], so[256 / D][D];
  int64_t srow[256];
};

// token t of sequence s, query head hq
template <int D, int QT>
__device__ inline void attend_row(const PageAttendArgs& a, RowLds<D>& L, const Seq& x, int s, int t, int hq) {
  const int Hq = a.pc.Hkv * a.G, h = hq / a.G;
  const int lim = max(0, min(x.len, (int)((int64_t)x.len - x.n + (t - x.q0) + 1)));
  const int32_t* trow = a.table + (int64_t)s * a.ld;
  for (int d = threadIdx.x; d < D; d += blockDim.x) L.sq[d] = q_val<QT>(a.q, (int64_t)t * a.q_ld + hq * D + d);
  const int ng = a.pc.ng, gsz = D / ng;
  const int dim = threadIdx.x % D, part = threadIdx.x / D;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = kNone, l = 0.0f, acc = 0.0f;
  bool bad = false;
  for (int j0 = 0; j0 < lim; j0 += 256) {
    const int j = j0 + threadIdx.x;
    float v = -INFINITY;
    int64_t row = -1;
    if (j < lim) {
      const int page = page_of(trow, j, a.pc.lgP, a.pc.n_pages);
      if (page < 0) bad = true;
      else row = page_row(page, a.pc.Hkv, h, a.pc.lgP, j);
    }
    __syncthreads();  // sq is written; sp and srow are no longer read
    if (row >= 0) {
      float sum = 0.0f;
      const uint32_t* codes = (const uint32_t*)a.pc.codes_k + row * (D / 8);
      for (int w = 0; w < D / 8; ++w) {
        const int c0 = 32 * (w % (D / 32)) + 8 * (w / (D / 32));  // first channel of the word
        const uint32_t cw = codes[w], sw = a.pc.scale_k[row * ng + c0 / gsz];
        for (int e = 0; e < 8; ++e)
          sum = fmaf(L.sq[c0 + e], fmaf((float)((cw >> (4 * e)) & 15u), word_step(sw), word_min(sw)), sum);
      }
      v = sum * a.scale_log2;
    }
    L.srow[threadIdx.x] = row;
    float mx = wave_max(v);
    if (lane == 0) L.red[wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(L.red[0], L.red[1]), fmaxf(L.red[2], L.red[3]));
    const float m_new = fmaxf(m, mx), alpha = exp2f(m - m_new);
    m = m_new;
    const float p = exp2f(v - m);
    L.sp[threadIdx.x] = p;
    l = l * alpha + p;  // this thread's keys
    acc *= alpha;
    __syncthreads();
    const int n = min(256, lim - j0);
    for (int i = part; i < n; i += 256 / D) {
      if (L.srow[i] < 0) continue;
      const uint8_t b = a.pc.codes_v[L.srow[i] * (D / 2) + dim / 2];
      const uint32_t sw = a.pc.scale_v[L.srow[i] * ng + dim / gsz];
      acc = fmaf(L.sp[i], fmaf((float)((b >> (4 * (dim & 1))) & 15), word_step(sw), word_min(sw)), acc);
    }
  }
  __syncthreads();
  L.so[part][dim] = acc;
  l = wave_sum(l);
  if (lane == 0) L.red[wave] = l;
  const int any_bad = __syncthreads_or(bad);
  l = (L.red[0] + L.red[1]) + (L.red[2] + L.red[3]);
  if (any_bad) l = __builtin_nanf("");
  if (threadIdx.x < D) {
    float y = 0.0f;
    for (int i = 0; i < 256 / D; ++i) y += L.so[i][threadIdx.x];
    put<QT>(a.o, ((int64_t)t * Hq + hq) * D + threadIdx.x, l == 0.0f ? 0.0f : y / l);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)t * Hq + hq] = lse_of(m, l);
}

template <int D, int QT>
__global__ __launch_bounds__(256) void page_attend_valu_kernel(PageAttendArgs a) {
  __shared__ RowLds<D> lds;
  __shared__ int s_seq;
  const int Hq = a.pc.Hkv * a.G;
  for (int row = blockIdx.x; row < a.T * Hq; row += gridDim.x) {
    const int t = row / Hq;
    // the sequence whose tokens include t
    __syncthreads();
    if (threadIdx.x == 0) s_seq = INT32_MAX;
    __syncthreads();
    for (int s = threadIdx.x; s < a.S; s += blockDim.x) {
      const Seq x = seq_of(a, s);
      if (t >= x.q0 && t < x.q0 + x.n) atomicMin(&s_seq, s);
    }
    __syncthreads();
    const int s = s_seq;
    if (s < INT32_MAX) attend_row<D, QT>(a, lds, seq_of(a, s), s, t, row % Hq);  // a row of no sequence stays as it was
    if (row > INT32_MAX - (int)gridDim.x) break;
  }
}

// inclusive sums over the lanes, without LDS
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}

// ---------------------------------------------------------------- the line of tiles
// U units cut into W pieces that differ by one unit at most, the longer ones
// first (a call has fewer than 2^31 units, checked on the host).
struct Line {
  int per, more, W;
  __device__ Line(int U, int pieces) : per(U / pieces), more(U % pieces), W(pieces) {}
  __device__ int first(int w) const { return w * per + min(w, more); }
  __device__ int piece_of(int u) const {  // the piece that holds unit u
    const int edge = more * (per + 1);
    return u < edge ? u / (per + 1) : more + (u - edge) / per;
  }
};

// The single-token kernel takes the query rows of a KV head in blocks of 16, of
// sequences with kFewBlocks of them at most; 0 where the prompt kernel takes
// it, which works on 256 rows whatever their number (64 sequences of 4096 rows
// with 21, 28, 42, 63 query rows for each of 4 heads: 69, 69, 104, 127 us here,
// 199 to 204 there).
__device__ inline int token_blocks(const Seq& x, int G) {
  const int64_t rows = (int64_t)x.n * G;
  return rows > 16 * kFewBlocks ? 0 : (int)(rows + 15) >> 4;
}
// units of a block: the sequence's tiles, at least one so that a row that sees
// nothing is written too, behind `start` units that stand for what a block
// costs beside them (kStart; kSoloStart where a wave takes it by itself)
constexpr int kSoloStart = 2;
__device__ inline int tiles_of(int rows) { return rows <= KT ? 1 : (int)(((uint32_t)rows + KT - 1) / KT); }

// a block of a sequence (its first row among the sequence's) cut into pieces
// first .. last
struct Cut {
  int seq, first, last, block;
};

// Records: piece w leaves at most two, [2 w] of a sequence it continues and
// [2 w + 1] of one it begins; ROWS rows of o (D floats, not yet divided by l),
// m and l.
template <int D>
constexpr int kRec = D + 4;
template <int D, int ROWS, class T>
__device__ inline T* record(T* rec, int w, int Hkv, int h, bool begins) {
  return rec + (((int64_t)w * Hkv + h) * 2 + begins) * ROWS * kRec<D>;
}

// the prompt kernel's cut: blocks of 256 query rows
constexpr int PWAVES = 8, QROWS = 32 * PWAVES;

// blocks of a sequence
__device__ inline int prompt_blocks(const Seq& x, int G) {
  const int64_t rows = (int64_t)x.n * G;
  return rows <= 16 * kFewBlocks ? 0 : (int)((rows + QROWS - 1) / QROWS);
}
// tiles of its block b, at least one
__device__ inline int prompt_tiles(const Seq& x, int G, int b) {
  const int64_t last = min((int64_t)x.n - 1, ((int64_t)b * QROWS + QROWS - 1) / G);
  const int64_t sees = max((int64_t)0, min((int64_t)x.len, (int64_t)x.len - x.n + last + 1));
  return tiles_of((int)sees);
}

// before[s]: units of the sequences ahead of s, before[S]: all of them (by one
// workgroup of 256).  Only starts by which sequences share tokens can give more
// than the host allows for: then there are none, and no prompt is taken.
__device__ inline void plan_prompts(const PageAttendArgs& a, int* __restrict__ before, int64_t* part) {
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  for (int s0 = 0; s0 < a.S; s0 += 256) {
    const int s = s0 + threadIdx.x;
    Seq x{0, 0, 0};
    if (s < a.S) x = seq_of(a, s);
    const int blocks = prompt_blocks(x, a.G);
    int mine = 0;
    // the wave counts one sequence after the other, a block per lane
    for (uint64_t todo = __builtin_amdgcn_ballot_w64(blocks > 0); todo; todo &= todo - 1) {
      const int from = __ffsll((unsigned long long)todo) - 1;
      const Seq y{0, __shfl(x.n, from, 64), __shfl(x.len, from, 64)};
      const int nb = __shfl(blocks, from, 64);
      int sum = 0;
      for (int b = lane; b < nb; b += 64) sum += prompt_tiles(y, a.G, b);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (lane == from) mine = sum;
    }
    int64_t total;
    const int64_t upto = block_scan((int64_t)mine, part, total);
    if (s < a.S) before[s] = (int)(base + upto - mine);
    base += total;
  }
  if (threadIdx.x == 0) before[a.S] = base > INT32_MAX ? 0 : (int)base;
}

// ---------------------------------------------------------------- single tokens
// codes of a word -> four pairs of bf16 (128 + code): pair i holds codes i
// and i + 4.  The two constants come in registers, where one instruction ands
// and ors.
struct Magic {
  uint32_t mask, base;
  __device__ Magic() : mask(opaque(0x000F000Fu)), base(opaque(0x43004300u)) {}
  __device__ u4 pairs(uint32_t w) const {
    return u4{(w & mask) | base, ((w >> 4) & mask) | base, ((w >> 8) & mask) | base, ((w >> 12) & mask) | base};
  }
};

template <int N>
__device__ inline void load_words(const uint32_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const u4 x = *reinterpret_cast<const u4*>(p);
    w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x, w[1] = x.y;
  } else {
    w[0] = *p;
  }
}

// D/32 words of codes, read once per call: past the caches
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
template <int N>
__device__ inline void load_codes(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const u4 x = __builtin_nontemporal_load(reinterpret_cast<const u4*>(p));
    w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
  } else {
    const u2 x = __builtin_nontemporal_load(reinterpret_cast<const u2*>(p));
    w[0] = x[0], w[1] = x[1];
  }
}

template <int D, int NG>
struct WaveLds {
  static constexpr int VROW = D / 2 + 8;  // bytes of a staged row of values
  float k[2][NG][KT];                     // steps and minima of the tile's keys
  float v[2][NG][KT];                     // steps and (minima - 128 steps) of its values
  uint8_t codes[KT * VROW];
};

// x * scale rounded, then less m
__device__ inline float scaled_less(float x, float scale, float m) {
#pragma clang fp contract(off)
  const float y = x * scale;
  return y - m;
}

// D, NG: head dim and groups of a row; QP: bf16 parts of a query element;
// SOLO: a piece is a wave's, not the workgroup's.
//
// A wave's tile is four blocks of 16 keys, each within one page (pages are 16
// rows or more), so a block's codes are one contiguous piece of the cache
// behind a scalar address.  Block b's product rows are its keys, and lane
// group g4 holds those of keys 16 b + 4 g4 + j; the transposing reads of the
// values take their rows in that order.
template <int D, int NG, int QP, bool SOLO>
__global__ __launch_bounds__(256, 2) void page_tokens_kernel(PageAttendArgs a, int W_all, float* __restrict__ rec,
                                                             Cut* __restrict__ cuts, int* __restrict__ units_out) {
  constexpr int KS = D / 32;  // matrix steps over the channels, words of a lane's codes of a row
  constexpr int DT = D / 16;  // tiles of 16 output channels
  constexpr int GS = KS / NG;
  constexpr int QT = QP == 1 ? UC_BF16 : UC_F16;
  constexpr int STEP = SOLO ? 1 : WAVES, START = SOLO ? kSoloStart : kStart;
  using Lds = WaveLds<D, NG>;
  constexpr size_t kTiles = sizeof(Lds) * WAVES, kMerge = sizeof(float) * WAVES * 16 * (D + 2);
  __shared__ __attribute__((aligned(16))) char lds[kTiles > kMerge ? kTiles : kMerge];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int Hkv = a.pc.Hkv, h = blockIdx.x % Hkv, w = blockIdx.x / Hkv * (SOLO ? WAVES : 1) + (SOLO ? wave : 0);
  const int G = a.G, Hq = G * Hkv, lgP = a.pc.lgP, P1 = (1 << lgP) - 1;
  const Magic magic;
  if ((int)(blockIdx.x / Hkv * (SOLO ? WAVES : 1)) == W_all) {  // one workgroup more where prompts follow: their plan
    plan_prompts(a, units_out, reinterpret_cast<int64_t*>(lds));
    return;
  }
  const int turn = SOLO ? 0 : wave;  // the wave's among a piece's tiles
  if (SOLO ? lane == 0 : threadIdx.x == 0) cuts[w * Hkv + h] = Cut{-1, 0, 0, 0};

  // This piece of the line: the units of 64 sequences at a time, a sum for each
  // lane's c times 64, so that two looks find the sequence that holds unit u0.
  const int c = (a.S + 4095) / 4096;
  auto count = [&](int s, Seq& x) {
    x = Seq{0, 0, 0};
    if (s < a.S) x = seq_of(a, s);
    return token_blocks(x, G) * (START + tiles_of(x.len));  // (no tokens: no blocks)
  };
  Seq x;
  int mine = 0;
  if (a.S <= 64) {
    mine = count(lane, x);
  } else {
#pragma unroll 4
    for (int k = 0; k * 64 < a.S; ++k) {
      const int sum = __builtin_amdgcn_readlane(wave_scan(count(k * 64 + lane, x)), 63);
      if (lane == k / c) mine += sum;
    }
  }
  int upto = wave_scan(mine);
  const int U = __builtin_amdgcn_readlane(upto, 63);
  if (U == 0) return;
  // a sequence and a tile per wave at least
  const Line line(U, max(1, min(W_all, U / (START + STEP))));
  if (w >= line.W) return;
  const int u0 = line.first(w), u1 = line.first(w + 1);
  int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > u0)), s = at;
  int before = __builtin_amdgcn_readlane(upto - mine, at);  // units before sequence s
  if (a.S > 64) {
    for (s = at * c * 64;; s += 64) {
      mine = count(s + lane, x);
      upto = before + wave_scan(mine);
      const int end = __builtin_amdgcn_readlane(upto, 63);
      if (end > u0 || s + 64 >= a.S) break;
      before = end;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(upto > u0);
    at = past ? __builtin_ctzll(past) : 0;
    s += at;
    before = __builtin_amdgcn_readlane(upto - mine, at);
  }
  x = Seq{__builtin_amdgcn_readlane(x.q0, at), __builtin_amdgcn_readlane(x.n, at),
          __builtin_amdgcn_readlane(x.len, at)};
  Lds& L = *reinterpret_cast<Lds*>(lds + wave * sizeof(Lds));

  // The block at hand, `blk` of the sequence's `blks`: tiles [t0, t1) of it lie
  // in this piece.
  int blk = 0, blks = 0, units = 0, t0 = 0, t1 = 0, page = 0, page_next = 0, last16 = 0;
  const int32_t* trow = nullptr;
  u4 raw[KS];                                    // the lane's query row
  uint32_t ck[4][KS], cv[4][KS], wk[NG], wv[NG];  // a tile
  bool bad = false;
  // page of the lane's block of a tile; tiles past the range repeat its last
  auto page_for = [&](int t) {
    return x.len > 0 ? page_of(trow, min(min(t, t1 - 1) * KT + g4 * 16, last16), lgP, a.pc.n_pages) : 0;
  };
  // cache row of block b of tile t
  auto block_row = [&](int t, int pg, int b) {
    const int pb = max(__builtin_amdgcn_readlane(pg, 16 * b), 0);
    return (((int64_t)pb * Hkv + h) << lgP) + (min(t * KT + 16 * b, last16) & P1);
  };
  auto issue_keys = [&](int t, int pg) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      load_codes<KS>(a.pc.codes_k + block_row(t, pg, b) * (D / 2) + (uint32_t)(i16 * (D / 2) + g4 * (D / 8)), ck[b]);
  };
  auto issue_values = [&](int t, int pg) {
    if (t * KT + g4 * 16 < x.len && pg < 0) bad = true;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      load_codes<KS>(a.pc.codes_v + block_row(t, pg, b) * (D / 2) + (uint32_t)(lane * (D / 8)), cv[b]);
    const int64_t row = (((int64_t)max(pg, 0) * Hkv + h) << lgP) + (min(t * KT + g4 * 16, last16) & P1) + i16;
    load_words<NG>(a.pc.scale_k + row * NG, wk);
    load_words<NG>(a.pc.scale_v + row * NG, wv);
  };
  // on to the first block from this one on with tiles in [u, u1); false if
  // there is none.  Its pages and queries are asked for.
  auto open = [&](int u) {
    for (;;) {
      blks = token_blocks(x, G);
      units = START + tiles_of(x.len);
      if (before + (blks - blk) * units > u) break;
      before += (blks - blk) * units;
      if (before >= u1 || s + 1 >= a.S) return false;
      x = seq_of(a, ++s);
      blk = 0;
    }
    const int ahead = (u - before) / units;
    blk += ahead;
    before += ahead * units;
    if (before + START >= u1) return false;
    t0 = max(0, u - before - START);
    t1 = min(units, u1 - before) - START;
    trow = a.table + (int64_t)s * a.ld;
    last16 = (x.len - 1) & ~15;  // first row of the last 16
    page = page_for(t0 + turn);
    page_next = page_for(t0 + turn + STEP);
    const int r = min(blk * 16 + i16, x.n * G - 1);
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(x.q0 + r / G) * a.q_ld +
                        (int64_t)(h * G + r % G) * D + g4 * 8;
#pragma unroll
    for (int t = 0; t < KS; ++t) raw[t] = *reinterpret_cast<const u4*>(q + t * 32);
    return true;
  };
  // its first tile's loads
  auto first = [&]() {
    bad = false;
    if (x.len > 0 && t0 + turn < t1) {
      issue_values(t0 + turn, page);
      issue_keys(t0 + turn, page);
    }
  };
  if (!open(u0)) return;
  first();

  for (;;) {
    const int nq = min(16, x.n * G - blk * 16);
    // queries: the operand's channel order pairs codes i and i + 4
    u4 qb[QP][KS];
    float sq[NG];  // sum of the group's channels, all of them in every lane
#pragma unroll
    for (int g = 0; g < NG; ++g) sq[g] = 0.0f;
    {
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        if (i16 >= nq) raw[t] = u4{0, 0, 0, 0};
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[2 * e] = QP == 1 ? __uint_as_float(raw[t][e] << 16) : f16_to_f32((uint16_t)raw[t][e]);
          f[2 * e + 1] = QP == 1 ? __uint_as_float(raw[t][e] & 0xFFFF0000u) : f16_to_f32((uint16_t)(raw[t][e] >> 16));
          sq[t / GS] += f[2 * e] + f[2 * e + 1];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t hi = bf2(f[e], f[e + 4]);
          qb[0][t][e] = hi;
          if constexpr (QP == 2)
            qb[1][t][e] = bf2(f[e] - __uint_as_float(hi << 16), f[e + 4] - __uint_as_float(hi & 0xFFFF0000u));
        }
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        sq[g] += __shfl_xor(sq[g], 16, 64);
        sq[g] += __shfl_xor(sq[g], 32, 64);
      }
    }
    // first row that the lane's query does not see, and the least of them all
    const int lim = max(0, min(x.len, (int)((int64_t)x.len - x.n + (blk * 16 + min(i16, nq - 1)) / G + 1)));
    const int lim_all = max(0, (int)min((int64_t)x.len, (int64_t)x.len - x.n + blk * 16 / G + 1));

    bool far = false;
    float m = kNone, l = 0.0f, low[NG];
    f4 acc[DT];
#pragma unroll
    for (int g = 0; g < NG; ++g) low[g] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f4{0.f, 0.f, 0.f, 0.f};

    if (x.len > 0) {
      int t = t0 + turn;
      for (; t < t1; t += STEP) {
        const int tn = t + STEP;
        const bool more = tn < t1;
        // stage the tile: values as codes, words as floats; rows behind the
        // sequence hold anything, so their words become zeros
        {
          const bool in = t * KT + lane < x.len;
          uint8_t* dst = L.codes + (lane >> 2) * Lds::VROW + (lane & 3) * (D / 8);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int e = 0; e < KS; e += 2)
              *reinterpret_cast<uint2*>(dst + b * 16 * Lds::VROW + e * 4) = uint2{cv[b][e], cv[b][e + 1]};
          }
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint32_t xk = in ? wk[g] : 0, xv = in ? wv[g] : 0;
            L.k[0][g][lane] = word_step(xk);
            L.k[1][g][lane] = word_min(xk);
            L.v[0][g][lane] = word_step(xv);
            // (held finite: a row that is not seen weighs it with zero)
            L.v[1][g][lane] = fmaxf(fmaf(-128.0f, word_step(xv), word_min(xv)), -3.4e38f);
          }
        }
        __builtin_amdgcn_wave_barrier();
        // the next tile's loads, as registers become free; its page was read a
        // tile ago
        const int page_now = page_next;
        if (more) {
          issue_values(tn, page_now);
          page_next = page_for(tn + STEP);
        }

        // logits: p[4 b + j] of key 16 b + 4 g4 + j
        float p[16];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          f4 sum = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const float z = -128.0f * sq[g];
            f4 dot = f4{z, z, z, z};
#pragma unroll
            for (int t2 = g * GS; t2 < (g + 1) * GS; ++t2) {
              const u4 kb = magic.pairs(ck[b][t2]);
#pragma unroll
              for (int qp = 0; qp < QP; ++qp) dot = mfma(kb, qb[qp][t2], dot);
            }
            const f4 st = *reinterpret_cast<const f4*>(&L.k[0][g][b * 16 + g4 * 4]);
            const f4 mn = *reinterpret_cast<const f4*>(&L.k[1][g][b * 16 + g4 * 4]);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = fmaf(st[j], dot[j], fmaf(mn[j], sq[g], sum[j]));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) p[b * 4 + j] = sum[j];
        }
        const int r0 = t * KT;
        if (r0 + KT > lim_all) {
          asm volatile("");  // a branch, not sixteen selects per tile
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (r0 + (e >> 2) * 16 + g4 * 4 + (e & 3) >= lim) p[e] = -INFINITY;
        }
        if (more) issue_keys(tn, page_now);

        // softmax against a lazily raised reference maximum
        float mx = p[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, p[e]);
        mx *= a.scale_log2;
        if (__builtin_amdgcn_ballot_w64(mx > m + kLazy)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - m_new);
          m = m_new;
          far = __builtin_amdgcn_ballot_w64(fabsf(m) > kFar) != 0;
          l *= alpha;
#pragma unroll
          for (int g = 0; g < NG; ++g) low[g] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[d] *= alpha;
        }
        if (far) {  // round the others alike
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = scaled_less(p[e], a.scale_log2, m);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = fmaf(p[e], a.scale_log2, -m);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          p[e] = __builtin_amdgcn_exp2f(p[e]);
          l += p[e];
        }
        // O^T += V^T P, group by group
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float e1[8], e2[8];  // pairs (j, j + 4) of a lane's keys 0 .. 7 and 8 .. 15
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const f4 st = *reinterpret_cast<const f4*>(&L.v[0][g][b * 16 + g4 * 4]);
            const f4 mn = *reinterpret_cast<const f4*>(&L.v[1][g][b * 16 + g4 * 4]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float ps = p[b * 4 + j] * st[j];
              (b < 2 ? e1 : e2)[2 * j + (b & 1)] = ps;
              low[g] = fmaf(p[b * 4 + j], mn[j], low[g]);
            }
          }
          u4 h1, l1, h2, l2;
          split_p(e1, h1, l1);
          split_p(e2, h2, l2);
          const uint8_t* row = L.codes + ((i16 >> 2) * 16 + g4 * 4 + (i16 & 3)) * Lds::VROW;
#pragma unroll
          for (int d = g * (DT / NG); d < (g + 1) * (DT / NG); ++d) {
            typedef int v2i __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) v2i lds_v2i;
            const v2i cw = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_v2i*)(row + d * 8));
            const u4 va = magic.pairs((uint32_t)cw[0]), vb = magic.pairs((uint32_t)cw[1]);
            acc[d] = mfma(va, h1, acc[d]);
            acc[d] = mfma(va, l1, acc[d]);
            acc[d] = mfma(vb, h2, acc[d]);
            acc[d] = mfma(vb, l2, acc[d]);
          }
        }
        __builtin_amdgcn_wave_barrier();  // the tile's LDS is written again
      }
    }

    // the next block's loads are under way while this one's waves merge
    const Seq now = x;
    const int s_now = s, r_now = blk * 16, from = before + START, to = before + units;  // its tiles' units
    bool more = to < u1;
    const bool any = bad;
    if (more) {
      before = to;
      ++blk;
      more = open(to);
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      low[g] += __shfl_xor(low[g], 16, 64);
      low[g] += __shfl_xor(low[g], 32, 64);
    }
    const bool begins = from >= u0, ends = to <= u1;
    float* out = record<D, 16>(rec, w, Hkv, h, begins);
    if (begins && !ends && (SOLO ? lane == 0 : threadIdx.x == 0))
      cuts[w * Hkv + h] = Cut{s_now, w, line.piece_of(to - 1), r_now};
    if constexpr (SOLO) {
      if (more) first();
      if (__builtin_amdgcn_ballot_w64(any)) l = __builtin_nanf("");
      if (i16 < nq) {
        const int64_t at = (int64_t)(now.q0 + (r_now + i16) / G) * Hq + h * G + (r_now + i16) % G;
        const bool whole = begins && ends;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f4 y = acc[d];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] += low[d / (DT / NG)];
          if (whole) {
            y *= inv;
            const uint2 z =
                QT == UC_BF16 ? uint2{bf2(y[0], y[1]), bf2(y[2], y[3])} : uint2{h2(y[0], y[1]), h2(y[2], y[3])};
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + at * D + d * 16 + g4 * 4) = z;
          } else {
            *reinterpret_cast<f4*>(out + i16 * kRec<D> + d * 16 + g4 * 4) = y;
          }
        }
        if (g4 == 0) {
          if (!whole) out[i16 * kRec<D> + D] = m, out[i16 * kRec<D> + D + 1] = l;
          else if (a.lse) a.lse[at] = lse_of(m, l);
        }
      }
      if (!more) break;
      continue;
    }
    const int any_bad = __syncthreads_or(any);
    float* mo = reinterpret_cast<float*>(lds);  // [WAVES][16][D]
    float* ml = mo + WAVES * 16 * D;            // [WAVES][16] m, then l
    if (g4 == 0) {
      ml[wave * 16 + i16] = m;
      ml[WAVES * 16 + wave * 16 + i16] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f4 y = acc[d];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += low[d / (DT / NG)];
      *reinterpret_cast<f4*>(&mo[(wave * 16 + i16) * D + d * 16 + g4 * 4]) = y;
    }
    if (more) first();
    __syncthreads();
    for (int e = threadIdx.x; e < nq * D; e += blockDim.x) {
      const int r = e / D, d = e % D;
      float M = kNone, ls = 0.0f, y = 0.0f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) M = fmaxf(M, ml[i * 16 + r]);
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        const float wt = exp2f(ml[i * 16 + r] - M);
        ls = fmaf(wt, ml[WAVES * 16 + i * 16 + r], ls);
        y = fmaf(wt, mo[(i * 16 + r) * D + d], y);
      }
      if (any_bad) ls = __builtin_nanf("");
      if (begins && ends) {
        const int64_t at = (int64_t)(now.q0 + (r_now + r) / G) * Hq + h * G + (r_now + r) % G;
        put<QT>(a.o, at * D + d, ls == 0.0f ? 0.0f : y / ls);
        if (d == 0 && a.lse) a.lse[at] = lse_of(M, ls);
      } else {
        out[r * kRec<D> + d] = y;
        if (d == 0) {
          out[r * kRec<D> + D] = M;
          out[r * kRec<D> + D + 1] = ls;
        }
      }
    }
    if (!more) break;
    __syncthreads();  // LDS is written again
  }
}

// ---------------------------------------------------------------- prompts
// Blocks of 256 query rows, 32 a wave, each over the tiles that its last row
// sees; the line is made of all blocks' tiles.  A workgroup's eight waves share
// the tile in LDS, where the 4-bit rows, read and unpacked once for all of
// them, stand as fp16: with the power of two 2^e of the largest step of 16 rows
// taken out, c * (s 2^-e) has 8 significant bits and is exact, and so is the
// minimum, down to steps of 2^-13 of the largest.  The powers return where they
// cost nothing: the keys' in the factor that turns a product into a logit, the
// values' in the exponent,
//   w_j = 2^(logit_j + e_j - m),  o ~ sum_j w_j (v_j 2^-e_j),  l = sum_j w_j 2^-e_j,
// with the reference m kept over logit + e, so that w_j, rounded to fp16 (11
// bits), is measured by what key j contributes whatever the values' sizes.  l
// is summed in binary32 before that rounding.  The reference puts a row's
// largest weight at 2^7 .. 2^15, so that the small ones of a long tail are fp16's
// too: what lies below its subnormal step is off by 2^-32 of the largest (with
// the largest at 1, a tail of 65500 keys of 2^-25.5 each, a 700th of the sum, was
// lost from o and not from l; 1 % faster).  The minima go through matrix
// instructions of their own, q . k += sum_g m_g sum(q_g) with sum(q_g) in three
// fp16 parts.  Queries enter as fp16 too, a row far from 1, or of sums that fp16
// does not hold, by a power of two: as such a row stands, its elements below
// 2^-14 are off by 2^-25 at most, 2^-21 of its largest; the others are exact.
//
// Rows of more different sizes within 16 (one of infinities, say, that earlier
// queries do not see), values beyond 2^-60 .. 2^76 and logits beyond 2^16 mark
// the workgroup's piece; every block that has a part in it is computed anew from
// the cache, a row per workgroup: right, but a hundred times as slow.  Looking
// for them costs 2 % of the kernel's time.
//
// Four prompts of 1500 tokens over up to 8192 rows, 28 query heads on 4, D 128
// (342 GFLOP): 465 us a call, 736 TFLOP/s.  A stage of 64 keys x 32 rows is 76
// matrix instructions a wave and five vector instructions to each of those,
// most of them for the softmax; the two do not overlap fully with the two waves
// a SIMD holds.  Tried: four waves a workgroup, each tile then staged for half
// the rows (709 us); two buffers and a barrier per tile instead of the
// pipeline of steps (530 us); bf16 planes (578 us); fixed orders of matrix and
// vector instructions (498 to 553 us) - the compiler's own is the best.

// A raised reference puts the largest weight at 2^kPeak; it is raised once a
// weight passes 2^kRaise, which is looked at where the eight weights of a lane
// together pass kTop = 8 * 2^kRaise, the last power that fp16 holds.
constexpr float kPeak = 7.0f, kRaise = 12.0f, kTop = 0x1p15f;

template <int D>
constexpr int kRow = 2 * D + 32;  // bytes of a staged row: 8 consecutive rows start in different 8-bank groups

typedef _Float16 half2 __attribute__((ext_vector_type(2)));

// Keys and values of a stage of KS keys, in rings of three: the loop is a
// pipeline over steps of 32 keys that takes, in step j, the products of step
// j + 1, the probabilities of step j and the output of step j - 1, which do
// not depend on one another; so a stage's keys are wanted from the stage
// before it to its own end, and its values from its beginning to the next
// one's.
template <int D, int KEYS>
struct PromptKeys {
  uint8_t k[KEYS * kRow<D>];  // c * s 2^-e in fp16; of eight channels in the order 0 4 1 5 2 6 3 7
  _Float16 m[KEYS][8];        // minima (2^-e) of a key, zeros behind them
  float f[KEYS / 16];         // logit of a product: scale * 2^e
};
template <int D, int KEYS>
struct PromptValues {
  uint8_t v[KEYS * kRow<D>];
  _Float16 m[4][KEYS + 8];            // minima (2^-e) of a group, by key
  float e[KEYS / 16], inv[KEYS / 16];  // e and 2^-e
};

// a word's eight codes times a step, as fp16: (1024 + c) s - 1024 s
struct Unpack {
  uint32_t mask, base;
  __device__ Unpack() : mask(opaque(0x000F000Fu)), base(opaque(0x64006400u)) {}
  __device__ u4 times(uint32_t w, half2 s, half2 off) const {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const half2 x = __builtin_bit_cast(half2, ((w >> (4 * i)) & mask) | base);
      r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, s, off));
    }
    return r;
  }
};

// Biased exponent of the power of two taken out of 16 rows (16 CH lanes, CH
// of a row): their largest step comes below 2 and their minima below 2^14.
// What does not fit beside it sets `wide`: a group whose step and minimum are
// both below 2^-13 of it (above, codes times steps are exact and a minimum is
// off by 2^-12 of the larger of both at most), or a power beyond the range.
template <int NG, int CH>
__device__ inline int rows_exponent(const uint32_t (&w)[NG], int ch, int least, int most, int& wide) {
  int e = 0;
#pragma unroll
  for (int n = 0; n < NG; ++n)
    e = max(e, max((int)(w[n] >> 7 & 0xFF), (int)(w[n] >> 23 & 0xFF) - 12));
  // over the lanes CH apart of a row of 16 lanes, then over the rows
  e = max(e, __builtin_amdgcn_update_dpp(e, e, 0x120 + 8, 0xF, 0xF, false));
  e = max(e, __builtin_amdgcn_update_dpp(e, e, 0x120 + 4, 0xF, 0xF, false));
  if constexpr (CH == 2) e = max(e, __builtin_amdgcn_update_dpp(e, e, 0x120 + 2, 0xF, 0xF, false));
  const auto r16 = __builtin_amdgcn_permlane16_swap(e, e, false, false);
  e = max((int)r16[0], (int)r16[1]);
  if constexpr (CH == 4) {
    const auto r32 = __builtin_amdgcn_permlane32_swap(e, e, false, false);
    e = max((int)r32[0], (int)r32[1]);
  }
  const int E = e == 0 ? 127 : min(max(e, least), most);  // rows of zeros: any
  uint32_t mine = w[0];  // the row's lanes look at a group each
#pragma unroll
  for (int n = 1; n < NG; ++n)
    if (ch * NG / CH == n) mine = w[n];
  const int own = max((int)(mine >> 7 & 0xFF), (int)(mine >> 23 & 0xFF));
  if (e > most || (uint32_t)(own - 1) < (uint32_t)(E - 14)) wide = 1;  // (a group of zeros fits)
  return E;
}

template <int D, int NG>
__global__ __launch_bounds__(64 * PWAVES, 2) void page_prompt_kernel(PageAttendArgs a, int W_all, bool q_f16,
                                                                 const int* __restrict__ units,
                                                                 float* __restrict__ rec, Cut* __restrict__ cuts,
                                                                 int* __restrict__ wide) {
  constexpr int KS = D / 32, DT = D / 16, THREADS = 64 * PWAVES;
  constexpr int KEYS = 64, SPS = KEYS / 32;  // keys and steps of a stage
  using Keys = PromptKeys<D, KEYS>;
  using Values = PromptValues<D, KEYS>;
  __shared__ __attribute__((aligned(16))) Keys keys[3];
  __shared__ __attribute__((aligned(16))) Values values[3];
  __shared__ float2 s_rows[2][THREADS];  // for the lanes' query rows: first row not seen (bits), power of two taken out
  __shared__ int s_part[16], s_block, s_before, s_wide;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int Hkv = a.pc.Hkv, h = blockIdx.x % Hkv, w = blockIdx.x / Hkv;
  const int G = a.G, Hq = G * Hkv, lgP = a.pc.lgP;
  const Unpack unpack;
  if (threadIdx.x == 0) {
    cuts[blockIdx.x] = Cut{-1, 0, 0, 0};
    wide[blockIdx.x] = s_wide = 0;
  }
  const int U = __builtin_amdgcn_readfirstlane(units[a.S]);
  if (U == 0) return;
  const Line line(U, min(W_all, U));
  if (w >= line.W) return;
  const int u0 = line.first(w), u1 = line.first(w + 1);
  // the sequence and the block that hold unit u0
  int s = 0;
  for (int hi = a.S; hi - s > 1;) {
    const int mid = (s + hi) >> 1;
    if (units[mid] <= u0) s = mid;
    else hi = mid;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  Seq x = scalar(seq_of(a, s));
  int nb = prompt_blocks(x, G);
  {
    int base = units[s];
    for (int b0 = 0; b0 < nb; b0 += THREADS) {
      const int b = b0 + threadIdx.x;
      const int mine = b < nb ? prompt_tiles(x, G, b) : 0;
      int total;
      const int upto = base + block_scan(mine, s_part, total);
      if (upto - mine <= u0 && u0 < upto) {
        s_block = b;
        s_before = upto - mine;
      }
      base += total;
    }
  }
  // the slots behind a key's minima stay zero
  for (int i = threadIdx.x; i < KEYS * 8; i += THREADS)
    (&keys[0].m[0][0])[i] = (&keys[1].m[0][0])[i] = (&keys[2].m[0][0])[i] = (_Float16)0.0f;
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(s_block);
  int before = __builtin_amdgcn_readfirstlane(s_before);

  // A thread's share of a stage: 16 bytes of codes of a row, of keys (the
  // first waves) or of values.
  constexpr int CH = D / 32;
  static_assert(2 * KEYS * CH <= THREADS, "a task a thread at most");
  const int kind = wave * 64 / (KEYS * CH), key = threadIdx.x % (KEYS * CH) / CH, ch = threadIdx.x % CH;
  u4 codes;
  uint32_t words[NG];

  for (int u = u0; u < u1;) {
    const int tiles = prompt_tiles(x, G, b);
    const int t0 = u - before, t1 = min(tiles, u1 - before);
    const int rows = (int)min((int64_t)QROWS, (int64_t)x.n * G - (int64_t)b * QROWS);
    const int32_t* trow = a.table + (int64_t)s * a.ld;
    bool bad = false;

    // the thread's codes of a stage; rows past the sequence repeat its last
    // one.  Its page is read a stage ahead.
    auto row_at = [&](int stage) { return min(t0 * KT + stage * KEYS + key, x.len - 1); };
    int page = x.len > 0 ? page_of(trow, row_at(0), lgP, a.pc.n_pages) : 0;
    auto issue = [&](int stage) {
      if (page < 0) bad = true;
      const int64_t row = page_row(max(page, 0), Hkv, h, lgP, row_at(stage));
      page = page_of(trow, row_at(stage + 1), lgP, a.pc.n_pages);
      if (kind > 1) return;
      codes = *reinterpret_cast<const u4*>((kind ? a.pc.codes_v : a.pc.codes_k) + row * (D / 2) + ch * 16);
      load_words<NG>((kind ? a.pc.scale_v : a.pc.scale_k) + row * NG, words);
    };
    auto store_keys = [&](Keys& L) {
      const int E = rows_exponent<NG, CH>(words, ch, 24, 230, s_wide);
      const float out = __uint_as_float((uint32_t)(254 - E) << 23);
      half2 st[NG], off[NG];
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        const float f = word_step(words[n]) * out;
        st[n] = __builtin_bit_cast(half2, h2(f, f));
        off[n] = __builtin_bit_cast(half2, h2(-1024.0f * f, -1024.0f * f));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // the word holds channels 32 step + 8 g ..
        const int step = KS == 4 ? j : j % KS, g = (ch * 4 + j) / KS, n = step * NG / KS;
        *reinterpret_cast<u4*>(L.k + key * kRow<D> + (step * 4 + g) * 16) = unpack.times(codes[j], st[n], off[n]);
      }
      if (ch == 0) {
#pragma unroll
        for (int n = 0; n < NG; ++n) L.m[key][n] = (_Float16)(word_min(words[n]) * out);
        L.f[key / 16] = __uint_as_float((uint32_t)E << 23) * a.scale_log2;
      }
    };
    auto store_values = [&](Values& L) {
      const int E = rows_exponent<NG, CH>(words, ch, 127 - 48, 127 + 76, s_wide);
      const float out = __uint_as_float((uint32_t)(254 - E) << 23);
      float f = word_step(words[0]);
#pragma unroll
      for (int n = 1; n < NG; ++n)
        if (ch * NG / CH == n) f = word_step(words[n]);
      f *= out;
      const half2 st = __builtin_bit_cast(half2, h2(f, f)), off = __builtin_bit_cast(half2, h2(-1024.0f * f, -1024.0f * f));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<u4*>(L.v + key * kRow<D> + (ch * 4 + j) * 16) = unpack.times(codes[j], st, off);
      if (ch == 0) {
#pragma unroll
        for (int n = 0; n < NG; ++n) L.m[n][key] = (_Float16)(word_min(words[n]) * out);
        L.e[key / 16] = (float)(E - 127);
        L.inv[key / 16] = out;
      }
    };
    if (x.len > 0) issue(0);

    u4 qb[2][KS], sqb[2];
    bool scaled = false;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = wave * 32 + c * 16 + i16;
      const int rr = b * QROWS + min(r, rows - 1), i = rr / G, gq = rr % G;
      const int lim = (int)max((int64_t)0, min((int64_t)x.len, (int64_t)x.len - x.n + i + 1));
      const int64_t base = (int64_t)(x.q0 + i) * a.q_ld + (int64_t)(h * G + gq) * D + g4 * 8;
      float f[KS][8], most = 0.0f;
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const u4 raw = *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(a.q) + base + t * 32);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[t][2 * e] = q_f16 ? f16_to_f32((uint16_t)raw[e]) : __uint_as_float(raw[e] << 16);
          f[t][2 * e + 1] = q_f16 ? f16_to_f32((uint16_t)(raw[e] >> 16)) : __uint_as_float(raw[e] & 0xFFFF0000u);
          most = fmaxf(most, fmaxf(fabsf(f[t][2 * e]), fabsf(f[t][2 * e + 1])));
        }
      }
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      // sums of the groups' channels, all of them in every lane
      float sq[NG];
      auto add_up = [&]() {
#pragma unroll
        for (int n = 0; n < NG; ++n) sq[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) sq[t * NG / KS] += f[t][e];
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          sq[n] += __shfl_xor(sq[n], 16, 64);
          sq[n] += __shfl_xor(sq[n], 32, 64);
        }
      };
      add_up();
      float most_sum = 0.0f;
#pragma unroll
      for (int n = 0; n < NG; ++n) most_sum = fmaxf(most_sum, fabsf(sq[n]));
      const int E = (int)(__float_as_uint(most) >> 23);  // 2^(E - 127) <= most
      // elements and sums have to fit fp16: a row whose elements or sums reach
      // 2^15 comes below 2, its sums below 2 D / NG
      const bool far = most > 0.0f && (E < 127 - 4 || E > 127 + 14 || !(most_sum < 0x1p15f));
      const float out = far ? __uint_as_float((uint32_t)(254 - min(max(E, 1), 253)) << 23) : 1.0f;
      s_rows[c][threadIdx.x] = float2{__int_as_float(lim), far ? __uint_as_float((uint32_t)min(max(E, 1), 253) << 23) : 1.0f};
      scaled |= far;
      if (__builtin_amdgcn_ballot_w64(far)) {
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) f[t][e] *= out;
        add_up();  // anew: sums of large elements may have passed binary32
      }
#pragma unroll
      for (int t = 0; t < KS; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) qb[c][t][e] = h2(f[t][e], f[t][e + 4]);
      // sums in three fp16 parts: part g4 in this lane's slots
      uint32_t bits[4] = {0, 0, 0, 0};
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        float y = sq[n];
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (p < g4) y -= f16_to_f32(f32_to_f16_bits(y));
        const uint32_t v = g4 < 3 ? f32_to_f16_bits(y) : 0;
        bits[n >> 1] |= v << (16 * (n & 1));
      }
      sqb[c] = u4{bits[0], bits[1], bits[2], bits[3]};
    }
    const bool always = __builtin_amdgcn_ballot_w64(scaled) != 0;
    // rows below it are seen by all of the wave's queries
    const int lim_all =
        (int)max((int64_t)0, (int64_t)x.len - x.n + min((int64_t)b * QROWS + wave * 32, (int64_t)x.n * G - 1) / G + 1);

    float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};
    f4 acc[2][DT], low[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      low[c] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[c][d] = f4{0.f, 0.f, 0.f, 0.f};
    }

    if (x.len > 0) {
      // products of both blocks of queries with 16 keys
      auto products = [&](const Keys& L, int first, f4& s0, f4& s1) {
        const u4 km = *reinterpret_cast<const u4*>(&L.m[first + i16][0]);
        s0 = mfma_f16(km, sqb[0], f4{0.f, 0.f, 0.f, 0.f});
        s1 = mfma_f16(km, sqb[1], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          const u4 ka = *reinterpret_cast<const u4*>(L.k + (first + i16) * kRow<D> + (st * 4 + g4) * 16);
          s0 = mfma_f16(ka, qb[0][st], s0);
          s1 = mfma_f16(ka, qb[1][st], s1);
        }
      };
      // weights of 32 keys for queries c: w = 2^(logit + e - m); their sum,
      // and that of l
      auto weigh = [&](const Keys& K, const Values& V, int sub, int c, const f4& s0, const f4& s1, float& sum,
                       float& sum_l) {
        float e[8], part[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float kf = K.f[sub * 2 + i], off = V.e[sub * 2 + i] - m[c];
#pragma unroll
          for (int j = 0; j < 4; ++j) e[i * 4 + j] = __builtin_amdgcn_exp2f(fmaf(i ? s1[j] : s0[j], kf, off));
          part[i] = (e[i * 4] + e[i * 4 + 1]) + (e[i * 4 + 2] + e[i * 4 + 3]);
        }
        sum = part[0] + part[1];
        sum_l = fmaf(part[0], V.inv[sub * 2], part[1] * V.inv[sub * 2 + 1]);
        return u4{h2(e[0], e[1]), h2(e[2], e[3]), h2(e[4], e[5]), h2(e[6], e[7])};
      };
      auto output = [&](const Values& L, int sub, const u4 (&p)[2], int d0, int d1) {
        if (d0 == 0) {
          const _Float16* vm = &L.m[i16 & (NG - 1)][sub * 32 + g4 * 4];
          const uint2 v0 = *reinterpret_cast<const uint2*>(vm), v1 = *reinterpret_cast<const uint2*>(vm + 16);
          const u4 va{v0.x, v0.y, v1.x, v1.y};
          low[0] = mfma_f16(va, p[0], low[0]);
          low[1] = mfma_f16(va, p[1], low[1]);
        }
        const char* vb = (const char*)L.v + (sub * 32 + g4 * 4 + (i16 >> 2)) * kRow<D> + (i16 & 3) * 8;
#pragma unroll
        for (int d = d0; d < d1; ++d) {
          const u4 vt = ds_tr(vb + d * 32, vb + 16 * kRow<D> + d * 32);
          acc[0][d] = mfma_f16(vt, p[0], acc[0][d]);
          acc[1][d] = mfma_f16(vt, p[1], acc[1][d]);
        }
      };

      const int stages = (t1 - t0) * (KT / KEYS);
      // keys of stages 0 and 1, values of stage 0; the thread then holds its
      // share of the keys of stage 2 or of the values of stage 1
      if (kind == 0) {
        store_keys(keys[0]);
        issue(1);
        store_keys(keys[1]);
        issue(2);
      } else if (kind == 1) {
        store_values(values[0]);
        issue(1);
      }
      __syncthreads();
      f4 sc[2][2];
      u4 p[2] = {u4{0, 0, 0, 0}, u4{0, 0, 0, 0}};
      products(keys[0], 0, sc[0][0], sc[1][0]);
      products(keys[0], 16, sc[0][1], sc[1][1]);
      int k0 = 0, k1 = 1, k2 = 2;  // slots of the stage at hand, the next and the one after
      int vp = 0, v0 = 0, v1 = 1;  // the one before (at first: any with finite values), at hand, the next
      for (int n = 0; n < stages; ++n) {
        __syncthreads();
        // a SIMD's two waves stage at different times
        if (kind == 0) {
          store_keys(keys[k2]);
          issue(n + 3);
        }
#pragma unroll 1
        for (int sub = 0; sub < SPS; ++sub) {
          if (sub == SPS - 1 && kind == 1) {
            store_values(values[v1]);
            issue(n + 2);
          }
          const Keys& K = keys[k0];
          const Values& V = values[v0];
          const Keys& Kn = keys[sub + 1 < SPS ? k0 : k1];
          const Values& Vp = values[sub == 0 ? vp : v0];
          const int next = sub + 1 < SPS ? sub + 1 : 0, prev = sub == 0 ? SPS - 1 : sub - 1;
          const int before_sub = n == 0 && sub == 0 ? 0 : prev;
          float sum[2], top[2];
          u4 pn[2];
          pn[0] = weigh(K, V, sub, 0, sc[0][0], sc[0][1], top[0], sum[0]);
          pn[1] = weigh(K, V, sub, 1, sc[1][0], sc[1][1], top[1], sum[1]);
          products(Kn, next * 32, sc[0][0], sc[1][0]);
          products(Kn, next * 32 + 16, sc[0][1], sc[1][1]);
          output(Vp, before_sub, p, 0, DT);
          const int r0 = t0 * KT + n * KEYS + sub * 32;
          const bool mask = always || r0 + 32 > lim_all;
          if (__builtin_amdgcn_ballot_w64(mask || !(top[0] <= kTop && top[1] <= kTop))) {
            // rare: the step's products again (its keys are still there),
            // masked, against a reference raised where it has to be
            f4 s2[2][2];
            products(K, sub * 32, s2[0][0], s2[1][0]);
            products(K, sub * 32 + 16, s2[0][1], s2[1][1]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const float2 lq = s_rows[c][threadIdx.x];  // the first row not seen, the power taken out
              const int lim = __float_as_int(lq.x);
              float mx = -INFINITY;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float kf = K.f[sub * 2 + i], ve = V.e[sub * 2 + i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  s2[c][i][j] = fmaf(s2[c][i][j] * lq.y, kf, ve);
                  if (r0 + i * 16 + g4 * 4 + j >= lim) s2[c][i][j] = -INFINITY;
                  mx = fmaxf(mx, s2[c][i][j]);
                }
              }
              mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
              mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
              if (mx > m[c] + kRaise) {
                const float m_new = mx - kPeak, alpha = __builtin_amdgcn_exp2f(m[c] - m_new);
                m[c] = m_new;
                if (fabsf(mx) > kFar) s_wide = 1;  // it would swallow e
                l[c] *= alpha;
                low[c] *= alpha;
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[c][d] *= alpha;
              }
              float e[8];
              sum[c] = 0.0f;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float vi = V.inv[sub * 2 + i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  e[i * 4 + j] = __builtin_amdgcn_exp2f(s2[c][i][j] - m[c]);
                  sum[c] = fmaf(e[i * 4 + j], vi, sum[c]);
                }
              }
              pn[c] = u4{h2(e[0], e[1]), h2(e[2], e[3]), h2(e[4], e[5]), h2(e[6], e[7])};
            }
          }
          l[0] += sum[0];
          l[1] += sum[1];
          p[0] = pn[0];
          p[1] = pn[1];
        }
        const int ko = k0, vo = n == 0 ? 2 : vp;  // the slots that fall free
        k0 = k1, k1 = k2, k2 = ko;
        vp = v0, v0 = v1, v1 = vo;
      }
      output(values[vp], SPS - 1, p, 0, DT);
    }

    const int any_bad = __syncthreads_or(bad);
    if (threadIdx.x == 0 && s_wide) wide[blockIdx.x] = 1;
    const bool begins = before >= u0, ends = before + tiles <= u1;
    float* out = record<D, QROWS>(rec, w, Hkv, h, begins);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float ls = l[c];
      ls += __shfl_xor(ls, 16, 64);
      ls += __shfl_xor(ls, 32, 64);
      if (any_bad) ls = __builtin_nanf("");
      const int r = wave * 32 + c * 16 + i16;
      const int rr = b * QROWS + min(r, rows - 1);
      const int64_t tok = (int64_t)(x.q0 + rr / G) * Hq + h * G + rr % G;  // among the rows of o
      const float inv = begins && ends ? (ls == 0.0f ? 0.0f : 1.0f / ls) : 1.0f;
      const bool odd = g4 & 1;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        f4 y = acc[c][d];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (y[j] + low[c][d * NG / DT]) * inv;
        // channels 0 4 1 5 and 2 6 3 7 of eight -> 0 .. 3 and 4 .. 7
        const float r0 = __shfl_xor(odd ? y[0] : y[1], 16, 64), r1 = __shfl_xor(odd ? y[2] : y[3], 16, 64);
        const f4 z = odd ? f4{r0, r1, y[1], y[3]} : f4{y[0], y[2], r0, r1};
        if (r >= rows) continue;
        if (begins && ends) {
          const uint2 v = q_f16 ? uint2{h2(z[0], z[1]), h2(z[2], z[3])} : uint2{bf2(z[0], z[1]), bf2(z[2], z[3])};
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + tok * D + d * 16 + g4 * 4) = v;
        } else {
          *reinterpret_cast<f4*>(out + r * kRec<D> + d * 16 + g4 * 4) = z;
        }
      }
      if (g4 == 0 && r < rows) {
        if (begins && ends) {
          if (a.lse) a.lse[tok] = lse_of(m[c], ls);
        } else {
          out[r * kRec<D> + D] = m[c];
          out[r * kRec<D> + D + 1] = ls;
        }
      }
    }
    if (begins && !ends && threadIdx.x == 0)
      cuts[blockIdx.x] = Cut{s, w, line.piece_of(before + tiles - 1), b * QROWS};
    before += tiles;
    u = before;
    if (u < u1 && ++b == nb) {  // on to the next sequence that has blocks
      b = 0;
      do {
        if (++s >= a.S) return;
        x = scalar(seq_of(a, s));
        nb = prompt_blocks(x, G);
      } while (nb == 0);
    }
  }
}

// A cut's pieces' records in order: ROWS query rows from row `block` of the
// sequence on, those that fall to workgroup y of `ys`.  A thread takes four
// channels; the loads of a few records do not wait for one another.
template <int D, int ROWS, int QT>
__device__ inline void merge_cut(const PageAttendArgs& a, const Cut& k, int h, const float* __restrict__ rec, int y0,
                                 int ys) {
  const int Hkv = a.pc.Hkv, G = a.G, Hq = G * Hkv;
  const Seq x = seq_of(a, k.seq);
  const int rows = (int)min((int64_t)ROWS, (int64_t)x.n * G - k.block);
  constexpr int TR = D / 4;  // threads of a row
  const int d = threadIdx.x % TR * 4;
  for (int r = y0 * (256 / TR) + threadIdx.x / TR; r < rows; r += ys * (256 / TR)) {
    float M = kNone, l = 0.0f;
    f4 y = f4{0.f, 0.f, 0.f, 0.f};
    constexpr int N = 6;  // records at a time
    for (int w0 = k.first; w0 <= k.last; w0 += N) {
      f4 v[N];
      float m[N], ls[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int w = min(w0 + i, k.last);
        const float* p = record<D, ROWS>(rec, w, Hkv, h, w == k.first) + r * kRec<D>;
        v[i] = *reinterpret_cast<const f4*>(p + d);
        m[i] = w0 + i <= k.last ? p[D] : kNone;
        ls[i] = w0 + i <= k.last ? p[D + 1] : 0.0f;
      }
      float m_new = M;
#pragma unroll
      for (int i = 0; i < N; ++i) m_new = fmaxf(m_new, m[i]);
      const float old = exp2f(M - m_new);
      l *= old;
      y *= old;
      M = m_new;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float wt = w0 + i <= k.last ? exp2f(m[i] - M) : 0.0f;
        l = fmaf(ls[i], wt, l);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = fmaf(v[i][j], wt, y[j]);
      }
    }
    const int i = (k.block + r) / G, g = (k.block + r) % G;
    const int64_t at = (int64_t)(x.q0 + i) * Hq + h * G + g;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    y *= inv;
    const uint2 z = QT == UC_BF16 ? uint2{bf2(y[0], y[1]), bf2(y[2], y[3])} : uint2{h2(y[0], y[1]), h2(y[2], y[3])};
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + at * D + d) = z;
    if (d == 0 && a.lse) a.lse[at] = lse_of(M, l);
  }
}

// the rows of a block that fall to workgroup y0 of `ys`, from the cache itself
template <int D, int QT>
__device__ inline void attend_block(const PageAttendArgs& a, RowLds<D>& lds, int s, int block, int h, int y0, int ys) {
  const Seq x = seq_of(a, s);
  const int rows = (int)min((int64_t)QROWS, (int64_t)x.n * a.G - block);
  for (int r = block + y0; r < block + rows; r += ys)
    attend_row<D, QT>(a, lds, x, s, x.q0 + r / a.G, h * a.G + r % a.G);
}

// Two workgroups a cut of the token kernel (blocks [0, 2 n_tokens) of the
// grid), sixteen a cut of the prompt kernel (those behind).  Blocks that a
// piece marked as wide has a part in are computed anew, whole ones of the piece
// by its own workgroups.
constexpr int kMergeT = 2, kMergeP = 16;
template <int D, int QT>
__global__ __launch_bounds__(256, 8) void page_merge_kernel(PageAttendArgs a, int n_tokens, const Cut* __restrict__ cuts_t,
                                                         const float* __restrict__ rec_t,
                                                         const Cut* __restrict__ cuts_p,
                                                         const float* __restrict__ rec_p, int Wp,
                                                         const int* __restrict__ units, const int* __restrict__ wide) {
  if ((int)blockIdx.x < n_tokens * kMergeT) {
    const int i = blockIdx.x / kMergeT;
    const Cut k = cuts_t[i];
    if (k.seq >= 0) merge_cut<D, 16, QT>(a, k, i % a.pc.Hkv, rec_t, blockIdx.x % kMergeT, kMergeT);
    return;
  }
  __shared__ RowLds<D> lds;
  const int at = blockIdx.x - n_tokens * kMergeT, i = at / kMergeP, y = at % kMergeP, Hkv = a.pc.Hkv, h = i % Hkv, w = i / Hkv;
  const Cut k = cuts_p[i];
  const int all = wide[i];
  if (k.seq >= 0) {
    int any = 0;
    for (int j = k.first + threadIdx.x; j <= k.last; j += blockDim.x) any |= wide[j * Hkv + h];
    if (__syncthreads_or(any)) attend_block<D, QT>(a, lds, k.seq, k.block, h, y, kMergeP);
    else merge_cut<D, QROWS, QT>(a, k, h, rec_p, y, kMergeP);
  }
  if (!all) return;
  const int U = units[a.S];
  const Line line(U, min(Wp, U));
  const int u0 = line.first(w), u1 = line.first(w + 1);
  for (int s = 0; s < a.S; ++s) {
    if (units[s + 1] <= u0 || units[s] >= u1) continue;
    const Seq x = seq_of(a, s);
    int before = units[s];
    for (int b = 0; b < prompt_blocks(x, a.G) && before < u1; ++b) {
      const int tiles = prompt_tiles(x, a.G, b);
      if (before >= u0 && before + tiles <= u1) attend_block<D, QT>(a, lds, s, b * QROWS, h, y, kMergeP);
      before += tiles;
    }
  }
}

}  // namespace

// Pieces of the line per KV head, each a workgroup's: for single tokens two
// workgroups per CU in one round, for prompts one (of twice the waves).  Where
// the sequences are many, each of a single-token workgroup's waves has a piece:
// then waves neither idle on sequences of fewer tiles than there are waves, nor
// meet at the end of every sequence.  28 heads on 4, us that way and the other:
// 1024 sequences of 128 rows 30 and 73, 512 of 2048 rows 123 and 142, 256 of 64
// rows 10 and 21; but 256 of 512 rows 34 and 32, 128 of 1024 rows 30 and 25, one
// of 65536 rows 66 and 33 (more records to merge).
static int prompt_pieces(const PageCache& pc) { return std::max(1, device_cus() / pc.Hkv); }
static bool solo_waves(const PageCache& pc, int S) { return S >= 2 * std::max(1, 2 * device_cus() / pc.Hkv); }
static int token_pieces(const PageCache& pc, int S) {
  return std::max(1, 2 * device_cus() / pc.Hkv) * (solo_waves(pc, S) ? WAVES : 1);
}

static size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

// cuts and records of both kernels (no records where there is one piece), the
// prompt kernel's sums of units and marks
struct PageWorkspace {
  size_t cuts_p, wide, units, rec_t, rec_p, end;
  PageWorkspace(const PageCache& pc, int S, bool prompts) {
    const size_t nt = (size_t)token_pieces(pc, S) * pc.Hkv, np = (size_t)prompt_pieces(pc) * pc.Hkv;
    cuts_p = align_up(nt * sizeof(Cut));
    wide = cuts_p + (prompts ? align_up(np * sizeof(Cut)) : 0);
    units = wide + (prompts ? align_up(np * sizeof(int)) : 0);
    rec_t = units + (prompts ? align_up(((size_t)S + 1) * sizeof(int)) : 0);
    const size_t row = (pc.D + 4) * sizeof(float);
    rec_p = rec_t + (nt > (size_t)pc.Hkv ? nt * 2 * 16 * row : 0);
    end = rec_p + (prompts && np > (size_t)pc.Hkv ? np * 2 * QROWS * row : 0);
  }
};

size_t page_attend_workspace(const PageCache& pc, int G, int S, int max_q) {
  return PageWorkspace(pc, S, (int64_t)max_q * G > 16 * kFewBlocks).end;
}

template <int D, int NG, int QP>
static void launch_matrix(const PageAttendArgs& a, int max_q, void* ws, hipStream_t st) {
  constexpr int QT = QP == 1 ? UC_BF16 : UC_F16;
  const bool prompts = (int64_t)max_q * a.G > 16 * kFewBlocks;
  const PageWorkspace at(a.pc, a.S, prompts);
  char* p = (char*)ws;
  Cut *cuts_t = (Cut*)p, *cuts_p = (Cut*)(p + at.cuts_p);
  int *units = (int*)(p + at.units), *wide = (int*)(p + at.wide);
  float *rec_t = (float*)(p + at.rec_t), *rec_p = (float*)(p + at.rec_p);
  // The tiles there can be: where they are no more than the pieces, a wave takes
  // each by itself as well (one sequence of 777 rows: 13.3 us, and 14.9 in one
  // workgroup); and no more pieces than there can be work for.
  const int64_t blocks = a.S * std::min<int64_t>(kFewBlocks, ((int64_t)max_q * a.G + 15) / 16);
  const int64_t tiles = std::max<int64_t>(1, (((int64_t)a.ld << a.pc.lgP) + KT - 1) / KT);
  int Wt = token_pieces(a.pc, a.S);
  const bool solo = solo_waves(a.pc, a.S) || (Wt >= WAVES && blocks * tiles <= Wt);
  if (solo) Wt &= ~(WAVES - 1);
  else Wt = (int)std::max<int64_t>(1, std::min<int64_t>(Wt, blocks * (kStart + tiles) / (kStart + WAVES)));
  const int nt = Wt * a.pc.Hkv, Wp = prompt_pieces(a.pc), np = prompts ? Wp * a.pc.Hkv : 0;
  const dim3 grid((solo ? nt / WAVES : nt) + (prompts ? 1 : 0));
  if (solo)
    hipLaunchKernelGGL((page_tokens_kernel<D, NG, QP, true>), grid, dim3(256), 0, st, a, Wt, rec_t, cuts_t, units);
  else
    hipLaunchKernelGGL((page_tokens_kernel<D, NG, QP, false>), grid, dim3(256), 0, st, a, Wt, rec_t, cuts_t, units);
  if (prompts)
    hipLaunchKernelGGL((page_prompt_kernel<D, NG>), dim3(np), dim3(64 * PWAVES), 0, st, a, Wp, QP == 2, units, rec_p,
                       cuts_p, wide);
  const int merge_t = Wt > 1 ? nt : 0;
  if (merge_t + np)
    hipLaunchKernelGGL((page_merge_kernel<D, QT>), dim3(merge_t * kMergeT + np * kMergeP), dim3(256), 0, st, a,
                       merge_t, cuts_t, rec_t, cuts_p, rec_p, Wp, units, wide);
}

static void launch_page_valu(const PageAttendArgs& a, int q_dt, hipStream_t st) {
  const dim3 grid(std::min<uint32_t>((uint32_t)a.T * a.pc.Hkv * a.G, 1 << 20));
#define UC_VALU(DIM, TYPE) \
  hipLaunchKernelGGL((page_attend_valu_kernel<DIM, TYPE>), grid, dim3(256), 0, st, a)
  if (a.pc.D == 128) {
    if (q_dt == UC_BF16) UC_VALU(128, UC_BF16);
    else if (q_dt == UC_F16) UC_VALU(128, UC_F16);
    else UC_VALU(128, UC_F32);
  } else {
    if (q_dt == UC_BF16) UC_VALU(64, UC_BF16);
    else if (q_dt == UC_F16) UC_VALU(64, UC_F16);
    else UC_VALU(64, UC_F32);
  }
#undef UC_VALU
}

hipError_t launch_page_attend(const PageAttendArgs& a, int q_dt, int max_q, bool valu, void* ws, hipStream_t st) {
#define UC_MATRIX(DIM, NGR) \
  q_dt == UC_BF16 ? launch_matrix<DIM, NGR, 1>(a, max_q, ws, st) : launch_matrix<DIM, NGR, 2>(a, max_q, ws, st)
  if (valu) {
    launch_page_valu(a, q_dt, st);
  } else if (a.pc.D == 128) {
    if (a.pc.ng == 4) UC_MATRIX(128, 4);
    else if (a.pc.ng == 2) UC_MATRIX(128, 2);
    else UC_MATRIX(128, 1);
  } else {
    if (a.pc.ng == 2) UC_MATRIX(64, 2);
    else UC_MATRIX(64, 1);
  }
#undef UC_MATRIX
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess)
    set_last_kernel(valu ? "page_valu" : (int64_t)max_q * a.G > 16 * kFewBlocks ? "page_prompt" : "page_tokens");
  return e;
}

}  // namespace uc
