// page_attend.hip -- attention over a paged cache held in 4 bits: single
// tokens (at most 16 query rows of a KV head), prompts (any number), and the
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
// equal pieces.  A sequence that lies within one piece is written by its
// workgroup; one cut into several leaves a record (m, l, o) per piece, merged
// by a second kernel in the order of the pieces.
#include <algorithm>
#include <type_traits>

#include "page_common.h"

namespace uc {
namespace {

using namespace mf;

constexpr int WAVES = 4;
constexpr int KT = 64;         // keys per tile
constexpr float kLazy = 8.0f;  // base-2 headroom before the reference maximum is raised
constexpr float kNone = -3.0e38f;  // the reference maximum before any visible key

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
// One workgroup per (token, query head); keys in chunks of 256, one per
// thread for the logits, one channel per thread for the values.
template <int D, int QT>
__global__ __launch_bounds__(256) void page_attend_valu_kernel(PageAttendArgs a) {
  __shared__ float sq[D], sp[256], red[WAVES], so[256 / D][D];
  __shared__ int64_t srow[256];
  const int Hq = a.pc.Hkv * a.G, hq = blockIdx.x % Hq, t = blockIdx.x / Hq, h = hq / a.G;
  // the sequence whose tokens include t
  __shared__ int s_seq;
  if (threadIdx.x == 0) s_seq = INT32_MAX;
  __syncthreads();
  for (int s = threadIdx.x; s < a.S; s += blockDim.x) {
    const Seq x = seq_of(a, s);
    if (t >= x.q0 && t < x.q0 + x.n) atomicMin(&s_seq, s);
  }
  __syncthreads();
  if (s_seq == INT32_MAX) return;  // a row of no sequence stays as it was
  const Seq x = seq_of(a, s_seq);
  const int lim = max(0, min(x.len, (int)((int64_t)x.len - x.n + (t - x.q0) + 1)));
  const int32_t* trow = a.table + (int64_t)s_seq * a.ld;
  for (int d = threadIdx.x; d < D; d += blockDim.x) sq[d] = q_val<QT>(a.q, (int64_t)t * a.q_ld + hq * D + d);
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
          sum = fmaf(sq[c0 + e], fmaf((float)((cw >> (4 * e)) & 15u), word_step(sw), word_min(sw)), sum);
      }
      v = sum * a.scale_log2;
    }
    srow[threadIdx.x] = row;
    float mx = wave_max(v);
    if (lane == 0) red[wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float m_new = fmaxf(m, mx), alpha = exp2f(m - m_new);
    m = m_new;
    const float p = exp2f(v - m);
    sp[threadIdx.x] = p;
    l = l * alpha + p;  // this thread's keys
    acc *= alpha;
    __syncthreads();
    const int n = min(256, lim - j0);
    for (int i = part; i < n; i += 256 / D) {
      if (srow[i] < 0) continue;
      const uint8_t b = a.pc.codes_v[srow[i] * (D / 2) + dim / 2];
      const uint32_t sw = a.pc.scale_v[srow[i] * ng + dim / gsz];
      acc = fmaf(sp[i], fmaf((float)((b >> (4 * (dim & 1))) & 15), word_step(sw), word_min(sw)), acc);
    }
  }
  __syncthreads();
  so[part][dim] = acc;
  l = wave_sum(l);
  if (lane == 0) red[wave] = l;
  const int any_bad = __syncthreads_or(bad);
  l = (red[0] + red[1]) + (red[2] + red[3]);
  if (any_bad) l = __builtin_nanf("");
  if (threadIdx.x < D) {
    float s = 0.0f;
    for (int i = 0; i < 256 / D; ++i) s += so[i][threadIdx.x];
    put<QT>(a.o, ((int64_t)t * Hq + hq) * D + threadIdx.x, l == 0.0f ? 0.0f : s / l);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)t * Hq + hq] = lse_of(m, l);
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

// units of a sequence in the single-token kernel: its tiles, at least one so
// that a row that sees nothing is written too, behind kStart units that stand
// for what a sequence costs beside them; none where the prompt kernel takes it
constexpr int kStart = 8;
__device__ inline int tiles_of(int rows) { return rows <= KT ? 1 : (int)(((uint32_t)rows + KT - 1) / KT); }
__device__ inline int token_units(const Seq& x, int G) {
  return x.n == 0 || (int64_t)x.n * G > 16 ? 0 : kStart + tiles_of(x.len);
}

// a sequence cut into pieces first .. last; rows of the call it stands for
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

// D, NG: head dim and groups of a row; QP: bf16 parts of a query element.
//
// A wave's tile is four blocks of 16 keys, each within one page (pages are 16
// rows or more), so a block's codes are one contiguous piece of the cache
// behind a scalar address.  Block b's product rows are its keys, and lane
// group g4 holds those of keys 16 b + 4 g4 + j; the transposing reads of the
// values take their rows in that order.
template <int D, int NG, int QP>
__global__ __launch_bounds__(256, 2) void page_tokens_kernel(PageAttendArgs a, int W_all, float* __restrict__ rec,
                                                             Cut* __restrict__ cuts) {
  constexpr int KS = D / 32;  // matrix steps over the channels, words of a lane's codes of a row
  constexpr int DT = D / 16;  // tiles of 16 output channels
  constexpr int GS = KS / NG;
  constexpr int QT = QP == 1 ? UC_BF16 : UC_F16;
  using Lds = WaveLds<D, NG>;
  constexpr size_t kTiles = sizeof(Lds) * WAVES, kMerge = sizeof(float) * WAVES * 16 * (D + 2);
  __shared__ __attribute__((aligned(16))) char lds[kTiles > kMerge ? kTiles : kMerge];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int Hkv = a.pc.Hkv, h = blockIdx.x % Hkv, w = blockIdx.x / Hkv;
  const int G = a.G, Hq = G * Hkv, lgP = a.pc.lgP, P1 = (1 << lgP) - 1;
  const Magic magic;
  if (threadIdx.x == 0) cuts[blockIdx.x] = Cut{-1, 0, 0, 0};

  // this piece of the line; lane i counts sequences i c .. i c + c - 1
  const int c = (a.S + 63) / 64;
  Seq x{0, 0, 0};
  int mine = 0;
  for (int s = lane * c; s < min(a.S, (lane + 1) * c); ++s) {
    x = seq_of(a, s);
    mine += token_units(x, G);
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(upto, o, 64);
    if (lane >= o) upto += y;
  }
  const int U = __builtin_amdgcn_readlane(upto, 63);
  if (U == 0) return;
  // a sequence and a tile per wave at least
  const Line line(U, max(1, min(W_all, U / (kStart + WAVES))));
  if (w >= line.W) return;
  const int u0 = line.first(w), u1 = line.first(w + 1);
  const int bucket = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > u0));
  int s = bucket * c, before = __builtin_amdgcn_readlane(upto - mine, bucket);  // units before sequence s
  if (c == 1) {
    x = Seq{__builtin_amdgcn_readlane(x.q0, bucket), __builtin_amdgcn_readlane(x.n, bucket),
            __builtin_amdgcn_readlane(x.len, bucket)};
  } else {
    x = seq_of(a, s);
  }
  Lds& L = *reinterpret_cast<Lds*>(lds + wave * sizeof(Lds));

  // The sequence at hand: tiles [t0, t1) of it lie in this piece.
  int units = 0, t0 = 0, t1 = 0, page = 0, page_next = 0, last16 = 0;
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
  // on to the first sequence from s on with tiles in [u, u1); false if there
  // is none.  Its pages and queries are asked for.
  auto open = [&](int u) {
    for (;;) {
      units = token_units(x, G);
      if (before + units > u) break;
      before += units;
      if (before >= u1 || s + 1 >= a.S) return false;
      x = seq_of(a, ++s);
    }
    if (before + kStart >= u1) return false;
    t0 = max(0, u - before - kStart);
    t1 = min(units, u1 - before) - kStart;
    trow = a.table + (int64_t)s * a.ld;
    last16 = (x.len - 1) & ~15;  // first row of the last 16
    page = page_for(t0 + wave);
    page_next = page_for(t0 + wave + WAVES);
    const int r = min(i16, x.n * G - 1);
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(x.q0 + r / G) * a.q_ld +
                        (int64_t)(h * G + r % G) * D + g4 * 8;
#pragma unroll
    for (int t = 0; t < KS; ++t) raw[t] = *reinterpret_cast<const u4*>(q + t * 32);
    return true;
  };
  // its first tile's loads
  auto first = [&]() {
    bad = false;
    if (x.len > 0 && t0 + wave < t1) {
      issue_values(t0 + wave, page);
      issue_keys(t0 + wave, page);
    }
  };
  if (!open(u0)) return;
  first();

  for (;;) {
    const int nq = x.n * G;
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
    const int lim = max(0, min(x.len, (int)((int64_t)x.len - x.n + min(i16, nq - 1) / G + 1)));
    const int lim_all = max(0, (int)((int64_t)x.len - x.n + 1));

    float m = kNone, l = 0.0f, low[NG];
    f4 acc[DT];
#pragma unroll
    for (int g = 0; g < NG; ++g) low[g] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f4{0.f, 0.f, 0.f, 0.f};

    if (x.len > 0) {
      int t = t0 + wave;
      for (; t < t1; t += WAVES) {
        const int tn = t + WAVES;
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
            L.v[1][g][lane] = fmaf(-128.0f, word_step(xv), word_min(xv));
          }
        }
        __builtin_amdgcn_wave_barrier();
        // the next tile's loads, as registers become free; its page was read a
        // tile ago
        const int page_now = page_next;
        if (more) {
          issue_values(tn, page_now);
          page_next = page_for(tn + WAVES);
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
          l *= alpha;
#pragma unroll
          for (int g = 0; g < NG; ++g) low[g] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[d] *= alpha;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], a.scale_log2, -m));
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

    // the next sequence's loads are under way while this one's waves merge
    const Seq now = x;
    const int s_now = s, from = before + kStart, to = before + units;  // its tiles' units
    bool more = to < u1 && s + 1 < a.S;
    const bool any = bad;
    if (more) {
      before = to;
      x = seq_of(a, ++s);
      more = open(to);
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      low[g] += __shfl_xor(low[g], 16, 64);
      low[g] += __shfl_xor(low[g], 32, 64);
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
    const bool begins = from >= u0, ends = to <= u1;
    float* out = record<D, 16>(rec, w, Hkv, h, begins);
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
        const int64_t at = (int64_t)(now.q0 + r / G) * Hq + h * G + r % G;
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
    if (begins && !ends && threadIdx.x == 0) cuts[blockIdx.x] = Cut{s_now, w, line.piece_of(to - 1), 0};
    if (!more) break;
    __syncthreads();  // LDS is written again
  }
}

// ---------------------------------------------------------------- prompts
// Blocks of 32 query rows a wave, each over the tiles that its last row sees;
// the line is made of all blocks' tiles.  A workgroup's waves share the tile
// in LDS, where the 4-bit rows, read and unpacked once for all of them, stand
// as fp16: with the power of two 2^e of the key's largest step taken out,
// c * (s 2^-e) has 8 significant bits and is exact, and so is the minimum.
// The powers return where they cost nothing: the keys' in the factor that
// turns a product into a logit, the values' in the exponent,
//   w_j = 2^(logit_j + e_j - m),  o ~ sum_j w_j (v_j 2^-e_j),  l = sum_j w_j 2^-e_j,
// with the reference m kept over logit + e, so that w_j, rounded to fp16 (11
// bits), is measured by what key j contributes whatever the values' sizes.  l
// is summed in binary32 before that rounding.  Steps of values from 2^-60 to
// 2^88 keep all their bits.  The minima go through matrix instructions of
// their own, q . k += sum_g m_g sum(q_g) with sum(q_g) in three fp16 parts.
// Queries enter as fp16 too, exactly (a row far from 1 by a power of two).
//
// Per 64 keys x 32 rows a wave issues 64 matrix instructions of 16 cycles for
// the two products and 12 for the minima, and some 400 vector instructions of
// 4 cycles; both bound it.
template <int WV>
constexpr int kQRows = 32 * WV;

// blocks of a sequence in the prompt kernel
template <int WV>
__device__ inline int prompt_blocks(const Seq& x, int G) {
  const int64_t rows = (int64_t)x.n * G;
  return rows <= 16 ? 0 : (int)((rows + kQRows<WV> - 1) / kQRows<WV>);
}
// tiles of its block b, at least one
template <int WV>
__device__ inline int prompt_tiles(const Seq& x, int G, int b) {
  const int64_t last = min((int64_t)x.n - 1, ((int64_t)b * kQRows<WV> + kQRows<WV> - 1) / G);
  const int64_t sees = max((int64_t)0, min((int64_t)x.len, (int64_t)x.len - x.n + last + 1));
  return tiles_of((int)sees);
}

// before[s]: units of the sequences ahead of s, before[S]: all of them
template <int WV>
__global__ __launch_bounds__(1024) void page_plan_kernel(PageAttendArgs a, int* __restrict__ before) {
  __shared__ int part[16];
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int s0 = 0; s0 < a.S; s0 += 1024) {
    const int s = s0 + threadIdx.x;
    Seq x{0, 0, 0};
    if (s < a.S) x = seq_of(a, s);
    const int blocks = prompt_blocks<WV>(x, a.G);
    int mine = 0;
    // the wave counts one sequence after the other, a block per lane
    for (uint64_t todo = __builtin_amdgcn_ballot_w64(blocks > 0); todo; todo &= todo - 1) {
      const int from = __ffsll((unsigned long long)todo) - 1;
      const Seq y{0, __shfl(x.n, from, 64), __shfl(x.len, from, 64)};
      const int nb = __shfl(blocks, from, 64);
      int sum = 0;
      for (int b = lane; b < nb; b += 64) sum += prompt_tiles<WV>(y, a.G, b);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (lane == from) mine = sum;
    }
    int total;
    const int upto = block_scan(mine, part, total);
    if (s < a.S) before[s] = base + upto - mine;
    base += total;
  }
  if (threadIdx.x == 0) before[a.S] = base;
}

template <int D>
constexpr int kRow = 2 * D + 32;  // bytes of a staged row: 8 consecutive rows start in different 8-bank groups

typedef _Float16 half2 __attribute__((ext_vector_type(2)));

template <int D>
struct PromptTile {
  uint8_t k[KT * kRow<D>];  // c * s 2^-e in fp16; of eight channels in the order 0 4 1 5 2 6 3 7
  uint8_t v[KT * kRow<D>];
  _Float16 km[KT][8];      // minima (2^-e) of a key, zeros behind them
  _Float16 vm[4][KT + 8];  // minima (2^-e) of a value group, by key
  float kf[KT];            // logit of a product: scale * 2^e
  float ve[KT], vi[KT];    // e and 2^-e of the values
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

// biased exponent of the power of two taken out of a row: its largest step
// comes below 2 and its minima below 2^14
template <int NG>
__device__ inline int row_exponent(const uint32_t (&w)[NG], int least, int most) {
  int e = 0;
#pragma unroll
  for (int n = 0; n < NG; ++n)
    e = max(e, max((int)(w[n] >> 7 & 0xFF), (int)(w[n] >> 23 & 0xFF) - 12));
  return e == 0 ? 127 : min(max(e, least), most);  // a row of zeros: any
}

template <int D, int NG, int WV>
__global__ __launch_bounds__(64 * WV, 2) void page_prompt_kernel(PageAttendArgs a, int W_all, bool q_f16,
                                                                 const int* __restrict__ units,
                                                                 float* __restrict__ rec, Cut* __restrict__ cuts) {
  constexpr int KS = D / 32, DT = D / 16, QROWS = kQRows<WV>, THREADS = 64 * WV;
  __shared__ __attribute__((aligned(16))) PromptTile<D> tiles_lds[2];
  __shared__ int s_part[16], s_block, s_before;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i16 = lane & 15, g4 = lane >> 4;
  const int Hkv = a.pc.Hkv, h = blockIdx.x % Hkv, w = blockIdx.x / Hkv;
  const int G = a.G, Hq = G * Hkv, lgP = a.pc.lgP;
  const Unpack unpack;
  if (threadIdx.x == 0) cuts[blockIdx.x] = Cut{-1, 0, 0, 0};
  const int U = units[a.S];
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
  Seq x = seq_of(a, s);
  int nb = prompt_blocks<WV>(x, G);
  if (threadIdx.x == 0) s_block = -1;
  {
    int base = units[s];
    for (int b0 = 0; b0 < nb; b0 += THREADS) {
      const int b = b0 + threadIdx.x;
      const int mine = b < nb ? prompt_tiles<WV>(x, G, b) : 0;
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
  for (int i = threadIdx.x; i < KT * 8; i += THREADS)
    (&tiles_lds[0].km[0][0])[i] = (&tiles_lds[1].km[0][0])[i] = (_Float16)0.0f;
  __syncthreads();
  int b = s_block;
  if (b < 0) return;  // starts that overlap so often that the sums passed their type
  int before = s_before;

  // A thread's share of a tile: 16 bytes of codes of a row of keys or values.
  constexpr int CH = D / 32, TASKS = 2 * KT * CH, PER = TASKS > THREADS ? TASKS / THREADS : 1;
  static_assert(PER <= 2, "one task of each kind at most");
  u4 codes[PER];
  uint32_t words[PER][NG];

  for (int u = u0; u < u1;) {
    const int tiles = prompt_tiles<WV>(x, G, b);
    const int t0 = u - before, t1 = min(tiles, u1 - before);
    const int rows = (int)min((int64_t)QROWS, (int64_t)x.n * G - (int64_t)b * QROWS);
    const int32_t* trow = a.table + (int64_t)s * a.ld;
    bool bad = false;

    auto issue = [&](int t) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int task = threadIdx.x + i * THREADS, kind = task / (KT * CH), key = task % (KT * CH) / CH;
        if (kind > 1) continue;
        const int r = min(t * KT + key, x.len - 1), page = page_of(trow, r, lgP, a.pc.n_pages);
        if (page < 0) bad = true;
        const int64_t row = page_row(max(page, 0), Hkv, h, lgP, r);
        codes[i] = *reinterpret_cast<const u4*>((kind ? a.pc.codes_v : a.pc.codes_k) + row * (D / 2) + task % CH * 16);
        load_words<NG>((kind ? a.pc.scale_v : a.pc.scale_k) + row * NG, words[i]);
      }
    };
    // the tile to LDS; rows past the sequence repeat its last one
    auto stage = [&](PromptTile<D>& L) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int task = threadIdx.x + i * THREADS, kind = task / (KT * CH), key = task % (KT * CH) / CH, ch = task % CH;
        if (kind > 1) continue;
        const int E = kind ? row_exponent<NG>(words[i], 127 - 48, 127 + 76) : row_exponent<NG>(words[i], 24, 230);
        const float out = __uint_as_float((uint32_t)(254 - E) << 23), in = __uint_as_float((uint32_t)E << 23);
        half2 st[NG], off[NG];
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const float f = word_step(words[i][n]) * out;
          st[n] = __builtin_bit_cast(half2, h2(f, f));
          off[n] = __builtin_bit_cast(half2, h2(-1024.0f * f, -1024.0f * f));
        }
        if (kind == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // the word holds channels 32 step + 8 g ..
            const int step = KS == 4 ? j : j % KS, g = (ch * 4 + j) / KS, n = step * NG / KS;
            *reinterpret_cast<u4*>(L.k + key * kRow<D> + (step * 4 + g) * 16) = unpack.times(codes[i][j], st[n], off[n]);
          }
          if (ch == 0) {
#pragma unroll
            for (int n = 0; n < NG; ++n) L.km[key][n] = (_Float16)(word_min(words[i][n]) * out);
            L.kf[key] = in * a.scale_log2;
          }
        } else {
          half2 sv = st[0], ov = off[0];
#pragma unroll
          for (int n = 1; n < NG; ++n)
            if (ch * NG / CH == n) sv = st[n], ov = off[n];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<u4*>(L.v + key * kRow<D> + (ch * 4 + j) * 16) = unpack.times(codes[i][j], sv, ov);
          if (ch == 0) {
#pragma unroll
            for (int n = 0; n < NG; ++n) L.vm[n][key] = (_Float16)(word_min(words[i][n]) * out);
            L.ve[key] = (float)(E - 127);
            L.vi[key] = out;
          }
        }
      }
    };
    if (x.len > 0) issue(t0);

    u4 qb[2][KS], sqb[2];
    int lim[2];
    float qf[2];      // power of two taken out of the lane's query row
    int64_t tok[2];   // the lane's query rows, among the rows of o
    bool scaled = false;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = wave * 32 + c * 16 + i16;
      const int rr = b * QROWS + min(r, rows - 1), i = rr / G, gq = rr % G;
      lim[c] = (int)max((int64_t)0, min((int64_t)x.len, (int64_t)x.len - x.n + i + 1));
      tok[c] = (int64_t)(x.q0 + i) * Hq + h * G + gq;
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
      const int E = (int)(__float_as_uint(most) >> 23);  // 2^(E - 127) <= most
      const bool far = most > 0.0f && (E < 127 - 4 || E > 127 + 14);
      const float out = far ? __uint_as_float((uint32_t)(254 - min(max(E, 1), 253)) << 23) : 1.0f;
      qf[c] = far ? __uint_as_float((uint32_t)min(max(E, 1), 253) << 23) : 1.0f;
      scaled |= far;
      float sq[NG];
#pragma unroll
      for (int n = 0; n < NG; ++n) sq[n] = 0.0f;
#pragma unroll
      for (int t = 0; t < KS; ++t) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[t][e] *= out;
          sq[t * NG / KS] += f[t][e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) qb[c][t][e] = h2(f[t][e], f[t][e + 4]);
      }
      // sums in three fp16 parts: part g4 in this lane's slots
      uint32_t bits[4] = {0, 0, 0, 0};
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        float y = sq[n];
        y += __shfl_xor(y, 16, 64);
        y += __shfl_xor(y, 32, 64);
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (p < g4) y -= f16_to_f32(f32_to_f16_bits(y));
        const uint32_t v = g4 < 3 ? f32_to_f16_bits(y) : 0;
        bits[n >> 1] |= v << (16 * (n & 1));
      }
      sqb[c] = u4{bits[0], bits[1], bits[2], bits[3]};
    }
    scaled = __builtin_amdgcn_ballot_w64(scaled) != 0;
    const int lim_all = (int)max((int64_t)0, (int64_t)x.len - x.n + (int64_t)b * QROWS / G + 1);

    float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};
    f4 acc[2][DT], low[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      low[c] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[c][d] = f4{0.f, 0.f, 0.f, 0.f};
    }

    if (x.len > 0) {
      stage(tiles_lds[0]);
      if (t0 + 1 < t1) issue(t0 + 1);
      for (int t = t0; t < t1; ++t) {
        PromptTile<D>& L = tiles_lds[(t - t0) & 1];
        __syncthreads();  // this tile is whole, and the other one is no longer read
        if (t + 1 < t1) stage(tiles_lds[(t - t0 + 1) & 1]);
        if (t + 2 < t1) issue(t + 2);

        // products with keys 16 k + 4 g4 + j
        f4 sc[2][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const u4 km = *reinterpret_cast<const u4*>(&L.km[k * 16 + i16][0]);
          sc[0][k] = mfma_f16(km, sqb[0], f4{0.f, 0.f, 0.f, 0.f});
          sc[1][k] = mfma_f16(km, sqb[1], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int st = 0; st < KS; ++st) {
            const u4 ka = *reinterpret_cast<const u4*>(L.k + (k * 16 + i16) * kRow<D> + (st * 4 + g4) * 16);
            sc[0][k] = mfma_f16(ka, qb[0][st], sc[0][k]);
            sc[1][k] = mfma_f16(ka, qb[1][st], sc[1][k]);
          }
        }
        if (scaled) {
          asm volatile("");
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) sc[c][k] *= qf[c];
        }
        // logits and the values' exponents
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f4 kf = *reinterpret_cast<const f4*>(&L.kf[k * 16 + g4 * 4]);
          const f4 ve = *reinterpret_cast<const f4*>(&L.ve[k * 16 + g4 * 4]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sc[0][k][j] = fmaf(sc[0][k][j], kf[j], ve[j]);
            sc[1][k][j] = fmaf(sc[1][k][j], kf[j], ve[j]);
          }
        }
        const int r0 = t * KT;
        if (r0 + KT > lim_all) {
          asm volatile("");
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (r0 + k * 16 + g4 * 4 + j >= lim[c]) sc[c][k][j] = -INFINITY;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float mx = -INFINITY;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[c][k][j]);
          if (__builtin_amdgcn_ballot_w64(mx > m[c] + kLazy)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m[c], mx), alpha = __builtin_amdgcn_exp2f(m[c] - m_new);
            m[c] = m_new;
            l[c] *= alpha;
            low[c] *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[c][d] *= alpha;
          }
        }
        u4 p[2][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f4 vi = *reinterpret_cast<const f4*>(&L.vi[k * 16 + g4 * 4]);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              e[j] = __builtin_amdgcn_exp2f(sc[c][k][j] - m[c]);
              l[c] = fmaf(e[j], vi[j], l[c]);
            }
            p[c][k >> 1][2 * (k & 1)] = h2(e[0], e[1]);
            p[c][k >> 1][2 * (k & 1) + 1] = h2(e[2], e[3]);
          }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const _Float16* vm = &L.vm[i16 & (NG - 1)][half * 32 + g4 * 4];
          const uint2 v0 = *reinterpret_cast<const uint2*>(vm), v1 = *reinterpret_cast<const uint2*>(vm + 16);
          const u4 va{v0.x, v0.y, v1.x, v1.y};
          low[0] = mfma_f16(va, p[0][half], low[0]);
          low[1] = mfma_f16(va, p[1][half], low[1]);
          const char* vb = (const char*)L.v + (half * 32 + g4 * 4 + (i16 >> 2)) * kRow<D> + (i16 & 3) * 8;
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const u4 vt = ds_tr(vb + d * 32, vb + 16 * kRow<D> + d * 32);
            acc[0][d] = mfma_f16(vt, p[0][half], acc[0][d]);
            acc[1][d] = mfma_f16(vt, p[1][half], acc[1][d]);
          }
        }
      }
    }

    const int any_bad = __syncthreads_or(bad);
    const bool begins = before >= u0, ends = before + tiles <= u1;
    float* out = record<D, QROWS>(rec, w, Hkv, h, begins);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float ls = l[c];
      ls += __shfl_xor(ls, 16, 64);
      ls += __shfl_xor(ls, 32, 64);
      if (any_bad) ls = __builtin_nanf("");
      const int r = wave * 32 + c * 16 + i16;
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
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + tok[c] * D + d * 16 + g4 * 4) = v;
        } else {
          *reinterpret_cast<f4*>(out + r * kRec<D> + d * 16 + g4 * 4) = z;
        }
      }
      if (g4 == 0 && r < rows) {
        if (begins && ends) {
          if (a.lse) a.lse[tok[c]] = lse_of(m[c], ls);
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
        x = seq_of(a, s);
        nb = prompt_blocks<WV>(x, G);
      } while (nb == 0);
    }
  }
}

// One workgroup per cut and group of its rows: its pieces' records in order,
// ROWS query rows from row `block` of the sequence on.  A thread takes four
// channels; a row's references and sums come first, so that the records' loads
// do not wait for one another.
template <int D, int ROWS, int QT>
__global__ __launch_bounds__(256) void page_merge_kernel(PageAttendArgs a, const float* __restrict__ rec,
                                                         const Cut* __restrict__ cuts) {
  const Cut k = cuts[blockIdx.x];
  if (k.seq < 0) return;
  const int Hkv = a.pc.Hkv, h = blockIdx.x % Hkv, G = a.G, Hq = G * Hkv;
  const Seq x = seq_of(a, k.seq);
  const int rows = (int)min((int64_t)ROWS, (int64_t)x.n * G - k.block);
  constexpr int TR = D / 4;  // threads of a row
  const int d = threadIdx.x % TR * 4;
  for (int r = blockIdx.y * (256 / TR) + threadIdx.x / TR; r < rows; r += gridDim.y * (256 / TR)) {
    float M = kNone, l = 0.0f;
    f4 y = f4{0.f, 0.f, 0.f, 0.f};
    constexpr int N = 8;  // records at a time
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

}  // namespace

// pieces of the line per KV head: two workgroups per CU in one round
static int pieces(const PageCache& pc) { return std::max(1, 2 * device_cus() / pc.Hkv); }

static size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

// cuts, the prompt kernel's sums of units, records (none where there is one
// piece); the two kernels of a call use it one after the other
static size_t records_at(const PageCache& pc, int S) {
  return align_up((size_t)pieces(pc) * pc.Hkv * sizeof(Cut)) + align_up(((size_t)S + 1) * sizeof(int));
}

// eight waves a workgroup where blocks of 256 rows are well filled
static bool wide_prompt(int max_q, int G) { return (int64_t)max_q * G >= 512; }

size_t page_attend_workspace(const PageCache& pc, int G, int S, int max_q) {
  const size_t W = pieces(pc);
  if (W == 1) return records_at(pc, S);
  // (prompts: half the workgroups where they have twice the rows)
  const size_t rows = (int64_t)max_q * G <= 16 ? 16 : kQRows<4>;
  return records_at(pc, S) + W * pc.Hkv * 2 * rows * (pc.D + 4) * sizeof(float);
}

template <int D, int NG, int QP>
static void launch_matrix(const PageAttendArgs& a, int max_q, void* ws, hipStream_t st) {
  constexpr int QT = QP == 1 ? UC_BF16 : UC_F16;
  const int W = pieces(a.pc);
  Cut* cuts = (Cut*)ws;
  int* units = (int*)((char*)ws + align_up((size_t)W * a.pc.Hkv * sizeof(Cut)));
  float* rec = (float*)((char*)ws + records_at(a.pc, a.S));
  const int64_t most = a.S * std::max<int64_t>(1, (((int64_t)a.ld << a.pc.lgP) + KT - 1) / KT);  // tiles there can be
  const int Wt = (int)std::max<int64_t>(1, std::min<int64_t>(W, (most + (int64_t)kStart * a.S) / (kStart + WAVES))), n = Wt * a.pc.Hkv;
  hipLaunchKernelGGL((page_tokens_kernel<D, NG, QP>), dim3(n), dim3(256), 0, st, a, Wt, rec, cuts);
  if (Wt > 1) hipLaunchKernelGGL((page_merge_kernel<D, 16, QT>), dim3(n, 2), dim3(256), 0, st, a, rec, cuts);
  if ((int64_t)max_q * a.G <= 16) return;
  auto prompts = [&](auto waves) {
    constexpr int WV = decltype(waves)::value;
    const int Wp = W * 4 / WV > 1 ? W * 4 / WV : 1, np = Wp * a.pc.Hkv;  // workgroups of WV waves: two waves per SIMD
    hipLaunchKernelGGL(page_plan_kernel<WV>, dim3(1), dim3(1024), 0, st, a, units);
    hipLaunchKernelGGL((page_prompt_kernel<D, NG, WV>), dim3(np), dim3(64 * WV), 0, st, a, Wp, QP == 2, units, rec, cuts);
    if (Wp > 1)
      hipLaunchKernelGGL((page_merge_kernel<D, kQRows<WV>, QT>), dim3(np, 16), dim3(256), 0, st, a, rec, cuts);
  };
  if (wide_prompt(max_q, a.G)) prompts(std::integral_constant<int, 8>{});
  else prompts(std::integral_constant<int, 4>{});
}

hipError_t launch_page_valu(const PageAttendArgs& a, int q_dt, hipStream_t st) {
  const dim3 grid((uint32_t)((int64_t)a.T * a.pc.Hkv * a.G));
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
  return hipGetLastError();
}

hipError_t launch_page_attend(const PageAttendArgs& a, int q_dt, int max_q, bool valu, void* ws, hipStream_t st) {
  if (valu) {
    set_last_kernel("page_valu");
    return launch_page_valu(a, q_dt, st);
  }
  set_last_kernel((int64_t)max_q * a.G > 16 ? "page_prompt" : "page_tokens");
#define UC_MATRIX(DIM, NGR) \
  q_dt == UC_BF16 ? launch_matrix<DIM, NGR, 1>(a, max_q, ws, st) : launch_matrix<DIM, NGR, 2>(a, max_q, ws, st)
  if (a.pc.D == 128) {
    if (a.pc.ng == 4) UC_MATRIX(128, 4);
    else if (a.pc.ng == 2) UC_MATRIX(128, 2);
    else UC_MATRIX(128, 1);
  } else {
    if (a.pc.ng == 2) UC_MATRIX(64, 2);
    else UC_MATRIX(64, 1);
  }
#undef UC_MATRIX
  return hipGetLastError();
}

}  // namespace uc
