// beam.hip -- one step of a beam search: the W best of a request's W * V
// continuations, and the reordering of its beams' tables and histories.
//
// Selection.  total = score + logit - log sum exp(logits of the beam).  Within
// a beam the totals are ordered as the logits, so one pass over the logits
// yields both the normaliser and the only W candidates that can be chosen;
// totals are formed for those alone, in 64 bits.  The pass should be bound by
// the bytes of the logits; rows are split where there are few.  A wave gathers
// the elements that pass a floor, which W elements are known to reach, and
// raises the floor when its list is full; so an element costs a multiply-add,
// an exponential, an addition and its share of a comparison.  384 rows of
// 131071 bf16, of which 308 are live (81 MB): 29 us, 2.8 TB/s.  (W best kept in
// order in the wave's lanes instead: 49 us.)  The choice among the candidates
// takes 8 us, most of it W dependent steps over a wave.  A whole selection of
// 384 live rows: 36 us, 44 where a mask leaves one logit in a thousand, 705 where
// rows rise all along.
//
// The first floor stands once each of the four waves has W / 4 vectors.  Shorter
// rows (below some 1550 elements of 16 bits, half of that in binary32) are
// gathered whole and ranked by comparing all pairs, which costs more than a long
// row: 384 rows of 300, 1000 and 1500 bf16 take 24, 83 and 170 us, of 2000 14.
//
// Reordering.  A beam's pages before the one being filled are full and may be
// shared; that last page is each beam's own.  The first child of a beam keeps
// it; another child takes over the last page of a beam without children, and
// the list of copies says which rows are to be copied there (every layer's
// append does so before attention).  So no page is taken or given up.
#include "mfma_util.h"
#include "uc_common.h"

namespace uc {
namespace {

constexpr int kMaxW = UC_MAX_BEAMS;

// Cross-lane steps without LDS.  `old` is what lanes without a source keep.
template <int CTRL, int ROWS = 0xF>
__device__ inline uint32_t dpp(uint32_t old, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xF, false);
}
__device__ inline float lane_of(float x, int i) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
}
__device__ inline int lane_of(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
// f over the wave in six steps, in lane 63 (then in every lane)
template <class F>
__device__ inline void wave_fold(F f) {
  f.template step<0x111, 0xF>();
  f.template step<0x112, 0xF>();
  f.template step<0x114, 0xF>();
  f.template step<0x118, 0xF>();
  f.template step<0x142, 0xA>();
  f.template step<0x143, 0xC>();
}
struct MaxStep {
  float& x;
  template <int CTRL, int ROWS>
  __device__ void step() {
    const uint32_t u = __float_as_uint(x);
    x = fmaxf(x, __uint_as_float(dpp<CTRL, ROWS>(u, u)));
  }
};
__device__ inline float max_of_wave(float x) {
  wave_fold(MaxStep{x});
  return lane_of(x, 63);
}

// An element as one number, the larger the earlier: value descending, then
// index ascending.
__device__ inline uint64_t key_of(float v, int i) {
  const uint32_t u = __float_as_uint(v + 0.0f);  // -0 is 0
  return (uint64_t)(u ^ ((uint32_t)((int)u >> 31) | 0x80000000u)) << 32 | (uint32_t)(INT32_MAX - i);
}
__device__ inline float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ inline int index_of(uint64_t key) { return INT32_MAX - (int)(uint32_t)key; }

struct KeyStep {
  uint64_t& k;
  template <int CTRL, int ROWS>
  __device__ void step() {
    const uint32_t lo = (uint32_t)k, hi = (uint32_t)(k >> 32);
    const uint64_t y = (uint64_t)dpp<CTRL, ROWS>(hi, hi) << 32 | dpp<CTRL, ROWS>(lo, lo);
    k = y > k ? y : k;
  }
};

// What a wave has gathered (LDS), and what an element has to reach to join: W
// elements of the split have keys of `key` or more.  v is the value below which
// none can: that of `key`, or the next above it where `key` is one that the
// wave has read, since its later vectors have larger indexes (a mask leaves
// most logits of a row equal).
constexpr int kCap = 576;  // W and eight elements of 64 lanes
struct Floor {
  float v;
  uint64_t key;
  int count;
};

// keeps the W best of what the wave has gathered (W of them at least)
__device__ inline void cut_down(uint64_t* g, Floor& f, int W, int lane) {
  __builtin_amdgcn_wave_barrier();
  uint64_t mine = 0;
  for (int k = 0; k < W; ++k) {
    uint64_t best = 0;
    for (int j = lane; j < f.count; j += 64) best = g[j] > best ? g[j] : best;
    uint64_t top = best;
    wave_fold(KeyStep{top});
    top = (uint64_t)(uint32_t)lane_of((int)(top >> 32), 63) << 32 | (uint32_t)lane_of((int)top, 63);
    if (best == top)
      for (int j = lane; j < f.count; j += 64)
        if (g[j] == top) g[j] = 0;
    if (lane == k) mine = top;
    f.key = top;
  }
  __builtin_amdgcn_wave_barrier();
  if (lane < W) g[lane] = mine;
  f.v = value_of((f.key | 0xFFFFFFFFu) + 1);
  f.count = W;
  __builtin_amdgcn_wave_barrier();
}

// The sum's terms are 2^(c x - r), c = log2(e) as a float and r the rounded
// product of c and the largest of the split's first logits: one multiply-add
// and one exponential an element.  r is taken as it is, so its rounding
// cancels; it must not grow past what an exponent holds, so it stands for at
// most 2^30.  Where the sum leaves its type (a logit beyond that, or 88 above
// the first ones, or a NaN) the split is summed again, by differences.
constexpr float kHeld = 1073741824.0f;
__device__ inline float held(float x) { return __builtin_amdgcn_fmed3f(x, -kHeld, kHeld); }  // NaN: -kHeld
__device__ inline float ranked(float x) { return x != x ? -INFINITY : x; }

// the n-th largest of the wave's values
__device__ inline float nth_largest(float x, int n, int lane) {
  for (;;) {
    const float t = max_of_wave(x);
    if (--n == 0) return t;
    const uint64_t who = __builtin_amdgcn_ballot_w64(x == t);
    if (lane == __ffsll((unsigned long long)who) - 1) x = -INFINITY;
  }
}

// N elements per lane, e-th one at index base + e (none of the lane's if !in)
template <int N>
__device__ inline void consume(const float (&x)[N], int base, bool in, int W, int lane, uint64_t* g, Floor& f, float r,
                               float& s) {
  float mx = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) mx = fmaxf(mx, x[e]);  // (a NaN loses)
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) sum += __builtin_amdgcn_exp2f(fmaf(x[e], kLog2e, -r));
  s += in ? sum : 0.0f;
  if (__builtin_amdgcn_ballot_w64(in && !(mx < f.v))) {
    if (f.count + 64 * N > kCap) cut_down(g, f, W, lane);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (!__builtin_amdgcn_ballot_w64(in && !(x[e] < f.v))) continue;
      const uint64_t key = key_of(ranked(x[e]), base + e);
      const uint64_t join = __builtin_amdgcn_ballot_w64(in && key > f.key);
      if (join >> lane & 1) g[f.count + __popcll(join & ((1ull << lane) - 1))] = key;
      f.count += __popcll(join);
    }
  }
}

struct SelectArgs {
  const void* logits;
  int64_t ld;
  const float* score;
  const uint8_t* done;
  float* score_out;
  int32_t* parent;
  int32_t* token;
  uint8_t* done_out;
  int R, W, V, eos, pad, splits, span;  // span: elements per split
  float* cand_v;  // [R W, splits, W]
  int32_t* cand_i;
  float2* norm;  // [R W, splits]: largest logit, sum of exponentials against it
};

template <int DT>
__device__ inline void unpack(const mf::u4& w, float* x) {
#pragma unroll
  for (int e = 0; e < (DT == UC_F32 ? 4 : 8); ++e) {
    if constexpr (DT == UC_F32) x[e] = __uint_as_float(w[e]);
    else if constexpr (DT == UC_BF16) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    else x[e] = f16_to_f32((uint16_t)(w[e / 2] >> (16 * (e & 1))));
  }
}

// The same of a vector that begins in the middle of a word: w starts an element
// early, `next` is the word behind it.
template <int DT>
__device__ inline void unpack_odd(const mf::u4& w, uint32_t next, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = e == 7 ? next : w[(e + 1) / 2];
    if constexpr (DT == UC_BF16) x[e] = __uint_as_float(e & 1 ? u << 16 : u & 0xFFFF0000u);
    else x[e] = f16_to_f32((uint16_t)(e & 1 ? u : u >> 16));
  }
}

// What a lane reads of its vectors: whole words (4-byte aligned).
typedef uint32_t u4_words __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kDepth = 4;  // vectors of a lane under way

// Reads a split's `vecs` vectors of N elements from element `first` of row p
// on: gathers into g and f, adds to s, returns r.  Vector i is read by thread
// i % 256 wherever the row lies.  ODD: the row's elements are the odd halves of
// the words; a lane then reads from the word that holds its first one, and has
// its last one from the next lane, the wave's last lane from a load of its own.
// (The first and the last word may hold an element that is not the row's: it is
// not used.)
template <int DT, bool ODD>
__device__ inline float read_vectors(const char* p, int first, int vecs, int W, int lane, int wave, uint64_t* g, Floor& f,
                                     float& s, float* s_nth, float* s_max) {
  constexpr int N = DT == UC_F32 ? 4 : 8;
  const char* from = p + (int64_t)first * (16 / N) - (ODD ? 2 : 0);
  mf::u4 w[kDepth];
  uint32_t edge[kDepth];
  int i = wave * 64 + lane;
  // loads without branches (past the end: the last vector again), so that
  // waiting for one leaves the others under way
  const int last = max(vecs - 1, 0);
  auto load = [&](int k, int at) {
    w[k] = __builtin_nontemporal_load(reinterpret_cast<const u4_words*>(from) + min(at, last));
    if constexpr (ODD)  // the word behind the wave's last vector
      edge[k] = reinterpret_cast<const uint32_t*>(from)[4 * (int64_t)(min(at - lane + 63, last) + 1)];
  };
  auto take = [&](int k, int at, float (&x)[N]) {
    if constexpr (ODD) {
      uint32_t next = dpp<0x130>(edge[k], w[k][0]);  // the next lane's first word
      if (at >= last) next = edge[k];
      unpack_odd<DT>(w[k], next, x);
    } else {
      unpack<DT>(w[k], x);
    }
  };
  if (vecs > 0) {
#pragma unroll
    for (int k = 0; k < kDepth; ++k) load(k, i + k * 256);
  }
  // W of the 256 lanes' maxima over their first vectors reach the least of the
  // four waves' (W/4)-th largest ones, so nothing below it is gathered: of
  // 8192 elements of one kind about W pass.
  float mx = -INFINITY;
  if (vecs > 0) {
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      float x[N], most = -INFINITY;
      take(k, i + k * 256, x);
#pragma unroll
      for (int e = 0; e < N; ++e) most = fmaxf(most, x[e]);
      if (i + k * 256 < vecs) mx = fmaxf(mx, most);
    }
  }
  const float most = max_of_wave(mx), nth = nth_largest(mx, (W + 3) / 4, lane);
  if (lane == 0) s_max[wave] = most, s_nth[wave] = nth;
  __syncthreads();
  f.v = fminf(fminf(s_nth[0], s_nth[1]), fminf(s_nth[2], s_nth[3]));
  f.key = key_of(f.v, INT32_MAX) - 1;  // one of this value joins, whatever its index
  const float r = held(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]))) * kLog2e;
  for (int done = 0; done < vecs; done += kDepth * 256) {
#pragma unroll
    for (int k = 0; k < kDepth; ++k, i += 256) {
      float x[N];
      take(k, i, x);
      load(k, i + kDepth * 256);
      consume<N>(x, first + i * N, i < vecs, W, lane, g, f, r, s);
    }
  }
  return r;
}

// One workgroup per (row, split); its waves take the vectors of the split in
// turn, the next one's load under way.  Which thread sums an element goes by
// its index in the row and not by its address, so that rows of the same logits
// have the same sum and equal totals stay equal.  (Vectors that begin on any
// element, read as such, instead of the words and their shift: 384 rows of
// 131071 bf16 in 40 us instead of 36.)
template <int DT>
__global__ __launch_bounds__(256) void beam_rows_kernel(SelectArgs a) {
  constexpr int N = DT == UC_F32 ? 4 : 8;
  constexpr int EB = DT == UC_F32 ? 4 : 2;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  if (a.done && a.done[row]) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = a.W;
  const char* p = (const char*)a.logits + (int64_t)row * a.ld * EB;
  const int first = split * a.span, end = first + min(a.V - first, a.span);
  // whole vectors of 16 bytes, and single elements behind them
  const int vecs = (end - first) / N, to = first + vecs * N;
  __shared__ uint64_t gathered[4][kCap];
  uint64_t* g = gathered[wave];
  Floor f{-INFINITY, 0, 0};
  float s = 0.0f;
  __shared__ float s_nth[4], s_max[4];
  float r;
  if (DT != UC_F32 && ((uintptr_t)p & 2))  // (a split begins at an even element)
    r = read_vectors<DT, DT != UC_F32>(p, first, vecs, W, lane, wave, g, f, s, s_nth, s_max);
  else
    r = read_vectors<DT, false>(p, first, vecs, W, lane, wave, g, f, s, s_nth, s_max);
  if (wave == 3) {  // at most 7 elements behind the vectors, one per lane
    const bool in = lane < end - to;
    const int at = in ? to + lane : 0;
    float x[1] = {in ? load_elem(p, DT, at) : -INFINITY};
    consume<1>(x, at, in, W, lane, g, f, r, s);
  }
  // the wave's sum, then the workgroup's lists and sums
  s = wave_sum(s);
  __shared__ float ls[4];
  __shared__ int counts[4];
  __shared__ float s_best;
  if (lane == 0) ls[wave] = s, counts[wave] = f.count;
  if (threadIdx.x == 0) s_best = -INFINITY;
  __syncthreads();
  // an element's rank is the number of those before it
  const int64_t out = (int64_t)blockIdx.x * W;
  const int c1 = counts[0], c2 = c1 + counts[1], c3 = c2 + counts[2], n = c3 + counts[3];
  for (int t = threadIdx.x; t - lane < n; t += 256) {
    const int h = (t >= c1) + (t >= c2) + (t >= c3), at = t - (h == 0 ? 0 : h == 1 ? c1 : h == 2 ? c2 : c3);
    const uint64_t key = t < n ? gathered[h][at] : 0;
    int rank = 0;
    for (int k = 0; k < 4; ++k) {
      const int count = counts[k];
#pragma unroll 4
      for (int j = 0; j < count; ++j) rank += gathered[k][j] > key;
    }
    if (t < n && rank < W) {
      a.cand_v[out + rank] = value_of(key);
      a.cand_i[out + rank] = index_of(key);
      if (rank == 0) s_best = value_of(key);
    }
  }
  if ((int)threadIdx.x >= n && (int)threadIdx.x < W) {  // a split of fewer elements
    a.cand_v[out + threadIdx.x] = -INFINITY;
    a.cand_i[out + threadIdx.x] = INT32_MAX;
  }
  __syncthreads();
  // the split's largest logit (none: -inf), and the sum of exp(x - it)
  const float top = s_best;
  float sum = ((ls[0] + ls[1]) + (ls[2] + ls[3])) * exp2f(-fmaf(top, kLog2e, -r));
  const bool fits = top >= -kHeld && top <= kHeld && sum >= 1e-6f && sum < INFINITY;  // (at least 1, but for rounding)
  if (!fits && top > -INFINITY && top < INFINITY) {
    sum = 0.0f;
    for (int k = first + threadIdx.x; k < end; k += 256) {
      const float x = load_elem(p, DT, k);
      sum += x == x ? exp2f((x - top) * kLog2e) : 0.0f;
    }
    sum = wave_sum(sum);
    __syncthreads();
    if (lane == 0) ls[wave] = sum;
    __syncthreads();
    sum = (ls[0] + ls[1]) + (ls[2] + ls[3]);
  }
  if (threadIdx.x == 0) a.norm[blockIdx.x] = float2{top, sum};
}

struct Total {
  double v;
  int flat;
};
__device__ inline bool before(const Total& x, const Total& y) { return x.v > y.v || (x.v == y.v && x.flat < y.flat); }
struct FirstStep {  // the total that comes first
  Total& t;
  template <int CTRL, int ROWS>
  __device__ void step() {
    const uint64_t u = (uint64_t)__double_as_longlong(t.v);
    const uint32_t lo = dpp<CTRL, ROWS>((uint32_t)u, (uint32_t)u), hi = dpp<CTRL, ROWS>(u >> 32, u >> 32);
    const Total y{__longlong_as_double((int64_t)((uint64_t)hi << 32 | lo)), (int)dpp<CTRL, ROWS>(t.flat, t.flat)};
    if (before(y, t)) t = y;
  }
};

// One workgroup per request: totals of the candidates in registers (at most
// kPer of a thread, by the choice of splits), then W rounds of the first among
// them.
constexpr int kMostPer = 16, kMaxRows = 512;  // splits of a request: W min(64, 4096 / W^2)
template <int kPer>
__global__ __launch_bounds__(256) void beam_pick_kernel(SelectArgs a) {
  __shared__ double log_sum[kMaxW];  // of a beam's exponentials against its largest logit
  __shared__ float top[kMaxW];
  __shared__ Total best[2][4];
  __shared__ float score[kMaxW];  // read whole first: the outputs may be the inputs
  __shared__ bool ended[kMaxW];
  const int q = blockIdx.x, W = a.W, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = a.splits * W, n = W * per;  // candidate c: beam c / per
  int ci[kPer];
  float cv[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int c = threadIdx.x + k * 256;
    ci[k] = INT32_MAX;
    cv[k] = -INFINITY;
    if (k * 256 < n && c < n) {  // (an ended beam's are not written; not used either)
      ci[k] = a.cand_i[(int64_t)q * n + c];
      cv[k] = a.cand_v[(int64_t)q * n + c];
    }
  }
  __shared__ float2 norm[kMaxRows];
  for (int i = threadIdx.x; i < W * a.splits; i += 256) norm[i] = a.norm[(int64_t)q * W * a.splits + i];
  __syncthreads();
  if ((int)threadIdx.x < W) {  // a lane per beam
    const int b = threadIdx.x;
    const int64_t row = (int64_t)q * W + b;
    const bool gone = a.done && a.done[row];
    double z = 0.0;
    float t = -INFINITY;
    if (!gone) {
      for (int k = 0; k < a.splits; ++k) t = fmaxf(t, norm[b * a.splits + k].x);
      // a beam without a finite logit, or with one of +inf, has no totals
      const bool some = t > -INFINITY && t < INFINITY;
      for (int k = 0; k < a.splits; ++k) {
        const float2 x = norm[b * a.splits + k];
        if (some && x.x > -INFINITY) z += (double)x.y * (double)exp2f((x.x - t) * kLog2e);
      }
      z = some ? log(z) : INFINITY;
    }
    log_sum[b] = z;
    top[b] = t;
    score[b] = a.score[row];
    ended[b] = gone;
  }
  __syncthreads();
  double tv[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    tv[k] = -INFINITY;
    const int c = threadIdx.x + k * 256;
    if (k * 256 >= n || c >= n) {
      ci[k] = INT32_MAX;
      continue;
    }
    const int b = c / per, j = c % per;
    const double sc = score[b], base = sc - log_sum[b];
    if (ended[b] || !(base > -INFINITY && base < INFINITY)) {
      // an ended beam goes on by its pad token alone; one without totals
      // offers its first tokens
      int tok = j < W ? j : a.V;
      if (ended[b] && j == 0) tok = a.pad, tv[k] = sc > -INFINITY && sc < INFINITY ? sc : -INFINITY;
      else if (ended[b] && j < W) tok = j - 1 < a.pad ? j - 1 : j;
      ci[k] = tok < a.V ? b * a.V + tok : INT32_MAX;
    } else if (ci[k] != INT32_MAX) {
      tv[k] = base + ((double)cv[k] - (double)top[b]);
      ci[k] += b * a.V;
    }
  }
  auto write = [&](int k, const Total& t) {
    const int b = t.flat / a.V, tok = t.flat % a.V;
    const int64_t to = (int64_t)q * W + k;
    a.score_out[to] = (float)t.v;
    a.parent[to] = b;
    a.token[to] = tok;
    if (a.done_out) a.done_out[to] = ended[b] || tok == a.eos;
  };
  if constexpr (kPer == 1) {  // one wave takes them all: no barriers
    __shared__ Total all[256];
    all[threadIdx.x] = Total{tv[0], ci[0]};
    __syncthreads();
    if (wave) return;
    Total c[4], chosen{-INFINITY, INT32_MAX};
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = all[lane + 64 * j];
    for (int k = 0; k < W; ++k) {
      Total t = c[0];
#pragma unroll
      for (int j = 1; j < 4; ++j)
        if (before(c[j], t)) t = c[j];
      wave_fold(FirstStep{t});
      const uint64_t u = (uint64_t)__double_as_longlong(t.v);
      const uint64_t v = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)u, 63);
      t = Total{__longlong_as_double((int64_t)v), __builtin_amdgcn_readlane(t.flat, 63)};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c[j].flat == t.flat) c[j] = Total{-INFINITY, INT32_MAX};
      if (lane == k) chosen = t;
    }
    if (lane < W) write(lane, chosen);
    return;
  }
  for (int k = 0; k < W; ++k) {
    Total t{-INFINITY, INT32_MAX};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const Total x{tv[j], ci[j]};
      if (before(x, t)) t = x;
    }
    wave_fold(FirstStep{t});
    if (lane == 63) best[k & 1][wave] = t;
    __syncthreads();
    t = best[k & 1][0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (before(best[k & 1][i], t)) t = best[k & 1][i];
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (ci[j] == t.flat) tv[j] = -INFINITY, ci[j] = INT32_MAX;
    if (threadIdx.x == 0) write(k, t);
  }
}

// ---------------------------------------------------------------- reordering
struct ReorderArgs {
  const int32_t* parent;
  const int32_t* token;
  const int32_t* table;
  const int32_t* len;
  int32_t* table_out;
  int32_t* copies;
  const int32_t* history;
  int32_t* history_out;
  int64_t history_ld;
  int R, W, ld, lgP, n_history, table_blocks;
};

// A thread moves one column of the request's W rows: read whole, then
// written, so the outputs may be the inputs.
template <int MAXW>
__global__ __launch_bounds__(256) void beam_reorder_kernel(ReorderArgs a) {
  __shared__ int s_from[kMaxW], s_last[kMaxW];  // a row's parent, and the row whose last page it takes (-1: its parent's)
  const int r = blockIdx.x, W = a.W;
  if (threadIdx.x < 64) {  // a lane per beam
    const int b = threadIdx.x;
    const int p = b < W ? min(max(a.parent[(int64_t)r * W + b], 0), W - 1) : -1;
    uint32_t has = 0;  // beams with a child
    bool again = false;
    for (int j = 0; j < W; ++j) {
      const int pj = __builtin_amdgcn_readlane(p, j);
      has |= 1u << pj;
      again |= j < b && pj == p;
    }
    const uint64_t extra = __builtin_amdgcn_ballot_w64(b < W && again);
    if (b < W) {
      uint32_t free = ~has & (W == 32 ? ~0u : (1u << W) - 1);
      for (int k = __popcll(extra & ((1ull << b) - 1)); k > 0; --k) free &= free - 1;
      s_from[b] = p;
      s_last[b] = again ? __ffs(free) - 1 : -1;
    }
  }
  __syncthreads();
  if ((int)blockIdx.y < a.table_blocks) {
    const int c = blockIdx.y * blockDim.x + threadIdx.x;
    const int rows = max(a.len[(int64_t)r * W], 0);
    const int full = rows >> a.lgP, part = rows & ((1 << a.lgP) - 1);
    int v[MAXW];
    if (c < a.ld && c < full + (part > 0)) {
#pragma unroll
      for (int b = 0; b < MAXW; ++b)
        if (b < W) {
          const int from = c == full && s_last[b] >= 0 ? s_last[b] : s_from[b];
          v[b] = a.table[((int64_t)r * W + from) * a.ld + c];
        }
      int src[MAXW];
      if (c == full) {
#pragma unroll
        for (int b = 0; b < MAXW; ++b)
          if (b < W) src[b] = a.table[((int64_t)r * W + s_from[b]) * a.ld + c];
      }
#pragma unroll
      for (int b = 0; b < MAXW; ++b)
        if (b < W) {
          a.table_out[((int64_t)r * W + b) * a.ld + c] = v[b];
          if (c == full) {
            const bool moved = s_last[b] >= 0;
            int32_t* cp = a.copies + ((int64_t)r * W + b) * 3;
            cp[0] = moved ? src[b] : -1;
            cp[1] = moved ? v[b] : -1;
            cp[2] = moved ? part : 0;
          }
        }
    }
    // no page in part: no copies
    if (blockIdx.y == 0 && (part == 0 || full >= a.ld) && (int)threadIdx.x < W) {
      int32_t* cp = a.copies + ((int64_t)r * W + threadIdx.x) * 3;
      cp[0] = cp[1] = -1;
      cp[2] = 0;
    }
    return;
  }
  const int c = (blockIdx.y - a.table_blocks) * blockDim.x + threadIdx.x;
  if (c > a.n_history) return;
  int v[MAXW];
#pragma unroll
  for (int b = 0; b < MAXW; ++b)
    if (b < W) {
      const int64_t row = (int64_t)r * W + s_from[b];
      v[b] = c < a.n_history ? a.history[row * a.history_ld + c] : a.token[(int64_t)r * W + b];
    }
#pragma unroll
  for (int b = 0; b < MAXW; ++b)
    if (b < W) a.history_out[((int64_t)r * W + b) * a.history_ld + c] = v[b];
}

// Splits of a row: six workgroups per CU over all rows at most, which run in one
// round (384 rows of 131071 in two, three, four and six splits: 45.1, 45.9, 39.6
// and 43.7 us a step with its reordering), a span of at least 2048 elements (a workgroup's
// fixed work is a few microseconds), and candidates that the second kernel
// holds in registers.
int beam_splits(int R, int W, int V) {
  const int want = 6 * device_cus() / (R * W);
  return max(1, min(min(want, min(64, 256 * kMostPer / (W * W))), V / 2048));
}
size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t beam_select_workspace(int R, int W, int V) {
  const size_t rows = (size_t)R * W * beam_splits(R, W, V);
  return align_up(rows * W * sizeof(float)) + align_up(rows * W * sizeof(int32_t)) + align_up(rows * sizeof(float2));
}

hipError_t launch_beam_select(const void* logits, int dt, int64_t ld, const float* score, const uint8_t* done, int R,
                              int W, int V, int eos, int pad, float* score_out, int32_t* parent, int32_t* token,
                              uint8_t* done_out, void* ws, hipStream_t st) {
  const int splits = beam_splits(R, W, V);
  const size_t rows = (size_t)R * W * splits;
  char* p = (char*)ws;
  const int span = ((V + splits - 1) / splits + 7) & ~7;  // whole vectors; none is empty, with 64 splits of 2048 at most
  SelectArgs a{logits, ld, score, done, score_out, parent, token, done_out, R, W, V, eos, pad, splits, span,
               (float*)p, (int32_t*)(p + align_up(rows * W * sizeof(float))),
               (float2*)(p + align_up(rows * W * sizeof(float)) + align_up(rows * W * sizeof(int32_t)))};
  if (dt == UC_BF16) hipLaunchKernelGGL(beam_rows_kernel<UC_BF16>, dim3(rows), dim3(256), 0, st, a);
  else if (dt == UC_F16) hipLaunchKernelGGL(beam_rows_kernel<UC_F16>, dim3(rows), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(beam_rows_kernel<UC_F32>, dim3(rows), dim3(256), 0, st, a);
  const int per = (W * W * splits + 255) / 256;
  if (per == 1) hipLaunchKernelGGL(beam_pick_kernel<1>, dim3(R), dim3(256), 0, st, a);
  else if (per <= 4) hipLaunchKernelGGL(beam_pick_kernel<4>, dim3(R), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(beam_pick_kernel<kMostPer>, dim3(R), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const int32_t* parent, const int32_t* token, const int32_t* table, const int32_t* len,
                               int R, int W, int ld, int lgP, int32_t* table_out, int32_t* copies,
                               const int32_t* history, int32_t* history_out, int64_t history_ld, int n_history,
                               hipStream_t st) {
  const int tb = (ld + 255) / 256, hb = history ? (int)(((int64_t)n_history + 1 + 255) / 256) : 0;
  const ReorderArgs a{parent, token, table, len, table_out, copies, history, history_out, history_ld,
                      R, W, ld, lgP, n_history, tb};
  if (W <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, dim3(R, tb + hb), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(beam_reorder_kernel<32>, dim3(R, tb + hb), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace uc
