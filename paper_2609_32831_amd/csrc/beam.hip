// beam.hip -- one step of a beam search: the W best of a request's W * V
// continuations, and the reordering of its beams' tables and histories.
//
// Selection.  total = score + logit - log sum exp(logits of the beam).  Within
// a beam the totals are ordered as the logits, so one pass over the logits
// yields both the normaliser and the only W candidates that can be chosen;
// totals are formed for those alone, in 64 bits.  The pass is bound by the
// bytes of the logits; rows are split where there are few.  A wave keeps the
// W best in its lanes in order, and looks at a vector of elements only where
// its largest passes the last of them, which soon is rare.
//
// Reordering.  A beam's pages before the one being filled are full and may be
// shared; that last page is each beam's own.  The first child of a beam keeps
// it; another child takes over the last page of a beam without children, and
// the list of copies says which rows are to be copied there (every layer's
// append does so before attention).  So no page is taken or given up.
#include <algorithm>

#include "mfma_util.h"
#include "uc_common.h"

namespace uc {
namespace {

constexpr int kMaxW = UC_MAX_BEAMS;

struct Best {  // lane i holds the i-th best of the wave (value descending, index ascending)
  float v;
  int i;
  float last_v;  // the W-th best, in every lane
  int last_i;
};

__device__ inline bool before(float v, int i, float v2, int i2) { return v > v2 || (v == v2 && i < i2); }

__device__ inline void insert(Best& b, int W, int lane, float v, int i) {
  const int at = __popcll(__builtin_amdgcn_ballot_w64(lane < W && before(b.v, b.i, v, i)));
  const float uv = __shfl_up(b.v, 1, 64);
  const int ui = __shfl_up(b.i, 1, 64);
  if (lane > at) b.v = uv, b.i = ui;
  if (lane == at) b.v = v, b.i = i;
  b.last_v = __shfl(b.v, W - 1, 64);
  b.last_i = __shfl(b.i, W - 1, 64);
}

template <int DT>
__device__ inline float elem(const void* p, int64_t i) {
  return fmaxf(load_elem(p, DT, i), -INFINITY);  // a NaN counts as -inf
}

// N elements per lane, e-th one at index base + e; those past n are -inf
template <int N>
__device__ inline void consume(const float (&x)[N], int base, int n, int W, int lane, Best& b, float& m, float& s) {
  float mx = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) mx = fmaxf(mx, x[e]);
  if (mx > m) {
    s *= exp2f((m - mx) * kLog2e);
    m = mx;
  }
  // differences first: the rounding of m * log2(e) would reach every term
  const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((x[e] - ref) * kLog2e);
  if (__builtin_amdgcn_ballot_w64(n > 0 && mx >= b.last_v)) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      uint64_t todo = __builtin_amdgcn_ballot_w64(e < n && before(x[e], base + e, b.last_v, b.last_i));
      while (todo) {
        const int from = __ffsll((unsigned long long)todo) - 1;
        todo &= todo - 1;
        const float v = __shfl(x[e], from, 64);
        const int i = __shfl(base, from, 64) + e;
        if (before(v, i, b.last_v, b.last_i)) insert(b, W, lane, v, i);
      }
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
  float2* norm;  // [R W, splits]: reference maximum, sum
};

// one workgroup per (row, split)
template <int DT>
__global__ __launch_bounds__(256) void beam_rows_kernel(SelectArgs a) {
  constexpr int N = DT == UC_F32 ? 4 : 8;
  constexpr int EB = DT == UC_F32 ? 4 : 2;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  if (a.done && a.done[row]) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = a.W;
  const char* p = (const char*)a.logits + (int64_t)row * a.ld * EB;
  const int first = split * a.span, end = min(a.V, first + a.span);
  // whole 16-byte vectors from `from` on; single elements before and behind
  const int from = min(end, first + (int)(((16 - ((uintptr_t)(p + (int64_t)first * EB) & 15)) & 15) / EB));
  const int vecs = (end - from) / N, to = from + vecs * N;
  Best b{-INFINITY, INT32_MAX, -INFINITY, INT32_MAX};
  float m = -INFINITY, s = 0.0f;
  {
    const int n_head = from - first, n_edge = n_head + end - to;  // at most 14, one per lane of wave 0
    float x[1] = {-INFINITY};
    int at = 0;
    const bool in = wave == 0 && lane < n_edge;
    if (in) {
      at = lane < n_head ? first + lane : to + lane - n_head;
      x[0] = elem<DT>(p, at);
    }
    consume<1>(x, at, in, W, lane, b, m, s);
  }
  const char* vec = p + (int64_t)from * EB;
  for (int i = threadIdx.x; i - lane < vecs; i += 256) {
    float x[N];
    const bool in = i < vecs;
    mf::u4 w = mf::u4{0, 0, 0, 0};
    if (in) w = __builtin_nontemporal_load(reinterpret_cast<const mf::u4*>(vec) + i);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f;
      if constexpr (DT == UC_F32) f = __uint_as_float(w[e]);
      else if constexpr (DT == UC_BF16) f = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
      else f = f16_to_f32((uint16_t)(w[e / 2] >> (16 * (e & 1))));
      x[e] = in ? fmaxf(f, -INFINITY) : -INFINITY;
    }
    consume<N>(x, from + i * N, in ? N : 0, W, lane, b, m, s);
  }
  // the wave's sum, then the workgroup's lists and sums
  const float mw = wave_max(m);
  s = wave_sum(m == -INFINITY ? 0.0f : s * exp2f((m - mw) * kLog2e));
  __shared__ float lv[4 * kMaxW], lm[4], ls[4];
  __shared__ int li[4 * kMaxW];
  if (lane < W) {
    lv[wave * W + lane] = b.v;
    li[wave * W + lane] = b.i;
  }
  if (lane == 0) lm[wave] = mw, ls[wave] = s;
  __syncthreads();
  const int64_t out = (int64_t)blockIdx.x * W;
  if ((int)threadIdx.x < 4 * W) {
    const float v = lv[threadIdx.x];
    const int i = li[threadIdx.x];
    int rank = 0;
    for (int k = 0; k < 4 * W; ++k)
      rank += before(lv[k], li[k], v, i) || (lv[k] == v && li[k] == i && k < (int)threadIdx.x);
    if (rank < W) a.cand_v[out + rank] = v, a.cand_i[out + rank] = i;
  }
  if (threadIdx.x == 0) {
    const float M = fmaxf(fmaxf(lm[0], lm[1]), fmaxf(lm[2], lm[3]));
    float sum = 0.0f;
    for (int k = 0; k < 4; ++k) sum += lm[k] == -INFINITY ? 0.0f : ls[k] * exp2f((lm[k] - M) * kLog2e);
    a.norm[blockIdx.x] = float2{M, sum};
  }
}

struct Total {
  double v;
  int flat;
};
__device__ inline bool before(const Total& x, const Total& y) { return x.v > y.v || (x.v == y.v && x.flat < y.flat); }

// one workgroup per request: totals of the candidates, W rounds of the best
__global__ __launch_bounds__(256) void beam_pick_kernel(SelectArgs a) {
  __shared__ double top[kMaxW], log_sum[kMaxW];  // a beam's largest logit, and the log of its sum of exponentials
  __shared__ Total best[4];
  __shared__ float score[kMaxW];  // read whole first: the outputs may be the inputs
  __shared__ bool ended[kMaxW];
  const int r = blockIdx.x, W = a.W, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = wave; b < W; b += 4) {  // a wave per beam; splits <= 64
    const int64_t row = (int64_t)r * W + b;
    const bool gone = a.done && a.done[row];
    double M = 0.0, z = 0.0;
    if (!gone) {
      const float2 n = lane < a.splits ? a.norm[row * a.splits + lane] : float2{-INFINITY, 0.0f};
      M = wave_max(n.x);
      const double part = n.x == -INFINITY ? 0.0 : (double)n.y * exp((double)n.x - M);
      z = log(wave_sum_d(part));  // not finite if no logit is, or one is +inf
    }
    if (lane == 0) {
      top[b] = M;
      log_sum[b] = z;
      score[b] = a.score[row];
      ended[b] = gone;
    }
  }
  __syncthreads();
  // candidate c of the request: beam c / (splits W)
  const int per = a.splits * W, n = W * per;
  auto total = [&](int c) {
    const int b = c / per, k = c % per;
    const int64_t row = (int64_t)r * W + b;
    const double sc = score[b];
    Total t{-INFINITY, INT32_MAX};
    const bool gone = ended[b];
    const double base = sc - log_sum[b];
    if (gone || !(base > -INFINITY && base < INFINITY)) {
      // an ended beam goes on by its pad token alone; one whose totals are
      // all -inf offers its first tokens
      if (k < W) {
        int tok = k;
        if (gone && k == 0) tok = a.pad, t.v = sc > -INFINITY && sc < INFINITY ? sc : -INFINITY;
        else if (gone) tok = k - 1 < a.pad ? k - 1 : k;
        if (tok < a.V) t.flat = b * a.V + tok;
      }
      return t;
    }
    const int i = a.cand_i[row * per + k];
    if (i == INT32_MAX) return t;
    t.v = base + ((double)a.cand_v[row * per + k] - top[b]);
    t.flat = b * a.V + i;
    return t;
  };
  Total last{INFINITY, -1};  // the one chosen before
  for (int k = 0; k < W; ++k) {
    Total t{-INFINITY, INT32_MAX};
    for (int c = threadIdx.x; c < n; c += 256) {
      const Total x = total(c);
      if (before(last, x) && before(x, t)) t = x;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      Total y;
      y.v = __shfl_xor(t.v, o, 64);
      y.flat = __shfl_xor(t.flat, o, 64);
      if (before(y, t)) t = y;
    }
    if (lane == 0) best[wave] = t;
    __syncthreads();
    t = best[0];
    for (int i = 1; i < 4; ++i)
      if (before(best[i], t)) t = best[i];
    __syncthreads();
    last = t;
    if (threadIdx.x == 0) {
      const int b = t.flat / a.V, tok = t.flat % a.V;
      const int64_t to = (int64_t)r * W + k;
      a.score_out[to] = (float)t.v;
      a.parent[to] = b;
      a.token[to] = tok;
      if (a.done_out) a.done_out[to] = ended[b] || tok == a.eos;
    }
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
  if (threadIdx.x == 0) {
    uint32_t has = 0;  // beams with a child
    for (int b = 0; b < W; ++b) {
      const int p = min(max(a.parent[(int64_t)r * W + b], 0), W - 1);
      s_from[b] = p;
      s_last[b] = has >> p & 1 ? -2 : -1;
      has |= 1u << p;
    }
    uint32_t free = ~has & (W == 32 ? ~0u : (1u << W) - 1);
    for (int b = 0; b < W; ++b)
      if (s_last[b] == -2) {
        s_last[b] = __ffs(free) - 1;
        free &= free - 1;
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

// Splits of a row: about four workgroups per CU over all rows, a span of at
// least 4096 elements (a workgroup's fixed work is a few microseconds).
int beam_splits(int R, int W, int V) {
  const int want = (4 * device_cus() + R * W - 1) / (R * W);
  return max(1, min(min(want, 64), V / 4096));
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
  SelectArgs a{logits, ld, score, done, score_out, parent, token, done_out, R, W, V, eos, pad, splits,
               (V + splits - 1) / splits, (float*)p, (int32_t*)(p + align_up(rows * W * sizeof(float))),
               (float2*)(p + align_up(rows * W * sizeof(float)) + align_up(rows * W * sizeof(int32_t)))};
  if (dt == UC_BF16) hipLaunchKernelGGL(beam_rows_kernel<UC_BF16>, dim3(rows), dim3(256), 0, st, a);
  else if (dt == UC_F16) hipLaunchKernelGGL(beam_rows_kernel<UC_F16>, dim3(rows), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(beam_rows_kernel<UC_F32>, dim3(rows), dim3(256), 0, st, a);
  hipLaunchKernelGGL(beam_pick_kernel, dim3(R), dim3(256), 0, st, a);
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
