// abi_page.hip -- the C entry points of the paged 4-bit cache and of beam
// search over it: argument checks, then the launches.  Every check runs before
// any launch, so a failing call writes nothing and enqueues nothing.
#include <limits.h>
#include <math.h>

#include "page_common.h"

using namespace uc;

namespace uc {
size_t page_free_workspace(int n_pages);
hipError_t launch_page_free(const int32_t* table, const int32_t* len, int S, int ld, int lgP, int n_pages,
                            int32_t* list, int32_t* pool, void* ws, hipStream_t st);
hipError_t launch_page_step(int S, const int32_t* len, const int32_t* more, int32_t* table, int ld, int lgP,
                            int n_pages, const int32_t* list, const int32_t* pool, int32_t* len_out,
                            int32_t* q_start, int32_t* slots, int n_slots, int32_t* pool_out, uint8_t* refused,
                            hipStream_t st);
hipError_t launch_page_append(const PageCache& pc, const void* k, const void* v, int dt, int64_t ld, int T,
                              const int32_t* slots, const int32_t* copies, int n_copies, hipStream_t st);
hipError_t launch_page_read(const PageCache& pc, const int32_t* slots, int T, void* kout, void* vout, int dt,
                            int64_t ld, hipStream_t st);
size_t page_attend_workspace(const PageCache& pc, int G, int S, int max_q);
hipError_t launch_page_attend(const PageAttendArgs& a, int q_dt, int max_q, bool valu, void* ws, hipStream_t st);
size_t beam_select_workspace(int R, int W, int V);
hipError_t launch_beam_select(const void* logits, int dt, int64_t ld, const float* score, const uint8_t* done, int R,
                              int W, int V, int eos, int pad, float* score_out, int32_t* parent, int32_t* token,
                              uint8_t* done_out, void* ws, hipStream_t st);
hipError_t launch_beam_reorder(const int32_t* parent, const int32_t* token, const int32_t* table, const int32_t* len,
                               int R, int W, int ld, int lgP, int32_t* table_out, int32_t* copies,
                               const int32_t* history, int32_t* history_out, int64_t history_ld, int n_history,
                               hipStream_t st);
}  // namespace uc

namespace {

// an append or a read: 16 heads' rows or more to a workgroup of 256, a page's
// head to another; a launch holds fewer than 2^24 of them
constexpr int64_t kMostRows = 1 << 27, kMostCopies = 1 << 22;
// sequences, table columns, slots, and continuations of a request: what the
// kernels' indexes pass by a grid's stride stays in 31 bits
constexpr int kMostIndex = 1 << 30;

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

uc_status check_paging(int page_rows, int64_t n_pages) {
  if (!pow2(page_rows) || page_rows < 16 || page_rows > 1024)
    return fail(UC_E_INVALID, "page_rows %d must be a power of two in [16,1024]", page_rows);
  if (n_pages < 1 || n_pages * page_rows > INT32_MAX)
    return fail(UC_E_INVALID, "n_pages %lld must be >= 1, n_pages * page_rows < 2^31", (long long)n_pages);
  return UC_OK;
}

// int32 arrays of the device: present and aligned
uc_status check_ints(const char* what, const void* p) {
  if (!p || !aligned4(p)) return fail(UC_E_INVALID, "%s is NULL or not 4-byte aligned", what);
  return UC_OK;
}

uc_status check_cache(const uc_page_cache* c, PageCache& pc) {
  if (!c) return fail(UC_E_INVALID, "cache is NULL");
  uc_status st = check_paging(c->page_rows, c->n_pages);
  if (st) return st;
  if (c->D != 64 && c->D != 128) return fail(UC_E_INVALID, "D must be 64 or 128 (got %d)", c->D);
  if (c->Hkv < 1 || c->Hkv > 4096) return fail(UC_E_INVALID, "Hkv %d not in [1,4096]", c->Hkv);
  if ((c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->D)
    return fail(UC_E_INVALID, "group %d must be 32, 64 or 128 and at most D", c->group);
  const void* ptrs[] = {c->codes_k, c->codes_v, c->scale_k, c->scale_v};
  for (const void* p : ptrs)
    if (!p || !aligned16(p)) return fail(UC_E_INVALID, "a cache pointer is NULL or not 16-byte aligned");
  pc = PageCache{c->codes_k, c->codes_v, c->scale_k, c->scale_v, c->n_pages, __builtin_ctz(c->page_rows),
                 c->Hkv, c->D, c->D / c->group};
  return UC_OK;
}

// rows of T tokens in dt, ld elements apart
uc_status check_rows(const char* what, const void* p, int dt, int64_t ld, int64_t width) {
  if (!dtype_ok(dt)) return fail(UC_E_INVALID, "bad dtype %d", dt);
  if (!p || !aligned16(p)) return fail(UC_E_INVALID, "%s is NULL or not 16-byte aligned", what);
  if (ld < width || ld % (dt == UC_F32 ? 4 : 8))
    return fail(UC_E_INVALID, "%s: row distance %lld must be at least %lld and a multiple of 16 bytes", what,
                (long long)ld, (long long)width);
  return UC_OK;
}

}  // namespace

extern "C" {

size_t uc_page_free_workspace_size(int n_pages) { return n_pages < 1 ? 0 : page_free_workspace(n_pages); }

uc_status uc_page_free(int S, int page_rows, int n_pages, const int32_t* table, int table_ld, const int32_t* len,
                       int32_t* free_list, int32_t* pool, void* ws, size_t ws_bytes, void* stream) {
  uc_status st = check_paging(page_rows, n_pages);
  if (st) return st;
  if (S < 1 || table_ld < 1) return fail(UC_E_INVALID, "S and table_ld must be >= 1 (got %d, %d)", S, table_ld);
  if (S > kMostIndex || table_ld > kMostIndex)
    return fail(UC_E_UNSUPPORTED, "more than 2^30 sequences or table columns (got %d, %d)", S, table_ld);
  if ((st = check_ints("table", table)) || (st = check_ints("len", len)) ||
      (st = check_ints("free_list", free_list)) || (st = check_ints("pool", pool)))
    return st;
  if (!ws || !aligned16(ws) || ws_bytes < page_free_workspace(n_pages))
    return fail(UC_E_WORKSPACE, "workspace %zu < %zu bytes, or not 16-byte aligned", ws_bytes,
                page_free_workspace(n_pages));
  return launched(launch_page_free(table, len, S, table_ld, __builtin_ctz(page_rows), n_pages, free_list, pool, ws,
                                   (hipStream_t)stream));
}

uc_status uc_page_step(int S, int page_rows, int n_pages, const int32_t* len, const int32_t* new_len, int32_t* table,
                       int table_ld, const int32_t* free_list, const int32_t* pool, int32_t* len_out,
                       int32_t* q_start, int32_t* slots, int n_slots, int32_t* pool_out, uint8_t* refused,
                       void* stream) {
  uc_status st = check_paging(page_rows, n_pages);
  if (st) return st;
  if (S < 1 || table_ld < 1 || n_slots < 0)
    return fail(UC_E_INVALID, "S and table_ld must be >= 1, n_slots >= 0 (got %d, %d, %d)", S, table_ld, n_slots);
  if (S > kMostIndex || table_ld > kMostIndex || n_slots > kMostIndex)
    return fail(UC_E_UNSUPPORTED, "more than 2^30 sequences, table columns or slots (got %d, %d, %d)", S, table_ld, n_slots);
  if ((st = check_ints("len", len)) || (st = check_ints("new_len", new_len)) || (st = check_ints("table", table)) ||
      (st = check_ints("free_list", free_list)) || (st = check_ints("pool", pool)) ||
      (st = check_ints("len_out", len_out)) || (st = check_ints("q_start", q_start)) ||
      (n_slots && (st = check_ints("slots", slots))) || (st = check_ints("pool_out", pool_out)))
    return st;
  if (!refused) return fail(UC_E_INVALID, "refused is NULL");
  return launched(launch_page_step(S, len, new_len, table, table_ld, __builtin_ctz(page_rows), n_pages, free_list,
                                   pool, len_out, q_start, slots, n_slots, pool_out, refused, (hipStream_t)stream));
}

uc_status uc_page_append(const uc_page_cache* cache, const void* k_new, const void* v_new, uc_dtype dt, int64_t ld,
                         int T, const int32_t* slots, const int32_t* copies, int n_copies, void* stream) {
  PageCache pc;
  uc_status st = check_cache(cache, pc);
  if (st) return st;
  if (T < 0 || n_copies < 0) return fail(UC_E_INVALID, "T and n_copies must be >= 0 (got %d, %d)", T, n_copies);
  if ((int64_t)T * pc.Hkv > kMostRows || (int64_t)n_copies * pc.Hkv > kMostCopies)
    return fail(UC_E_UNSUPPORTED, "too many rows or copies for one call");
  if (T > 0 && ((st = check_rows("k_new", k_new, dt, ld, (int64_t)pc.Hkv * pc.D)) ||
                (st = check_rows("v_new", v_new, dt, ld, (int64_t)pc.Hkv * pc.D)) || (st = check_ints("slots", slots))))
    return st;
  if (T == 0 && !dtype_ok(dt)) return fail(UC_E_INVALID, "bad dtype %d", dt);
  if (n_copies > 0 && (st = check_ints("copies", copies))) return st;
  return launched(launch_page_append(pc, k_new, v_new, dt, ld, T, slots, copies, n_copies, (hipStream_t)stream));
}

uc_status uc_page_read(const uc_page_cache* cache, const int32_t* slots, int T, void* k_out, void* v_out, uc_dtype dt,
                       int64_t ld, void* stream) {
  PageCache pc;
  uc_status st = check_cache(cache, pc);
  if (st) return st;
  if (T < 0) return fail(UC_E_INVALID, "T must be >= 0 (got %d)", T);
  if ((int64_t)T * pc.Hkv > kMostRows) return fail(UC_E_UNSUPPORTED, "too many rows for one call");
  if (T == 0 && !dtype_ok(dt)) return fail(UC_E_INVALID, "bad dtype %d", dt);
  if (T > 0 && ((st = check_rows("k_out", k_out, dt, ld, (int64_t)pc.Hkv * pc.D)) ||
                (st = check_rows("v_out", v_out, dt, ld, (int64_t)pc.Hkv * pc.D)) || (st = check_ints("slots", slots))))
    return st;
  return launched(launch_page_read(pc, slots, T, k_out, v_out, dt, ld, (hipStream_t)stream));
}

size_t uc_page_attend_workspace_size(const uc_page_cache* cache, int Hq, int T, int S, int max_q) {
  PageCache pc;
  if (check_cache(cache, pc) || Hq < 1 || Hq % pc.Hkv || T < 0 || S < 1 || max_q < 1) return 0;
  return page_attend_workspace(pc, Hq / pc.Hkv, S, max_q);
}

uc_status uc_page_attend(const uc_page_cache* cache, int Hq, const void* q, uc_dtype q_dt, int64_t q_ld, int T, int S,
                         int max_q, const int32_t* q_start, const int32_t* len, const int32_t* table, int table_ld,
                         float sm_scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  PageCache pc;
  uc_status st = check_cache(cache, pc);
  if (st) return st;
  if (Hq < 1 || Hq % pc.Hkv) return fail(UC_E_INVALID, "Hq %d is not a multiple of Hkv %d", Hq, pc.Hkv);
  if (T < 0 || S < 1 || max_q < 1 || table_ld < 1)
    return fail(UC_E_INVALID, "T must be >= 0, S, max_q and table_ld >= 1 (got %d, %d, %d, %d)", T, S, max_q, table_ld);
  if (!dtype_ok(q_dt)) return fail(UC_E_INVALID, "bad q dtype %d", q_dt);
  if (!(sm_scale > 0.0f) || !isfinite(sm_scale * kLog2e)) return fail(UC_E_INVALID, "sm_scale must be finite and > 0");
  if ((int64_t)T * Hq > INT32_MAX) return fail(UC_E_UNSUPPORTED, "too many query rows");
  // units of work: tiles of 64 rows and what a block counts beside them, for
  // every block of few query rows and of 256, taken as 128
  const int64_t tiles = ((int64_t)table_ld * cache->page_rows + 63) / 64 + kStart;
  if (tiles > INT32_MAX / 64 || tiles * ((int64_t)S * kFewBlocks + (int64_t)T * (Hq / pc.Hkv) / 128) > INT32_MAX)
    return fail(UC_E_UNSUPPORTED, "tables of %d pages for %d sequences and %d tokens hold too much work for one call",
                table_ld, S, T);
  if ((st = check_ints("q_start", q_start)) || (st = check_ints("len", len)) || (st = check_ints("table", table)))
    return st;
  if (T == 0) return ok();
  if ((st = check_rows("q", q, q_dt, q_ld, (int64_t)Hq * pc.D)) ||
      (st = check_rows("o", o, q_dt, (int64_t)Hq * pc.D, (int64_t)Hq * pc.D)))
    return st;
  const char *q0 = (const char*)q, *o0 = (const char*)o;
  const int64_t size = q_dt == UC_F32 ? 4 : 2, row = (int64_t)Hq * pc.D;
  if (q0 < o0 + T * row * size && o0 < q0 + ((T - 1) * q_ld + row) * size)
    return fail(UC_E_INVALID, "q and o overlap");
  if (lse && !aligned4(lse)) return fail(UC_E_INVALID, "lse is not 4-byte aligned");
  const size_t need = page_attend_workspace(pc, Hq / pc.Hkv, S, max_q);
  if (!ws || !aligned16(ws) || ws_bytes < need)
    return fail(UC_E_WORKSPACE, "workspace %zu < %zu bytes, or not 16-byte aligned", ws_bytes, need);
  const PageAttendArgs a{pc, q_start, len, table, q, o, lse, q_ld, S, T, table_ld, Hq / pc.Hkv, sm_scale * kLog2e};
  const bool valu = q_dt == UC_F32 || current_path() == UC_PATH_VALU;
  return launched(launch_page_attend(a, q_dt, max_q, valu, ws, (hipStream_t)stream));
}

size_t uc_beam_select_workspace_size(int R, int W, int V) {
  if (R < 1 || W < 1 || W > UC_MAX_BEAMS || V < W || (int64_t)W * V > kMostIndex || (int64_t)R * W > (1 << 23)) return 0;
  return beam_select_workspace(R, W, V);
}

uc_status uc_beam_select(int R, int W, int V, const void* logits, uc_dtype dt, int64_t ld, const float* score,
                         const uint8_t* done, int eos, int pad, float* score_out, int32_t* parent, int32_t* token,
                         uint8_t* done_out, void* ws, size_t ws_bytes, void* stream) {
  if (R < 1 || W < 1 || W > UC_MAX_BEAMS)
    return fail(UC_E_INVALID, "R %d must be >= 1 and W %d in [1,%d]", R, W, UC_MAX_BEAMS);
  if (V < W || (int64_t)W * V > kMostIndex) return fail(UC_E_INVALID, "V %d must be at least W, W * V <= 2^30", V);
  if ((int64_t)R * W > (1 << 23)) return fail(UC_E_UNSUPPORTED, "more than 2^23 beams");
  if (!dtype_ok(dt)) return fail(UC_E_INVALID, "bad dtype %d", dt);
  if (!logits || ((uintptr_t)logits & (dt == UC_F32 ? 3u : 1u)))
    return fail(UC_E_INVALID, "logits is NULL or not aligned to its type");
  if (ld < V) return fail(UC_E_INVALID, "ld %lld < V %d", (long long)ld, V);
  if (pad < 0 || pad >= V) return fail(UC_E_INVALID, "pad %d not in [0,%d)", pad, V);
  if (eos < -1 || eos >= V) return fail(UC_E_INVALID, "eos %d not in [-1,%d)", eos, V);
  uc_status st;
  if ((st = check_ints("score", score)) || (st = check_ints("score_out", score_out)) ||
      (st = check_ints("parent", parent)) || (st = check_ints("token", token)))
    return st;
  const size_t need = beam_select_workspace(R, W, V);
  if (!ws || !aligned16(ws) || ws_bytes < need)
    return fail(UC_E_WORKSPACE, "workspace %zu < %zu bytes, or not 16-byte aligned", ws_bytes, need);
  return launched(launch_beam_select(logits, dt, ld, score, done, R, W, V, eos, pad, score_out, parent, token,
                                     done_out, ws, (hipStream_t)stream));
}

uc_status uc_beam_reorder(int R, int W, const int32_t* parent, const int32_t* token, const int32_t* table,
                          int table_ld, const int32_t* len, int page_rows, int32_t* table_out, int32_t* copies,
                          const int32_t* history, int32_t* history_out, int64_t history_ld, int n_history,
                          void* stream) {
  uc_status st = check_paging(page_rows, 1);
  if (st) return st;
  if (R < 1 || W < 1 || W > UC_MAX_BEAMS)
    return fail(UC_E_INVALID, "R %d must be >= 1 and W %d in [1,%d]", R, W, UC_MAX_BEAMS);
  if ((int64_t)R * W > (1 << 23)) return fail(UC_E_UNSUPPORTED, "more than 2^23 beams");
  if (table_ld < 1 || table_ld > (1 << 22)) return fail(UC_E_INVALID, "table_ld %d not in [1,2^22]", table_ld);
  if ((st = check_ints("parent", parent)) || (st = check_ints("table", table)) || (st = check_ints("len", len)) ||
      (st = check_ints("table_out", table_out)) || (st = check_ints("copies", copies)))
    return st;
  if (history) {
    if ((st = check_ints("history", history)) || (st = check_ints("history_out", history_out)) ||
        (st = check_ints("token", token)))
      return st;
    if (n_history < 0 || n_history >= history_ld || n_history > (1 << 22))
      return fail(UC_E_INVALID, "n_history %d must be >= 0, below history_ld %lld and at most 2^22", n_history,
                  (long long)history_ld);
  }
  return launched(launch_beam_reorder(parent, token, table, len, R, W, table_ld, __builtin_ctz(page_rows), table_out,
                                      copies, history, history_out, history_ld, n_history, (hipStream_t)stream));
}

}  // extern "C"
