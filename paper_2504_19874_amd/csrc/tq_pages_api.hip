// The C ABI of the paged 8-bit cache: checks of arguments, workspaces, launches (include/turboquant.h).
#include <algorithm>
#include <climits>
#include <cstdint>

#include "tq_pages.h"

using namespace tq;

namespace {

constexpr int64_t kMaxPoolPages = 1 << 22;

bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

tq_status check_pages(const tq_pages* c) {
  if (c == nullptr || c->d <= 0 || c->n_heads <= 0 || c->page_tokens <= 0 || c->n_pages <= 0) return TQ_ERR_INVALID_ARG;
  if (c->type != TQ_PAGE_E4M3 && c->type != TQ_PAGE_I8) return TQ_ERR_INVALID_ARG;
  if (c->d != 64 && c->d != 128 && c->d != 256) return TQ_ERR_UNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return TQ_ERR_UNSUPPORTED;
  if (c->n_heads > 65535 / 2 || c->n_pages > INT_MAX) return TQ_ERR_UNSUPPORTED;
  if (c->n_pages > (int64_t(1) << 34) / ((int64_t)c->n_heads * c->page_tokens)) return TQ_ERR_UNSUPPORTED;
  return TQ_OK;
}
tq_status check_store(const tq_pages* c) {
  if (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return TQ_ERR_INVALID_ARG;
  if (misaligned(c->k) || misaligned(c->v) || misaligned(c->k_scale, 4) || misaligned(c->v_scale, 4) || misaligned(c->bounds)) return TQ_ERR_UNSUPPORTED;
  return TQ_OK;
}

tq_status check_batch(const tq_batch* b) {
  if (b == nullptr || b->n_seqs < 0 || b->max_new < 0 || b->n_rows < 0 || b->width < 0 || b->table_stride < b->width) return TQ_ERR_INVALID_ARG;
  if (b->n_rows > INT_MAX) return TQ_ERR_UNSUPPORTED;
  return TQ_OK;
}
bool batch_arrays(const tq_batch* b) { return (b->table != nullptr || b->width == 0) && b->lens != nullptr; }

tq_status check_rows(const void* p, int32_t dtype, int64_t ld_row, int64_t ld_head, int d) {
  if (p == nullptr || ld_row < 0 || ld_head < 0) return TQ_ERR_INVALID_ARG;
  const int64_t unit = dtype == TQ_F32 ? 4 : 8;
  if (misaligned(p) || ld_row % unit != 0 || ld_head % unit != 0) return TQ_ERR_UNSUPPORTED;
  return TQ_OK;
}

int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

PagesView view(const tq_pages* c) {
  PagesView v;
  v.k = static_cast<uint8_t*>(c->k), v.v = static_cast<uint8_t*>(c->v);
  v.k_scale = c->k_scale, v.v_scale = c->v_scale;
  v.bounds = c->bounds, v.refs = c->refs;
  v.n_pages = (int)c->n_pages, v.heads = c->n_heads, v.log2_page = log2_of(c->page_tokens);
  return v;
}
BatchView view(const tq_batch* b) {
  BatchView v;
  v.table = b->table, v.lens = b->lens, v.starts = b->starts;
  v.table_stride = b->table_stride, v.n_rows = b->n_rows;
  v.width = b->width, v.n_seqs = b->n_seqs, v.max_new = b->max_new;
  return v;
}

// (what a launch does not take is refused before any is made)
tq_status from_hip(hipError_t e) { return e == hipSuccess ? TQ_OK : e == hipErrorInvalidConfiguration ? TQ_ERR_UNSUPPORTED : TQ_ERR_HIP; }

// what attend, its workspace and select share
tq_status check_queries(const tq_pages* c, const tq_batch* b, int32_t n_heads_q) {
  tq_status st = check_pages(c);
  if (st != TQ_OK) return st;
  st = check_batch(b);
  if (st != TQ_OK) return st;
  if (n_heads_q <= 0 || n_heads_q % c->n_heads != 0) return TQ_ERR_INVALID_ARG;
  return TQ_OK;
}

// products of sizes that the kernels hold in an int
bool launchable(int64_t a, int64_t b, int64_t c) {
  const int64_t most = INT_MAX;
  return a <= most && b <= most && a * b <= most && c <= most && a * b * c <= most;
}

// the grids of attend: ranges of keys at most 64
bool attend_fits(const tq_batch* b, int heads, int group, bool chosen) {
  const int64_t rows = (chosen ? 1 : (int64_t)b->max_new) * group;
  return rows <= INT_MAX - 16 && launchable((int64_t)b->n_seqs * (chosen ? b->max_new : 1), heads, (rows + 15) / 16) &&
         launchable((int64_t)b->n_seqs * b->max_new, (int64_t)heads * group, 1);
}
size_t attend_part_bytes(const tq_pages* c, const tq_batch* b, bool f32, int group, bool chosen, int n_chosen, int window, PagesAttendPlan* plan) {
  const BatchView v = view(b);
  const PagesAttendPlan n = pages_attend_plan(
      c->d, f32, pages_attend_sizes(v, c->n_heads, group, chosen, n_chosen, log2_of(c->page_tokens), window > 0 ? window : INT_MAX), device_cu_count());
  if (plan != nullptr) *plan = n;
  return pages_attend_part_bytes(c->d, v, c->n_heads, group, n.splits);
}

size_t pool_bytes(const tq_pages* c, int64_t n) { return (size_t)(3 * c->n_pages + 2 * n + 64) * sizeof(int32_t); }

tq_status check_pool(const tq_pages* c, const tq_batch* b, int64_t n) {
  tq_status st = check_pages(c);
  if (st != TQ_OK) return st;
  st = check_store(c);
  if (st != TQ_OK) return st;
  if (b != nullptr) {
    st = check_batch(b);
    if (st != TQ_OK) return st;
  }
  if (c->refs == nullptr) return TQ_ERR_INVALID_ARG;
  if (c->n_pages > kMaxPoolPages || (int64_t)c->n_heads * c->page_tokens * c->d > (1 << 28)) return TQ_ERR_UNSUPPORTED;
  if (n >= 0 && (c->workspace == nullptr || c->workspace_bytes < pool_bytes(c, n) || misaligned(c->workspace))) return TQ_ERR_WORKSPACE;
  return TQ_OK;
}

}  // namespace

extern "C" {

tq_status tq_pages_append(const tq_pages* c, const tq_batch* b, const void* k, const void* v, int32_t dtype, int64_t ld_row, int64_t ld_head,
                          void* stream) {
  tq_status st = check_pages(c);
  if (st != TQ_OK) return st;
  st = check_batch(b);
  if (st != TQ_OK) return st;
  if (dtype != TQ_F32 && dtype != TQ_BF16) return TQ_ERR_INVALID_ARG;
  if (b->n_seqs == 0 || b->max_new == 0 || b->n_rows == 0 || b->width == 0) return TQ_OK;
  st = check_store(c);
  if (st != TQ_OK) return st;
  if (!batch_arrays(b)) return TQ_ERR_INVALID_ARG;
  st = check_rows(k, dtype, ld_row, ld_head, c->d);
  if (st != TQ_OK) return st;
  st = check_rows(v, dtype, ld_row, ld_head, c->d);
  if (st != TQ_OK) return st;
  if (!launchable(b->n_seqs, std::min<int64_t>(((int64_t)b->max_new + c->page_tokens - 2) / c->page_tokens + 1, b->width), 1)) return TQ_ERR_UNSUPPORTED;
  return from_hip(launch_pages_append(c->d, c->type, dtype == TQ_F32, view(c), view(b), PagesRows{k, ld_row, ld_head}, PagesRows{v, ld_row, ld_head},
                                      static_cast<hipStream_t>(stream)));
}

size_t tq_pages_attend_workspace_bytes(const tq_pages* c, const tq_batch* b, int32_t n_heads_q, int32_t n_chosen, int32_t window) {
  if (check_queries(c, b, n_heads_q) != TQ_OK || n_chosen < 0 || window < 0) return 0;
  if (!attend_fits(b, c->n_heads, n_heads_q / c->n_heads, n_chosen > 0)) return 0;
  const int group = n_heads_q / c->n_heads;
  const size_t f32 = attend_part_bytes(c, b, true, group, n_chosen > 0, n_chosen, window, nullptr);
  const size_t bf16 = attend_part_bytes(c, b, false, group, n_chosen > 0, n_chosen, window, nullptr);
  return f32 > bf16 ? f32 : bf16;
}

tq_status tq_pages_attend(const tq_pages* c, const tq_batch* b, const void* q, int32_t dtype, int64_t ldq_row, int64_t ldq_head, int32_t n_heads_q,
                          float scale, int32_t window, const int32_t* chosen, int32_t n_chosen, void* out, int64_t ldo_row, int64_t ldo_head,
                          float* lse, void* stream) {
  tq_status st = check_queries(c, b, n_heads_q);
  if (st != TQ_OK) return st;
  if ((dtype != TQ_F32 && dtype != TQ_BF16) || window < 0 || n_chosen < 0) return TQ_ERR_INVALID_ARG;
  if (chosen != nullptr && (int64_t)n_chosen * c->page_tokens > INT_MAX - 127) return TQ_ERR_UNSUPPORTED;
  if (b->n_seqs == 0 || b->max_new == 0 || b->n_rows == 0) return TQ_OK;
  st = check_store(c);
  if (st != TQ_OK) return st;
  if (!batch_arrays(b)) return TQ_ERR_INVALID_ARG;
  st = check_rows(q, dtype, ldq_row, ldq_head, c->d);
  if (st != TQ_OK) return st;
  st = check_rows(out, dtype, ldo_row, ldo_head, c->d);
  if (st != TQ_OK) return st;
  PagesAttendArgs a;
  a.c = view(c), a.b = view(b);
  a.q = PagesRows{q, ldq_row, ldq_head}, a.out = PagesRows{out, ldo_row, ldo_head};
  a.lse = lse, a.chosen = chosen, a.n_chosen = n_chosen, a.group = n_heads_q / c->n_heads;
  const double scale2 = (double)scale * 1.4426950408889634074;
  a.scale2 = (float)scale2, a.scale2_rest = (float)(scale2 - (double)a.scale2);
  a.window = window > 0 ? window : INT_MAX;
  if (!attend_fits(b, c->n_heads, a.group, chosen != nullptr)) return TQ_ERR_UNSUPPORTED;
  PagesAttendPlan plan;
  const size_t need = attend_part_bytes(c, b, dtype == TQ_F32, a.group, chosen != nullptr, n_chosen, window, &plan);
  a.splits = plan.splits, a.prompt = plan.prompt, a.tiles = plan.tiles;
  if (need > 0 && (c->workspace == nullptr || c->workspace_bytes < need || misaligned(c->workspace))) return TQ_ERR_WORKSPACE;
  a.part = static_cast<float*>(c->workspace);
  return from_hip(launch_pages_attend(c->d, c->type, dtype == TQ_F32, a, static_cast<hipStream_t>(stream)));
}

size_t tq_pages_select_workspace_bytes(const tq_pages* c, const tq_batch* b) {
  if (check_pages(c) != TQ_OK || check_batch(b) != TQ_OK) return 0;
  if (!launchable((int64_t)b->n_seqs * b->max_new, c->n_heads, 1) || !pages_pick_fits(view(b), c->n_heads)) return 0;
  return (size_t)b->n_rows * c->n_heads * b->width * sizeof(float);
}

tq_status tq_pages_select(const tq_pages* c, const tq_batch* b, const void* q, int32_t dtype, int64_t ldq_row, int64_t ldq_head, int32_t n_heads_q,
                          int32_t keep_first, int32_t keep_last, int32_t* chosen, int32_t n_chosen, void* stream) {
  tq_status st = check_queries(c, b, n_heads_q);
  if (st != TQ_OK) return st;
  if ((dtype != TQ_F32 && dtype != TQ_BF16) || n_chosen < 1 || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > n_chosen)
    return TQ_ERR_INVALID_ARG;
  if (n_chosen > 1024 || b->width > 65536) return TQ_ERR_UNSUPPORTED;
  if (b->n_seqs == 0 || b->max_new == 0 || b->n_rows == 0) return TQ_OK;
  if (chosen == nullptr || c->bounds == nullptr || !batch_arrays(b)) return TQ_ERR_INVALID_ARG;
  if (misaligned(c->bounds)) return TQ_ERR_UNSUPPORTED;
  st = check_rows(q, dtype, ldq_row, ldq_head, c->d);
  if (st != TQ_OK) return st;
  if (!launchable((int64_t)b->n_seqs * b->max_new, c->n_heads, (b->width + 63) / 64) || !pages_pick_fits(view(b), c->n_heads)) return TQ_ERR_UNSUPPORTED;
  const size_t need = tq_pages_select_workspace_bytes(c, b);
  if (need > 0 && (c->workspace == nullptr || c->workspace_bytes < need || misaligned(c->workspace))) return TQ_ERR_WORKSPACE;
  PagesSelectArgs a;
  a.c = view(c), a.b = view(b), a.q = PagesRows{q, ldq_row, ldq_head};
  a.group = n_heads_q / c->n_heads, a.keep_first = keep_first, a.keep_last = keep_last, a.n_chosen = n_chosen, a.chosen = chosen;
  a.scores = static_cast<float*>(c->workspace);
  return from_hip(launch_pages_select(c->d, dtype == TQ_F32, a, static_cast<hipStream_t>(stream)));
}

size_t tq_pages_pool_workspace_bytes(const tq_pages* c, int64_t n) {
  if (check_pages(c) != TQ_OK || n < 0 || n > INT_MAX) return 0;
  return pool_bytes(c, n);
}

tq_status tq_pages_reserve(const tq_pages* c, const tq_batch* b, int32_t* missing, void* stream) {
  if (b == nullptr) return TQ_ERR_INVALID_ARG;
  tq_status st = check_pool(c, b, 0);
  if (st != TQ_OK) return st;
  if (b->n_seqs > 0 && !batch_arrays(b)) return TQ_ERR_INVALID_ARG;
  if (!launchable((int64_t)b->n_seqs + 1024, std::min<int64_t>(b->max_new / c->page_tokens + 2, std::max(b->width, 1)), 1)) return TQ_ERR_UNSUPPORTED;
  return from_hip(launch_pages_reserve(view(c), view(b), static_cast<int32_t*>(c->workspace), missing, static_cast<hipStream_t>(stream)));
}

tq_status tq_pages_fork(const tq_pages* c, const tq_batch* b, const int32_t* parents, const int32_t* children, int32_t n, int32_t* missing,
                        void* stream) {
  if (b == nullptr || n < 0) return TQ_ERR_INVALID_ARG;
  tq_status st = check_pool(c, b, n);
  if (st != TQ_OK) return st;
  if (!grid_fits(n, 256)) return TQ_ERR_UNSUPPORTED;
  if (n > 0 && (parents == nullptr || children == nullptr || !batch_arrays(b))) return TQ_ERR_INVALID_ARG;
  int32_t* const list = static_cast<int32_t*>(c->workspace);
  return from_hip(launch_pages_fork(view(c), view(b), c->d, parents, children, n, list, list + (c->n_pages + 1) / 2 * 2, missing, static_cast<hipStream_t>(stream)));
}

tq_status tq_pages_free(const tq_pages* c, const tq_batch* b, const int32_t* rows, int32_t n, void* stream) {
  if (b == nullptr || n < 0) return TQ_ERR_INVALID_ARG;
  tq_status st = check_pool(c, b, -1);
  if (st != TQ_OK) return st;
  if (n == 0) return TQ_OK;
  if (!grid_fits(n, 256)) return TQ_ERR_UNSUPPORTED;
  if (rows == nullptr || !batch_arrays(b)) return TQ_ERR_INVALID_ARG;
  return from_hip(launch_pages_free(view(c), view(b), rows, n, static_cast<hipStream_t>(stream)));
}

tq_status tq_pages_compact(const tq_pages* c, const tq_batch* b, int32_t* n_live, void* stream) {
  if (b == nullptr) return TQ_ERR_INVALID_ARG;
  tq_status st = check_pool(c, b, 0);
  if (st != TQ_OK) return st;
  if (b->n_seqs > 0 && b->width > 0 && b->table == nullptr) return TQ_ERR_INVALID_ARG;
  int32_t* const plan = static_cast<int32_t*>(c->workspace);
  return from_hip(launch_pages_compact(view(c), view(b), c->d, plan, plan + 64, plan + 64 + 2 * c->n_pages, n_live, static_cast<hipStream_t>(stream)));
}

tq_status tq_pages_copy(const tq_pages* c, const int32_t* src, const int32_t* dst, int64_t n, void* stream) {
  tq_status st = check_pages(c);
  if (st != TQ_OK) return st;
  if (n < 0) return TQ_ERR_INVALID_ARG;
  if ((int64_t)c->n_heads * c->page_tokens * c->d > (1 << 28)) return TQ_ERR_UNSUPPORTED;
  if (n == 0) return TQ_OK;
  st = check_store(c);
  if (st != TQ_OK) return st;
  if (src == nullptr || dst == nullptr) return TQ_ERR_INVALID_ARG;
  return from_hip(launch_pages_copy(view(c), c->d, src, dst, n, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
