// Host side of the cache in pages (ckv_paged_* in include/ckv.h): argument checks and launches.  Nothing is kept between calls.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ckv_paged_host.h"
#include "ckv_paged_kernels.h"

using namespace ckv;

static_assert(CKV_PAGED_BAD_PAGE == PAGED_BAD_PAGE && CKV_PAGED_BAD_LENGTH == PAGED_BAD_LENGTH && CKV_PAGED_BAD_PICK == PAGED_BAD_PICK, "status bits");

namespace {

int check_query(const ckv_pages* p, const ckv_query* q) {
  if (!q || !q->q || !aligned(q->q, 16)) return fail(CKV_EINVAL, "q must be a 16-byte aligned device address");
  if (int rc = check_heads(p, q->n_q_heads)) return rc;
  if (!stride_ok(q->seq_stride, kDim, 8) || !stride_ok(q->head_stride, kDim, 8)) return fail(CKV_EINVAL, "strides of q must be at least 128 elements and multiples of 8");
  return CKV_OK;
}

// How an attention is cut, and what its pieces leave in the workspace.
struct Split {
  AttendPlan plan;
  size_t partial, ml, parts;    // bytes
  size_t bytes() const { return partial + ml + parts; }
};
// Entries of a unit at most.
long long unit_entries(const ckv_pages* p, const ckv_seqs* s, int n_picked) { return n_picked > 0 ? (long long)n_picked * p->page_size : s->max_length; }
int check_entries(const ckv_pages* p, const ckv_seqs* s, int n_picked) {
  if ((long long)n_picked * p->page_size > kMaxLength) return fail(CKV_EINVAL, "too many pages picked");
  if ((long long)s->batch * p->n_kv_heads * unit_blocks((int)unit_entries(p, s, n_picked)) > (1ll << 30)) return fail(CKV_EINVAL, "too many entries in all (2^35)");
  return CKV_OK;
}
Split split_entries(const ckv_pages* p, const ckv_seqs* s, int n_q_heads, int entries, bool same, int n_cu) {
  const long long units = (long long)s->batch * p->n_kv_heads;
  Split r{};
  r.plan = attend_plan(units, entries, same, n_cu);
  if (r.plan.split) {
    const size_t G = (size_t)(n_q_heads / p->n_kv_heads);
    r.partial = up256((size_t)r.plan.pieces * G * kDim * 4);
    r.ml = up256((size_t)r.plan.pieces * G * 8);
    r.parts = up256((size_t)units * 8);
  }
  return r;
}
Split split_of(const ckv_pages* p, const ckv_seqs* s, int n_q_heads, int n_picked, int n_cu) {
  return split_entries(p, s, n_q_heads, (int)unit_entries(p, s, n_picked), n_picked > 0, n_cu);
}
// Of tokens that look back through a window: units whose window is shorter than sequences may be have as much to do each, as a rule.
Split split_window(const ckv_pages* p, const ckv_seqs* s, int n_q_heads, const ckv_mask* m, int n_cu) {
  const long long seen = m->window ? 32 * (((long long)m->sinks + 31) / 32 + ((long long)m->window + 31) / 32 + 1) : s->max_length;
  return split_entries(p, s, n_q_heads, (int)std::min<long long>(seen, s->max_length), m->window > 0 && m->window < s->max_length, n_cu);
}
int score_columns(const ckv_pages* p, const ckv_seqs* s) { return (int)(((long long)s->max_length + p->page_size - 1) / p->page_size); }
size_t score_bytes(const ckv_pages* p, const ckv_seqs* s, int n_cu) {
  const int units = s->batch * p->n_kv_heads, columns = score_columns(p, s);
  return selects_whole(units, columns, n_cu) ? 0 : up256((size_t)units * columns * 4);
}

// `c`: what is the call's own of pages picked or a window.
int attend(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_query* query, const Split& s, Attend c, bool window, float scale_log2e, void* out, int32_t out_dtype, float* lse,
           void* workspace, size_t workspace_bytes, void* stream, const char* what) {
  const int G = query->n_q_heads / pages->n_kv_heads;
  if (!launches(s.plan.pieces, kThreads)) return fail(CKV_EINVAL, "too many sequences times KV heads for one attention (2^24)");
  if (s.bytes() > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes())) return fail(CKV_EWORKSPACE, "workspace too small or misaligned");
  const Paged p = paged_of(pages, seqs);
  c.q = (const uint8_t*)query->q;
  c.q_seq_stride = query->seq_stride * 2;
  c.q_head_stride = query->head_stride * 2;
  c.out = (uint8_t*)out;
  c.out_bf16 = out_dtype == CKV_BF16;
  c.lse = lse;
  c.partial = (float*)workspace;
  c.ml = (float*)((char*)workspace + s.partial);
  c.scale_log2e = scale_log2e;
  c.G = G;
  if (s.plan.split) c.parts = (int32_t*)((char*)workspace + s.partial + s.ml);
  c.share = s.plan.share;
  c.places = s.plan.places;
  c.workers = s.plan.workers;
  const dim3 grid((unsigned)s.plan.pieces);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, p, c); };
  auto attend = [&](auto windowed) {
    constexpr bool WINDOW = decltype(windowed)::value;
    if (pages->dtype == CKV_E4M3) G > 8 ? launch(paged_attend_kernel<true, true, WINDOW>) : launch(paged_attend_kernel<true, false, WINDOW>);
    else G > 8 ? launch(paged_attend_kernel<false, true, WINDOW>) : launch(paged_attend_kernel<false, false, WINDOW>);
  };
  window ? attend(std::true_type()) : attend(std::false_type());
  if (int rc = launched(what)) return rc;
  if (!s.plan.split) return CKV_OK;
  const unsigned units = (unsigned)(seqs->batch * pages->n_kv_heads);
  const int heads = (int)units > compute_units() ? std::min(G, kJoinRows) : 1;
  auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(units, (unsigned)((G + heads - 1) / heads)), dim3(32 * kJoinRows), 0, (hipStream_t)stream, c, heads); };
  window ? join(paged_join_kernel<true>) : join(paged_join_kernel<false>);
  return launched(what);
}

}  // namespace

namespace ckv {
size_t one_row_workspace(const ckv_pages* pages, const ckv_seqs* seqs, int n_q_heads, const ckv_mask* mask) {
  return split_window(pages, seqs, n_q_heads, mask, compute_units()).bytes();
}
int attend_one_row(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_query* query, const int32_t* first, const ckv_mask* mask, float scale_log2e, void* out, int32_t out_dtype,
                   float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Attend c{};
  c.first = first;
  c.window = mask->window;
  c.sinks = mask->sinks;
  c.lower = lowered_by(seqs->max_length);
  return attend(pages, seqs, query, split_window(pages, seqs, query->n_q_heads, mask, compute_units()), c, true, scale_log2e, out, out_dtype, lse, workspace, workspace_bytes, stream,
                "ckv_paged_attend_rows");
}
}  // namespace ckv

namespace ckv {
const char* thread_error() { return t_error; }
}  // namespace ckv

extern "C" {

int ckv_paged_append(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_rows* rows, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (int rc = check_rows(rows)) return rc;
  if (seqs->max_length == 0 || nothing(rows)) return CKV_OK;
  const Paged p = paged_of(pages, seqs);
  const Rows r = rows_of(rows);
  unsigned touched;
  if (int rc = touched_pages(pages, seqs, rows, touched)) return rc;
  const dim3 grid((unsigned)(seqs->batch * pages->n_kv_heads), touched);
  auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3((unsigned)threads), 0, (hipStream_t)stream, p, r); };
  const bool e4m3 = pages->dtype == CKV_E4M3;
  if (appends_by_wave(pages->page_size, rows->rows, (long long)grid.x * grid.y, compute_units())) e4m3 ? launch(paged_append_kernel<true, 64>, 64) : launch(paged_append_kernel<false, 64>, 64);
  else e4m3 ? launch(paged_append_kernel<true, kThreads>, kThreads) : launch(paged_append_kernel<false, kThreads>, kThreads);
  return launched("ckv_paged_append");
}

int ckv_paged_read(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_rows* rows, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (int rc = check_rows(rows)) return rc;
  if (seqs->max_length == 0 || nothing(rows)) return CKV_OK;
  const Paged p = paged_of(pages, seqs);
  const Rows r = rows_of(rows);
  const long long pieces = (std::min<long long>(rows->rows, seqs->max_length) + kReadRows - 1) / kReadRows;
  if (pieces > kMaxGrid) return fail(CKV_EINVAL, "too many rows for one call");
  const dim3 grid((unsigned)(seqs->batch * pages->n_kv_heads), (unsigned)pieces);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, p, r); };
  const bool past = reads_past_caches((rows->starts ? (long long)rows->total : (long long)seqs->batch * std::min(rows->rows, seqs->max_length)) * pages->n_kv_heads);
  if (pages->dtype == CKV_E4M3) past ? launch(paged_read_kernel<true, true>) : launch(paged_read_kernel<true, false>);
  else past ? launch(paged_read_kernel<false, true>) : launch(paged_read_kernel<false, false>);
  return launched("ckv_paged_read");
}

size_t ckv_paged_workspace_bytes(const ckv_pages* pages, const ckv_seqs* seqs, int32_t n_q_heads, int32_t n_picked) {
  if (check(pages, seqs) != CKV_OK) return 0;
  if (check_heads(pages, n_q_heads) != CKV_OK) return 0;
  if (n_picked == -1) return std::max<size_t>(256, score_bytes(pages, seqs, compute_units()));
  if (n_picked < 0) {
    fail(CKV_EINVAL, "n_picked must be -1 (a selection), 0 (all entries) or a number of pages");
    return 0;
  }
  if (check_entries(pages, seqs, n_picked) != CKV_OK) return 0;
  return std::max<size_t>(256, split_of(pages, seqs, n_q_heads, n_picked, compute_units()).bytes());
}

int ckv_paged_attend(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_query* query, float softmax_scale, const int32_t* picked, int32_t n_picked, void* out,
                     int32_t out_dtype, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (int rc = check_query(pages, query)) return rc;
  if (!out || !aligned(out, 16)) return fail(CKV_EINVAL, "out must be a 16-byte aligned device address");
  if (out_dtype != CKV_F32 && out_dtype != CKV_BF16) return fail(CKV_EINVAL, "out_dtype must be CKV_F32 or CKV_BF16");
  const float scale_log2e = softmax_scale * 1.44269504088896340736f;
  if (!(softmax_scale > 0.0f) || !std::isfinite(scale_log2e)) return fail(CKV_EINVAL, "softmax_scale must be positive and below 2.3e38");
  if (picked ? n_picked < 1 : n_picked != 0) return fail(CKV_EINVAL, "n_picked must be positive with a list of pages and 0 without");
  if (int rc = check_entries(pages, seqs, n_picked)) return rc;
  Attend c{};
  c.picked = picked;
  c.n_picked = n_picked;
  return attend(pages, seqs, query, split_of(pages, seqs, query->n_q_heads, n_picked, compute_units()), c, false, scale_log2e, out, out_dtype, lse, workspace, workspace_bytes, stream,
                "ckv_paged_attend");
}

int ckv_paged_select(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_query* query, int32_t keep, int32_t keep_first, int32_t keep_last, int32_t* picked,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (int rc = check_query(pages, query)) return rc;
  if (!pages->bounds) return fail(CKV_EINVAL, "the cache keeps no bounds");
  if (!picked) return fail(CKV_EINVAL, "picked is NULL");
  if (keep < 1 || keep > kMaxPicked || keep_first < 0 || keep_last < 0 || keep_first > keep || keep_last > keep - keep_first)
    return fail(CKV_EINVAL, "need 1 <= keep <= 32768 and keep_first + keep_last <= keep");
  const int columns = score_columns(pages, seqs);
  if (columns > kMaxPicked) return fail(CKV_EINVAL, "a selection chooses from 32768 pages of a sequence at most");
  const Paged p = paged_of(pages, seqs);
  Select c{};
  c.q = (const uint8_t*)query->q;
  c.q_seq_stride = query->seq_stride * 2;
  c.q_head_stride = query->head_stride * 2;
  c.scores = (float*)workspace;
  c.picked = picked;
  c.G = query->n_q_heads / pages->n_kv_heads;
  c.keep = keep;
  c.keep_first = keep_first;
  c.keep_last = keep_last;
  c.score_stride = columns;
  const unsigned units = (unsigned)(seqs->batch * pages->n_kv_heads);
  if (!launches(units, columns > 4 * kPickThreads ? kWideThreads : kPickThreads)) return fail(CKV_EINVAL, "too many sequences times KV heads for one selection (2^23; 2^22 of more than 2048 pages)");
  const int n_cu = compute_units();
  const bool past = bounds_past_caches(units, columns);
  if (selects_whole((int)units, columns, n_cu)) {
    auto select = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(units), dim3(kPickThreads), 0, (hipStream_t)stream, p, c); };
    past ? select(paged_select_kernel<true>) : select(paged_select_kernel<false>);
    return launched("ckv_paged_select");
  }
  if (columns > keep) {
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < score_bytes(pages, seqs, n_cu)) return fail(CKV_EWORKSPACE, "workspace too small or misaligned");
    const int each = score_pages_each((int)units, columns, n_cu);
    const dim3 grid(units, (unsigned)((columns + each - 1) / each));
    auto score = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, p, c, each); };
    past ? score(paged_score_kernel<true>) : score(paged_score_kernel<false>);
    if (int rc = launched("ckv_paged_select")) return rc;
  }
  auto pick = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(units), dim3((unsigned)threads), 0, (hipStream_t)stream, p, c); };
  if (columns <= 2 * kPickThreads) pick(paged_pick_kernel<2, kPickThreads>, kPickThreads);
  else if (columns <= 4 * kPickThreads) pick(paged_pick_kernel<4, kPickThreads>, kPickThreads);
  else if (columns <= 4 * kWideThreads) pick(paged_pick_kernel<4, kWideThreads>, kWideThreads);
  else if (columns <= 8 * kWideThreads) pick(paged_pick_kernel<8, kWideThreads>, kWideThreads);
  else pick(paged_pick_kernel<32, kWideThreads>, kWideThreads);
  return launched("ckv_paged_select");
}

}  // extern "C"
