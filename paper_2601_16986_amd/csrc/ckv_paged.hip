// Host side of the cache in pages (ckv_paged_* in include/ckv.h): argument checks and launches.  Nothing is kept between calls.
#include "../../include/ckv.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "ckv_paged_kernels.h"

using namespace ckv;

static_assert(CKV_PAGED_BAD_PAGE == PAGED_BAD_PAGE && CKV_PAGED_BAD_LENGTH == PAGED_BAD_LENGTH && CKV_PAGED_BAD_PICK == PAGED_BAD_PICK, "status bits");

namespace {

// What the last failed call of this thread complained about (these calls have no context to keep it in).
thread_local char t_error[256];

int fail(int code, const char* what) {
  std::snprintf(t_error, sizeof t_error, "%s", what);
  return code;
}
int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return CKV_OK;
  std::snprintf(t_error, sizeof t_error, "%s: %s", what, hipGetErrorString(e));
  return CKV_EHIP;
}

constexpr long long kMaxLength = 1ll << 30;
constexpr int64_t kMaxStride = 1ll << 40;
constexpr int kMaxGrid = 65535;          // of the second and third axis

bool aligned(const void* p, uintptr_t to) { return (uintptr_t)p % to == 0; }
// a stride of so many elements, a multiple of `of`
bool stride_ok(int64_t s, int64_t least, int64_t of) { return s >= least && s % of == 0 && s < kMaxStride; }

int element(const ckv_pages* p) { return p->dtype == CKV_E4M3 ? 1 : 2; }

// Whether a launch of so many workgroups has fewer than 2^32 threads, the most that one axis takes.
bool launches(long long groups, int threads) { return groups * threads < (1ll << 32); }

int check(const ckv_pages* p, const ckv_seqs* s) {
  if (!p || !s) return fail(CKV_EINVAL, "pages or sequences are NULL");
  if (p->dtype != CKV_BF16 && p->dtype != CKV_E4M3) return fail(CKV_EINVAL, "dtype must be CKV_BF16 or CKV_E4M3");
  if (p->head_dim != kDim) return fail(CKV_EINVAL, "head_dim must be 128");
  if (p->n_pages < 1) return fail(CKV_EINVAL, "n_pages must be >= 1");
  if (p->page_size < kMinPage || p->page_size > kMaxPage || (p->page_size & (p->page_size - 1)) != 0) return fail(CKV_EINVAL, "page_size must be 16, 32, 64, 128 or 256");
  if (p->n_kv_heads < 1 || p->n_kv_heads > 1024) return fail(CKV_EINVAL, "n_kv_heads must be in [1, 1024]");
  if (!p->k || !p->v || !aligned(p->k, 16) || !aligned(p->v, 16)) return fail(CKV_EINVAL, "k and v must be 16-byte aligned device addresses");
  const int64_t of = 16 / element(p);
  if (!stride_ok(p->page_stride, kDim, of) || !stride_ok(p->head_stride, kDim, of) || !stride_ok(p->slot_stride, kDim, of))
    return fail(CKV_EINVAL, "strides of k and v must be at least a row and multiples of 16 bytes");
  if (p->slot_stride * element(p) * p->page_size >= (1ll << 31)) return fail(CKV_EINVAL, "a page's slots must lie within 2 GiB");
  if (p->dtype == CKV_E4M3) {
    if (!p->scales || !aligned(p->scales, 8)) return fail(CKV_EINVAL, "an e4m3 cache needs 8-byte aligned scales");
    if (!stride_ok(p->scale_page_stride, 2 * p->page_size, 8) || !stride_ok(p->scale_head_stride, 2 * p->page_size, 8))
      return fail(CKV_EINVAL, "strides of the scales must be at least a page's and multiples of 8 bytes");
  }
  if (p->bounds) {
    if (!aligned(p->bounds, 16)) return fail(CKV_EINVAL, "bounds must be 16-byte aligned");
    if (!stride_ok(p->bounds_page_stride, 2 * kDim, 8) || !stride_ok(p->bounds_head_stride, 2 * kDim, 8))
      return fail(CKV_EINVAL, "strides of the bounds must be at least 256 elements and multiples of 8");
  }
  if (!s->table || !s->lengths) return fail(CKV_EINVAL, "table or lengths is NULL");
  if (s->batch < 1 || s->columns < 1 || s->table_stride < s->columns || s->table_stride >= kMaxStride) return fail(CKV_EINVAL, "the table needs a row per sequence and a column per page");
  if (s->max_length < 0 || s->max_length > kMaxLength || s->max_length > (long long)s->columns * p->page_size)
    return fail(CKV_EINVAL, "max_length must be in [0, columns * page_size], at most 2^30");
  if (!launches((long long)s->batch * p->n_kv_heads, kThreads)) return fail(CKV_EINVAL, "too many sequences times KV heads (2^24)");
  return CKV_OK;
}

Paged paged_of(const ckv_pages* p, const ckv_seqs* s) {
  const int64_t e = element(p);
  Paged d{};
  d.k = (uint8_t*)p->k;
  d.v = (uint8_t*)p->v;
  d.scales = p->scales;
  d.bounds = (uint8_t*)p->bounds;
  d.status = p->status;
  d.table = s->table;
  d.lengths = s->lengths;
  d.page_stride = p->page_stride * e;
  d.head_stride = p->head_stride * e;
  d.slot_stride = (int32_t)(p->slot_stride * e);
  d.scale_page_stride = p->scale_page_stride;
  d.scale_head_stride = p->scale_head_stride;
  d.bounds_page_stride = p->bounds_page_stride * 2;
  d.bounds_head_stride = p->bounds_head_stride * 2;
  d.table_stride = s->table_stride;
  d.n_pages = p->n_pages;
  d.shift = __builtin_ctz((unsigned)p->page_size);
  d.hkv = p->n_kv_heads;
  d.batch = s->batch;
  d.columns = s->columns;
  d.max_length = s->max_length;
  return d;
}

// Packed rows of which there are none.
bool nothing(const ckv_rows* r) { return r->starts && r->total == 0; }

int check_rows(const ckv_rows* r) {
  if (!r) return fail(CKV_EINVAL, "rows are NULL");
  if (nothing(r)) return CKV_OK;
  if (!r->k || !r->v) return fail(CKV_EINVAL, "rows are NULL");
  if (!aligned(r->k, 16) || !aligned(r->v, 16)) return fail(CKV_EINVAL, "rows must be 16-byte aligned");
  if (r->rows < 1 || r->rows > kMaxLength) return fail(CKV_EINVAL, "rows must be in [1, 2^30]");
  if (!stride_ok(r->row_stride, kDim, 8) || !stride_ok(r->head_stride, kDim, 8) || (r->starts ? r->total < 0 : !stride_ok(r->seq_stride, kDim, 8)))
    return fail(CKV_EINVAL, "strides of the rows must be at least 128 elements and multiples of 8");
  return CKV_OK;
}

Rows rows_of(const ckv_rows* r) {
  return Rows{(uint8_t*)r->k, (uint8_t*)r->v, r->first, r->starts, r->seq_stride * 2, r->row_stride * 2, r->head_stride * 2, r->rows, r->total};
}

int check_heads(const ckv_pages* p, int n_q_heads) {
  if (n_q_heads < p->n_kv_heads || n_q_heads % p->n_kv_heads != 0) return fail(CKV_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
  if (n_q_heads / p->n_kv_heads > kPagedGroup) return fail(CKV_EINVAL, "at most 16 query heads per KV head");
  return CKV_OK;
}

int check_query(const ckv_pages* p, const ckv_query* q) {
  if (!q || !q->q || !aligned(q->q, 16)) return fail(CKV_EINVAL, "q must be a 16-byte aligned device address");
  if (int rc = check_heads(p, q->n_q_heads)) return rc;
  if (!stride_ok(q->seq_stride, kDim, 8) || !stride_ok(q->head_stride, kDim, 8)) return fail(CKV_EINVAL, "strides of q must be at least 128 elements and multiples of 8");
  return CKV_OK;
}

// Compute units of the current device.
int compute_units() {
  static int known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  n = __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
  if (n > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
  return n;
}

constexpr size_t up256(size_t x) { return (x + 255) / 256 * 256; }

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
Split split_of(const ckv_pages* p, const ckv_seqs* s, int n_q_heads, int n_picked, int n_cu) {
  const long long units = (long long)s->batch * p->n_kv_heads;
  Split r{};
  r.plan = attend_plan(units, (int)unit_entries(p, s, n_picked), n_picked > 0, n_cu);
  if (r.plan.split) {
    const size_t G = (size_t)(n_q_heads / p->n_kv_heads);
    r.partial = up256((size_t)r.plan.pieces * G * kDim * 4);
    r.ml = up256((size_t)r.plan.pieces * G * 8);
    r.parts = up256((size_t)units * 8);
  }
  return r;
}
int score_columns(const ckv_pages* p, const ckv_seqs* s) { return (int)(((long long)s->max_length + p->page_size - 1) / p->page_size); }
size_t score_bytes(const ckv_pages* p, const ckv_seqs* s, int n_cu) {
  const int units = s->batch * p->n_kv_heads, columns = score_columns(p, s);
  return selects_whole(units, columns, n_cu) ? 0 : up256((size_t)units * columns * 4);
}

}  // namespace

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
  const long long reach = std::min<long long>(rows->rows, seqs->max_length), touched = std::min<long long>((reach + pages->page_size - 2) / pages->page_size + 1, seqs->columns);
  if (touched > kMaxGrid) return fail(CKV_EINVAL, "rows of a call may reach 65535 pages of a sequence at most");
  const dim3 grid((unsigned)(seqs->batch * pages->n_kv_heads), (unsigned)touched);
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
  const int G = query->n_q_heads / pages->n_kv_heads;
  const Split s = split_of(pages, seqs, query->n_q_heads, n_picked, compute_units());
  if (!launches(s.plan.pieces, kThreads)) return fail(CKV_EINVAL, "too many sequences times KV heads for one attention (2^24)");
  if (s.bytes() > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes())) return fail(CKV_EWORKSPACE, "workspace too small or misaligned");
  const Paged p = paged_of(pages, seqs);
  Attend c{};
  c.q = (const uint8_t*)query->q;
  c.q_seq_stride = query->seq_stride * 2;
  c.q_head_stride = query->head_stride * 2;
  c.picked = picked;
  c.n_picked = n_picked;
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
  const bool wide = G > 8;
  if (pages->dtype == CKV_E4M3) wide ? launch(paged_attend_kernel<true, true>) : launch(paged_attend_kernel<true, false>);
  else wide ? launch(paged_attend_kernel<false, true>) : launch(paged_attend_kernel<false, false>);
  if (int rc = launched("ckv_paged_attend")) return rc;
  if (!s.plan.split) return CKV_OK;
  const unsigned units = (unsigned)(seqs->batch * pages->n_kv_heads);
  const int heads = (int)units > compute_units() ? std::min(G, kJoinRows) : 1;
  hipLaunchKernelGGL(paged_join_kernel, dim3(units, (unsigned)((G + heads - 1) / heads)), dim3(32 * kJoinRows), 0, (hipStream_t)stream, c, heads);
  return launched("ckv_paged_attend");
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
