// Host side of the calls on several rows of each sequence of a cache in pages: argument checks and launches.  Nothing is kept between calls.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ckv_paged_host.h"
#include "ckv_rotate_kernels.h"
#include "ckv_rows_kernels.h"

using namespace ckv;

namespace {

int check_row_heads(const ckv_pages* p, const ckv_heads* q, bool packed) {
  if (!q->q || !aligned(q->q, 16)) return fail(CKV_EINVAL, "q must be a 16-byte aligned device address");
  if (int rc = check_heads(p, q->n_q_heads)) return rc;
  if (!stride_ok(q->row_stride, kDim, 8) || !stride_ok(q->head_stride, kDim, 8) || (!packed && !stride_ok(q->seq_stride, kDim, 8)))
    return fail(CKV_EINVAL, "strides of q must be at least 128 elements and multiples of 8");
  return CKV_OK;
}

int check_rotation(const ckv_rotation* r) {
  if (!r || !r->frequencies || !aligned(r->frequencies, 8)) return fail(CKV_EINVAL, "frequencies must be 8-byte aligned doubles on the device");
  if (r->n_pairs < 8 || r->n_pairs > kDim / 2 || r->n_pairs % 8 != 0) return fail(CKV_EINVAL, "n_pairs must be a multiple of 8, at most 64");
  if (r->interleaved != 0 && r->interleaved != 1) return fail(CKV_EINVAL, "interleaved must be 0 or 1");
  if (!(r->magnitude > 0.0f) || !std::isfinite(r->magnitude)) return fail(CKV_EINVAL, "magnitude must be positive and finite");
  return CKV_OK;
}

int check_queries(const ckv_pages* p, const ckv_row_queries* q) {
  if (!q) return fail(CKV_EINVAL, "queries are NULL");
  const ckv_heads heads = {const_cast<void*>(q->q), q->seq_stride, q->row_stride, q->head_stride, q->n_q_heads};
  if (int rc = check_row_heads(p, &heads, q->starts)) return rc;
  if (q->starts && q->total < 0) return fail(CKV_EINVAL, "total must not be negative");
  return CKV_OK;
}

// Sizes of a call on several rows, without its buffers.
int check_sizes(const ckv_pages* p, const ckv_seqs* s, int rows, int n_q_heads, const ckv_mask* m) {
  if (int rc = check_heads(p, n_q_heads)) return rc;
  if (!m) return fail(CKV_EINVAL, "mask is NULL");
  if (rows < 1 || rows > kMaxLength) return fail(CKV_EINVAL, "rows must be in [1, 2^30]");
  if (std::min<long long>(rows, s->max_length) * (n_q_heads / p->n_kv_heads) >= (1ll << 31)) return fail(CKV_EINVAL, "too many rows times query heads per KV head (2^31)");
  if (m->window < 0 || m->sinks < 0 || (m->window == 0 && m->sinks != 0)) return fail(CKV_EINVAL, "window and sinks must not be negative, and sinks belong to a window");
  if (m->tree) {
    if (rows > kMaxDrafts) return fail(CKV_EINVAL, "a tree has at most 512 rows");
    if (m->window && m->window < rows) return fail(CKV_EINVAL, "a tree's window must hold all of its rows");
    if (m->tree_seq_stride < 0 || m->tree_seq_stride >= kMaxStride || m->tree_row_stride < rows || m->tree_row_stride >= kMaxStride)
      return fail(CKV_EINVAL, "strides of the tree must be at least a row (0 for one tree for all)");
  }
  return CKV_OK;
}

// Whether rows are a token of each sequence, without a tree: bound by memory, the attention of one token takes them (unless they are packed, when some sequence may have none).  By it and as blocks of
// rows, us: 32 sequences x 8 KV heads x 4 heads, window 4096, 8 bits 55 and 83, bf16 92 and 116; of 16 heads 66 and 86, 102 and 121; one sequence of 131072 55 and 89, 94 and 119; 4 x 4 of 777 10 and 16.
bool one_row(const ckv_pages* p, const ckv_seqs* s, int rows, const ckv_mask* m) {
  return rows == 1 && !m->tree && (long long)s->batch * p->n_kv_heads * unit_blocks(s->max_length) <= (1ll << 30);
}

// How a call is cut, and what its pieces leave in the workspace.
struct RowsSplit {
  RowsPlan plan;
  size_t partial, ml, parts, cut;      // bytes
  size_t bytes() const { return partial + ml + parts + cut; }
};
RowsSplit rows_split(const ckv_pages* p, const ckv_seqs* s, int rows, int n_q_heads, const ckv_mask* m, int n_cu) {
  const long long units = (long long)s->batch * p->n_kv_heads;
  const int G = n_q_heads / p->n_kv_heads, most = std::max(std::min(rows, s->max_length), 1);
  const long long spread = m->tree ? most : std::min(most, 128 / G + 2), seen = m->window ? (long long)m->window + m->sinks + spread : s->max_length;
  RowsSplit r{};
  r.plan = rows_plan(units, most, G, (int)std::min<long long>(seen, s->max_length), n_cu, s->batch);
  if (r.plan.places > 1 || r.plan.more) {
    const size_t held = (size_t)(r.plan.pieces + r.plan.more) * 32 * r.plan.wide;
    r.partial = up256(held * kDim * 4);
    r.ml = up256(held * 8);
    r.parts = up256((size_t)units * r.plan.blocks * 8);
    r.cut = r.plan.more ? up256(((size_t)s->batch + 2) * 4) : 0;
  }
  return r;
}

}  // namespace

extern "C" {

size_t ckv_paged_rows_workspace_bytes(const ckv_pages* pages, const ckv_seqs* seqs, int32_t rows, int32_t n_q_heads, const ckv_mask* mask) {
  if (check(pages, seqs) != CKV_OK || check_sizes(pages, seqs, rows, n_q_heads, mask) != CKV_OK) return 0;
  size_t bytes = rows_split(pages, seqs, rows, n_q_heads, mask, compute_units()).bytes();
  if (one_row(pages, seqs, rows, mask)) bytes = std::max(bytes, one_row_workspace(pages, seqs, n_q_heads, mask));
  return std::max<size_t>(256, bytes);
}

int ckv_paged_attend_rows(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_row_queries* queries, const ckv_mask* mask, float softmax_scale, void* out,
                          int32_t out_dtype, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (!queries) return fail(CKV_EINVAL, "queries are NULL");
  if (int rc = check_sizes(pages, seqs, queries->rows, queries->n_q_heads, mask)) return rc;
  if (out_dtype != CKV_F32 && out_dtype != CKV_BF16) return fail(CKV_EINVAL, "out_dtype must be CKV_F32 or CKV_BF16");
  const float scale_log2e = softmax_scale * 1.44269504088896340736f;
  if (!(softmax_scale > 0.0f) || !std::isfinite(scale_log2e)) return fail(CKV_EINVAL, "softmax_scale must be positive and below 2.3e38");
  if (seqs->max_length == 0 || (queries->starts && queries->total == 0)) return CKV_OK;
  if (int rc = check_queries(pages, queries)) return rc;
  if (!out || !aligned(out, 16)) return fail(CKV_EINVAL, "out must be a 16-byte aligned device address");
  if (one_row(pages, seqs, queries->rows, mask) && !queries->starts) {
    const ckv_query query = {queries->q, queries->seq_stride, queries->head_stride, queries->n_q_heads};
    return attend_one_row(pages, seqs, &query, queries->first, mask, scale_log2e, out, out_dtype, lse, workspace, workspace_bytes, stream);
  }
  const RowsSplit s = rows_split(pages, seqs, queries->rows, queries->n_q_heads, mask, compute_units());
  const long long units = (long long)seqs->batch * pages->n_kv_heads, first = rows_grid(units * s.plan.places, (long long)s.plan.blocks), grid = first + s.plan.more;
  if (!launches(grid, kThreads) || !launches(units * s.plan.blocks, 32 * kRowsJoined)) return fail(CKV_EINVAL, "too many rows for one attention (2^24 blocks of 128, a row per query head)");
  if (s.bytes() > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes())) return fail(CKV_EWORKSPACE, "workspace too small or misaligned");
  const Paged p = paged_of(pages, seqs);
  RowsAttend c{};
  c.rows = Rows{(uint8_t*)queries->q, nullptr, queries->first, queries->starts, queries->seq_stride * 2, queries->row_stride * 2, queries->head_stride * 2, queries->rows, queries->total};
  c.tree = mask->tree;
  c.tree_seq = mask->tree_seq_stride;
  c.tree_row = mask->tree_row_stride;
  c.out = (uint8_t*)out;
  c.lse = lse;
  c.units = units;
  c.scale_log2e = scale_log2e;
  c.G = queries->n_q_heads / pages->n_kv_heads;
  c.window = mask->window;
  c.sinks = mask->sinks;
  c.out_bf16 = out_dtype == CKV_BF16;
  c.blocks = s.plan.blocks;
  c.least = s.plan.least;
  c.places = s.plan.places;
  c.workers = s.plan.workers;
  c.more = s.plan.more;
  c.grid = (int)first;
  c.lower = lowered_by(seqs->max_length);
  if (s.bytes() > 0) {
    c.partial = (float*)workspace;
    c.ml = (float*)((char*)workspace + s.partial);
    c.parts = (int32_t*)((char*)workspace + s.partial + s.ml);
    c.cut = (int32_t*)((char*)workspace + s.partial + s.ml + s.parts);
  }
  if (c.more) {
    auto cut = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(1), dim3(kCutThreads), 0, (hipStream_t)stream, RowsCall{p, c}); };
    s.plan.wide == 2 ? cut(paged_rows_cut_kernel<2>) : cut(paged_rows_cut_kernel<4>);
    if (int rc = launched("ckv_paged_attend_rows")) return rc;
  }
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), 0, (hipStream_t)stream, RowsCall{p, c}); };
  auto typed = [&](auto e4m3, auto wide) {
    constexpr bool E4M3 = decltype(e4m3)::value;
    constexpr int WIDE = decltype(wide)::value;
    c.more ? launch(paged_rows_kernel<E4M3, WIDE, true>) : launch(paged_rows_kernel<E4M3, WIDE, false>);
  };
  auto attend = [&](auto wide) { pages->dtype == CKV_E4M3 ? typed(std::true_type(), wide) : typed(std::false_type(), wide); };
  s.plan.wide == 2 ? attend(std::integral_constant<int, 2>()) : attend(std::integral_constant<int, 4>());
  if (int rc = launched("ckv_paged_attend_rows")) return rc;
  if (s.bytes() == 0) return CKV_OK;
  const long long blocks = units * s.plan.blocks, most = 32 * s.plan.wide / kRowsJoined;
  const dim3 joins((unsigned)blocks, (unsigned)std::max(1ll, std::min(most, 8192 / blocks)));
  auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, joins, dim3(32 * kRowsJoined), 0, (hipStream_t)stream, RowsCall{p, c}); };
  if (c.more) s.plan.wide == 2 ? join(paged_rows_join_kernel<2, true>) : join(paged_rows_join_kernel<4, true>);
  else s.plan.wide == 2 ? join(paged_rows_join_kernel<2, false>) : join(paged_rows_join_kernel<4, false>);
  return launched("ckv_paged_attend_rows");
}

int ckv_paged_append_rotated(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_rows* rows, const ckv_rotation* rotation, const int32_t* positions,
                             const ckv_heads* q, const ckv_heads* q_out, void* stream) {
  if (int rc = check(pages, seqs)) return rc;
  if (int rc = check_rows(rows)) return rc;
  if (int rc = check_rotation(rotation)) return rc;
  if (!q != !q_out) return fail(CKV_EINVAL, "q and q_out belong together");
  if (seqs->max_length == 0 || nothing(rows)) return CKV_OK;
  if (q) {
    if (int rc = check_row_heads(pages, q, rows->starts)) return rc;
    if (int rc = check_row_heads(pages, q_out, rows->starts)) return rc;
    if (q->n_q_heads != q_out->n_q_heads) return fail(CKV_EINVAL, "q and q_out must have as many heads");
  }
  const Paged p = paged_of(pages, seqs);
  const Rows r = rows_of(rows);
  unsigned touched;
  if (int rc = touched_pages(pages, seqs, rows, touched)) return rc;
  Turned c{};
  if (q) {
    c.q = (const uint8_t*)q->q;
    c.out = (uint8_t*)q_out->q;
    c.q_seq = q->seq_stride * 2;
    c.q_row = q->row_stride * 2;
    c.q_head = q->head_stride * 2;
    c.out_seq = q_out->seq_stride * 2;
    c.out_row = q_out->row_stride * 2;
    c.out_head = q_out->head_stride * 2;
    c.G = q->n_q_heads / pages->n_kv_heads;
  }
  c.frequencies = rotation->frequencies;
  c.positions = positions;
  c.magnitude = rotation->magnitude;
  c.pairs = rotation->n_pairs;
  c.interleaved = rotation->interleaved;
  const long long units = (long long)seqs->batch * pages->n_kv_heads;
  const dim3 grid((unsigned)units, touched, (unsigned)turned_by(units * touched, rows->rows, c.G, compute_units()));
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, p, r, c); };
  if (grid.z > 1) pages->dtype == CKV_E4M3 ? launch(paged_append_rotated_kernel<true, true>) : launch(paged_append_rotated_kernel<false, true>);
  else pages->dtype == CKV_E4M3 ? launch(paged_append_rotated_kernel<true, false>) : launch(paged_append_rotated_kernel<false, false>);
  return launched("ckv_paged_append_rotated");
}

}  // extern "C"
