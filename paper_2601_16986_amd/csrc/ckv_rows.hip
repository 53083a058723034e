// Host side of the calls on several rows of each sequence of a cache in pages: argument checks and launches.  Nothing is kept between calls.
#include <algorithm>
#include <cmath>

#include "ckv_paged_host.h"
#include "ckv_rotate_kernels.h"

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

}  // namespace

extern "C" {

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
  const dim3 grid((unsigned)(seqs->batch * pages->n_kv_heads), touched);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, (hipStream_t)stream, p, r, c); };
  pages->dtype == CKV_E4M3 ? launch(paged_append_rotated_kernel<true>) : launch(paged_append_rotated_kernel<false>);
  return launched("ckv_paged_append_rotated");
}

}  // extern "C"
