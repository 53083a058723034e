// What the entry points of the cache in pages (ckv_paged_*) share on the host: what a thread's last refused call complained about, the checks of
// pools, sequences and rows, and what kernels get of them.
#pragma once
#include "../../include/ckv.h"

#include <hip/hip_runtime.h>

#include <cstdio>

#include "ckv_paged_device.h"

namespace ckv {

// What the last failed call of this thread complained about (these calls have no context to keep it in).
inline thread_local char t_error[256];

inline int fail(int code, const char* what) {
  std::snprintf(t_error, sizeof t_error, "%s", what);
  return code;
}
inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return CKV_OK;
  std::snprintf(t_error, sizeof t_error, "%s: %s", what, hipGetErrorString(e));
  return CKV_EHIP;
}

constexpr long long kMaxLength = 1ll << 30;
constexpr int64_t kMaxStride = 1ll << 40;
constexpr int kMaxGrid = 65535;          // of the second and third axis

inline bool aligned(const void* p, uintptr_t to) { return (uintptr_t)p % to == 0; }
// a stride of so many elements, a multiple of `of`
inline bool stride_ok(int64_t s, int64_t least, int64_t of) { return s >= least && s % of == 0 && s < kMaxStride; }

inline int element(const ckv_pages* p) { return p->dtype == CKV_E4M3 ? 1 : 2; }

// Whether a launch of so many workgroups has fewer than 2^32 threads, the most that one axis takes.
inline bool launches(long long groups, int threads) { return groups * threads < (1ll << 32); }

inline int check(const ckv_pages* p, const ckv_seqs* s) {
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

inline Paged paged_of(const ckv_pages* p, const ckv_seqs* s) {
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
inline bool nothing(const ckv_rows* r) { return r->starts && r->total == 0; }

inline int check_rows(const ckv_rows* r) {
  if (!r) return fail(CKV_EINVAL, "rows are NULL");
  if (nothing(r)) return CKV_OK;
  if (!r->k || !r->v) return fail(CKV_EINVAL, "rows are NULL");
  if (!aligned(r->k, 16) || !aligned(r->v, 16)) return fail(CKV_EINVAL, "rows must be 16-byte aligned");
  if (r->rows < 1 || r->rows > kMaxLength) return fail(CKV_EINVAL, "rows must be in [1, 2^30]");
  if (!stride_ok(r->row_stride, kDim, 8) || !stride_ok(r->head_stride, kDim, 8) || (r->starts ? r->total < 0 : !stride_ok(r->seq_stride, kDim, 8)))
    return fail(CKV_EINVAL, "strides of the rows must be at least 128 elements and multiples of 8");
  return CKV_OK;
}

inline Rows rows_of(const ckv_rows* r) {
  return Rows{(uint8_t*)r->k, (uint8_t*)r->v, r->first, r->starts, r->seq_stride * 2, r->row_stride * 2, r->head_stride * 2, r->rows, r->total};
}

// Pages of a sequence that the rows of a call may reach.
inline int touched_pages(const ckv_pages* p, const ckv_seqs* s, const ckv_rows* r, unsigned& touched) {
  const long long reach = r->rows < s->max_length ? r->rows : s->max_length, pages = (reach + p->page_size - 2) / p->page_size + 1, most = pages < s->columns ? pages : s->columns;
  if (most > kMaxGrid) return fail(CKV_EINVAL, "rows of a call may reach 65535 pages of a sequence at most");
  touched = (unsigned)most;
  return CKV_OK;
}

inline int check_heads(const ckv_pages* p, int n_q_heads) {
  if (n_q_heads < p->n_kv_heads || n_q_heads % p->n_kv_heads != 0) return fail(CKV_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
  if (n_q_heads / p->n_kv_heads > kPagedGroup) return fail(CKV_EINVAL, "at most 16 query heads per KV head");
  return CKV_OK;
}

// Compute units of the current device.
inline int compute_units() {
  static int known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  n = __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
  if (n > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
  return n;
}

// One row of each sequence as ckv_paged_attend_rows takes it (ckv_paged.hip, where the attention of one token is): its workspace, 0 if it needs none, and the call, its arguments checked.
size_t one_row_workspace(const ckv_pages* pages, const ckv_seqs* seqs, int n_q_heads, const ckv_mask* mask);
int attend_one_row(const ckv_pages* pages, const ckv_seqs* seqs, const ckv_query* query, const int32_t* first, const ckv_mask* mask, float scale_log2e, void* out, int32_t out_dtype,
                   float* lse, void* workspace, size_t workspace_bytes, void* stream);

constexpr size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace ckv
