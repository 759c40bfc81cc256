// extern "C" entry points of the 4-bit cache: argument checks, then one launcher each.
#include <cmath>

#include "slkv_internal.cuh"

namespace slkv {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr int kMaxSegments = 16384;

// What every call asks of a cache.
int check_cache(const slkv_q4_cache* c, Q4CacheView* view) {
  if (!c || !c->records || !c->pos || !c->starts || !c->lens) return SLKV_ERR_NULL_PTR;
  if (c->n_seqs < 1 || c->n_kv_heads < 1 || (int64_t)c->n_seqs * c->n_kv_heads > kMaxSegments) return SLKV_ERR_BAD_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return SLKV_ERR_BAD_SHAPE;
  if (c->capacity_rows < 1 || c->capacity_rows >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (!aligned16(c->records)) return SLKV_ERR_BAD_ALIGN;
  view->records = static_cast<unsigned char*>(c->records);
  view->pos = c->pos; view->weight = c->weight; view->starts = c->starts; view->lens = c->lens;
  view->capacity = c->capacity_rows;
  view->n_seg = c->n_seqs * c->n_kv_heads;
  return SLKV_OK;
}

bool dtype_ok(int dtype) { return dtype == SLKV_F32 || dtype == SLKV_BF16; }

int check_strides(const int64_t* strides, int n, int head_dim, int dtype) {
  const int elem = dtype == SLKV_F32 ? 4 : 2;
  for (int i = 0; i < n; ++i) {
    if (strides[i] < head_dim) return SLKV_ERR_BAD_SHAPE;
    if (strides[i] * elem % 16 != 0) return SLKV_ERR_BAD_ALIGN;
  }
  return SLKV_OK;
}

int check_attend(const slkv_q4_cache* c, const slkv_q4_attend_params* p, Q4CacheView* view) {
  const int rc = check_cache(c, view);
  if (rc != SLKV_OK) return rc;
  if (!p) return SLKV_ERR_NULL_PTR;
  if (!dtype_ok(p->dtype) || (p->lse_units != SLKV_LSE_LN && p->lse_units != SLKV_LSE_LOG2)) return SLKV_ERR_BAD_DTYPE;
  if (p->n_tokens < 1 || p->n_q_heads < c->n_kv_heads || p->n_q_heads % c->n_kv_heads != 0) return SLKV_ERR_BAD_SHAPE;
  const int64_t columns = (int64_t)(p->n_q_heads / c->n_kv_heads) * p->n_tokens;
  if (columns > kMaxQ4Columns) return SLKV_ERR_BAD_SHAPE;
  // the tiles of all units are counted in 32 bits
  if ((c->capacity_rows / 32 + view->n_seg) * ((columns + 7) / 8) >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  // the kernel multiplies with 2^73 log2(e) scale
  if (!(std::fabs(p->scale) <= 0x1p54f) || !std::isfinite(p->softcap) || (p->softcap != 0.0f && p->softcap < 1e-20f) ||
      !std::isfinite(p->weight_decay))
    return SLKV_ERR_BAD_SHAPE;
  const int64_t strides[] = {p->q_stride_seq, p->q_stride_tok, p->q_stride_head, p->o_stride_seq, p->o_stride_tok, p->o_stride_head};
  return check_strides(strides, 6, c->head_dim, p->dtype);
}

bool overlap(const void* a, const void* b, size_t a_bytes, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

}  // namespace
}  // namespace slkv

using namespace slkv;

extern "C" {

size_t slkv_q4_record_bytes(int32_t head_dim) { return head_dim == 64 || head_dim == 128 ? (size_t)head_dim + head_dim / 4 : 0; }

int slkv_q4_pack(const slkv_q4_cache* c, int32_t dtype, const void* k, const void* v, int64_t n_rows, const int32_t* offsets,
                 const int32_t* kept_idx, int32_t* status, void* stream) {
  Q4CacheView view;
  const int rc = check_cache(c, &view);
  if (rc != SLKV_OK) return rc;
  if (!dtype_ok(dtype)) return SLKV_ERR_BAD_DTYPE;
  if (!offsets) return SLKV_ERR_NULL_PTR;
  if (n_rows < 0 || n_rows >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (n_rows > 0 && (!k || !v || !kept_idx)) return SLKV_ERR_NULL_PTR;
  if (!aligned16(k) || !aligned16(v)) return SLKV_ERR_BAD_ALIGN;
  // the rows may be those of a layer that is still queued
  int launches = 0;
  cudaError_t e = send_queued_layers((cudaStream_t)stream, &launches);
  if (e == cudaSuccess) e = launch_q4_pack(view, c->head_dim, dtype == SLKV_F32, k, v, n_rows, offsets, kept_idx, status, (cudaStream_t)stream, &launches);
  return report(e, launches);
}

int slkv_q4_append(const slkv_q4_cache* c, int32_t dtype, const void* k, const void* v, int32_t n_tokens, int64_t k_stride_seq,
                   int64_t k_stride_tok, int64_t k_stride_head, int64_t v_stride_seq, int64_t v_stride_tok, int64_t v_stride_head,
                   const int32_t* pos, int32_t* lens_out, int32_t* status, void* stream) {
  Q4CacheView view;
  int rc = check_cache(c, &view);
  if (rc != SLKV_OK) return rc;
  if (!dtype_ok(dtype)) return SLKV_ERR_BAD_DTYPE;
  if (!k || !v || !pos) return SLKV_ERR_NULL_PTR;
  if (n_tokens < 1 || n_tokens > 65536) return SLKV_ERR_BAD_SHAPE;
  const int64_t strides[6] = {k_stride_seq, k_stride_tok, k_stride_head, v_stride_seq, v_stride_tok, v_stride_head};
  rc = check_strides(strides, 6, c->head_dim, dtype);
  if (rc != SLKV_OK) return rc;
  if (!aligned16(k) || !aligned16(v)) return SLKV_ERR_BAD_ALIGN;
  const size_t len_bytes = view.n_seg * sizeof(int32_t);
  if (lens_out && lens_out != c->lens && overlap(lens_out, c->lens, len_bytes, len_bytes)) return SLKV_ERR_BAD_SHAPE;
  int launches = 0;
  const cudaError_t e = launch_q4_append(view, c->n_kv_heads, c->head_dim, dtype == SLKV_F32, k, v, n_tokens, strides, pos,
                                         lens_out ? lens_out : c->lens, status, (cudaStream_t)stream, &launches);
  return report(e, launches);
}

int slkv_q4_unpack(const slkv_q4_cache* c, int32_t dtype, const int32_t* slots_opt, int64_t n, void* k_out, void* v_out, void* stream) {
  Q4CacheView view;
  const int rc = check_cache(c, &view);
  if (rc != SLKV_OK) return rc;
  if (!dtype_ok(dtype)) return SLKV_ERR_BAD_DTYPE;
  if (!slots_opt) n = c->capacity_rows;
  if (n < 0 || n >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (n == 0) return report(cudaSuccess, 0);
  if (!k_out || !v_out) return SLKV_ERR_NULL_PTR;
  if (!aligned16(k_out) || !aligned16(v_out)) return SLKV_ERR_BAD_ALIGN;
  int launches = 0;
  const cudaError_t e = launch_q4_unpack(view, c->head_dim, dtype == SLKV_F32, slots_opt, n, k_out, v_out, (cudaStream_t)stream, &launches);
  return report(e, launches);
}

size_t slkv_q4_attend_workspace_bytes(const slkv_q4_cache* c, const slkv_q4_attend_params* p, int32_t accumulate) {
  Q4CacheView view;
  if (check_attend(c, p, &view) != SLKV_OK) return 0;
  return q4_attend_workspace(view.n_seg, c->head_dim, p->n_q_heads / c->n_kv_heads * p->n_tokens, view.capacity, accumulate != 0);
}

int slkv_q4_attend(const slkv_q4_cache* c, const slkv_q4_attend_params* p, const void* q, const int32_t* q_pos_opt,
                   const float* slopes_opt, void* out, float* lse_opt, int32_t accumulate, int32_t* status, void* workspace,
                   size_t workspace_bytes, void* stream) {
  Q4CacheView view;
  const int rc = check_attend(c, p, &view);
  if (rc != SLKV_OK) return rc;
  if (!q || !out || (slopes_opt && !q_pos_opt) || (accumulate && !c->weight)) return SLKV_ERR_NULL_PTR;
  if (!aligned16(q) || !aligned16(out)) return SLKV_ERR_BAD_ALIGN;
  if (!workspace || workspace_bytes < slkv_q4_attend_workspace_bytes(c, p, accumulate)) return SLKV_ERR_WORKSPACE;
  if (!aligned16(workspace)) return SLKV_ERR_BAD_ALIGN;
  int launches = 0;
  const cudaError_t e = launch_q4_attend(view, *c, *p, q, q_pos_opt, slopes_opt, out, lse_opt, accumulate != 0, status, workspace,
                                         (cudaStream_t)stream, &launches);
  return report(e, launches);
}

size_t slkv_q4_evict_workspace_bytes(const slkv_q4_cache* from) {
  Q4CacheView view;
  if (check_cache(from, &view) != SLKV_OK) return 0;
  return q4_evict_workspace(view.n_seg, view.capacity);
}

int slkv_q4_evict(const slkv_q4_cache* from, const slkv_q4_cache* to, const int32_t* budgets, int32_t window, const int32_t* newest,
                  int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  Q4CacheView a, b;
  int rc = check_cache(from, &a);
  if (rc == SLKV_OK) rc = check_cache(to, &b);
  if (rc != SLKV_OK) return rc;
  if (!budgets || !newest || !from->weight || !to->weight) return SLKV_ERR_NULL_PTR;
  if (from->n_seqs != to->n_seqs || from->n_kv_heads != to->n_kv_heads || from->head_dim != to->head_dim) return SLKV_ERR_BAD_SHAPE;
  if (window < 1) return SLKV_ERR_BAD_SHAPE;
  const size_t len_bytes = a.n_seg * sizeof(int32_t);
  if (from->lens != to->lens && overlap(from->lens, to->lens, len_bytes, len_bytes)) return SLKV_ERR_BAD_SHAPE;
  if (from->records == to->records) {                      // in place: the same cache throughout, only the lengths may be elsewhere
    if (from->pos != to->pos || from->weight != to->weight || from->starts != to->starts || from->capacity_rows != to->capacity_rows)
      return SLKV_ERR_BAD_SHAPE;
  } else {
    const size_t m = (size_t)from->capacity_rows, n = (size_t)to->capacity_rows, rec = slkv_q4_record_bytes(from->head_dim);
    if (overlap(from->records, to->records, m * rec, n * rec) || overlap(from->pos, to->pos, m * 4, n * 4) ||
        overlap(from->weight, to->weight, m * 4, n * 4))
      return SLKV_ERR_BAD_SHAPE;
  }
  if (!workspace || workspace_bytes < slkv_q4_evict_workspace_bytes(from)) return SLKV_ERR_WORKSPACE;
  if (!aligned16(workspace)) return SLKV_ERR_BAD_ALIGN;
  int launches = 0;
  const cudaError_t e = launch_q4_evict(a, b, from->n_kv_heads, from->head_dim, budgets, window, newest, status, workspace,
                                        (cudaStream_t)stream, &launches);
  return report(e, launches);
}

}  // extern "C"
