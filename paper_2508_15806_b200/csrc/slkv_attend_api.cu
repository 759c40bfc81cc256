// extern "C" entry points of the prompt attention and of the paged cache: argument checks, then one launcher each.

#include "slkv_attend.cuh"
#include "slkv_paged.cuh"

namespace slkv {
namespace {

constexpr long long kMaxRows = (1ll << 31) - 512;      // tokens, rows of a pool: a tile behind the last one still has 32-bit coordinates
constexpr int kMaxSegments = 1 << 20, kMaxLayerSegments = 16384;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool dtype_ok(int dtype) { return dtype == SLKV_F32 || dtype == SLKV_BF16; }
int elem_of(int dtype) { return dtype == SLKV_F32 ? 4 : 2; }

// Strides of axes with their lengths: at least a row, whole 16 bytes, below what a tensor map takes.  Of an axis of length 1 the stride
// says nothing: it becomes the row.
struct Axis { long long* stride; long long length; };
int check_axes(const Axis* axes, int n, int head_dim, int dtype) {
  for (int i = 0; i < n; ++i) {
    if (axes[i].length <= 1) { *axes[i].stride = head_dim; continue; }
    const long long s = *axes[i].stride;
    if (s < head_dim || s >= (1ll << 38)) return SLKV_ERR_BAD_SHAPE;
    if (s * elem_of(dtype) % 16 != 0) return SLKV_ERR_BAD_ALIGN;
  }
  return SLKV_OK;
}

int check_heads(int n_q_heads, int n_kv_heads, int head_dim, int dtype, int lse_units, float scale) {
  if (!dtype_ok(dtype) || (lse_units != SLKV_LSE_LN && lse_units != SLKV_LSE_LOG2)) return SLKV_ERR_BAD_DTYPE;
  if (head_dim != 64 && head_dim != 128) return SLKV_ERR_BAD_SHAPE;
  if (n_kv_heads < 1 || n_q_heads < n_kv_heads || n_q_heads % n_kv_heads != 0 || n_q_heads / n_kv_heads > kMaxGroup) return SLKV_ERR_BAD_SHAPE;
  if (!(scale >= 0x1p-54f && scale <= 0x1p54f)) return SLKV_ERR_BAD_SHAPE;
  return SLKV_OK;
}

// What follows from the types and shapes for both kernels: blocks, units, tiles.  max_tokens: of a sequence.
void set_blocks(AttendShape* a, int dtype, long long max_tokens) {
  a->ml_unit = a->scale * kLog2e;
  const int blocks = dtype == SLKV_F32 ? 1 : 2;    // of 128 query rows in a unit
  a->block_tokens = kAttendTile / a->G;
  a->unit_tokens = blocks * a->block_tokens;
  a->part_rows = max_tokens <= a->block_tokens ? kAttendTile : blocks * kAttendTile;
  a->box_tokens = a->paged && max_tokens < a->block_tokens ? (int)max_tokens : a->block_tokens;
  a->used_rows = a->part_rows == kAttendTile ? a->box_tokens * a->G : a->part_rows;
  a->tile_bits = dtype == SLKV_F32 ? kF32TileBits : kAttendTileBits;
  a->n_cta = sm_count();
  a->q_head_inner = dtype == SLKV_F32 || a->q_head <= a->q_tok;
  const int inner = a->q_head_inner ? a->G : a->box_tokens;
  a->row_inverse = (65536 + inner - 1) / inner;
}

// Segments of so many tiles are not cut: the second launch costs more.
constexpr int kWholeTiles = 4;
// What pieces and the launch that joins them cost, in the time of a tile.
constexpr int kJoinCost = 8;

// ---- prompts
// Whole units dealt out, or equal shares of all tiles whose pieces another launch joins?  By the time of the CTA that has the most to do,
// in tiles: for few units it is added up, in the order in which they are dealt out; many are always dealt out.  Both sides, us: 1000 tokens
// (128 units) 33 / 39, 2000 51 / 71, 3000 90 / 114; four chunks behind 24000 tokens 400 / 223.  Returns the number of units.
long long spread_or_share(const int32_t* cu_q, const int32_t* cu_k, AttendShape* a) {
  const int tile = 1 << a->tile_bits;
  long long units = 0;
  for (int s = 0; s < a->n_seqs; ++s) units += (cu_q[s + 1] - cu_q[s] + a->unit_tokens - 1) / a->unit_tokens;
  units *= a->n_kv_heads;
  a->spread = 1;
  constexpr int kMostCtas = 512;
  if (units >= 3ll * a->n_cta || (long long)a->n_seqs * a->levels > (1 << 16) || a->n_cta > kMostCtas) return units;
  long long load[kMostCtas] = {};
  long long total = 0, item = 0, most = 0;
  for (int level = a->levels - 1; level >= 0; --level)
    for (int s = 0; s < a->n_seqs; ++s) {
      const long long nq = cu_q[s + 1] - cu_q[s], nk = cu_k[s + 1] - cu_k[s], first = (long long)level * a->unit_tokens;
      if (first >= nq) continue;
      const long long seen = (first + a->unit_tokens < nq ? first + a->unit_tokens : nq) + nk - nq;
      const long long length = (seen > 0 ? (seen + tile - 1) / tile : 0) + kUnitCost;
      total += length * a->n_kv_heads;
      for (int h = 0; h < a->n_kv_heads; ++h, ++item) {
        const long long round = item / a->n_cta, place = item % a->n_cta;
        long long& l = load[round & 1 ? a->n_cta - 1 - place : place];
        l += length;
        if (l > most) most = l;
      }
    }
  if (most > total / a->n_cta + kJoinCost && total < (1ll << 31)) a->spread = 0;
  return units;
}

int check_prompt(const slkv_prompt_params* p, const int32_t* cu_q, const int32_t* cu_k, AttendShape* a) {
  if (!p || !cu_q) return SLKV_ERR_NULL_PTR;
  if (!cu_k) cu_k = cu_q;
  int rc = check_heads(p->n_q_heads, p->n_kv_heads, p->head_dim, p->dtype, p->lse_units, p->scale);
  if (rc != SLKV_OK) return rc;
  if (p->n_seqs < 1 || p->window < 1 || (long long)p->n_seqs * p->n_kv_heads >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (cu_q[0] != 0 || cu_k[0] != 0) return SLKV_ERR_BAD_SHAPE;
  long long longest = 0;
  for (int s = 0; s < p->n_seqs; ++s) {
    if (cu_q[s + 1] < cu_q[s] || cu_k[s + 1] < cu_k[s]) return SLKV_ERR_BAD_SHAPE;
    if (cu_q[s + 1] - cu_q[s] > longest) longest = cu_q[s + 1] - cu_q[s];
  }
  *a = AttendShape{};
  a->n_seqs = p->n_seqs; a->n_kv_heads = p->n_kv_heads; a->n_q_heads = p->n_q_heads; a->G = p->n_q_heads / p->n_kv_heads;
  a->head_dim = p->head_dim;
  a->window = p->window;
  a->rows_q = cu_q[p->n_seqs];
  a->rows_k = cu_k[p->n_seqs];
  if (a->rows_q > kMaxRows || a->rows_k > kMaxRows) return SLKV_ERR_BAD_SHAPE;
  a->q_tok = p->q_stride_tok; a->q_head = p->q_stride_head; a->o_tok = p->o_stride_tok; a->o_head = p->o_stride_head;
  a->k_tok = p->k_stride_tok; a->k_head = p->k_stride_head; a->v_tok = p->v_stride_tok; a->v_head = p->v_stride_head;
  const Axis axes[] = {{&a->q_tok, a->rows_q}, {&a->q_head, a->n_q_heads}, {&a->o_tok, a->rows_q}, {&a->o_head, a->n_q_heads},
                       {&a->k_tok, a->rows_k}, {&a->k_head, a->n_kv_heads}, {&a->v_tok, a->rows_k}, {&a->v_head, a->n_kv_heads}};
  rc = check_axes(axes, 8, p->head_dim, p->dtype);
  if (rc != SLKV_OK) return rc;
  a->scale = p->scale;
  set_blocks(a, p->dtype, longest);
  a->lse_unit = p->lse_units == SLKV_LSE_LOG2 ? 1.0f : 0.69314718055994531f;
  a->levels = (int)((longest + a->unit_tokens - 1) / a->unit_tokens);
  const long long units = spread_or_share(cu_q, cu_k, a);
  if (a->spread && units < a->n_cta) a->n_cta = (int)(units > 0 ? units : 1);
  return SLKV_OK;
}

// ---- the paged cache
int check_cache(const slkv_paged_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->tables || !c->lens || !c->free_pages || !c->n_free) return SLKV_ERR_NULL_PTR;
  if (!dtype_ok(c->dtype)) return SLKV_ERR_BAD_DTYPE;
  if (c->head_dim != 64 && c->head_dim != 128) return SLKV_ERR_BAD_SHAPE;
  if (c->n_layers < 1 || c->n_seqs < 1 || c->n_kv_heads < 1 || (long long)c->n_seqs * c->n_kv_heads > kMaxLayerSegments ||
      (long long)c->n_layers * c->n_seqs * c->n_kv_heads > kMaxSegments)
    return SLKV_ERR_BAD_SHAPE;
  if (c->page_rows != 16 && c->page_rows != 32 && c->page_rows != 64 && c->page_rows != 128) return SLKV_ERR_BAD_SHAPE;
  if (c->n_pages < 1 || (long long)c->n_pages * c->page_rows > kMaxRows) return SLKV_ERR_BAD_SHAPE;
  if (c->max_pages < 1 || (long long)c->max_pages * c->page_rows > kMaxRows) return SLKV_ERR_BAD_SHAPE;
  if ((long long)c->n_layers * c->n_seqs * c->n_kv_heads * c->max_pages >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return SLKV_ERR_BAD_ALIGN;
  return SLKV_OK;
}

int check_paged_attend(const slkv_paged_cache* c, const slkv_paged_attend_params* p, AttendShape* a) {
  int rc = check_cache(c);
  if (rc != SLKV_OK) return rc;
  if (!p) return SLKV_ERR_NULL_PTR;
  rc = check_heads(p->n_q_heads, c->n_kv_heads, c->head_dim, c->dtype, p->lse_units, p->scale);
  if (rc != SLKV_OK) return rc;
  if (p->layer < 0 || p->layer >= c->n_layers || p->n_tokens < 1 || p->n_tokens > kMaxDrafted) return SLKV_ERR_BAD_SHAPE;
  *a = AttendShape{};
  a->paged = 1;
  a->n_seqs = c->n_seqs; a->n_kv_heads = c->n_kv_heads; a->n_q_heads = p->n_q_heads; a->G = p->n_q_heads / c->n_kv_heads;
  a->head_dim = c->head_dim;
  const long long first = (long long)p->layer * c->n_seqs * c->n_kv_heads;
  a->tables = c->tables + first * c->max_pages;
  a->lens = c->lens + first;
  a->page_rows = c->page_rows; a->max_pages = c->max_pages; a->n_pages = c->n_pages;
  a->rows_k = (long long)c->n_pages * c->page_rows;
  a->k = c->k_pages; a->v = c->v_pages;
  a->n_tokens = p->n_tokens;
  a->q_seq = p->q_stride_seq; a->q_tok = p->q_stride_tok; a->q_head = p->q_stride_head;
  a->o_seq = p->o_stride_seq; a->o_tok = p->o_stride_tok; a->o_head = p->o_stride_head;
  a->kn_seq = p->k_stride_seq; a->kn_tok = p->k_stride_tok; a->kn_head = p->k_stride_head;
  a->vn_seq = p->v_stride_seq; a->vn_tok = p->v_stride_tok; a->vn_head = p->v_stride_head;
  const Axis axes[] = {{&a->q_seq, a->n_seqs}, {&a->q_tok, a->n_tokens}, {&a->q_head, a->n_q_heads}, {&a->o_seq, a->n_seqs},
                       {&a->o_tok, a->n_tokens}, {&a->o_head, a->n_q_heads}, {&a->kn_seq, a->n_seqs}, {&a->kn_tok, a->n_tokens},
                       {&a->kn_head, a->n_kv_heads}, {&a->vn_seq, a->n_seqs}, {&a->vn_tok, a->n_tokens}, {&a->vn_head, a->n_kv_heads}};
  rc = check_axes(axes, p->has_new ? 12 : 6, c->head_dim, c->dtype);
  if (rc != SLKV_OK) return rc;
  a->has_new = p->has_new != 0;
  a->scale = p->scale;
  set_blocks(a, c->dtype, a->n_tokens);
  a->lse_unit = p->lse_units == SLKV_LSE_LOG2 ? 1.0f : 0.69314718055994531f;
  const long long blocks = (a->n_tokens + a->unit_tokens - 1) / a->unit_tokens, longest = (long long)c->max_pages * c->page_rows;
  const long long units = blocks * a->n_seqs * a->n_kv_heads, tiles = ((longest + (1 << a->tile_bits) - 1) >> a->tile_bits) + a->has_new;
  if (units * (tiles + kUnitCost) >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;             // counted in 32 bits
  a->whole = tiles <= kWholeTiles ? (units <= a->n_cta ? 2 : 1) : 0;
  if (a->whole && units < a->n_cta) a->n_cta = (int)units;
  return SLKV_OK;
}

size_t workspace_of(const AttendShape& a) { return a.spread || a.whole ? 256 : attend_workspace(a.n_cta, a.part_rows, a.head_dim); }

int attend(AttendShape* a, int dtype, void* workspace, size_t workspace_bytes, cudaStream_t st) {
  if (!workspace || workspace_bytes < workspace_of(*a)) return SLKV_ERR_WORKSPACE;
  if (!aligned16(workspace)) return SLKV_ERR_BAD_ALIGN;
  if (!a->spread && !a->whole) attend_bind(a, workspace);
  int launches = 0;
  const size_t lse_rows = (size_t)a->n_seqs * a->n_q_heads * (a->paged ? a->n_tokens : a->window);
  cudaError_t e = send_layers_using(workspace, a->spread || a->whole ? 0 : workspace_of(*a), a->lse, lse_rows * sizeof(float), st, &launches);
  if (e == cudaSuccess) e = dtype == SLKV_F32 ? launch_attend_f32(*a, st, &launches) : launch_attend_tensor(*a, st, &launches);
  if (e == cudaSuccess) e = launch_attend_join(*a, dtype == SLKV_F32, st, &launches);
  return report(e, launches);
}

}  // namespace
}  // namespace slkv

using namespace slkv;

extern "C" {

size_t slkv_prompt_attend_workspace_bytes(const slkv_prompt_params* p, const int32_t* cu_q_host, const int32_t* cu_k_host_opt) {
  AttendShape a;
  return check_prompt(p, cu_q_host, cu_k_host_opt, &a) == SLKV_OK ? workspace_of(a) : 0;
}

int slkv_prompt_attend(const slkv_prompt_params* p, const void* q, const void* k, const void* v, const int32_t* cu_q_dev,
                       const int32_t* cu_q_host, const int32_t* cu_k_dev_opt, const int32_t* cu_k_host_opt, void* out, float* lse_opt,
                       int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  AttendShape a;
  const int rc = check_prompt(p, cu_q_host, cu_k_host_opt, &a);
  if (rc != SLKV_OK) return rc;
  if ((cu_k_dev_opt == nullptr) != (cu_k_host_opt == nullptr) || !cu_q_dev) return SLKV_ERR_NULL_PTR;
  if (a.rows_q == 0) return report(cudaSuccess, 0);
  if (!q || !out || (a.rows_k > 0 && (!k || !v))) return SLKV_ERR_NULL_PTR;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return SLKV_ERR_BAD_ALIGN;
  a.cu_q = cu_q_dev;
  a.cu_k = cu_k_dev_opt ? cu_k_dev_opt : cu_q_dev;
  a.q = q; a.k = k; a.v = v; a.out = out; a.lse = lse_opt; a.status = status;
  if (a.rows_k == 0) {                           // no key at all: nothing is loaded, but a tensor map wants a row
    a.k = a.v = q;
    a.rows_k = 1;
  }
  return attend(&a, p->dtype, workspace, workspace_bytes, (cudaStream_t)stream);
}

int slkv_paged_plan(const slkv_paged_cache* c, int32_t mode, const int32_t* want, int32_t* slots_opt, int64_t n_slots, int32_t slot_width,
                    int32_t* slot_offsets_opt, int32_t* lens_out, int32_t* n_free_out, int32_t* status, void* stream) {
  const int rc = check_cache(c);
  if (rc != SLKV_OK) return rc;
  if (mode != SLKV_PAGED_LENGTHS && mode != SLKV_PAGED_OFFSETS && mode != SLKV_PAGED_ADD) return SLKV_ERR_BAD_DTYPE;
  if (!want) return SLKV_ERR_NULL_PTR;
  const long long n_seg = (long long)c->n_layers * c->n_seqs * c->n_kv_heads;
  if (slots_opt) {
    if (n_slots < 0 || n_slots >= (1ll << 31) || slot_width < 0) return SLKV_ERR_BAD_SHAPE;
    if (slot_width > 0 && n_slots < n_seg * slot_width) return SLKV_ERR_BAD_SHAPE;
    if (slot_width == 0 && !slot_offsets_opt) return SLKV_ERR_NULL_PTR;
  }
  if ((lens_out == nullptr) != (n_free_out == nullptr)) return SLKV_ERR_NULL_PTR;
  if (lens_out && lens_out != c->lens && lens_out < c->lens + n_seg && c->lens < lens_out + n_seg) return SLKV_ERR_BAD_SHAPE;
  PagedPlanArgs a = {};
  a.n_seqs = c->n_seqs; a.n_kv_heads = c->n_kv_heads; a.n_seg = (int)n_seg;
  for (a.page_bits = 0; (1 << a.page_bits) < c->page_rows;) ++a.page_bits;
  a.n_pages = c->n_pages; a.max_pages = c->max_pages;
  a.mode = mode; a.slot_width = slot_width;
  a.tables = c->tables; a.lens = c->lens; a.lens_out = lens_out ? lens_out : c->lens;
  a.free_pages = c->free_pages; a.n_free = c->n_free; a.n_free_out = n_free_out ? n_free_out : c->n_free;
  a.want = want; a.slots = slots_opt; a.n_slots = n_slots; a.slot_offsets = slot_offsets_opt; a.status = status;
  int launches = 0;
  // the offsets may be those of layers that are still queued
  cudaError_t e = send_queued_layers((cudaStream_t)stream, &launches);
  if (e == cudaSuccess) e = launch_paged_plan(a, (cudaStream_t)stream, &launches);
  return report(e, launches);
}

int slkv_paged_write(const slkv_paged_cache* c, const void* k, const void* v, int32_t n_seqs, int32_t n_heads, int32_t n_tokens,
                     int64_t k_stride_seq, int64_t k_stride_tok, int64_t k_stride_head, int64_t v_stride_seq, int64_t v_stride_tok,
                     int64_t v_stride_head, const int32_t* slots, int32_t n_slots, const int32_t* take_opt, void* stream) {
  int rc = check_cache(c);
  if (rc != SLKV_OK) return rc;
  if (n_seqs < 1 || n_heads < 1 || n_tokens < 0 || n_slots < 0 || (long long)n_seqs * n_heads * n_slots >= (1ll << 31)) return SLKV_ERR_BAD_SHAPE;
  if (n_slots == 0 || n_tokens == 0) return report(cudaSuccess, 0);
  if (!k || !v || !slots) return SLKV_ERR_NULL_PTR;
  long long s[6] = {k_stride_seq, k_stride_tok, k_stride_head, v_stride_seq, v_stride_tok, v_stride_head};
  const long long len[3] = {n_seqs, n_tokens, n_heads};
  const Axis axes[6] = {{&s[0], len[0]}, {&s[1], len[1]}, {&s[2], len[2]}, {&s[3], len[0]}, {&s[4], len[1]}, {&s[5], len[2]}};
  rc = check_axes(axes, 6, c->head_dim, c->dtype);
  if (rc != SLKV_OK) return rc;
  if (!aligned16(k) || !aligned16(v)) return SLKV_ERR_BAD_ALIGN;
  const int elem = elem_of(c->dtype), chunks = c->head_dim * elem / 16;
  PagedWriteArgs a = {};
  a.k = static_cast<const char*>(k); a.v = static_cast<const char*>(v);
  for (int i = 0; i < 6; ++i) a.stride[i] = s[i] * elem;
  a.slots = slots; a.take = take_opt;
  a.k_pages = static_cast<uint4*>(c->k_pages); a.v_pages = static_cast<uint4*>(c->v_pages);
  a.n_rows = (unsigned)((long long)n_seqs * n_heads * n_slots);
  a.pool_rows = (unsigned)((long long)c->n_pages * c->page_rows);
  a.n_heads = (unsigned)n_heads; a.n_slots = (unsigned)n_slots; a.n_tokens = (unsigned)n_tokens;
  for (a.chunk_bits = 0; (1 << a.chunk_bits) < chunks;) ++a.chunk_bits;
  int launches = 0;
  // the rows may be those of a layer that is still queued
  cudaError_t e = send_queued_layers((cudaStream_t)stream, &launches);
  if (e == cudaSuccess) e = launch_paged_write(a, (cudaStream_t)stream, &launches);
  return report(e, launches);
}

size_t slkv_paged_attend_workspace_bytes(const slkv_paged_cache* c, const slkv_paged_attend_params* p) {
  AttendShape a;
  return check_paged_attend(c, p, &a) == SLKV_OK ? workspace_of(a) : 0;
}

int slkv_paged_attend(const slkv_paged_cache* c, const slkv_paged_attend_params* p, const void* q, const void* k_new, const void* v_new,
                      const uint64_t* tree_opt, const int32_t* n_new_opt, void* out, float* lse_opt, int32_t* status, void* workspace,
                      size_t workspace_bytes, void* stream) {
  AttendShape a;
  const int rc = check_paged_attend(c, p, &a);
  if (rc != SLKV_OK) return rc;
  if (!q || !out || (p->has_new && (!k_new || !v_new))) return SLKV_ERR_NULL_PTR;
  if (!aligned16(q) || !aligned16(out) || (p->has_new && (!aligned16(k_new) || !aligned16(v_new)))) return SLKV_ERR_BAD_ALIGN;
  a.q = q; a.k_new = k_new; a.v_new = v_new; a.out = out; a.lse = lse_opt; a.status = status;
  a.tree = reinterpret_cast<const unsigned long long*>(tree_opt);
  a.n_new = n_new_opt;
  return attend(&a, c->dtype, workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // extern "C"
