// Launches on a paged cache (slkv_paged.cu).
#pragma once

#include "slkv_internal.cuh"

namespace slkv {

struct PagedPlanArgs {
  int n_seqs, n_kv_heads, n_seg, page_bits, n_pages, max_pages, mode, slot_width;     // page_bits: log2 of a page's rows
  int32_t* tables;
  const int32_t* lens;
  int32_t* lens_out;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* n_free_out;
  const int32_t* want;
  int32_t *slots, *slot_offsets;                 // may be null
  long long n_slots;
  int32_t* status;
};
struct PagedWriteArgs {
  const char *k, *v;
  long long stride[6];                           // bytes: k and v by sequence, token, head
  const int32_t *slots, *take;                   // take may be null
  uint4 *k_pages, *v_pages;
  unsigned n_rows, pool_rows;                    // n_rows: slots of all sequences and heads
  unsigned n_heads, n_slots, n_tokens;           // n_slots: of a sequence and head
  int chunk_bits;                                // log2 of a row's chunks of 16 bytes
};
cudaError_t launch_paged_plan(const PagedPlanArgs& a, cudaStream_t st, int* launches);
cudaError_t launch_paged_write(const PagedWriteArgs& a, cudaStream_t st, int* launches);

}  // namespace slkv
