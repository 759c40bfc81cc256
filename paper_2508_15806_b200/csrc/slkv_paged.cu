// Pages of a 16-bit or fp32 cache whose segments have lengths of their own: planning (which pages a segment gets or gives back, where its
// new rows go) and writing rows through the resulting slots.
#include <cooperative_groups.h>

#include "slkv_paged.cuh"

namespace slkv {
namespace {

namespace cg = cooperative_groups;

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32, kPlanCluster = 8;
constexpr int kSlotsHere = 1 << 16;              // ragged slots that the planning launch writes itself

// Exclusive prefix over the block of one value a thread; *total: of all.
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  long long w = lane < kPlanWarps ? warp_sums[lane] : 0, wi = w;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long o = __shfl_up_sync(0xffffffffu, wi, d);
    if (lane >= d) wi += o;
  }
  *total = __shfl_sync(0xffffffffu, wi, 31);
  const long long before = __shfl_sync(0xffffffffu, wi - w, warp);
  __syncthreads();                               // warp_sums may be written again
  return before + incl - v;
}

struct Segment { int len, want, have, need; };

__device__ __forceinline__ Segment segment(const PagedPlanArgs& a, int seg) {
  Segment x;
  const long long most = (long long)a.max_pages * a.page_rows;
  x.len = (int)min((long long)max(a.lens[seg], 0), most);
  long long want;
  if (a.mode == SLKV_PAGED_LENGTHS) {
    want = a.want[seg];
  } else if (a.mode == SLKV_PAGED_OFFSETS) {
    const int per = a.n_seqs * a.n_kv_heads, layer = seg / per;
    const int32_t* o = a.want + (long long)layer * (per + 1) + (seg - layer * per);
    want = (long long)o[1] - o[0];
  } else {
    want = (long long)x.len + max(a.want[seg / a.n_kv_heads % a.n_seqs], 0);
  }
  x.want = (int)min(max(want, 0ll), most);
  x.have = (x.len + a.page_rows - 1) / a.page_rows;
  x.need = (x.want + a.page_rows - 1) / a.page_rows;
  return x;
}

// One cluster.  A CTA has a run of segments, 1024 at a time a thread each; what lies before a segment is what the CTAs before this one
// come to (exchanged through their shared memory) and a scan.  Pages are moved by the segment's thread, or by its warp where there are
// many.  What bounds it: three or four dependent reads of L2 and the barriers between them, the data is a few hundred KB.
__global__ void __launch_bounds__(kPlanThreads) k_paged_plan(const __grid_constant__ PagedPlanArgs a) {
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ long long warp_sums[kPlanWarps];
  __shared__ long long totals[3];                // of this CTA: pages returned, pages wanted, rows that come in
  const int rank = (int)cluster.block_rank(), n_cta = (int)cluster.num_blocks();
  const int tid = threadIdx.x, lane = tid & 31;
  pdl_launch_dependents();
  pdl_wait();
  const int first = (int)((long long)a.n_seg * rank / n_cta), last = (int)((long long)a.n_seg * (rank + 1) / n_cta);

  long long gone = 0, more = 0;
  for (int seg = first + tid; seg < last; seg += kPlanThreads) {
    const Segment x = segment(a, seg);
    gone += max(x.have - x.need, 0);
    more += max(x.need - x.have, 0);
  }
  long long sum;
  block_scan(gone, warp_sums, &sum);
  if (tid == 0) totals[0] = sum;
  block_scan(more, warp_sums, &sum);
  if (tid == 0) totals[1] = sum;
  const long long n_free = min(max(a.n_free[0], 0), a.n_pages);
  cluster.sync();
  long long gone_before = 0, gone_all = 0, more_before = 0, more_all = 0;
  for (int r = 0; r < n_cta; ++r) {
    const long long* t = cluster.map_shared_rank(totals, r);
    if (r == rank) { gone_before = gone_all; more_before = more_all; }
    gone_all += t[0];
    more_all += t[1];
  }
  const long long stack = n_free + gone_all;     // pages on it once all are returned

  if (gone_all > 0) {                            // the first segment's first page ends up on top
    long long before = gone_before;
    for (int s0 = first; s0 < last; s0 += kPlanThreads) {
      const int seg = s0 + tid;
      Segment x = {};
      if (seg < last) x = segment(a, seg);
      const int n = max(x.have - x.need, 0);
      const long long at = before + block_scan(n, warp_sums, &sum);
      before += sum;
      unsigned todo = __ballot_sync(0xffffffffu, n > 0);
      for (; todo; todo &= todo - 1) {
        const int l = __ffs(todo) - 1;
        const int m = __shfl_sync(0xffffffffu, n, l), need = __shfl_sync(0xffffffffu, x.need, l);
        const long long to = stack - 1 - __shfl_sync(0xffffffffu, at, l);
        const int32_t* row = a.tables + (long long)(seg - lane + l) * a.max_pages + need;
        for (int i = lane; i < m; i += 32)
          if (to - i >= 0 && to - i < a.n_pages) a.free_pages[to - i] = row[i];
      }
    }
    cluster.sync();                              // some are taken again below
  }

  // pages taken and new lengths; rows that come in
  const long long fits = min(stack, (long long)a.n_pages);
  bool short_of = false;
  auto new_length = [&](const Segment& x, long long at, int* granted) {
    const int wanted = max(x.need - x.have, 0);
    *granted = (int)min(max(fits - at, 0ll), (long long)wanted);
    return (int)min((long long)x.want, (long long)(min(x.have, x.need) + *granted) * a.page_rows);
  };
  const bool ragged = a.slots && a.slot_width == 0;
  long long rows_before = 0, rows_all = 0;
  if (ragged) {
    long long before = more_before, rows = 0;
    for (int s0 = first; s0 < last; s0 += kPlanThreads) {
      const int seg = s0 + tid;
      Segment x = {};
      if (seg < last) x = segment(a, seg);
      const long long at = before + block_scan(max(x.need - x.have, 0), warp_sums, &sum);
      before += sum;
      int granted;
      rows += max(new_length(x, at, &granted) - x.len, 0);
    }
    block_scan(rows, warp_sums, &sum);
    if (tid == 0) totals[2] = sum;
    cluster.sync();
    for (int r = 0; r < n_cta; ++r) {
      if (r == rank) rows_before = rows_all;
      rows_all += cluster.map_shared_rank(totals, r)[2];
    }
  }
  long long before = more_before;
  for (int s0 = first; s0 < last; s0 += kPlanThreads) {
    const int seg = s0 + tid;
    Segment x = {};
    if (seg < last) x = segment(a, seg);
    const long long at = before + block_scan(max(x.need - x.have, 0), warp_sums, &sum);
    before += sum;
    int granted = 0;
    const int len = new_length(x, at, &granted);
    const int added = max(len - x.len, 0);
    if (seg < last) {
      short_of |= len < x.want;
      a.lens_out[seg] = len;
    }
    unsigned todo = __ballot_sync(0xffffffffu, granted > 0);
    for (; todo; todo &= todo - 1) {
      const int l = __ffs(todo) - 1;
      const int m = __shfl_sync(0xffffffffu, granted, l), have = __shfl_sync(0xffffffffu, x.have, l);
      const long long from = fits - 1 - __shfl_sync(0xffffffffu, at, l);
      int32_t* row = a.tables + (long long)(seg - lane + l) * a.max_pages + have;
      for (int i = lane; i < m; i += 32) row[i] = __ldcg(a.free_pages + from - i);
    }
    if (ragged) {
      const long long to = rows_before + block_scan(added, warp_sums, &sum);
      rows_before += sum;
      if (seg < last) {
        a.slot_offsets[seg] = (int)min(to, (long long)0x7fffffff);
        if (seg == a.n_seg - 1) a.slot_offsets[a.n_seg] = (int)min(to + added, (long long)0x7fffffff);
      }
      if (a.n_slots <= kSlotsHere) {
        todo = __ballot_sync(0xffffffffu, added > 0);
        for (; todo; todo &= todo - 1) {
          const int l = __ffs(todo) - 1;
          const int m = __shfl_sync(0xffffffffu, added, l), r0 = __shfl_sync(0xffffffffu, x.len, l);
          const long long t0 = __shfl_sync(0xffffffffu, to, l);
          const int32_t* row = a.tables + (long long)(seg - lane + l) * a.max_pages;
          __syncwarp();
          for (int i = lane; i < m && t0 + i < a.n_slots; i += 32) {
            const int pg = (r0 + i) / a.page_rows;
            a.slots[t0 + i] = row[pg] * a.page_rows + r0 + i - pg * a.page_rows;
          }
        }
      }
    } else if (a.slots) {
      // 32 segments' slots are one run of the output
      __syncwarp();
      const int here = min(last - (seg - lane), 32);
      for (int i0 = 0; i0 < here * a.slot_width; i0 += 32) {
        const int i = i0 + lane, l = min(i / a.slot_width, 31), e = i - l * a.slot_width;
        const int m = __shfl_sync(0xffffffffu, added, l), r = __shfl_sync(0xffffffffu, x.len, l) + e;
        if (i >= here * a.slot_width) continue;
        const long long sg = seg - lane + l;
        const int pg = r / a.page_rows;
        a.slots[sg * a.slot_width + e] = e < m ? a.tables[sg * a.max_pages + pg] * a.page_rows + r - pg * a.page_rows : -1;
      }
      short_of |= seg < last && added > a.slot_width;
    }
  }
  if (ragged) {
    short_of |= rows_all > a.n_slots;
    if (a.n_slots <= kSlotsHere)
      for (long long i = rows_all + rank * kPlanThreads + tid; i < a.n_slots; i += (long long)n_cta * kPlanThreads) a.slots[i] = -1;
  }
  if (short_of && a.status) *a.status = SLKV_ERR_CAPACITY;
  if (rank == 0 && tid == 0) a.n_free_out[0] = (int)max(fits - more_all, 0ll);
  cluster.sync();                                // no CTA's shared memory goes while another reads it
}

// Ragged slots, where there are many: a thread each, its segment by bisection.
__global__ void __launch_bounds__(256) k_paged_slots(const __grid_constant__ PagedPlanArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n_slots) return;
  if (i >= a.slot_offsets[a.n_seg]) { a.slots[i] = -1; return; }
  int lo = 0, hi = a.n_seg;                      // the last segment whose offset is not above i
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.slot_offsets[mid] <= i) lo = mid; else hi = mid;
  }
  const int r = a.lens_out[lo] - a.slot_offsets[lo + 1] + (int)i, pg = r / a.page_rows;
  a.slots[i] = a.tables[(long long)lo * a.max_pages + pg] * a.page_rows + r - pg * a.page_rows;
}

// 16 bytes of a K and a V row a thread, of kWriteRows rows at once: their slots are read first, then the rows.
constexpr int kWriteThreads = 256, kWriteRows = 4;
__global__ void __launch_bounds__(kWriteThreads) k_paged_write(const __grid_constant__ PagedWriteArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned ch = threadIdx.x & ((1u << a.chunk_bits) - 1), per = kWriteThreads >> a.chunk_bits;
  const unsigned row0 = blockIdx.x * per * kWriteRows + (threadIdx.x >> a.chunk_bits);
  unsigned slot[kWriteRows];
  uint4 x[kWriteRows], y[kWriteRows];
#pragma unroll
  for (int i = 0; i < kWriteRows; ++i) {
    const unsigned row = row0 + i * per;
    slot[i] = row < a.n_rows ? (unsigned)a.slots[row] : 0xffffffffu;
  }
#pragma unroll
  for (int i = 0; i < kWriteRows; ++i) {
    if (slot[i] >= a.pool_rows) continue;        // padding
    const unsigned row = row0 + i * per, seg = row / a.n_slots, r = row - seg * a.n_slots, s = seg / a.n_heads, h = seg - s * a.n_heads;
    const unsigned tok = a.take ? (unsigned)a.take[(size_t)s * a.n_slots + r] : r;
    if (tok >= a.n_tokens) { slot[i] = 0xffffffffu; continue; }
    x[i] = *reinterpret_cast<const uint4*>(a.k + s * a.stride[0] + tok * a.stride[1] + h * a.stride[2] + 16 * ch);
    y[i] = *reinterpret_cast<const uint4*>(a.v + s * a.stride[3] + tok * a.stride[4] + h * a.stride[5] + 16 * ch);
  }
#pragma unroll
  for (int i = 0; i < kWriteRows; ++i) {
    if (slot[i] >= a.pool_rows) continue;
    const size_t at = ((size_t)slot[i] << a.chunk_bits) + ch;
    a.k_pages[at] = x[i];
    a.v_pages[at] = y[i];
  }
}

}  // namespace

cudaError_t launch_paged_plan(const PagedPlanArgs& a, cudaStream_t st, int* launches) {
  {
    int ctas = 1;
    while (ctas < kPlanCluster && (long long)ctas * 256 < a.n_seg) ctas *= 2;
    LaunchScope scope(KID_PAGED_PLAN, st, launches);
    const cudaError_t e = launch_pdl(k_paged_plan, dim3((unsigned)ctas), dim3(kPlanThreads), 0, st, ctas, a);
    if (e != cudaSuccess) return e;
  }
  if (!a.slots || a.slot_width != 0 || a.n_slots <= kSlotsHere) return cudaSuccess;
  LaunchScope scope(KID_PAGED_PLAN, st, launches);
  return launch_pdl(k_paged_slots, dim3((unsigned)((a.n_slots + 255) / 256)), dim3(256), 0, st, 1, a);
}

cudaError_t launch_paged_write(const PagedWriteArgs& a, cudaStream_t st, int* launches) {
  LaunchScope scope(KID_PAGED_ROWS, st, launches);
  const unsigned rows = (kWriteThreads >> a.chunk_bits) * kWriteRows;
  return launch_pdl(k_paged_write, dim3((a.n_rows + rows - 1) / rows), dim3(kWriteThreads), 0, st, 1, a);
}

}  // namespace slkv
