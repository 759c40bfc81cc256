// Pages of a 16-bit or fp32 cache whose segments have lengths of their own: planning (which pages a segment gets or gives back, where its
// new rows go) and writing rows through the resulting slots.
#include <cooperative_groups.h>

#include "slkv_paged.cuh"

namespace slkv {
namespace {

namespace cg = cooperative_groups;

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32, kPlanCluster = 8;

// Exclusive prefix over the block of two values a thread (32 bits each, sums below 2^31 of the lower one); *total: of all.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* warp_sums, unsigned long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  unsigned long long incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (n_warps == 1) {
    *total = __shfl_sync(0xffffffffu, incl, 31);
    return incl - v;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  unsigned long long before = 0, all = 0;
#pragma unroll 4
  for (int w = 0; w < n_warps; ++w) {
    const unsigned long long x = warp_sums[w];
    if (w < warp) before += x;
    all += x;
  }
  *total = all;
  __syncthreads();                               // warp_sums may be written again
  return before + incl - v;
}
__device__ __forceinline__ unsigned long long pack(unsigned hi, unsigned lo) { return (unsigned long long)hi << 32 | lo; }

struct Segment { int len, want, have, need; };

__device__ __forceinline__ Segment segment(const PagedPlanArgs& a, int seg) {
  Segment x;
  const int most = a.max_pages << a.page_bits;
  x.len = min(max(a.lens[seg], 0), most);
  long long want;
  if (a.mode == SLKV_PAGED_LENGTHS) {
    want = a.want[seg];
  } else if (a.mode == SLKV_PAGED_OFFSETS) {
    const int per = a.n_seqs * a.n_kv_heads, layer = (unsigned)seg / (unsigned)per;
    const int32_t* o = a.want + seg + layer;     // a layer has one offset more than segments
    want = (long long)o[1] - o[0];
  } else {
    want = (long long)x.len + max(a.want[(unsigned)seg / (unsigned)a.n_kv_heads % (unsigned)a.n_seqs], 0);
  }
  x.want = (int)min(max(want, 0ll), (long long)most);
  const int mask = (1 << a.page_bits) - 1;
  x.have = (x.len + mask) >> a.page_bits;
  x.need = (x.want + mask) >> a.page_bits;
  return x;
}

__device__ __forceinline__ int slot_of(const PagedPlanArgs& a, long long table, int row) {
  return (a.tables[table + (row >> a.page_bits)] << a.page_bits) + (row & ((1 << a.page_bits) - 1));
}

// dst[to + TO i] = src[from + FROM i] for i below each thread's count, where that lies below `limit`: by the thread itself where all have
// few, else by all warps of the CTA, each at a thread's run or, where only the first n_runs threads have one and they are few, several.
struct Run { long long to, from; int count; };
template <int TO, int FROM>
__device__ __forceinline__ void move_runs(int32_t* dst, long long limit, const int32_t* src, Run mine, Run* runs, int n_runs) {
  constexpr int kFew = 4;
  auto move = [&](const Run& r, int i) {
    if ((unsigned long long)(r.to + TO * i) < (unsigned long long)limit) dst[r.to + TO * i] = __ldcg(src + r.from + FROM * i);
  };
  if (!__syncthreads_or(mine.count > kFew)) {
#pragma unroll
    for (int i = 0; i < kFew; ++i)
      if (i < mine.count) move(mine, i);
  } else {
    runs[threadIdx.x] = mine;
    __syncthreads();
    const int warps = (int)blockDim.x >> 5, group = max(warps / max(n_runs, 1), 1) << 5, at = threadIdx.x % group;
    for (int t = threadIdx.x / group; t < n_runs; t += (int)blockDim.x / group) {
      const Run r = runs[t];
#pragma unroll 4
      for (int i = at; i < r.count; i += group) move(r, i);
    }
  }
  __syncthreads();                               // the entries are there for the slots; runs may be written again
}

// One cluster, or one CTA where that does.  A CTA has a run of segments, a thread each at a time; what lies before a segment is what the
// CTAs before this one come to (exchanged through their shared memory) and a scan.  What bounds it: three or four dependent reads of L2
// and the barriers between them, the data is a few hundred KB at most; so lengths are read once where a thread has one segment, and
// pages returned and taken are counted in one scan.  A step's accepted rows (128 segments) 6.7 us, 4096 segments in a cluster of 8 7.9;
// 128 segments of up to 12000 rows that come in 15, most of it their pages, which go from the stack to the tables.
__global__ void __launch_bounds__(kPlanThreads) k_paged_plan(const __grid_constant__ PagedPlanArgs a) {
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ unsigned long long warp_sums[kPlanWarps];
  __shared__ Run runs[kPlanThreads];
  __shared__ unsigned long long totals[2];       // of this CTA: pages returned and wanted; rows that come in
  const int rank = (int)cluster.block_rank(), n_cta = (int)cluster.num_blocks();
  const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
  auto sync = [&] {
    if (n_cta == 1) __syncthreads();
    else cluster.sync();
  };
  pdl_launch_dependents();
  pdl_wait();
  const int first = (int)((long long)a.n_seg * rank / n_cta), last = (int)((long long)a.n_seg * (rank + 1) / n_cta);
  const bool once = last - first <= threads;     // a segment a thread: x and its place stay in registers
  const long long n_free = min(max(a.n_free[0], 0), a.n_pages);

  Segment x = {};
  unsigned long long place = 0, sum = 0, all = 0;
  for (int s0 = first; s0 < last; s0 += threads) {
    x = Segment{};
    if (s0 + tid < last) x = segment(a, s0 + tid);
    place = all + block_scan(pack(max(x.have - x.need, 0), max(x.need - x.have, 0)), warp_sums, &sum);
    all += sum;
  }
  unsigned long long before = 0, total = all;
  if (n_cta > 1) {
    if (tid == 0) totals[0] = all;
    cluster.sync();
    total = 0;
    for (int r = 0; r < n_cta; ++r) {
      if (r == rank) before = total;
      total += cluster.map_shared_rank(totals, r)[0];
    }
  }
  const long long gone_all = total >> 32, more_all = total & 0xffffffffu;
  const long long stack = n_free + gone_all;     // pages on it once all are returned
  // The segments again, with what lies before each: returned pages in the upper word, wanted ones in the lower.
  auto again = [&](auto body) {
    if (once) {
      body(first + tid, x, before + place);
      return;
    }
    unsigned long long run = before;
    for (int s0 = first; s0 < last; s0 += threads) {
      Segment y = {};
      if (s0 + tid < last) y = segment(a, s0 + tid);
      const unsigned long long at = run + block_scan(pack(max(y.have - y.need, 0), max(y.need - y.have, 0)), warp_sums, &sum);
      run += sum;
      body(s0 + tid, y, at);
    }
  };

  if (gone_all > 0) {                            // the first segment's first page ends up on top
    again([&](int seg, const Segment& y, unsigned long long at) {
      move_runs<-1, 1>(a.free_pages, a.n_pages, a.tables,
                       {stack - 1 - (long long)(at >> 32), (long long)seg * a.max_pages + y.need, max(y.have - y.need, 0)}, runs,
                       min(last - first, threads));
    });
    sync();                                      // some are taken again below
  }

  // pages taken and new lengths; rows that come in
  const long long fits = min(stack, (long long)a.n_pages), entries = (long long)a.n_seg * a.max_pages;
  auto new_length = [&](const Segment& y, unsigned long long at, int* granted) {
    const int wanted = max(y.need - y.have, 0);
    *granted = (int)min(max(fits - (long long)(at & 0xffffffffu), 0ll), (long long)wanted);
    return min(y.want, (min(y.have, y.need) + *granted) << a.page_bits);
  };
  const bool ragged = a.slots && a.slot_width == 0;
  unsigned long long rows_before = 0, rows_all = 0;
  if (ragged && n_cta > 1) {
    unsigned long long rows = 0;
    again([&](int, const Segment& y, unsigned long long at) {
      int granted;
      block_scan((unsigned long long)max(new_length(y, at, &granted) - y.len, 0), warp_sums, &sum);
      rows += sum;
    });
    if (tid == 0) totals[1] = rows;
    cluster.sync();
    for (int r = 0; r < n_cta; ++r) {
      if (r == rank) rows_before = rows_all;
      rows_all += cluster.map_shared_rank(totals, r)[1];
    }
  }
  bool short_of = false;
  again([&](int seg, const Segment& y, unsigned long long at) {
    int granted;
    const int len = new_length(y, at, &granted), added = max(len - y.len, 0);
    const bool mine = seg < last;
    if (mine) {
      short_of |= len < y.want;
      a.lens_out[seg] = len;
    }
    const long long row0 = (long long)seg * a.max_pages;
    move_runs<1, -1>(a.tables, entries, a.free_pages, {row0 + y.have, fits - 1 - (long long)(at & 0xffffffffu), mine ? granted : 0}, runs,
                     min(last - first, threads));
    if (ragged) {
      const unsigned long long to = rows_before + block_scan((unsigned long long)added, warp_sums, &sum);
      rows_before += sum;
      if (mine) {
        a.slot_offsets[seg] = (int)min(to, 0x7fffffffull);
        if (seg == a.n_seg - 1) a.slot_offsets[a.n_seg] = (int)min(to + added, 0x7fffffffull);
      }
    } else if (a.slots) {
      short_of |= mine && added > a.slot_width;
      if (a.slot_width <= 16) {                  // a lane its own segment's
        if (mine)
          for (int e = 0; e < a.slot_width; ++e) a.slots[(long long)seg * a.slot_width + e] = e < added ? slot_of(a, row0, y.len + e) : -1;
      } else {
        for (unsigned todo = __ballot_sync(0xffffffffu, mine); todo; todo &= todo - 1) {
          const int l = __ffs(todo) - 1, m = __shfl_sync(0xffffffffu, added, l), r0 = __shfl_sync(0xffffffffu, y.len, l);
          const long long table = __shfl_sync(0xffffffffu, row0, l), to = (long long)(seg - lane + l) * a.slot_width;
          for (int e = lane; e < a.slot_width; e += 32) a.slots[to + e] = e < m ? slot_of(a, table, r0 + e) : -1;
        }
      }
    }
  });
  if (ragged) {
    if (n_cta == 1) rows_all = rows_before;
    short_of |= rows_all > (unsigned long long)a.n_slots;
  }
  if (short_of && a.status) *a.status = SLKV_ERR_CAPACITY;
  if (rank == 0 && tid == 0) a.n_free_out[0] = (int)max(fits - more_all, 0ll);
  if (n_cta > 1) cluster.sync();                 // no CTA's shared memory goes while another reads it
}

// Ragged slots, a launch of their own (in the one that plans, 23000 of 32 segments took 40 us more): 256 in a row to a warp, which finds the
// first one's segment by bisection; from there each lane goes on.  667000 slots take 6.4 us, most of it the bisection's dependent reads.
constexpr int kSlotThreads = 256, kSlotsOfWarp = 256;
__global__ void __launch_bounds__(kSlotThreads) k_paged_slots(const __grid_constant__ PagedPlanArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const long long first = ((long long)blockIdx.x * (kSlotThreads / 32) + (threadIdx.x >> 5)) * kSlotsOfWarp;
  if (first >= a.n_slots) return;
  const int rows = a.slot_offsets[a.n_seg];
  int lo = 0, hi = a.n_seg;                      // the last segment whose offset is not above the first slot
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.slot_offsets[mid] <= first) lo = mid; else hi = mid;
  }
#pragma unroll 2
  for (long long i = first + (threadIdx.x & 31); i < first + kSlotsOfWarp && i < a.n_slots; i += 32) {
    int slot = -1;
    if (i < rows) {
      while (a.slot_offsets[lo + 1] <= i) ++lo;
      slot = slot_of(a, (long long)lo * a.max_pages, a.lens_out[lo] - a.slot_offsets[lo + 1] + (int)i);
    }
    a.slots[i] = slot;
  }
}

// 16 bytes of a K and a V row a thread, of kWriteRows rows at once: their slots are read first, then the rows.  Bound by DRAM: 667000 rows of
// 256 bytes, read and written, take 100 us (6.8 TB/s, 104 % of a plain copy's rate).
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
    // A segment a thread as far as a cluster goes, or, where whole segments come and go, 32 a CTA, which moves their pages.  Both sides of
    // that, with slots and rows, us: 32 segments of 1200 rows 16.3 in one CTA, 19.3 in two; 128 of 7000 126 in one, 122 in eight;
    // 512 of 600 67 / 59.
    int ctas = 1;
    const int each = a.mode != SLKV_PAGED_ADD ? 32 : kPlanThreads / 2;
    while (ctas < kPlanCluster && ctas * each < a.n_seg) ctas *= 2;
    int threads = (a.n_seg + ctas - 1) / ctas;
    threads = threads >= kPlanThreads ? kPlanThreads : (threads + 31) / 32 * 32;
    if (a.mode != SLKV_PAGED_ADD) threads = kPlanThreads;      // whole segments come and go: the warps move their pages
    LaunchScope scope(KID_PAGED_PLAN, st, launches);
    const cudaError_t e = launch_pdl(k_paged_plan, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, ctas, a);
    if (e != cudaSuccess) return e;
  }
  if (!a.slots || a.slot_width != 0 || a.n_slots == 0) return cudaSuccess;
  LaunchScope scope(KID_PAGED_PLAN, st, launches);
  const long long per = kSlotThreads / 32 * kSlotsOfWarp;
  return launch_pdl(k_paged_slots, dim3((unsigned)((a.n_slots + per - 1) / per)), dim3(kSlotThreads), 0, st, 1, a);
}

cudaError_t launch_paged_write(const PagedWriteArgs& a, cudaStream_t st, int* launches) {
  LaunchScope scope(KID_PAGED_ROWS, st, launches);
  const unsigned rows = (kWriteThreads >> a.chunk_bits) * kWriteRows;
  return launch_pdl(k_paged_write, dim3((a.n_rows + rows - 1) / rows), dim3(kWriteThreads), 0, st, 1, a);
}

}  // namespace slkv
