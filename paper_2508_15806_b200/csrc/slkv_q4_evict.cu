// Eviction from the 4-bit cache: every segment keeps as many rows as its head's budget allows, the newest and those with the
// largest accumulated weights.
//
// Rows are ranked by 32-bit keys -- the newest rows first, then by weight, NaN last -- and a segment's kept rows are the
// `kept` largest, ties to the lower slot.  The kept-th largest key comes from a histogram with 64 bins to an octave -- that many, so
// that few lanes of a warp meet in a bin -- and from counting, for each of the keys in its bin, how many are above it.  Where a
// bin holds too many for that (weights that are all alike, or far out) their bits are descended, 11 + 11 + 10 of them.
// The kept rows that lie behind the first `kept` slots then fill the holes before them, in order, so that as few rows move as
// can, no row is read that another one overwrites, and a cache can be evicted from in place.
// A cluster of CTAs per segment (one CTA where there are many segments or few rows), each with a contiguous share of the slots, keys in
// shared memory; they share the moves evenly.  Where that is a handful of CTAs, a second launch moves the rows.
// What bounds it: for few rows the chain of passes over the keys, for many the rows' bytes.
#include <algorithm>
#include <atomic>

#include <cooperative_groups.h>

#include "slkv_q4_device.cuh"

namespace slkv {
namespace {

namespace cg = cooperative_groups;

constexpr int kEvictThreads = 512, kEvictBins = 2048, kEvictCluster = 8;
constexpr int kMostKeys = 40960;        // that shared memory holds beside the rest
// Keys that are ranked by counting, one for each thread: 128 of them take 0.5 us, 512 2 us; another histogram takes 1.5 us, and 8
// in a cluster.
template <bool CLUSTER> constexpr unsigned kFewKeys = CLUSTER ? kEvictThreads : 128;

struct Q4EvictArgs {
  Q4CacheView from, to;
  const int32_t *budgets, *newest;
  int32_t* status;
  int32_t* source;                      // [capacity of from] per kept slot, from its segment's first: the slot its row is in, or
                                        // ~i: the i-th of `movers`
  int32_t *holes, *movers;              // likewise: slots whose rows go, slots whose rows move
  int n_kv_heads, window, key_room;     // key_room: keys that the launch's shared memory holds
  int in_place, apart, ctas;            // apart: a second launch moves the rows; ctas: of a cluster
};

__device__ __forceinline__ unsigned evict_key(float weight, int pos, long long newest_kept) {
  if (pos > newest_kept) return 0xffffffffu;
  if (weight != weight) return 0u;
  const unsigned b = __float_as_uint(weight + 0.0f);       // -0 as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// First histogram: bins between 2^-22 and 2^10, the lowest for everything below, the highest for everything above.
__device__ __forceinline__ unsigned octave_bin(unsigned key) {
  constexpr unsigned kShift = 17, kFloor = 0x80000000u + ((127u - 22u) << 23) - (1u << kShift);
  return min((max(key, kFloor) - kFloor) >> kShift, kEvictBins - 1u);
}

// Adds one to the lanes' bins; all lanes in one bin (rows that nobody looked at) as one.  Whole warp.
__device__ __forceinline__ void count_bin(unsigned* hist, unsigned bin, bool valid) {
  const unsigned all = __ballot_sync(0xffffffffu, valid), lead = all ? __ffs(all) - 1 : 0;
  const unsigned of_lead = __shfl_sync(0xffffffffu, bin, lead);               // by all lanes, valid or not
  const bool alike = __all_sync(0xffffffffu, !valid || bin == of_lead);
  if (alike) {
    if (all && (threadIdx.x & 31) == lead) atomicAdd(&hist[bin], (unsigned)__popc(all));
  } else if (valid) {
    atomicAdd(&hist[bin], 1u);
  }
}

// Exclusive prefix sum over the CTA; *total: of all.
__device__ __forceinline__ unsigned cta_scan(unsigned x, unsigned* warp_sums, unsigned* total) {
  constexpr int kWarps = kEvictThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();                                         // the sums of the scan before are read
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  unsigned w = lane < kWarps ? warp_sums[lane] : 0u;
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, kWarps - 1);
  const unsigned upto = __shfl_sync(0xffffffffu, w, warp), own = __shfl_sync(0xffffffffu, inc, 31);
  return upto - own + inc - x;
}

// A row of each lane: from slot `src` of one cache to slot `dst` of the other, if that is not < 0.  The loads of ROUND 16-byte pieces
// to a lane come before their stores, and what `meanwhile` does in between; lanes without a row of their own read another's, since
// loads under a condition were not issued together (256 segments of 600 to 2400 rows: 27 us, 24 so).  Whole warp.
template <int HD, int ROUND, class F>
__device__ __forceinline__ void move_rows(const Q4EvictArgs& a, int src, int dst, int lane, F meanwhile) {
  constexpr int RB = q4_record_bytes(HD), kPieces = RB / 16;
  static_assert(kPieces % ROUND == 0, "whole rounds");
  const int pos = a.from.pos[src];
  const float weight = a.from.weight[src];
#pragma unroll
  for (int i0 = 0; i0 < kPieces; i0 += ROUND) {
    uint4 x[ROUND];
#pragma unroll
    for (int i = 0; i < ROUND; ++i) {
      const int piece = lane + 32 * (i0 + i), row = piece / kPieces, s = __shfl_sync(0xffffffffu, src, row);
      x[i] = __ldcs(reinterpret_cast<const uint4*>(a.from.records + (long long)s * RB) + (piece - row * kPieces));
    }
    meanwhile();
#pragma unroll
    for (int i = 0; i < ROUND; ++i) {
      const int piece = lane + 32 * (i0 + i), row = piece / kPieces, d = __shfl_sync(0xffffffffu, dst, row);
      if (d >= 0) *(reinterpret_cast<uint4*>(a.to.records + (long long)d * RB) + (piece - row * kPieces)) = x[i];
    }
  }
  if (dst >= 0) {
    a.to.pos[dst] = pos;
    a.to.weight[dst] = weight;
  }
}
constexpr int kRound = 5;               // of the evicting kernel: more would take registers that a second CTA per SM needs

struct EvictShared {
  alignas(16) unsigned hist[kEvictBins];   // of the CTA's keys
  unsigned few[kEvictThreads];               // the first CTA's: the keys that share the prefix
  unsigned warp_sums[32];
  unsigned found[3], n_few;
  alignas(16) unsigned counts[4];
};

template <int HD, bool CLUSTER>
__global__ void __launch_bounds__(kEvictThreads, 2) k_q4_evict(const __grid_constant__ Q4EvictArgs a) {
  extern __shared__ unsigned keys[];
  __shared__ EvictShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  auto sync = [&] {
    if constexpr (CLUSTER) cluster.sync();
    else __syncthreads();
  };
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = CLUSTER ? a.ctas : 1, rank = CLUSTER ? (int)cluster.block_rank() : 0, seg = blockIdx.x / ctas;
  EvictShared* first = CLUSTER ? cluster.map_shared_rank(&sh, 0) : &sh;
  const Q4Segment s = q4_segment(a.from.starts, a.from.lens, seg, a.from.capacity);
  const int sq = seg / a.n_kv_heads, h = seg - sq * a.n_kv_heads;
  const int kept = min(s.len, max(a.budgets[h], a.window));
  const Q4Segment d = a.in_place ? s : q4_segment(a.to.starts, a.to.starts, seg, a.to.capacity);
  sync();                                                  // the length is read by all before it changes
  if (rank == 0 && tid == 0) {
    a.to.lens[seg] = min(kept, d.room);
    if (kept > d.room && a.status) *a.status = SLKV_ERR_CAPACITY;
  }
  const int per_warp = 32, n_warps = ctas * (kEvictThreads / 32), my_warp = rank * (kEvictThreads / 32) + warp;
  if (kept == s.len) {                                     // everything stays
    if (!a.in_place)
      for (int i = my_warp * per_warp; i < min(kept, d.room); i += n_warps * per_warp) {
        const bool mine = i + lane < min(kept, d.room);
        if (!a.apart) move_rows<HD, kRound>(a, s.begin + min(i + lane, kept - 1), mine ? d.begin + i + lane : -1, lane, [] {});
        else if (mine) a.source[s.begin + i + lane] = i + lane;
      }
    return;
  }
  const float* weight = a.from.weight + s.begin;
  const int32_t* pos = a.from.pos + s.begin;
  const long long newest_kept = (long long)a.newest[sq] - a.window;
  // the CTA's slots [c0, c1)
  const int share = ((s.len + ctas - 1) / ctas + 3) & ~3, c0 = min(rank * share, s.len), c1 = min(c0 + share, s.len), n = c1 - c0;
  const bool cached = share <= a.key_room;
  auto key_at = [&](int i) { return cached ? keys[i] : evict_key(weight[c0 + i], pos[c0 + i], newest_kept); };

  // ---- the kept-th largest key
  unsigned prefix = 0, need = kept, equal = 0;             // need: of the keys that are looked at; equal: how many there are
  unsigned octave = 0;                                     // those in this bin of the first histogram
  int known = 0;                                           // and with this many bits of the prefix
  for (int level = 0;; ++level) {
    const int bits = level == 3 ? 10 : 11, shift = 32 - known - bits;
    for (int i = tid; i < kEvictBins; i += kEvictThreads) sh.hist[i] = 0;
    if (tid == 0) sh.n_few = 0;
    sync();
    constexpr int kAtOnce = CLUSTER ? 8 : 4;                 // loads on their way before the first is counted
    for (int i0 = 0; i0 < n; i0 += kAtOnce * kEvictThreads) {
      unsigned k[kAtOnce];
      if (level == 0) {
        float w[kAtOnce];
        int p[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
          const int i = min(i0 + e * kEvictThreads + tid, n - 1);
          w[e] = weight[c0 + i];
          p[e] = pos[c0 + i];
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) k[e] = evict_key(w[e], p[e], newest_kept);
      }
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const int i = i0 + e * kEvictThreads + tid;
        if (i0 + e * kEvictThreads >= n) break;
        if (level == 0) {
          if (cached && i < n) keys[i] = k[e];
          count_bin(sh.hist, octave_bin(k[e]), i < n);
        } else {
          const unsigned x = i < n ? key_at(i) : 0u;
          const bool in = i < n && octave_bin(x) == octave && (known == 0 || (x >> (32 - known)) == prefix);
          count_bin(sh.hist, (x >> shift) & ((1u << bits) - 1), in);
        }
      }
    }
    sync();
    // bins from the top, four to a thread: each CTA reads and adds up all CTAs' (adding into the first CTA's instead took 12 us)
    constexpr int kPer = kEvictBins / kEvictThreads;
    static_assert(kPer == 4, "one 16-byte load");
    const int top = kEvictBins - 1 - tid * kPer;
    unsigned bin[kPer] = {0, 0, 0, 0}, total;
#pragma unroll
    for (int r0 = 0; r0 < (CLUSTER ? kEvictCluster : 1); r0 += 4) {          // four loads under way at once
      uint4 x[4];
#pragma unroll
      for (int r = r0; r < r0 + 4; ++r) {
        x[r - r0] = make_uint4(0, 0, 0, 0);
        if (r < ctas) x[r - r0] = *reinterpret_cast<const uint4*>(&(CLUSTER ? cluster.map_shared_rank(&sh, r) : &sh)->hist[top - 3]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) { bin[0] += x[r].w; bin[1] += x[r].z; bin[2] += x[r].y; bin[3] += x[r].x; }
    }
    const unsigned mine = (bin[0] + bin[1]) + (bin[2] + bin[3]);
    unsigned above = cta_scan(mine, sh.warp_sums, &total);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (above < need && need <= above + bin[i]) {
        sh.found[0] = top - i;
        sh.found[1] = need - above;
        sh.found[2] = bin[i];
      }
      above += bin[i];
    }
    __syncthreads();
    if (level == 0) {
      octave = sh.found[0];
    } else {
      prefix = (prefix << bits) | sh.found[0];
      known += bits;
    }
    need = sh.found[1];
    equal = sh.found[2];
    if (known == 32 || equal <= kFewKeys<CLUSTER>) break;
    sync();                                                  // the histograms are read
  }
  if (known < 32) {                                          // few keys: which of them has need - 1 others above it?
    for (int i = tid; i < n; i += kEvictThreads) {
      const unsigned k = key_at(i);
      if (octave_bin(k) == octave && (known == 0 || (k >> (32 - known)) == prefix)) first->few[atomicAdd(&first->n_few, 1u)] = k;
    }
    sync();
    unsigned mine = 0, above = 0, same = 0;
    if (tid < (int)equal) mine = first->few[tid];
    const unsigned* few = CLUSTER ? sh.hist : sh.few;
    if constexpr (CLUSTER) {                                 // a copy nearby: nobody reads a histogram any more
      if (tid < (int)equal) sh.hist[tid] = mine;
      __syncthreads();
    }
    if (tid < (int)equal) {
      for (unsigned i = 0; i < equal; ++i) {
        above += few[i] > mine;
        same += few[i] == mine;
      }
      if (above < need && need <= above + same) {            // the same from every thread that has this key
        sh.found[0] = mine;
        sh.found[1] = need - above;
        sh.found[2] = same;
      }
    }
    __syncthreads();
    prefix = sh.found[0];
    need = sh.found[1];
    equal = sh.found[2];
  }

  // ---- kept or not, in the order of the slots: holes among the first `kept`, rows to move behind them.  Where a CTA's begin
  // follows from how many keys above and at the bound each CTA has on either side of slot `kept`.
  const bool ties = need < equal;
  unsigned n_equal = 0, n_holes = 0, n_moves = 0, all_moves = 0;      // of the CTAs before; then so far
  if constexpr (CLUSTER) {
    unsigned c[4] = {0, 0, 0, 0};                            // above / equal, before slot `kept` / behind
    for (int i = tid; i < n; i += kEvictThreads) {
      const unsigned k = key_at(i);
      const int behind = c0 + i >= kept;
      if (k > prefix) c[behind] += 1;
      else if (k == prefix) c[2 + behind] += 1;
    }
    if (tid < 4) sh.counts[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned x = __reduce_add_sync(0xffffffffu, c[e]);
      if (lane == 0 && x) atomicAdd(&sh.counts[e], x);
    }
    cluster.sync();
    unsigned eq = 0;                                         // keys at the bound so far
    uint4 of_cta = make_uint4(0, 0, 0, 0);                   // lane r: CTA r's
    if (lane < ctas) of_cta = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(&sh, lane)->counts);
    for (int r = 0; r < ctas; ++r) {
      const unsigned rc[4] = {__shfl_sync(0xffffffffu, of_cta.x, r), __shfl_sync(0xffffffffu, of_cta.y, r),
                              __shfl_sync(0xffffffffu, of_cta.z, r), __shfl_sync(0xffffffffu, of_cta.w, r)};
      const int b = min(r * share, s.len), e = min(b + share, s.len);
      const unsigned front = max(min(e, kept) - b, 0);       // its slots before `kept`
      const unsigned eq_front = min(rc[2], need - min(eq, need)), eq_back = min(rc[3], need - min(eq + rc[2], need));
      if (r == rank) n_equal = eq;
      if (r < rank) {
        n_holes += front - rc[0] - eq_front;
        n_moves += rc[1] + eq_back;
      }
      all_moves += rc[1] + eq_back;
      eq += rc[2] + rc[3];
    }
  }
  int32_t *holes = a.holes + s.begin, *movers = a.movers + s.begin, *source = a.source + s.begin;
  constexpr int kItems = 4;
  for (int i0 = 0; i0 < n; i0 += kEvictThreads * kItems) {
    const int at = i0 + tid * kItems;
    unsigned k[kItems], eq = 0;
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      k[e] = at + e < n ? key_at(at + e) : 0u;
      if (at + e < n && k[e] == prefix) eq |= 1u << e;
    }
    unsigned rank_of = 0, total;
    if (ties) {
      rank_of = n_equal + cta_scan(__popc(eq), sh.warp_sums, &total);
      n_equal += total;
    }
    unsigned hole = 0, mover = 0;
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      if (at + e >= n) break;
      bool keep = k[e] > prefix;
      if (eq >> e & 1) {
        keep = !ties || rank_of < need;
        ++rank_of;
      }
      if (c0 + at + e < kept) {
        if (!keep) hole |= 1u << e;
      } else if (keep) {
        mover |= 1u << e;
      }
    }
    const unsigned before = cta_scan(__popc(hole) | (__popc(mover) << 16), sh.warp_sums, &total);      // at most 2048 of either
    unsigned nh = n_holes + (before & 0xffffu), nm = n_moves + (before >> 16);
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      const int slot = c0 + at + e;
      if (at + e >= n) break;
      if (mover >> e & 1) movers[nm++] = slot;
      if (a.in_place) {
        if (hole >> e & 1) holes[nh++] = slot;
      } else if (slot < kept) {
        source[slot] = hole >> e & 1 ? ~(int)nh++ : slot;
      }
    }
    n_holes += total & 0xffffu;
    n_moves += total >> 16;
  }
  if (!CLUSTER) all_moves = n_moves;
  __threadfence();                                           // the lists are read by other CTAs of the cluster
  sync();
  if (a.apart) return;

  // ---- the rows
  if (a.in_place) {
    for (int i = my_warp * per_warp; i < (int)all_moves; i += n_warps * per_warp) {
      const int j = min(i + lane, (int)all_moves - 1);
      move_rows<HD, kRound>(a, s.begin + movers[j], i + lane == j ? s.begin + holes[j] : -1, lane, [] {});
    }
  } else {
    const int rows = min(kept, d.room);
    for (int i = my_warp * per_warp; i < rows; i += n_warps * per_warp) {
      const int j = min(i + lane, rows - 1);
      int src = source[j];
      if (src < 0) src = movers[~src];
      move_rows<HD, kRound>(a, s.begin + src, i + lane == j ? d.begin + j : -1, lane, [] {});
    }
  }
}

// The rows of an eviction into another cache, over that one's slots.
constexpr int kMoveWarps = 8;
template <int HD>
__global__ void __launch_bounds__(kMoveWarps * 32) k_q4_move(const __grid_constant__ Q4EvictArgs a) {
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_seg = a.to.n_seg;
  // where the row of slot r0 + lane comes from; < 0: from nowhere
  auto source_of = [&](long long r0) {
    const long long r = r0 + lane;
    int src = -1;
    if (r0 >= a.to.capacity) return src;
    int seg = q4_find(a.to.starts, n_seg, (int)r0, lane);
    if (r < a.to.capacity) {
      while (seg + 1 < n_seg && a.to.starts[seg + 1] <= r) ++seg;
      const Q4Segment d = q4_segment(a.to.starts, a.to.lens, seg, a.to.capacity);
      if (r >= d.begin && r < (long long)d.begin + d.len) {
        const int begin = q4_segment(a.from.starts, a.from.starts, seg, a.from.capacity).begin;
        src = a.source[begin + (int)(r - d.begin)];
        if (src < 0) src = a.movers[begin + ~src];
        src += begin;
      }
    }
    return src;
  };
  const long long step = (long long)gridDim.x * kMoveWarps * 32;
  long long r0 = ((long long)blockIdx.x * kMoveWarps + warp) * 32;
  int next = source_of(r0);
  for (; r0 < a.to.capacity; r0 += step) {
    const int src = next;
    const unsigned some = __ballot_sync(0xffffffffu, src >= 0);
    if (some) {
      const int any = __shfl_sync(0xffffffffu, src, __ffs(some) - 1);      // for lanes that have none to read, too
      move_rows<HD, q4_record_bytes(HD) / 16>(a, src >= 0 ? src : any, src >= 0 ? (int)(r0 + lane) : -1, lane,
                                              [&] { next = source_of(r0 + step); });
    } else {
      next = source_of(r0 + step);
    }
  }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

template <int HD, bool CLUSTER>
cudaError_t launch_evict(const Q4EvictArgs& a, cudaStream_t st) {
  auto kernel = k_q4_evict<HD, CLUSTER>;
  static std::atomic<unsigned> allowed{0};                 // devices on which the kernel may have that much shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 32 || !(allowed.load(std::memory_order_relaxed) >> dev & 1u)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKeys * (int)sizeof(unsigned));
    if (e != cudaSuccess) return e;
    if (dev < 32) allowed.fetch_or(1u << dev, std::memory_order_relaxed);
  }
  return launch_pdl(kernel, dim3((unsigned)(a.from.n_seg * a.ctas)), dim3(kEvictThreads), (size_t)a.key_room * sizeof(unsigned), st, a.ctas, a);
}

}  // namespace

size_t q4_evict_workspace(int n_seg, long long capacity) { return 3 * up256((size_t)capacity * sizeof(int32_t)); }

cudaError_t launch_q4_evict(const Q4CacheView& from, const Q4CacheView& to, int n_kv_heads, int head_dim, const int32_t* budgets,
                            int window, const int32_t* newest, int32_t* status, void* workspace, cudaStream_t st, int* launches) {
  Q4EvictArgs a = {};
  a.from = from; a.to = to; a.budgets = budgets; a.newest = newest; a.status = status;
  char* ws = static_cast<char*>(workspace);
  const size_t rows = up256((size_t)from.capacity * sizeof(int32_t));
  a.source = reinterpret_cast<int32_t*>(ws);
  a.holes = reinterpret_cast<int32_t*>(ws + rows);
  a.movers = reinterpret_cast<int32_t*>(ws + 2 * rows);
  a.n_kv_heads = n_kv_heads; a.window = window;
  a.in_place = from.records == to.records;
  const long long room = from.capacity / from.n_seg;       // of an average segment
  // CTAs per segment: as many as the device holds beside the other segments, but some 2000 slots for each
  a.ctas = 1;
  while (a.ctas < kEvictCluster && 2ll * a.ctas * from.n_seg <= 2 * sm_count() && room >= 4096ll * a.ctas) a.ctas *= 2;
  a.key_room = 2048;                                       // for segments of up to twice the average
  while (a.key_room < 2 * room / a.ctas && a.key_room < kMostKeys) a.key_room *= 2;
  if (a.key_room > kMostKeys) a.key_room = kMostKeys;
  // A second launch for the rows where the clusters have only a few SMs to move them with (into another cache, half of the rows kept
  // where nothing else is said): 1 segment of 300000 rows 102 us against 185, 2 of 65536 35 against 50, 8 of 8192 with four CTAs
  // each 17 either way, 16 against 20 with 95 % kept; 8 of 32768 with eight CTAs each 37 against 35, 64 of 8192 36 against 27.
  a.apart = !a.in_place && a.ctas > 1 && (long long)from.n_seg * a.ctas <= sm_count() / 4;
  {
    LaunchScope scope(KID_Q4_EVICT, st, launches);
    const cudaError_t e = head_dim == 128 ? (a.ctas > 1 ? launch_evict<128, true>(a, st) : launch_evict<128, false>(a, st))
                                          : (a.ctas > 1 ? launch_evict<64, true>(a, st) : launch_evict<64, false>(a, st));
    if (e != cudaSuccess || !a.apart) return e;
  }
  LaunchScope scope(KID_Q4_MOVE, st, launches);
  const long long chunks = (to.capacity + kMoveWarps * 32 - 1) / (kMoveWarps * 32);
  const dim3 grid((unsigned)std::min(chunks, 6ll * sm_count())), block(kMoveWarps * 32);
  return head_dim == 128 ? launch_pdl(k_q4_move<128>, grid, block, 0, st, 1, a) : launch_pdl(k_q4_move<64>, grid, block, 0, st, 1, a);
}

}  // namespace slkv
