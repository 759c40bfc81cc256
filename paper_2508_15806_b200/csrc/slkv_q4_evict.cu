// Eviction from the 4-bit cache: every segment keeps as many rows as its head's budget allows, the newest and those with the
// largest accumulated weights.
//
// Rows are ranked by 32-bit keys -- the newest rows first, then by weight, NaN last -- and a segment's kept rows are the
// `kept` largest, ties to the lower slot: a descent over the keys' bits, 11 + 11 + 10 of them, with a histogram each.  The kept
// rows that lie behind the first `kept` slots then fill the holes before them, in order, so that as few rows move as can, no
// row is read that another one overwrites, and a cache can be evicted from in place.
// Two launches: the selection, a CTA per segment, leaves for every kept slot where its row comes from; the moves are spread
// over the whole device.  What bounds it: for few rows the selection's chain of passes over its keys, for many the rows' bytes.
#include "slkv_q4_device.cuh"

namespace slkv {
namespace {

constexpr int kEvictBins = 2048;
constexpr int kMostKeys = 49152;        // that shared memory holds

struct Q4EvictArgs {
  Q4CacheView from, to;
  const int32_t *budgets, *newest;
  int32_t* status;
  int32_t* source;                      // [capacity of from] per kept slot, from its segment's first: the slot its row is in
  int32_t *holes, *movers;              // likewise
  int32_t* kept;                        // [n_seg] rows to write
  int n_kv_heads, window, key_room;     // key_room: keys that the launch's shared memory holds
  int in_place, splits;
};

__device__ __forceinline__ unsigned evict_key(float weight, int pos, long long newest_kept) {
  if (pos > newest_kept) return 0xffffffffu;
  if (weight != weight) return 0u;
  const unsigned b = __float_as_uint(weight + 0.0f);       // -0 as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive prefix sum over the CTA; *total: of all.
__device__ __forceinline__ unsigned cta_scan(unsigned x, unsigned* warp_sums, unsigned* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  unsigned inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();                                         // the sums of the scan before are read
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  unsigned w = lane < n_warps ? warp_sums[lane] : 0u;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const unsigned before = __shfl_sync(0xffffffffu, w, warp) - __shfl_sync(0xffffffffu, inc, 31);
  return before + inc - x;
}

__global__ void __launch_bounds__(1024) k_q4_evict_select(const __grid_constant__ Q4EvictArgs a) {
  extern __shared__ unsigned keys[];
  __shared__ unsigned hist[kEvictBins];
  __shared__ unsigned warp_sums[32];
  __shared__ unsigned found[3];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, seg = blockIdx.x, threads = blockDim.x;
  const Q4Segment s = q4_segment(a.from.starts, a.from.lens, seg, a.from.capacity);
  const int sq = seg / a.n_kv_heads, h = seg - sq * a.n_kv_heads;
  const int kept = min(s.len, max(a.budgets[h], a.window));
  const int room = a.in_place ? s.room : q4_segment(a.to.starts, a.to.starts, seg, a.to.capacity).room;
  __syncthreads();                                         // the length is read by all before it changes
  if (tid == 0) {
    a.to.lens[seg] = min(kept, room);
    a.kept[seg] = a.in_place && kept == s.len ? 0 : min(kept, room);
    if (kept > room && a.status) *a.status = SLKV_ERR_CAPACITY;
  }
  int32_t* source = a.source + s.begin;
  if (kept == s.len) {                                     // everything stays
    if (!a.in_place)
      for (int i = tid; i < kept; i += threads) source[i] = i;
    return;
  }
  const float* weight = a.from.weight + s.begin;
  const int32_t* pos = a.from.pos + s.begin;
  const long long newest_kept = (long long)a.newest[sq] - a.window;
  const bool cached = s.len <= a.key_room;
  auto key_at = [&](int i) { return cached ? keys[i] : evict_key(weight[i], pos[i], newest_kept); };
  if (cached)
    for (int i = tid; i < s.len; i += threads) keys[i] = evict_key(weight[i], pos[i], newest_kept);

  // ---- the kept-th largest key: its bits from the top
  unsigned prefix = 0, need = kept, equal = 0;             // need: of the keys that share the prefix; equal: how many do
#pragma unroll
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    for (int i = tid; i < kEvictBins; i += threads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < s.len; i += threads) {
      const unsigned k = key_at(i);
      if (level == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // bins from the top, consecutive ones to a thread
    const int per = kEvictBins / threads, top = kEvictBins - 1 - tid * per;
    unsigned mine = 0;
    for (int i = 0; i < per; ++i) mine += hist[top - i];
    unsigned total;
    unsigned above = cta_scan(mine, warp_sums, &total);
    if (above < need && need <= above + mine) {
      int i = 0;
      unsigned c = hist[top];
      while (above + c < need) {
        above += c;
        ++i;
        c = hist[top - i];
      }
      found[0] = top - i;
      found[1] = need - above;
      found[2] = c;
    }
    __syncthreads();
    prefix = (prefix << bits) | found[0];
    need = found[1];
    equal = found[2];
    __syncthreads();
  }

  // ---- kept or not, in the order of the slots: holes among the first `kept`, rows to move behind them
  int32_t *holes = a.holes + s.begin, *movers = a.movers + s.begin;
  const bool ties = need < equal;
  unsigned n_equal = 0, n_holes = 0, n_moves = 0;          // so far
  constexpr int kItems = 4;
  for (int i0 = 0; i0 < s.len; i0 += threads * kItems) {
    const int at = i0 + tid * kItems;
    unsigned k[kItems], eq = 0;
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      k[e] = at + e < s.len ? key_at(at + e) : 0u;
      if (at + e < s.len && k[e] == prefix) eq |= 1u << e;
    }
    unsigned rank = 0, total;
    if (ties) {
      rank = n_equal + cta_scan(__popc(eq), warp_sums, &total);
      n_equal += total;
    }
    unsigned hole = 0, mover = 0;
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      if (at + e >= s.len) break;
      bool keep = k[e] > prefix;
      if (eq >> e & 1) {
        keep = !ties || rank < need;
        ++rank;
      }
      if (at + e < kept) {
        if (!keep) hole |= 1u << e;
        source[at + e] = at + e;
      } else if (keep) {
        mover |= 1u << e;
      }
    }
    const unsigned before = cta_scan(__popc(hole) | (__popc(mover) << 16), warp_sums, &total);   // at most 4096 of either
    unsigned nh = n_holes + (before & 0xffffu), nm = n_moves + (before >> 16);
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      if (hole >> e & 1) holes[nh++] = at + e;
      if (mover >> e & 1) movers[nm++] = at + e;
    }
    n_holes += total & 0xffffu;
    n_moves += total >> 16;
  }
  __syncthreads();
  for (unsigned i = tid; i < n_moves; i += threads) source[holes[i]] = movers[i];
}

// Kept rows to their places.  A warp looks at 32 slots; those whose row comes from elsewhere are moved together.
template <int HD>
__global__ void __launch_bounds__(256) k_q4_evict_move(const __grid_constant__ Q4EvictArgs a) {
  constexpr int RB = q4_record_bytes(HD), kLanes = RB / 16, kAtOnce = 32 / kLanes;      // lanes per record, records at once
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int seg = blockIdx.x / a.splits, split = blockIdx.x - seg * a.splits;
  const int kept = a.kept[seg];
  if (kept == 0) return;
  const int from0 = q4_segment(a.from.starts, a.to.lens, seg, a.from.capacity).begin;
  const int to0 = a.in_place ? from0 : q4_segment(a.to.starts, a.to.lens, seg, a.to.capacity).begin;
  const int sub = lane / kLanes, part = lane - sub * kLanes;
  for (int i0 = (split * 8 + warp) * 32; i0 < kept; i0 += a.splits * 256) {
    const int i = i0 + lane;
    const int src = i < kept ? a.source[from0 + i] : 0;
    const bool moves = i < kept && !(a.in_place && src == i);
    if (moves) {
      a.to.pos[to0 + i] = a.from.pos[from0 + src];
      a.to.weight[to0 + i] = a.from.weight[from0 + src];
    }
    unsigned todo = __ballot_sync(0xffffffffu, moves);
    while (todo) {
      unsigned mine = todo;                                // the sub-th of them
      for (int e = 0; e < sub && mine; ++e) mine &= mine - 1;
      const int which = mine ? __ffs(mine) - 1 : 0;
      const int row_src = __shfl_sync(0xffffffffu, src, which);
      if (mine && sub < kAtOnce)
        *reinterpret_cast<uint4*>(a.to.records + (long long)(to0 + i0 + which) * RB + part * 16) =
            *reinterpret_cast<const uint4*>(a.from.records + (long long)(from0 + row_src) * RB + part * 16);
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) todo &= todo - 1;
    }
  }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t q4_evict_workspace(int n_seg, long long capacity) {
  return 3 * up256((size_t)capacity * sizeof(int32_t)) + up256((size_t)n_seg * sizeof(int32_t));
}

cudaError_t launch_q4_evict(const Q4CacheView& from, const Q4CacheView& to, int n_kv_heads, int head_dim, const int32_t* budgets,
                            int window, const int32_t* newest, int32_t* status, void* workspace, cudaStream_t st, int* launches) {
  Q4EvictArgs a = {};
  a.from = from; a.to = to; a.budgets = budgets; a.newest = newest; a.status = status;
  char* ws = static_cast<char*>(workspace);
  const size_t rows = up256((size_t)from.capacity * sizeof(int32_t));
  a.source = reinterpret_cast<int32_t*>(ws);
  a.holes = reinterpret_cast<int32_t*>(ws + rows);
  a.movers = reinterpret_cast<int32_t*>(ws + 2 * rows);
  a.kept = reinterpret_cast<int32_t*>(ws + 3 * rows);
  a.n_kv_heads = n_kv_heads; a.window = window;
  a.in_place = from.records == to.records;
  const long long room = from.capacity / from.n_seg;       // of an average segment
  const int threads = room <= 2048 ? 256 : room <= 16384 ? 512 : 1024;
  a.key_room = 2048;
  while (a.key_room < 2 * room && a.key_room < kMostKeys) a.key_room *= 2;
  if (a.key_room > kMostKeys) a.key_room = kMostKeys;
  cudaError_t e = cudaFuncSetAttribute(k_q4_evict_select, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKeys * (int)sizeof(unsigned));
  if (e != cudaSuccess) return e;
  {
    LaunchScope scope(KID_Q4_EVICT, st, launches);
    e = launch_pdl(k_q4_evict_select, dim3((unsigned)from.n_seg), dim3((unsigned)threads), (size_t)a.key_room * sizeof(unsigned), st, 1, a);
  }
  if (e != cudaSuccess) return e;
  const long long want = (room + 255) / 256, most = 65535ll * 16 / from.n_seg;
  a.splits = (int)(want < 1 ? 1 : want < 256 ? want : 256);
  if (a.splits > most) a.splits = (int)(most < 1 ? 1 : most);
  LaunchScope scope(KID_Q4_EVICT, st, launches);
  return launch_pdl(head_dim == 128 ? k_q4_evict_move<128> : k_q4_evict_move<64>, dim3((unsigned)(from.n_seg * a.splits)), dim3(256),
                    0, st, 1, a);
}

}  // namespace slkv
