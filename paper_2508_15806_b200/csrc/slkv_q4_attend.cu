// Attention of new tokens over the 4-bit cache: out = softmax(f(scale q.k)) v per query head, its log-sum-exp, and the rows'
// accumulated weights.
//
// One pass over the records with a running maximum and sum (base 2, fp32).  Four bits become matrix operands in registers.  The
// low eight bits of a bf16 with nothing above them are an integer times 2^-133 -- subnormal up to 127, the first normal numbers
// from there on -- so a nibble needs no more than a mask where it lies in them, the lower one as it is, the upper one as 16 times
// itself: one shift and four masks make eight operands.
//   scores  the queries are scaled by 2^60, those that meet upper nibbles by 2^56: exact, and every product of one of 2^-50 or more
//           is a normal fp32 number.  A score is the sum over groups of scale * product, plus the sum over groups of zero *
//           (sum of the group's queries), which is one more product: the zeros as they lie in the record, the query sums in three
//           bf16 parts.
//   output  one packed multiply-add makes (c - 8) / 128 of a value nibble, exactly.  Probabilities times the group's scale,
//           rounded to bf16, are the other operand.  zero + 8 scale goes with the unrounded probabilities, in fp32.  With a second
//           bf16 part of the operand, a relative error of 0.0023 over 64 long segments became the 0.0017 of the bf16 output itself, at
//           105 us instead of 93 (256 segments of 256 to 4096 rows: 0.0020, 0.0017, 32.8 us instead of 30.5); one part it is, as fp32
//           rows are there for those who want more.  (A branch round the second part where no row of 16 has much weight: 110 us.)
// Keys are the products' long side (m16), the query heads of a KV head and its tokens the short one (n8): with four heads to a
// KV head nothing wider would be used.  The scores' accumulators hold keys along the lanes, the second product wants
// them along the other axis: one 8 x 8 transposition by the matrix unit's own instruction per 8 keys and group.
// fp32 queries and probabilities go through the same products in three bf16 parts, which is exact (8 + 8 + 8 bits); sums over
// 16 keys are then added in fp32 outside the matrix unit, whose own accumulation cuts off.
//
// Work: a (segment, block of columns) is a unit of 32-row tiles.  Units longer than a share of the work that leaves about as many
// pieces as CTAs are cut into equal pieces of whole tiles; a CTA takes a piece, and further ones where there are more.  A unit of
// one piece is finished by its CTA; the others leave a maximum, a sum and an unscaled output per piece, which a second launch
// joins.  In a CTA each warp takes every fourth tile with its own ring of bulk copies, so that no warp waits for another before
// a piece ends.  (Cutting the line of all tiles evenly instead, pieces running across units, took 8 us more for 256 segments of 256 to
// 4096 rows: a CTA's second piece starts with 3.4 us of latencies.)
// Where units are few and short one launch does it all: a cluster of CTAs per unit, equal shares of its tiles, the shares joined
// through the cluster's shared memory.  (One user, 8 heads of 129 to 1031 rows: 8.4 us with two launches, 7.4 with one.)  The rule goes by
// the room of an average segment, since the host does not know lengths: the same rows with four times the room take two launches.
// A block of columns reads and unpacks the cache for itself: 256 segments of 256 to 4096 rows take 26 us with 4 columns, 56 with
// 16, 208 with 64 (masked).
// The weights need the final log-sum-exps: the scores are kept in the workspace, the second launch turns them into
// probabilities (the same CTA, behind the cluster's exchange, where there is one launch).
// What bounds it: instructions, 400 of them per 16 rows, from few warps -- their registers leave four CTAs to an SM, 3.5 warps to a
// scheduler, and those find an instruction to issue in 59 % of the cycles (64 long segments; ALU pipe 49 %, matrix pipe 20 %, DRAM 44 %).
// The masked forms for head_dim 128 spill 24 to 36 bytes around the loop at these 128 registers.
#include <atomic>

#include <cooperative_groups.h>

#include "slkv_q4_device.cuh"

namespace slkv {
namespace {

namespace cg = cooperative_groups;

constexpr int kAttendCluster = 8;       // CTAs of a cluster, at most
constexpr int kAttendWarps = 4, kTileRows = 32, kCols = 8;
constexpr unsigned kLower = 0x000f000fu, kUpper = 0x00f000f0u;
constexpr unsigned kQueryScales = 0x5b805d80u;            // bf16: 2^60 for even channels, which meet lower nibbles, 2^56 for odd ones
constexpr float kLowest = -3e38f;       // a maximum over nothing: below every score, and differences of two stay numbers
constexpr float kSlack = 8.0f;
constexpr int kFewestTiles = 4;         // of a piece, where its unit has as many: one for each warp
constexpr unsigned long long kQ4WaitNs = 1000ull * 1000ull * 1000ull;

// What the second launch wants to know of a piece: its rows, its segment, and its unit's pieces (of the first block of columns).
struct Q4Piece { int row0, rows, seg, cb, n, place; };

struct Q4AttendArgs {
  Q4CacheView c;
  const void* q;
  void* out;
  float* lse;                           // optional, [n_seqs][n_q_heads][n_tokens]
  const int32_t* q_pos;                 // optional
  const float* slopes;                  // optional
  int32_t* status;
  long long q_seq, q_tok, q_head, o_seq, o_tok, o_head;      // elements
  int n_kv_heads, n_q_heads, n_tokens, G, R, n_cb, n_cta, ctas, accumulate;         // ctas: of a cluster
  int arrivals;                         // of a phase of the first CTA's barriers: 1; diagnostics: 2, and its waits run out
  float scale, softcap, decay, lse_unit;                     // lse_unit: of a base-2 logarithm
  // workspace
  int* head;                            // pieces
  int2* unit;                           // [n_units] pieces of a unit, and the first one's place in ml and part
  Q4Piece* piece;                       // [pieces]
  float2* ml;                           // [places][8] maximum and sum of a piece's columns
  float* part;                          // [places][8][HD] their unscaled outputs
  float* lse2;                          // [n_seg][R] of units of one piece, base 2
  float* scores;                        // [capacity][R] base 2 (accumulate)
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// generic accesses to shared memory before it, bulk copies after it
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Whether the copies of a barrier's phase are there, within a second.
__device__ __forceinline__ bool copies_there(uint32_t bar, uint32_t parity) {
  unsigned long long began = 0;
  for (;;) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    unsigned long long now;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
    if (!began) began = now;
    if (now - began > kQ4WaitNs) return false;
  }
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_from_zero(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ unsigned transpose8(unsigned x) {
  unsigned y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ unsigned pack2(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&b);
}
__device__ __forceinline__ unsigned times2(unsigned a, unsigned b) {
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const unsigned*>(&y);
}
__device__ __forceinline__ float lo_f(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
// A constant that stays in a register: the loop has no room for instructions that bring it there again and again.
__device__ __forceinline__ unsigned held(unsigned x) {
  unsigned y;
  asm volatile("mov.b32 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Nibble I of both halves of a word as (c - 8) / 128.
struct Q4Centre { unsigned lower, upper, minus; };         // 2^126, 2^122, -1/16: a nibble c is c 2^-133 or c 2^-129
template <int I>
__device__ __forceinline__ unsigned v_pair(unsigned w, const Q4Centre& c) {
  unsigned y;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(y) : "r"((I & 2 ? w >> 8 : w) & (I & 1 ? 0x00f000f0u : 0x000f000fu)), "r"(I & 1 ? c.upper : c.lower), "r"(c.minus));
  return y;
}
// Key of a product's row r: neighbours apart, so that the lanes of one shared-memory access meet all banks.
__device__ __forceinline__ int key_of(int r) { return (r & 8) | ((0x57463120u >> (4 * (r & 7))) & 7); }      // 0 2 1 3 6 4 7 5
// Tiles [*from, *to) of the nth of n equal pieces: the first ones have a tile more.
__device__ __forceinline__ void piece_tiles(int tiles, int nth, int n, int* from, int* to) {
  int even = (int)((float)tiles / (float)n);               // near: put right
  while ((long long)even * n > tiles) --even;
  while ((long long)(even + 1) * n <= tiles) ++even;
  const int more = tiles - even * n;
  *from = even * nth + min(nth, more);
  *to = *from + even + (nth < more);
}
__device__ __forceinline__ int tiles_of(int len) { return (len + kTileRows - 1) / kTileRows; }
// N 32-bit words from shared memory
template <int N>
__device__ __forceinline__ void load_words(uint32_t at, unsigned (&w)[N]) {
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (N == 2)
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}

// Pieces of a unit, by the reciprocal of their size: to the nearest rounding up, at least one for a unit that has a tile, no more
// than tiles.  Every thread of the launch gets the same.
__device__ __forceinline__ int pieces_of(int tiles, float inverse) { return tiles > 0 ? 1 + (int)((float)(tiles - 1) * inverse) : 0; }
// What the threads before this one have of x and of y.  sums: 2 words for each warp.
__device__ __forceinline__ void cta_before2(int x, int y, int* x_before, int* y_before, int* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sx = x, sy = y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int ux = __shfl_up_sync(0xffffffffu, sx, o), uy = __shfl_up_sync(0xffffffffu, sy, o);
    if (lane >= o) { sx += ux; sy += uy; }
  }
  __syncthreads();
  if (lane == 31) { sums[2 * warp] = sx; sums[2 * warp + 1] = sy; }
  __syncthreads();
  for (int w = 0; w < warp; ++w) { sx += sums[2 * w]; sy += sums[2 * w + 1]; }
  *x_before = sx - x;
  *y_before = sy - y;
}
__device__ __forceinline__ float cta_total(float x, int* sums) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = __float_as_int(x);
  __syncthreads();
  float sum = 0.0f;
  for (int w = 0; w < kAttendWarps; ++w) sum += __int_as_float(sums[w]);
  return sum;
}

template <int HD> constexpr int kQ4Stages = HD == 128 ? 2 : 4;
template <int HD> constexpr int kQ4Smem = kAttendWarps * kQ4Stages<HD> * kTileRows * q4_record_bytes(HD);

// What a CTA of a cluster shows the others: its share's maximum, sum and unscaled output per column.
template <int HD>
struct Q4Share {
  float2 ml[kCols];
  float out[kCols][HD];
};

template <int HD, int PARTS, bool MASK, bool CLUSTER>
__global__ void __launch_bounds__(kAttendWarps * 32, PARTS == 1 ? 4 : HD == 64 ? 3 : 2) k_q4_attend(const __grid_constant__ Q4AttendArgs a) {
  constexpr int NG = HD / 32, RB = q4_record_bytes(HD), kStages = kQ4Stages<HD>, kStageBytes = kTileRows * RB;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ __align__(8) unsigned long long bars[kAttendWarps][kStages];
  __shared__ int found[9], wholes[kAttendWarps * 32 + 1], splits[kAttendWarps * 32 + 1];
  __shared__ float merge_m[kAttendWarps][kCols], merge_l[kAttendWarps][kCols];
  __shared__ __align__(16) unsigned char share_room[CLUSTER ? sizeof(Q4Share<HD>) : 16];
  __shared__ float2 shares_ml[CLUSTER ? kAttendCluster : 1][kCols];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  unsigned char* ring = smem + warp * (kStages * kStageBytes);
  const uint32_t bar0 = smem_at(bars[warp]), ring_at = smem_at(ring);
  const Q4Centre centre = {held(0x7e807e80u), held(0x7c807c80u), held(0xbd80bd80u)};
  // where a lane finds its keys in 16 rows: rows key_of(g) and that + 8 of the first product, key_of(2 t), key_of(2 t + 1) and
  // those + 8 of the second
  const uint32_t key_row = key_of(g) * RB, value_row[2] = {uint32_t(key_of(2 * t) * RB + HD / 2 + g * (HD / 16)),
                                                          uint32_t(key_of(2 * t + 1) * RB + HD / 2 + g * (HD / 16))};
  if (lane < kStages)
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar0 + 8 * lane), "r"(blockIdx.x ? 1 : a.arrivals) : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
  pdl_wait();

  // ---- tiles of all units, the size of a piece, how many pieces come before those of each thread's segments
  const int n_seg = a.c.n_seg;
  unsigned issued = 0, used = 0, lost = 0;                 // copies of this warp's ring
  bool dead = false;
  const int per_thread = CLUSTER ? 0 : (n_seg + kAttendWarps * 32 - 1) / (kAttendWarps * 32);
  const int first = min(tid * per_thread, n_seg), last = min(first + per_thread, n_seg);
  int all = 1, all_split = 0;
  float inverse_per = 1.0f;
  // Loops as they are written: this code runs once, and what it costs is bringing it into the instruction cache.
  auto each = [&](auto f) {                                // f(segment, its tiles) until it says false
#pragma unroll 1
    for (int i = first; i < last; ++i)
      if (!f(i, tiles_of(q4_segment(a.c.starts, a.c.lens, i, a.c.capacity).len))) break;
  };
  if constexpr (!CLUSTER) {
    float mine = 0.0f;                                     // near enough, and whatever starts holds it does not wrap around
    each([&](int, int n) { mine += (float)n; return true; });
    const float total = cta_total(mine, found) * (float)a.n_cb;
    const int units = n_seg * a.n_cb;
    // The size of a piece: the smallest of five between an even share and what leaves a CTA to each unit's odd rest that makes no
    // more pieces than CTAs (a further wave of a few would take as long as the first).  Reciprocals are near enough, too: they are
    // the same in every thread of the launch.
    auto share = [&](int n) { return max((int)fminf(total * rcp((float)n), 1e8f) + 1, kFewestTiles); };   // no unit has 1e8 tiles
    const int least = share(a.n_cta), most = share(max(a.n_cta - units, a.n_cta / 4));
    constexpr int kSizes = 5;
    float inverse[kSizes];
    int pieces[kSizes], several[kSizes];                   // of this thread's segments; of those cut into several
#pragma unroll
    for (int k = 0; k < kSizes; ++k) {
      inverse[k] = rcp((float)(least + ((most - least) * k >> 2)));
      pieces[k] = several[k] = 0;
    }
    each([&](int, int t) {
#pragma unroll
      for (int k = 0; k < kSizes; ++k) {
        const int n = pieces_of(t, inverse[k]);
        pieces[k] += n;
        several[k] += n > 1 ? n : 0;
      }
      return true;
    });
#pragma unroll
    for (int k = 0; k < kSizes - 1; ++k) {
      const int n = __reduce_add_sync(0xffffffffu, pieces[k]);
      if (lane == 0) wholes[warp * 4 + k] = n;
    }
    __syncthreads();
    inverse_per = inverse[kSizes - 1];
    int whole = pieces[kSizes - 1], split = several[kSizes - 1];
#pragma unroll
    for (int k = kSizes - 2; k >= 0; --k) {
      int n = 0;
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) n += wholes[w * 4 + k];
      if (n * a.n_cb <= a.n_cta) { inverse_per = inverse[k]; whole = pieces[k]; split = several[k]; }
    }
    // Pieces of units of several come first, all of some size, then the units of one piece, many of them small: CTAs that share an
    // SM lie far apart in this order, and so have some of either.
    whole = (whole - split) * a.n_cb;
    split *= a.n_cb;
    cta_before2(whole, split, &wholes[tid], &splits[tid], found);
    if (tid == kAttendWarps * 32 - 1) { wholes[tid + 1] = wholes[tid] + whole; splits[tid + 1] = splits[tid] + split; }
    __syncthreads();
    all_split = splits[kAttendWarps * 32];
    all = all_split + wholes[kAttendWarps * 32];
    if (blockIdx.x == 0 && tid == 0) a.head[0] = all;
  }

  for (int index = CLUSTER ? 0 : blockIdx.x; index < all; index += a.n_cta) {
    int seg, cb, nth, n_pieces, place = 0, from, to;
    Q4Segment sg;
    if constexpr (CLUSTER) {                               // once: all is 1
      const int unit = blockIdx.x / a.ctas;
      seg = unit / a.n_cb; cb = unit - seg * a.n_cb; nth = blockIdx.x - unit * a.ctas; n_pieces = a.ctas;
      sg = q4_segment(a.c.starts, a.c.lens, seg, a.c.capacity);
      piece_tiles(tiles_of(sg.len), nth, n_pieces, &from, &to);
    } else {
      const bool of_several = index < all_split;
      const int* before = of_several ? splits : wholes;
      const int nth_of = of_several ? index : index - all_split;
      if (before[tid] <= nth_of && nth_of < before[tid + 1]) {     // the one thread that has the piece's segment
        int u = before[tid], s = first, n = 1, tiles = 0;
        each([&](int segment, int t) {
          s = segment;
          tiles = t;
          n = pieces_of(t, inverse_per);
          if (n == 0 || of_several != (n > 1)) return true;
          if (nth_of < u + n * a.n_cb) return false;
          u += n * a.n_cb;
          return true;
        });
        const Q4Segment found_sg = q4_segment(a.c.starts, a.c.lens, s, a.c.capacity);
        int block = 0, rest = nth_of - u;
        for (; rest >= n; rest -= n) ++block;
        found[0] = s; found[1] = block; found[2] = rest; found[3] = n; found[4] = u;
        found[5] = found_sg.begin; found[6] = found_sg.len;
        piece_tiles(tiles, rest, n, &found[7], &found[8]);
      }
      __syncthreads();
      seg = found[0]; cb = found[1]; nth = found[2]; n_pieces = found[3]; place = found[4] + cb * n_pieces;           // of a unit of several: its pieces' own order
      sg.begin = found[5]; sg.len = found[6];
      from = found[7]; to = found[8];
    }
    const unsigned char* rows = a.c.records + (long long)sg.begin * RB;
    if (!CLUSTER && tid == 0) {
      if (nth == 0) a.unit[seg * a.n_cb + cb] = make_int2(n_pieces, place);
      if (a.accumulate)
        a.piece[index] = {sg.begin + from * kTileRows, min(to * kTileRows, sg.len) - from * kTileRows, seg, cb, n_pieces, found[4]};
    }

    // the ring's first copies
    auto issue = [&](int tile) {
      const int n = min(kTileRows, sg.len - tile * kTileRows), slot = issued % kStages;
      if (lane == 0) {
        const uint32_t bar = bar0 + 8 * slot;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n * RB) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         smem_at(ring + slot * kStageBytes)),
                     "l"(rows + (long long)tile * kStageBytes), "r"(n * RB), "r"(bar) : "memory");
      }
      ++issued;
    };
    int next = from + warp;
    if (!dead)
      for (int i = 0; i < kStages && next < to; ++i, next += kAttendWarps) issue(next);

    // ---- the unit's queries: fragments, and sums per group
    const int s = seg / a.n_kv_heads, h = seg - s * a.n_kv_heads;
    unsigned bq[PARTS][NG][2][2], bz[2] = {0u, 0u};
    {
      const int col = cb * kCols + g;
      const bool there = col < a.R;
      const int tok = there ? col / a.G : 0, qh = h * a.G + (there ? col - tok * a.G : 0);
      const long long at = s * a.q_seq + tok * a.q_tok + qh * a.q_head + 8 * t;
      float qs[NG];                                        // a group's sum, before the scaling: that leaves no room for 32 of them
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        if constexpr (PARTS == 1) {
          uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + at + 32 * j);
          if (!there) w = make_uint4(0, 0, 0, 0);
          qs[j] = ((hi_f(w.x) + hi_f(w.y)) + (hi_f(w.z) + hi_f(w.w))) + ((lo_f(w.x) + lo_f(w.y)) + (lo_f(w.z) + lo_f(w.w)));
          w.x = times2(w.x, kQueryScales); w.y = times2(w.y, kQueryScales);
          w.z = times2(w.z, kQueryScales); w.w = times2(w.w, kQueryScales);
          bq[0][j][0][0] = __byte_perm(w.x, w.z, 0x5410); bq[0][j][0][1] = __byte_perm(w.x, w.z, 0x7632);
          bq[0][j][1][0] = __byte_perm(w.y, w.w, 0x5410); bq[0][j][1][1] = __byte_perm(w.y, w.w, 0x7632);
        } else {
          float4 u = make_float4(0, 0, 0, 0), v = u;
          if (there) {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + 32 * j);
            u = p[0]; v = p[1];
          }
          qs[j] = ((u.x + u.y) + (u.z + u.w)) + ((v.x + v.y) + (v.z + v.w));
          float x[8] = {u.x * 0x1p60f, u.y * 0x1p56f, u.z * 0x1p60f, u.w * 0x1p56f, v.x * 0x1p60f, v.y * 0x1p56f, v.z * 0x1p60f, v.w * 0x1p56f};
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned w = pack2(x[e], x[e + 4]);
              bq[p][j][e >> 1][e & 1] = w;
              x[e] -= lo_f(w);
              x[e + 4] -= hi_f(w);
            }
        }
        qs[j] += __shfl_xor_sync(0xffffffffu, qs[j], 1);
        qs[j] += __shfl_xor_sync(0xffffffffu, qs[j], 2);
      }
      // the query sums in the products' units, 2^(60 - 133), in three parts: lane t holds part t of all groups, where the zeros'
      // fragment expects them
#pragma unroll
      for (int jj = 0; jj < NG / 2; ++jj) {
        float y0 = qs[2 * jj] * 0x1p-73f, y1 = qs[2 * jj + 1] * 0x1p-73f;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const unsigned v = pack2(y0, y1);
          if (p == t) bz[jj] = v;                          // lane t = 3: zeros
          y0 -= lo_f(v);
          y1 -= hi_f(v);
        }
      }
    }
    const float to_log2 = a.scale * kLog2e * 0x1p73f;      // from the products' units
    // softcap tanh(x / softcap) as softcap (1 - 2 / (1 + e^(2 x / softcap))), in base 2: off by 2^-22 of the cap at most.  Under a
    // quarter of the cap that could be more than the score itself: there x (1 - y^2 / 3 + 2 y^4 / 15 - 17 y^6 / 315 + 62 y^8 / 2835),
    // y = x / softcap, tanh's Taylor series, whose next term is below 2^-26.  (tanhf is exact to the last place, which a softmax
    // does not notice, and takes several times the instructions.)
    const float cap = a.softcap * kLog2e, per_cap = a.softcap > 0.0f ? 2.0f / a.softcap : 0.0f;
    int qp[2] = {0, 0};
    float slope[2] = {0.0f, 0.0f};
    if (MASK) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = cb * kCols + 2 * t + c, tok = col < a.R ? col / a.G : 0;
        qp[c] = a.q_pos[s * a.n_tokens + tok];
        if (a.slopes) slope[c] = a.slopes[h * a.G + (col < a.R ? col - tok * a.G : 0)] * kLog2e;
      }
    }

    float m[2] = {kLowest, kLowest}, l[2] = {0.0f, 0.0f};
    float o[NG][2][4], zacc[NG][2];
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      zacc[j][0] = zacc[j][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[j][i >> 2][i & 3] = 0.0f;
    }
    const bool pairs = (a.R & 1) == 0;
    const int* pos_rows = a.c.pos + sg.begin;
    int pos_next = 0;
    if (MASK && from + warp < to) pos_next = pos_rows[min((from + warp) * kTileRows + lane, sg.len - 1)];

    for (int tile = from + warp; tile < to; tile += kAttendWarps) {
      const int n = min(kTileRows, sg.len - tile * kTileRows), slot = used % kStages;
      const int pos_here = pos_next;
      if (MASK && tile + kAttendWarps < to) pos_next = pos_rows[min((tile + kAttendWarps) * kTileRows + lane, sg.len - 1)];
      const uint32_t buf = ring_at + slot * kStageBytes;
      if (!dead) {                                         // a copy that does not come in a second is not waited for again
        dead = __any_sync(0xffffffffu, !copies_there(bar0 + 8 * slot, (used / kStages) & 1));
        if (dead) {
          lost = used;
          if (lane == 0 && a.status) *a.status = SLKV_ERR_DEVICE_TIMEOUT;
        }
      }
      ++used;
      if (n < kTileRows) {                                 // what lies behind the last row must be finite: scales and zeros
        if (lane >= n && lane < kTileRows) {
#pragma unroll
          for (int i = 0; i < RB - HD; i += 16)
            *reinterpret_cast<uint4*>(ring + slot * kStageBytes + lane * RB + HD + i) = make_uint4(0, 0, 0, 0);
          async_fence();
        }
        __syncwarp();
      }
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 16) {
        // ---- scores: rows key_of(g) and key_of(g + 8), columns 2 t and 2 t + 1
        const int r0 = k0 + key_of(g), r1 = r0 + 8;
        const uint32_t rows16 = buf + k0 * RB, p0 = rows16 + key_row, p1 = p0 + 8 * RB;
        float x[4];
        {
          unsigned w0[NG], w1[NG], x0[NG], x1[NG];         // codes; scales and zeros
          load_words(p0 + HD, x0);
          load_words(p1 + HD, x1);
          load_words(p0 + 4 * NG * t, w0);
          load_words(p1 + 4 * NG * t, w1);
          mma16816_from_zero(x, x0[NG / 2], x1[NG / 2], NG == 4 ? x0[NG - 1] : 0u, NG == 4 ? x1[NG - 1] : 0u, bz[0], bz[1]);
#pragma unroll
          for (int j = 0; j < NG; ++j) {
            float d[4];
            const unsigned u0 = w0[j] >> 8, u1 = w1[j] >> 8;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
              if (p == 0) mma16816_from_zero(d, w0[j] & kLower, w1[j] & kLower, w0[j] & kUpper, w1[j] & kUpper, bq[p][j][0][0], bq[p][j][0][1]);
              else mma16816(d, w0[j] & kLower, w1[j] & kLower, w0[j] & kUpper, w1[j] & kUpper, bq[p][j][0][0], bq[p][j][0][1]);
              mma16816(d, u0 & kLower, u1 & kLower, u0 & kUpper, u1 & kUpper, bq[p][j][1][0], bq[p][j][1][1]);
            }
            const float s0 = j & 1 ? hi_f(x0[j >> 1]) : lo_f(x0[j >> 1]), s1 = j & 1 ? hi_f(x1[j >> 1]) : lo_f(x1[j >> 1]);
            x[0] = fmaf(s0, d[0], x[0]); x[1] = fmaf(s0, d[1], x[1]);
            x[2] = fmaf(s1, d[2], x[2]); x[3] = fmaf(s1, d[3], x[3]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= to_log2;
        if (a.softcap > 0.0f) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            constexpr float kUnit = 0.34657359027997265f * 0.34657359027997265f;         // (ln 2 / 2)^2: from u^2 to y^2
            const float u = x[i] * per_cap, z = u * u * kUnit;
            const float near = fmaf(x[i] * z, fmaf(z, fmaf(z, fmaf(z, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), x[i]);
            const float far = fmaf(cap * -2.0f, rcp(1.0f + ex2(u)), cap);
            x[i] = fabsf(u) < 0.72f ? near : far;
          }
        }
        if (MASK) {
          const int pos0 = __shfl_sync(0xffffffffu, pos_here, r0), pos1 = __shfl_sync(0xffffffffu, pos_here, r1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int pos = i < 2 ? pos0 : pos1;
            if (a.slopes) x[i] = fmaf(slope[i & 1], (float)(pos - qp[i & 1]), x[i]);
            if (pos > qp[i & 1]) x[i] = -INFINITY;
          }
        }
        if (k0 + 16 > n) {                                 // the last rows of a segment
          if (r0 >= n) x[0] = x[1] = -INFINITY;
          if (r1 >= n) x[2] = x[3] = -INFINITY;
        }
        if (a.accumulate) {
          const int col = cb * kCols + 2 * t;
          float* to_row = a.scores + ((long long)sg.begin + tile * kTileRows) * a.R + col;
          if (pairs) {
            if (r0 < n && col < a.R) *reinterpret_cast<float2*>(to_row + r0 * a.R) = make_float2(x[0], x[1]);
            if (r1 < n && col < a.R) *reinterpret_cast<float2*>(to_row + r1 * a.R) = make_float2(x[2], x[3]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = i < 2 ? r0 : r1;
              if (r < n && col + (i & 1) < a.R) to_row[r * a.R + (i & 1)] = x[i];
            }
          }
        }
        // ---- running maximum and sum.  The maximum need not be the largest score, only near it: it moves when a score is
        // over it by a factor of 2^8, and then to the largest, so that most steps exchange nothing between the lanes.
        const float top0 = fmaxf(x[0], x[2]), top1 = fmaxf(x[1], x[3]);
        if (__any_sync(0xffffffffu, top0 > m[0] + kSlack || top1 > m[1] + kSlack)) {
          float up[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float y = c ? top1 : top0;
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
            y = fmaxf(y, m[c]);
            up[c] = ex2(m[c] - y);
            m[c] = y;
            l[c] *= up[c];
          }
#pragma unroll
          for (int j = 0; j < NG; ++j) {
            zacc[j][0] *= up[0]; zacc[j][1] *= up[1];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[j][i >> 2][i & 3] *= up[i & 1];
          }
        }
        bool seen[4];
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          seen[i] = !MASK || x[i] != -INFINITY;
          p[i] = ex2(x[i] - m[i & 1]);
          l[i & 1] += p[i];
        }
        // ---- output
        unsigned x0[NG], x1[NG];
        load_words(p0 + HD + 4 * NG, x0);
        load_words(p1 + HD + 4 * NG, x1);
        unsigned va[4][NG / 2];                            // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int i = 0; i < 4; ++i)
          load_words(rows16 + value_row[i & 1] + (i & 2 ? 8 * RB : 0), va[i]);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const float s0 = j & 1 ? hi_f(x0[j >> 1]) : lo_f(x0[j >> 1]), s1 = j & 1 ? hi_f(x1[j >> 1]) : lo_f(x1[j >> 1]);
          const unsigned zw0 = x0[(NG + j) >> 1], zw1 = x1[(NG + j) >> 1];
          const float z0 = fmaf(8.0f, s0, j & 1 ? hi_f(zw0) : lo_f(zw0)), z1 = fmaf(8.0f, s1, j & 1 ? hi_f(zw1) : lo_f(zw1));
          float y[4];
          // a row that a column does not see gives it nothing, whatever its scales hold
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float zz = seen[i] ? (i < 2 ? z0 : z1) : 0.0f;
            zacc[j][i & 1] = fmaf(p[i], zz, zacc[j][i & 1]);
            y[i] = seen[i] ? p[i] * (i < 2 ? s0 : s1) : 0.0f;
          }
          const unsigned t01 = __byte_perm(va[0][j >> 1], va[1][j >> 1], j & 1 ? 0x7632 : 0x5410);
          const unsigned t89 = __byte_perm(va[2][j >> 1], va[3][j >> 1], j & 1 ? 0x7632 : 0x5410);
          const unsigned f0[4] = {v_pair<0>(t01, centre), v_pair<1>(t01, centre), v_pair<0>(t89, centre), v_pair<1>(t89, centre)};
          const unsigned f1[4] = {v_pair<2>(t01, centre), v_pair<3>(t01, centre), v_pair<2>(t89, centre), v_pair<3>(t89, centre)};
          if constexpr (PARTS == 1) {
            const unsigned b0 = transpose8(pack2(y[0], y[1])), b1 = transpose8(pack2(y[2], y[3]));
            mma16816(o[j][0], f0[0], f0[1], f0[2], f0[3], b0, b1);
            mma16816(o[j][1], f1[0], f1[1], f1[2], f1[3], b0, b1);
          } else {
            float d0[4] = {0.0f, 0.0f, 0.0f, 0.0f}, d1[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const unsigned w0 = pack2(y[0], y[1]), w1 = pack2(y[2], y[3]);
              y[0] -= lo_f(w0); y[1] -= hi_f(w0); y[2] -= lo_f(w1); y[3] -= hi_f(w1);
              const unsigned b0 = transpose8(w0), b1 = transpose8(w1);
              mma16816(d0, f0[0], f0[1], f0[2], f0[3], b0, b1);
              mma16816(d1, f1[0], f1[1], f1[2], f1[3], b0, b1);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { o[j][0][i] += d0[i]; o[j][1][i] += d1[i]; }
          }
        }
      }
      __syncwarp();
      if (next < to) {
        if (!dead) issue(next);
        next += kAttendWarps;
      }
    }
    // ---- the piece's end: the warps' shares together.  A warp's ring is empty now and takes its output.
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        l[c] += __shfl_xor_sync(0xffffffffu, l[c], d);
#pragma unroll
        for (int j = 0; j < NG; ++j) zacc[j][c] += __shfl_xor_sync(0xffffffffu, zacc[j][c], d);
      }
      if (g == 0) {
        merge_m[warp][2 * t + c] = m[c];
        merge_l[warp][2 * t + c] = dead ? __int_as_float(0x7fffffff) : l[c];       // rows that did not come: their unit is NaN throughout
      }
    }
    float* mine_o = reinterpret_cast<float*>(ring);        // [column][HD + 4]
    constexpr int kPitch = HD + 4;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        *reinterpret_cast<float4*>(mine_o + (2 * t + c) * kPitch + 32 * j + 4 * g) =
            make_float4(fmaf(128.0f, o[j][0][c], zacc[j][c]), fmaf(128.0f, o[j][0][c + 2], zacc[j][c]),
                        fmaf(128.0f, o[j][1][c], zacc[j][c]), fmaf(128.0f, o[j][1][c + 2], zacc[j][c]));
    async_fence();
    __syncthreads();
    const bool whole = !CLUSTER && n_pieces == 1;
    Q4Share<HD>& share = *reinterpret_cast<Q4Share<HD>*>(share_room);
    for (int i = tid; i < kCols * HD / 4; i += kAttendWarps * 32) {
      const int c = i / (HD / 4), ch = 4 * (i % (HD / 4)), col = cb * kCols + c;
      if (col >= a.R) continue;
      float top = merge_m[0][c];                           // kLowest, and a sum of 0, where no row is seen
#pragma unroll
      for (int w = 1; w < kAttendWarps; ++w) top = fmaxf(top, merge_m[w][c]);
      float sum_l = 0.0f;
      float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) {
        const float f = ex2(merge_m[w][c] - top);
        const float4 x = *reinterpret_cast<const float4*>(smem + w * (kStages * kStageBytes) + (c * kPitch + ch) * 4);
        sum_l = fmaf(merge_l[w][c], f, sum_l);
        v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
      }
      if (whole) {
        const int tok = col / a.G, qh = h * a.G + col - tok * a.G;
        const float inv = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;             // no visible row: zeros
        const long long at = s * a.o_seq + tok * a.o_tok + qh * a.o_head + ch;
        if constexpr (PARTS == 1) {
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) = make_uint2(pack2(v.x * inv, v.y * inv), pack2(v.z * inv, v.w * inv));
        } else {
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        }
        if (ch == 0) {
          const float z = top + log2f(sum_l);
          if (a.lse) a.lse[((long long)s * a.n_q_heads + qh) * a.n_tokens + tok] = z * a.lse_unit;
          a.lse2[(long long)seg * a.R + col] = z;
        }
      } else if constexpr (CLUSTER) {
        if (ch == 0) share.ml[c] = make_float2(top, sum_l);
        *reinterpret_cast<float4*>(&share.out[c][ch]) = v;
      } else {
        const long long at = (long long)(place + nth) * kCols + c;
        if (ch == 0) a.ml[at] = make_float2(top, sum_l);
        *reinterpret_cast<float4*>(a.part + at * HD + ch) = v;
      }
    }
    if constexpr (CLUSTER) {
      cg::cluster_group cluster = cg::this_cluster();
      cluster.sync();
      const int cols = min(kCols, a.R - cb * kCols);       // the block's
      if (tid < a.ctas * kCols && (tid & (kCols - 1)) < cols)
        shares_ml[tid / kCols][tid & (kCols - 1)] = cluster.map_shared_rank(&share, tid / kCols)->ml[tid & (kCols - 1)];
      __syncthreads();
      float* lse_of = merge_m[0];                          // [8]
      if (tid < cols) {
        float top = kLowest, sum_l = 0.0f;
        for (int r = 0; r < a.ctas; ++r) top = fmaxf(top, shares_ml[r][tid].x);
        for (int r = 0; r < a.ctas; ++r) sum_l = fmaf(shares_ml[r][tid].y, ex2(shares_ml[r][tid].x - top), sum_l);
        const float z = top + log2f(sum_l);
        merge_l[0][tid] = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;             // no visible row: zeros
        merge_l[1][tid] = top;
        lse_of[tid] = z == -INFINITY ? INFINITY : z;
        const int col = cb * kCols + tid, tok = col / a.G;
        if (a.lse && nth == 0) a.lse[((long long)s * a.n_q_heads + h * a.G + col - tok * a.G) * a.n_tokens + tok] = z * a.lse_unit;
      }
      __syncthreads();
      for (int i = tid; i < cols * HD; i += kAttendWarps * 32) {           // each CTA its share of the columns
        const int c = i / HD, ch = i - c * HD;
        if (c % a.ctas != nth) continue;
        float v = 0.0f;
#pragma unroll 4
        for (int r = 0; r < a.ctas; ++r) v = fmaf(cluster.map_shared_rank(&share, r)->out[c][ch], ex2(shares_ml[r][c].x - merge_l[1][c]), v);
        v *= merge_l[0][c];
        const int col = cb * kCols + c, tok = col / a.G;
        const long long at = s * a.o_seq + tok * a.o_tok + (h * a.G + col - tok * a.G) * a.o_head + ch;
        if constexpr (PARTS == 1) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.out)[at] = v;
      }
      if (a.accumulate) {                                  // one block of columns: the CTA has its rows' scores of all of them
        const float inv_g = 1.0f / (float)a.G;
        for (int r = from * kTileRows + tid; r < min(to * kTileRows, sg.len); r += kAttendWarps * 32) {
          const float* x = a.scores + ((long long)sg.begin + r) * a.R;
          float sum = 0.0f;
          for (int c = 0; c < a.R; ++c) sum += ex2(x[c] - lse_of[c]);
          float* w = a.c.weight + sg.begin + r;
          *w = fmaf(a.decay, *w, sum * inv_g);
        }
      }
      cluster.sync();                                      // nobody reads this CTA's share any more
    } else {
      __syncthreads();                                     // the rings and the sums are free again
    }
  }
  if (dead)                                                // what is still in flight lands before the memory is another CTA's
    for (unsigned i = lost; i < issued; ++i) copies_there(bar0 + 8 * (i % kStages), (i / kStages) & 1);
}

// ---- the pieces of units that lie in several CTAs, and the weights ---------------------------------------------------
constexpr int kJoinThreads = 128;

// Maximum and sum over a unit's n pieces for one column; whole warp.
__device__ __forceinline__ float2 join_ml(const float2* ml, int n, int lane) {
  float m = kLowest, l = 0.0f;
  for (int i = lane; i < n; i += 32) {
    const float2 x = ml[i * kCols];
    const float top = fmaxf(m, x.x);
    l = l * ex2(m - top) + x.y * ex2(x.x - top);
    m = top;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, m, o), ol = __shfl_xor_sync(0xffffffffu, l, o);
    const float top = fmaxf(m, om);
    l = l * ex2(m - top) + ol * ex2(om - top);
    m = top;
  }
  return make_float2(m, l);
}

template <int HD, bool F32>
__global__ void __launch_bounds__(kJoinThreads) k_q4_join(const __grid_constant__ Q4AttendArgs a) {
  constexpr int kWarps = kJoinThreads / 32, V = HD / 32;   // channels per lane
  __shared__ __align__(16) float shares[kWarps][HD], lse_of[kMaxQ4Columns];
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_out = a.c.n_seg * a.R;
  if ((int)blockIdx.x < n_out) {                           // one segment's column
    const int seg = blockIdx.x / a.R, col = blockIdx.x - seg * a.R, cb = col / kCols, c = col - cb * kCols;
    const int2 u = a.unit[seg * a.n_cb + cb];              // not written for a segment without rows
    const int n = q4_segment(a.c.starts, a.c.lens, seg, a.c.capacity).len > 0 ? u.x : 0;
    if (n == 1) return;
    const int s = seg / a.n_kv_heads, h = seg - s * a.n_kv_heads, tok = col / a.G, qh = h * a.G + col - tok * a.G;
    const long long first = n > 0 ? (long long)u.y * kCols + c : 0;
    const float2 ml = join_ml(a.ml + first, n, lane);
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
#pragma unroll 4
    for (int i = warp; i < n; i += kWarps) {
      const long long at = first + i * kCols;
      const float f = ex2(a.ml[at].x - ml.x);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fmaf(a.part[at * HD + lane + 32 * e], f, acc[e]);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) shares[warp][lane + 32 * e] = acc[e];
    __syncthreads();
    if (tid < HD) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += shares[w][tid];
      v *= ml.y == 0.0f ? 0.0f : 1.0f / ml.y;
      const long long at = s * a.o_seq + tok * a.o_tok + qh * a.o_head + tid;
      if (F32) static_cast<float*>(a.out)[at] = v;
      else static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
    }
    if (tid == 0 && a.lse) a.lse[((long long)s * a.n_q_heads + qh) * a.n_tokens + tok] = (ml.x + log2f(ml.y)) * a.lse_unit;
    return;
  }
  // The weights of a piece's rows: a row has its scores of all columns, so the first block of columns does it.  Rows are taken
  // four to a thread; the first ones' loads do not wait for the log-sum-exps.
  constexpr int kRowsAtOnce = 4;
  const float inv_g = 1.0f / (float)a.G;
  const int all = a.head[0];
  const bool quads = (a.R & 3) == 0;
  for (int index = blockIdx.x - n_out; index < all; index += a.n_cta) {
    const Q4Piece p = a.piece[index];
    if (p.cb != 0) continue;
    float4 x[kRowsAtOnce];
    float old[kRowsAtOnce];
    auto row = [&](int r0, int e) { return (long long)p.row0 + min(r0 + e * kJoinThreads, p.rows - 1); };
    auto load = [&](int r0, int c) {
#pragma unroll
      for (int e = 0; e < kRowsAtOnce; ++e) {
        const float* at = a.scores + row(r0, e) * a.R + c;
        if (quads) x[e] = *reinterpret_cast<const float4*>(at);
        else x[e] = make_float4(at[0], c + 1 < a.R ? at[1] : -INFINITY, c + 2 < a.R ? at[2] : -INFINITY, c + 3 < a.R ? at[3] : -INFINITY);
      }
    };
    load(tid, 0);
#pragma unroll
    for (int e = 0; e < kRowsAtOnce; ++e) old[e] = a.c.weight[row(tid, e)];
    __syncthreads();                                       // the log-sum-exps of the piece before are read
    for (int col = warp; col < ((a.R + 3) & ~3); col += kWarps) {
      float z = INFINITY;                                  // a column that is none, or sees nothing, gives nothing
      if (col < a.R) {
        if (p.n == 1) {
          z = a.lse2[(long long)p.seg * a.R + col];
        } else {
          const float2 ml = join_ml(a.ml + ((long long)p.place + col / kCols * p.n) * kCols + col % kCols, p.n, lane);
          z = ml.x + log2f(ml.y);
        }
        if (z == -INFINITY) z = INFINITY;
      }
      if (lane == 0) lse_of[col] = z;
    }
    __syncthreads();
    for (int r0 = tid; r0 < p.rows; r0 += kRowsAtOnce * kJoinThreads) {
      float sum[kRowsAtOnce] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (r0 != tid) {
        load(r0, 0);
#pragma unroll
        for (int e = 0; e < kRowsAtOnce; ++e) old[e] = a.c.weight[row(r0, e)];
      }
      for (int c = 0;;) {
        const float4 z = *reinterpret_cast<const float4*>(lse_of + c);
#pragma unroll
        for (int e = 0; e < kRowsAtOnce; ++e)
          sum[e] += (ex2(x[e].x - z.x) + ex2(x[e].y - z.y)) + (ex2(x[e].z - z.z) + ex2(x[e].w - z.w));
        c += 4;
        if (c >= a.R) break;
        load(r0, c);
      }
#pragma unroll
      for (int e = 0; e < kRowsAtOnce; ++e)
        if (r0 + e * kJoinThreads < p.rows) a.c.weight[row(r0, e)] = fmaf(a.decay, old[e], sum[e] * inv_g);
    }
  }
}

constexpr size_t kAlign = 256;
size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct Q4Workspace {
  size_t unit, piece, ml, part, lse2, scores, total;
  Q4Workspace(int n_seg, int head_dim, int R, long long capacity, bool accumulate) {
    const size_t units = (size_t)n_seg * ((R + kCols - 1) / kCols), places = 2 * kMaxQ4Ctas;      // of units of several pieces
    unit = kAlign;
    piece = unit + up(units * sizeof(int2));
    ml = piece + up((kMaxQ4Ctas + units) * sizeof(Q4Piece));
    part = ml + up(places * kCols * sizeof(float2));
    lse2 = part + up(places * kCols * head_dim * sizeof(float));
    scores = lse2 + up((size_t)n_seg * R * sizeof(float));
    total = scores + (accumulate ? up((size_t)capacity * R * sizeof(float)) : 0);
  }
};

// CTAs of one SM, and its dynamic shared memory allowed; found once for each device.
template <int HD, int PARTS, bool MASK, bool CLUSTER>
cudaError_t attend_ctas(int* per_sm) {
  auto kernel = k_q4_attend<HD, PARTS, MASK, CLUSTER>;
  static std::atomic<int> known[16];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  int n = dev < 16 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kQ4Smem<HD>);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kAttendWarps * 32, kQ4Smem<HD>);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    if (dev < 16) known[dev].store(n, std::memory_order_relaxed);
  }
  *per_sm = n;
  return cudaSuccess;
}

template <int HD, int PARTS, bool MASK>
cudaError_t launch_attend(Q4AttendArgs& a, cudaStream_t st, int* launches) {
  int per_sm = 0;
  const dim3 block(kAttendWarps * 32);
  // One launch: units that fit on the device with four or eight CTAs each, of 64 to 128 slots per CTA on average.  A cluster takes
  // its whole unit, however long: with more slots the longest unit costs more than the second launch (60 units of 33 to 3001
  // rows, 171 to a CTA: 13.7 us against 11).
  const long long units = (long long)a.c.n_seg * a.n_cb, room = a.c.capacity / a.c.n_seg;
  int ctas = kAttendCluster;
  while (ctas > 1 && (units * ctas > 3ll * sm_count() || room < 64 * ctas)) ctas /= 2;
  if (ctas >= 4 && room <= 128 * ctas && (a.n_cb == 1 || !a.accumulate)) {
    cudaError_t e = attend_ctas<HD, PARTS, MASK, true>(&per_sm);
    if (e != cudaSuccess) return e;
    a.ctas = ctas;
    a.n_cta = 1;
    LaunchScope scope(KID_Q4_ATTEND, st, launches);
    return launch_pdl(k_q4_attend<HD, PARTS, MASK, true>, dim3((unsigned)(units * ctas)), block, kQ4Smem<HD>, st, ctas, a);
  }
  cudaError_t e = attend_ctas<HD, PARTS, MASK, false>(&per_sm);
  if (e != cudaSuccess) return e;
  const int most = sm_count() * per_sm;
  a.n_cta = most < kMaxQ4Ctas ? most : kMaxQ4Ctas;
  {
    LaunchScope scope(KID_Q4_ATTEND, st, launches);
    e = launch_pdl(k_q4_attend<HD, PARTS, MASK, false>, dim3((unsigned)a.n_cta), block, kQ4Smem<HD>, st, 1, a);
  }
  if (e != cudaSuccess) return e;
  LaunchScope scope(KID_Q4_JOIN, st, launches);
  const unsigned grid = (unsigned)(a.c.n_seg * a.R + (a.accumulate ? a.n_cta : 0));
  return launch_pdl(k_q4_join<HD, (PARTS > 1)>, dim3(grid), dim3(kJoinThreads), 0, st, 1, a);
}

template <int HD>
cudaError_t launch_attend_of(Q4AttendArgs& a, bool f32, cudaStream_t st, int* launches) {
  if (f32) return a.q_pos ? launch_attend<HD, 3, true>(a, st, launches) : launch_attend<HD, 3, false>(a, st, launches);
  return a.q_pos ? launch_attend<HD, 1, true>(a, st, launches) : launch_attend<HD, 1, false>(a, st, launches);
}

}  // namespace

size_t q4_attend_workspace(int n_seg, int head_dim, int columns, long long capacity, bool accumulate) {
  return Q4Workspace(n_seg, head_dim, columns, capacity, accumulate).total;
}

cudaError_t launch_q4_attend(const Q4CacheView& c, const slkv_q4_cache& cache, const slkv_q4_attend_params& p, const void* q,
                             const int32_t* q_pos, const float* slopes, void* out, float* lse, bool accumulate, int32_t* status,
                             void* workspace, cudaStream_t st, int* launches) {
  Q4AttendArgs a = {};
  a.c = c; a.q = q; a.out = out; a.lse = lse; a.q_pos = q_pos; a.slopes = slopes; a.status = status;
  a.q_seq = p.q_stride_seq; a.q_tok = p.q_stride_tok; a.q_head = p.q_stride_head;
  a.o_seq = p.o_stride_seq; a.o_tok = p.o_stride_tok; a.o_head = p.o_stride_head;
  a.n_kv_heads = cache.n_kv_heads; a.n_q_heads = p.n_q_heads; a.n_tokens = p.n_tokens;
  a.G = p.n_q_heads / cache.n_kv_heads; a.R = a.G * p.n_tokens; a.n_cb = (a.R + kCols - 1) / kCols;
  a.accumulate = accumulate;
  a.arrivals = take_expire_next_copy_wait() ? 2 : 1;
  a.scale = p.scale; a.softcap = p.softcap; a.decay = p.weight_decay;
  a.lse_unit = p.lse_units == SLKV_LSE_LOG2 ? 1.0f : 0.69314718055994531f;
  const Q4Workspace w(c.n_seg, cache.head_dim, a.R, c.capacity, accumulate);
  char* ws = static_cast<char*>(workspace);
  a.head = reinterpret_cast<int*>(ws);
  a.unit = reinterpret_cast<int2*>(ws + w.unit);
  a.piece = reinterpret_cast<Q4Piece*>(ws + w.piece);
  a.ml = reinterpret_cast<float2*>(ws + w.ml);
  a.part = reinterpret_cast<float*>(ws + w.part);
  a.lse2 = reinterpret_cast<float*>(ws + w.lse2);
  a.scores = accumulate ? reinterpret_cast<float*>(ws + w.scores) : nullptr;
  return cache.head_dim == 128 ? launch_attend_of<128>(a, p.dtype == SLKV_F32, st, launches)
                               : launch_attend_of<64>(a, p.dtype == SLKV_F32, st, launches);
}

}  // namespace slkv
