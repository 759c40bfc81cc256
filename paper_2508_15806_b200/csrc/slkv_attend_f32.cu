// Attention of prompts and of tokens over a paged cache for fp32 rows, on the tensor cores.
//
// An fp32 number is the sum of three bf16 numbers, its significand in three parts of eight bits: x = x0 + x1 + x2 exactly.  A product
// of two such sums needs six of the nine products (x0 y0, x0 y1, x1 y0, x1 y1, x0 y2, x2 y0; the others are below 2^-24 of it), which the
// tensor cores add up in fp32: 278 TFLOP/s at six products each (a sixth of cuBLAS' measured bf16 rate), against 74 on the FMA pipe.  Scores and outputs are made this way:
//   K, V, Q   come in as fp32, are split by the warps that load them into three planes each; K and V lie in shared memory, Q in TMEM but
//             for its third plane, which one product in six needs: with all of it in shared memory a product of 64 keys takes 48 cycles
//             for its operands instead of 32
//   S = Q K^T in TMEM, two buffers; a thread has a row, 64 keys a tile, with a running reference and sum in fp32
//   P         = 2^(sc (x - m)) goes back to TMEM as three planes; O += P V, rescaled only where m rises by more than 2^8
// The tensor cores cut off what they add to an accumulator: over 16000 keys the outputs came out 2 10^-5 too small.  So O holds one tile's
// products, the small ones first, and the softmax warps, which have 240 registers for it, add it to the sum of the tiles before, rounded to
// nearest (4 10^-7 off).
// A CTA takes pieces of units (AttendSchedule) of one block of 128 query rows.
//   warps 0-3  softmax, results      warps 4-7  K      warps 8-11  Q, V      warp 12  MMAs      warp 13  schedule
// K and V are handed over in blocks of 64 channels, four buffers each; while one is split and stored, the one behind it is on its way into
// registers.
//
// Measured (B200, 32 query heads on 8 KV heads): 8000 tokens 2.53 ms (207 TFLOP/s counted once, 1240 as products of planes), head_dim 64
// 1.63 ms; one token each of 8 sequences over 8000 to 32000 rows 410 us (2.6 TB/s).  A tile of head_dim 128 takes 5700 cycles, its products
// 3450 of them: the warps of V, and behind them those of K, have 4600 cycles of loading, splitting and storing to do.  One softmax
// warp, one of K and one of V share a scheduler, which issues in about half of the cycles.
//
// A key that a row does not see gives it nothing: scores are replaced; keys behind the last one are rows of zeros; values that are not
// finite, which 0 would not cancel, are left out of V, and rows that see them add them at the end.
#include <atomic>

#include "slkv_attend_device.cuh"

namespace slkv {
namespace {

constexpr int kKeys = 1 << kF32TileBits;
constexpr int kThreads = 512;
constexpr int kKWarp = 4, kVWarp = 8, kMmaWarp = 12, kPlanWarp = 13;
constexpr int kUnits = 3;                        // pieces the schedule is ahead by: nobody is more than these ahead of a warp that is at one
constexpr int kAhead = 2 * kUnits;
constexpr float kLift = 8.0f;                    // log2 of how far P may exceed 1 before the reference is raised
constexpr int kTmemS = 0, kTmemP = 2 * kKeys, kPlaneCols = kKeys / 2, kTmemO = 256, kTmemQ = 384;   // P has 3 kPlaneCols columns
static_assert(kTmemP + 3 * kPlaneCols <= kTmemO, "columns");
constexpr int kPlane = kKeys * 128;              // bytes of a block of K or V, 64 channels of a tile's rows, one plane

template <int D>
struct Smem {
  static constexpr int kHalves = D / 64;
  static constexpr int kK = 4, kV = 4;           // buffers
  alignas(1024) unsigned char q[kHalves * kHalfBytes];         // Q's third plane; the others are in TMEM
  alignas(1024) unsigned char k[kK][3][kPlane];
  alignas(1024) unsigned char v[kV][3][kPlane];
  AttendPiece piece[kUnits];
  unsigned long long unit_full[kUnits], unit_empty[kUnits], q_full, q_empty, k_full[kK], k_empty[kK], v_full[kV], v_empty[kV], s_full[2], p_ready,
      pv_done, drain;
  int odd_lo[kAhead][4], odd_hi[kAhead][4];      // tiles of a piece where a warp of V met values that are not finite
  int abort;
  uint32_t tmem;
  AttendStart start;
};

struct AttendF32 {
  AttendShape a;
  int page_bits;
  int wide, wide_k, wide_v;                      // rows of out, of K, of V (drafted ones too) begin at 32-byte boundaries
  int extra_arrival;                             // 1: a test makes the waits for P run out
};

// Row j of a piece's tile, as it lies in memory; where there is none, another one that there is.
__device__ __forceinline__ const float* key_row(const AttendF32& t, const AttendPiece& p, bool v, int tile, int j, bool* there) {
  const AttendShape& a = t.a;
  if (a.has_new && tile == p.n_all - 1) {
    *there = j < p.n_seq_tok;
    j = min(j, p.n_seq_tok - 1);
    return static_cast<const float*>(v ? a.v_new : a.k_new) + p.s * (v ? a.vn_seq : a.kn_seq) + j * (v ? a.vn_tok : a.kn_tok) +
           p.h * (v ? a.vn_head : a.kn_head);
  }
  int row = tile * kKeys + j;
  *there = row < p.nk;
  row = min(row, p.nk - 1);
  const float* const base = static_cast<const float*>(v ? a.v : a.k);
  if (!a.paged) return base + (long long)(p.k_row + row) * (v ? a.v_tok : a.k_tok) + p.h * (v ? a.v_head : a.k_head);
  int id = __ldg(a.tables + (long long)(p.s * a.n_kv_heads + p.h) * a.max_pages + (row >> t.page_bits));
  if ((unsigned)id >= (unsigned)a.n_pages) {
    if (*there && a.status) *a.status = SLKV_ERR_BAD_SHAPE;
    *there = false;
    id = 0;
  }
  return base + (((long long)id << t.page_bits) + (row & (a.page_rows - 1))) * a.head_dim;
}

// Three planes of eight numbers: the upper 16 bits of x, of what is left of it, and of what is left then.
__device__ __forceinline__ void split8(const float (&x)[8], uint4& p0, uint4& p1, uint4& p2) {
  uint32_t w[3][4];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t b0[2], b1[2], b2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float v = x[e + i];
      b0[i] = __float_as_uint(v);
      const float r = v - __uint_as_float(b0[i] & 0xffff0000u);
      b1[i] = __float_as_uint(r);
      b2[i] = __float_as_uint(r - __uint_as_float(b1[i] & 0xffff0000u));
    }
    w[0][e / 2] = __byte_perm(b0[0], b0[1], 0x7632);
    w[1][e / 2] = __byte_perm(b1[0], b1[1], 0x7632);
    w[2][e / 2] = __byte_perm(b2[0], b2[1], 0x7632);
  }
  p0 = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
  p1 = make_uint4(w[1][0], w[1][1], w[1][2], w[1][3]);
  p2 = make_uint4(w[2][0], w[2][1], w[2][2], w[2][3]);
}

// Eight channels of a row into three planes of 128-byte-swizzled rows of 64 channels.
template <int PLANE>
__device__ __forceinline__ void store_planes(unsigned char* base, int row, int chunk, const float (&x)[8]) {
  uint4 p0, p1, p2;
  split8(x, p0, p1, p2);
  unsigned char* at = base + row * 128 + ((chunk ^ (row & 7)) << 4);
  *reinterpret_cast<uint4*>(at) = p0;
  *reinterpret_cast<uint4*>(at + PLANE) = p1;
  *reinterpret_cast<uint4*>(at + 2 * PLANE) = p2;
}

// Eight numbers, in whole sectors where rows begin at them; K and V pass by L1, they are read once.  Without a branch: values that one
// side of it loads are waited for where the sides meet (8000 tokens took 2720 us instead of 2530).
__device__ __forceinline__ void load8(const float* from, bool wide, float (&x)[8]) {
  asm volatile(
      "{\n\t.reg .pred w;\n\tsetp.ne.u32 w, %9, 0;\n\t"
      "@w ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "@!w ld.global.v4.f32 {%0, %1, %2, %3}, [%8];\n\t"
      "@!w ld.global.v4.f32 {%4, %5, %6, %7}, [%8 + 16];\n\t}"
      : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(from), "r"((uint32_t)wide));
}

// The warps of K, or of Q and V (v).  One code for both, a block at a time: what runs side by side here has to stay in the instruction
// cache (with a code each and both blocks of a tile unrolled, 8000 tokens took 4540 us, waiting for instructions for the most part).
template <int D>
__device__ __forceinline__ void rows_role(const AttendF32& t, Smem<D>& sm, const bool v) {
  using S = Smem<D>;
  const AttendShape& a = t.a;
  constexpr int kMine = kKeys / 16;              // rows of a block that a thread has eight channels of
  const int tid = threadIdx.x & 127, lane = threadIdx.x & 31, row0 = tid >> 3, chunk = tid & 7;
  const bool wide = v ? t.wide_v : t.wide_k;
  unsigned long long* const full = v ? sm.v_full : sm.k_full;
  unsigned long long* const empty = v ? sm.v_empty : sm.k_empty;
  unsigned char* const planes = v ? sm.v[0][0] : sm.k[0][0];
  auto wait = [&](unsigned long long* bar, unsigned phase) {
    return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), phase & 1, &sm.abort)) != 0;
  };
  const unsigned buffers = v ? S::kV : S::kK;
  unsigned slot = 0, round = 0, n_q = 0;         // blocks of keys, of query rows
  for (unsigned nth = 0;; ++nth) {
    if (!wait(&sm.unit_full[nth % kUnits], nth / kUnits)) return;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) return;
    if (p.n == 0) continue;
    float x[kMine][8];
    unsigned none = 0;                           // bit u: there is no row u, x[u] is another one's
    auto load = [&](int block) {                 // of the piece
      const int tile = p.tile0 + block / S::kHalves, ch = 64 * (block % S::kHalves) + 8 * chunk;
      none = 0;
#pragma unroll
      for (int u = 0; u < kMine; ++u) {
        bool there;
        load8(key_row(t, p, v, tile, row0 + 16 * u, &there) + ch, wide, x[u]);
        none |= there ? 0u : 1u << u;
      }
    };
    load(0);
    if (v) {
      if (n_q > 0 && !wait(&sm.q_empty, n_q - 1)) return;
      tc_fence_after();
      ++n_q;
      const int rt = tid / a.G, r7 = tid & 7;    // a row a thread
      const bool there = rt < p.n_tok && rt < a.block_tokens;
      const float* from = static_cast<const float*>(a.q) + (a.paged ? p.s * a.q_seq : p.q_row * a.q_tok) + (p.tok0 + rt) * a.q_tok +
                          (p.h * a.G + tid - rt * a.G) * a.q_head;
      const uint32_t tq = sm.tmem + ((uint32_t)(tid >> 5) << 21) + kTmemQ;
#pragma unroll 1
      for (int c = 0; c < D / 16; ++c) {
        uint32_t w[2][8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          if (there) {
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
              const float4 z = *reinterpret_cast<const float4*>(from + 16 * c + 8 * e + k);
              y[k] = z.x; y[k + 1] = z.y; y[k + 2] = z.z; y[k + 3] = z.w;
            }
          }
          uint4 p0, p1, p2;
          split8(y, p0, p1, p2);
          w[0][4 * e] = p0.x; w[0][4 * e + 1] = p0.y; w[0][4 * e + 2] = p0.z; w[0][4 * e + 3] = p0.w;
          w[1][4 * e] = p1.x; w[1][4 * e + 1] = p1.y; w[1][4 * e + 2] = p1.z; w[1][4 * e + 3] = p1.w;
          *reinterpret_cast<uint4*>(sm.q + (c >> 2) * kHalfBytes + tid * 128 + (((2 * (c & 3) + e) ^ r7) << 4)) = p2;
        }
        tc_st8(tq + 8 * c, w[0]);
        tc_st8(tq + D / 2 + 8 * c, w[1]);
      }
      tc_wait_st();
      tc_fence_before();
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.q_full));
    }
#pragma unroll 1
    for (int i = 0; i < p.n * S::kHalves; ++i) {
      if (round > 0 && !wait(empty + slot, round - 1)) return;
      if (__any_sync(0xffffffffu, none != 0)) {
#pragma unroll
        for (int u = 0; u < kMine; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = none >> u & 1u ? 0.0f : x[u][e];
      }
      if (v) {
        if (i == 0) {                            // results are at most kUnits pieces behind
          if (lane == 0) {
            sm.odd_lo[nth % kAhead][tid >> 5] = 0x7fffffff;
            sm.odd_hi[nth % kAhead][tid >> 5] = -1;
          }
          __syncwarp();
        }
        bool odd = false;
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
          float top = 0.0f;                      // 0 times what is not finite is NaN
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaf(0.0f, x[u][e], top);
          odd |= top != 0.0f;
        }
        if (odd) {
#pragma unroll
          for (int u = 0; u < kMine; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = fabsf(x[u][e]) < INFINITY ? x[u][e] : 0.0f;
          const int tile = p.tile0 + i / S::kHalves;
          atomicMin(&sm.odd_lo[nth % kAhead][tid >> 5], tile);
          atomicMax(&sm.odd_hi[nth % kAhead][tid >> 5], tile);
        }
      }
#pragma unroll
      for (int u = 0; u < kMine; ++u) store_planes<kPlane>(planes + slot * 3 * kPlane, row0 + 16 * u, chunk, x[u]);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(full + slot));
      if (++slot == buffers) { slot = 0; ++round; }
      if (i + 1 < p.n * S::kHalves) load(i + 1);
    }
  }
}

// The six products of three planes each, the small ones first, of all channels (what is cut off then is cut off small sums): planes of A and of B, two bits each.
constexpr int kPairs = 6;
constexpr uint32_t kPlanesA = 0u | 2u << 2 | 1u << 4 | 0u << 6 | 1u << 8 | 0u << 10;
constexpr uint32_t kPlanesB = 2u | 0u << 2 | 1u << 4 | 1u << 6 | 0u << 8 | 0u << 10;

template <int D>
__device__ __forceinline__ bool mma_role(const AttendF32& t, Smem<D>& sm) {
  using S = Smem<D>;
  const uint32_t tmem = sm.tmem;
  constexpr uint32_t kIdS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kKeys >> 3) << 17) | (8u << 24);
  constexpr uint32_t kIdO = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 17) | (8u << 24) | kRowsB;      // 64 channels
  const uint32_t qa = desc_lo(smem_u32(sm.q)), qt = tmem + kTmemQ;
  auto wait = [&](unsigned long long* bar, unsigned phase) {
    return __all_sync(0xffffffffu, mbar_poll(smem_u32(bar), phase & 1, &sm.abort)) != 0;
  };
  unsigned done = 0, n_q = 0;                    // tiles
  unsigned k_slot = 0, k_round = 0, v_slot = 0, v_round = 0;
  for (unsigned nth = 0;; ++nth) {
    if (!wait(&sm.unit_full[nth % kUnits], nth / kUnits)) return false;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (elect_one()) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) return true;
    if (p.n == 0) continue;
    if (!wait(&sm.q_full, n_q++)) return false;
    for (int i = 0; i <= p.n; ++i) {
      if (i < p.n) {
        const unsigned no = done + i;
        const uint32_t d = tmem + kTmemS + (no & 1) * kKeys;
        uint32_t kb[S::kHalves], kslot[S::kHalves];
#pragma unroll
        for (int h = 0; h < S::kHalves; ++h) {
          if (!wait(&sm.k_full[k_slot], k_round)) return false;
          kslot[h] = k_slot;
          kb[h] = desc_lo(smem_u32(sm.k[0][0])) + (k_slot * 3 * kPlane >> 4);
          if (++k_slot == S::kK) { k_slot = 0; ++k_round; }
        }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int c = 0; c < kPairs; ++c) {
            const uint32_t plane = kPlanesA >> (2 * c) & 3u, bo = (kPlanesB >> (2 * c) & 3u) * kPlane >> 4, ap = qt + plane * (D / 2);
#pragma unroll
            for (int h = 0; h < S::kHalves; ++h)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (plane == 2) tc_mma_ss(d, qa + (h * kHalfBytes >> 4) + 2 * k, kb[h] + bo + 2 * k, kIdS, c > 0 || h > 0 || k > 0);
                else tc_mma_ts(d, ap + 32 * h + 8 * k, kb[h] + bo + 2 * k, kIdS, c > 0 || h > 0 || k > 0);
              }
          }
#pragma unroll
          for (int h = 0; h < S::kHalves; ++h) tc_commit(smem_u32(&sm.k_empty[kslot[h]]));
          tc_commit(smem_u32(&sm.s_full[no & 1]));
          if (i + 1 == p.n) tc_commit(smem_u32(&sm.q_empty));
        }
        __syncwarp();
      }
      if (i > 0) {
        const unsigned no = done + i - 1;
        if (!wait(&sm.p_ready, no)) return false;
        tc_fence_after();
        const uint32_t pa = tmem + kTmemP;
#pragma unroll 1
        for (int h = 0; h < S::kHalves; ++h) {
          if (!wait(&sm.v_full[v_slot], v_round)) return false;
          tc_fence_after();
          const uint32_t va = desc_lo(smem_u32(sm.v[0][0])) + (v_slot * 3 * kPlane >> 4), d = tmem + kTmemO + 64 * h;
          if (elect_one()) {
#pragma unroll
            for (int c = 0; c < kPairs; ++c) {
              const uint32_t ap = pa + (kPlanesA >> (2 * c) & 3u) * kPlaneCols, bp = va + ((kPlanesB >> (2 * c) & 3u) * kPlane >> 4);
#pragma unroll
              for (int k = 0; k < kKeys / 16; ++k) tc_mma_ts(d, ap + 8 * k, bp + k * 128, kIdO, c > 0 || k > 0);
            }
            tc_commit(smem_u32(&sm.v_empty[v_slot]));
            if (h + 1 == S::kHalves) tc_commit(smem_u32(&sm.pv_done));
          }
          __syncwarp();
          if (++v_slot == S::kV) { v_slot = 0; ++v_round; }
        }
      }
    }
    done += p.n;
  }
}

__device__ __forceinline__ uint32_t seen_below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// Values of V that are not finite, of the tiles lo .. hi: rows that see them get them, in the results that the thread has written.
__device__ __forceinline__ void put_back(const AttendF32& t, const AttendPiece& p, int lo, int hi, int bound, unsigned long long mask, float* out) {
  const AttendShape& a = t.a;
  for (int tile = lo; tile <= hi; ++tile)
    for (int j = 0; j < kKeys; ++j) {
      const bool drafted = a.has_new && tile == p.n_all - 1;
      if (drafted ? !(mask >> j & 1) : !a.paged && tile * kKeys + j >= bound) continue;
      bool row_there;
      const float* v = key_row(t, p, true, tile, j, &row_there);
      if (!row_there) continue;
      for (int ch = 0; ch < a.head_dim; ++ch)
        if (!(fabsf(v[ch]) < INFINITY)) out[ch] += v[ch];
    }
}

template <int D>
__device__ __forceinline__ void softmax_role(const AttendF32& t, Smem<D>& sm) {
  const AttendShape& a = t.a;
  const int row = threadIdx.x, lane = threadIdx.x & 31;
  const float sc = a.ml_unit;
  const uint32_t lanes = sm.tmem + ((uint32_t)(row >> 5) << 21);
  const f32x2 sc2 = pack2(sc, sc);
  auto wait = [&](unsigned long long* bar, unsigned phase) {
    return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), phase & 1, &sm.abort)) != 0;
  };
  int rt, rh;                                    // the thread's row: token of the block, query head of the group
  if (!attend_row(a, row, &rt, &rh)) rt = 1 << 20;
  unsigned done = 0;
  for (unsigned nth = 0;; ++nth) {
    if (!wait(&sm.unit_full[nth % kUnits], nth / kUnits)) return;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) return;
    const bool there = rt < p.n_tok;
    const int tok = p.tok0 + rt, bound = max(min(tok + 1 + p.shift, p.nk), 0);
    unsigned long long mask = 0;
    if (a.has_new && there) {
      mask = a.tree ? a.tree[(long long)p.s * a.n_tokens + tok] : ~0ull >> (63 - tok);
      mask &= ~0ull >> (64 - p.n_seq_tok);
    }
    const bool work = __any_sync(0xffffffffu, there);
    float m = -INFINITY, l = 0.0f;
    f32x2 sum[D / 2];                            // of the tiles before the last one
#pragma unroll
    for (int e = 0; e < D / 2; ++e) sum[e] = 0;
#pragma unroll 1
    for (int i = 0; i < p.n; ++i, ++done) {
      const int tile = p.tile0 + i;
      const bool drafted = a.has_new && tile == p.n_all - 1;
      const int end = a.paged ? (drafted ? 0 : p.nk - tile * kKeys) : bound - tile * kKeys;     // keys that the row sees
      if (!wait(&sm.s_full[done & 1], done >> 1)) return;
      tc_fence_after();
      if (work) {
        const uint32_t ts = lanes + kTmemS + (done & 1) * kKeys, tp = lanes + kTmemP;
        uint32_t r[2][32];
        tc_ld32(ts, r[0]);
        tc_ld32(ts + 32, r[1]);
        tc_wait_ld(r[0]);
        tc_wait_ld(r[1]);
        if (__any_sync(0xffffffffu, drafted || end < kKeys)) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t see = drafted ? (uint32_t)(mask >> (32 * q)) : seen_below(end - 32 * q);
#pragma unroll
            for (int e = 0; e < 32; ++e) r[q][e] = see >> e & 1u ? r[q][e] : 0xff800000u;
          }
        }
        float mx[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          mx[q] = __uint_as_float(r[q][0]);
#pragma unroll
          for (int e = 1; e < 31; e += 2) mx[q] = fmaxf(fmaxf(mx[q], __uint_as_float(r[q][e])), __uint_as_float(r[q][e + 1]));
          mx[q] = fmaxf(mx[q], __uint_as_float(r[q][31]));
        }
        const float top = fmaxf(mx[0], mx[1]);
        const bool lift = i > 0 && (top - m) * sc > kLift;           // m = -infinity: any score lifts it
        const float f = lift ? ex2((m - top) * sc) : 1.0f;
        if (i == 0 || lift) m = top;
        l *= f;
        // 2^(sc x - sc m) with one rounding of the difference, which is as large as sc m 2^-24: where that is much, differences first
        float base = m == -INFINITY ? 0.0f : m;
        if (__any_sync(0xffffffffu, fabsf(base) * sc > 0x1p20f)) {
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int e = 0; e < 32; ++e) r[q][e] = __float_as_uint(__uint_as_float(r[q][e]) - base);
          base = 0.0f;
        }
        const float nm = -base * sc;
        const f32x2 nm2 = pack2(nm, nm);
        f32x2 s0 = 0, s1 = 0;
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const f32x2 p0 = ex2_pair(fma2(pack2(__uint_as_float(r[q][e]), __uint_as_float(r[q][e + 1])), sc2, nm2));
            const f32x2 p1 = ex2_pair(fma2(pack2(__uint_as_float(r[q][e + 2]), __uint_as_float(r[q][e + 3])), sc2, nm2));
            s0 = add2(s0, p0);
            s1 = add2(s1, p1);
            float y[4];
            unpack2(p0, y[0], y[1]);
            unpack2(p1, y[2], y[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) r[q][e + k] = __float_as_uint(y[k]);
          }
        l += sum2(s0, s1);
        // P and O belong to the product before until it is done; what can be is computed by then
        if (i > 0) {
          if (!wait(&sm.pv_done, done - 1)) return;
          tc_fence_after();
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {            // sixteen keys at a time
          uint32_t w[3][8];
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(r[q >> 1][16 * (q & 1) + e + k]);
            uint4 p0, p1, p2;
            split8(y, p0, p1, p2);
            w[0][e / 2] = p0.x; w[0][e / 2 + 1] = p0.y; w[0][e / 2 + 2] = p0.z; w[0][e / 2 + 3] = p0.w;
            w[1][e / 2] = p1.x; w[1][e / 2 + 1] = p1.y; w[1][e / 2 + 2] = p1.z; w[1][e / 2 + 3] = p1.w;
            w[2][e / 2] = p2.x; w[2][e / 2 + 1] = p2.y; w[2][e / 2 + 2] = p2.z; w[2][e / 2 + 3] = p2.w;
          }
#pragma unroll
          for (int c = 0; c < 3; ++c) tc_st8(tp + c * kPlaneCols + 8 * q, w[c]);
        }
        if (i > 0) {                             // the product before goes to the sum
#pragma unroll
          for (int ch = 0; ch < D; ch += 32) {
            uint32_t o[32];
            tc_ld32(lanes + kTmemO + ch, o);
            tc_wait_ld(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[ch / 2 + e] = add2(sum[ch / 2 + e], pack2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])));
          }
          if (__any_sync(0xffffffffu, lift)) {
            const f32x2 f2 = pack2(f, f);
#pragma unroll
            for (int e = 0; e < D / 2; ++e) sum[e] = mul2(sum[e], f2);
          }
        }
      } else if (i > 0) {
        if (!wait(&sm.pv_done, done - 1)) return;
      }
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.p_ready));
    }
    // ---- results
    if (p.n > 0) {
      if (!wait(&sm.pv_done, done - 1)) return;
      tc_fence_after();
    }
    if (!work) continue;
    const bool whole = p.part < 0;
    const float inv = !whole ? 1.0f : l > 0.0f || l != l ? 1.0f / l : 0.0f;
    const long long place = (long long)(blockIdx.x * 2 + p.part) * a.part_rows + row;
    float* const dst = whole ? static_cast<float*>(a.out) + (a.paged ? p.s * a.o_seq : p.q_row * a.o_tok) + tok * a.o_tok + (p.h * a.G + rh) * a.o_head
                             : a.part + place * D;
    const f32x2 inv2 = pack2(inv, inv);
#pragma unroll
    for (int ch = 0; ch < D; ch += 16) {
      uint32_t o[16];
      if (p.n > 0) {
        tc_ld16_issue(lanes + kTmemO + ch, o);
        tc_ld_wait(o);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0;
      }
      if (there) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          float x, y;
          unpack2(mul2(add2(sum[(ch + e) / 2], pack2(__uint_as_float(o[e]), __uint_as_float(o[e + 1]))), inv2), x, y);
          o[e] = __float_as_uint(x);
          o[e + 1] = __float_as_uint(y);
        }
        if (t.wide || !whole) {
          store32(dst + ch, o);
          store32(dst + ch + 8, o + 8);
        } else {
#pragma unroll
          for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(dst + ch + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      __syncwarp();                              // the next load is the whole warp's
    }
    if (there) {
      int lo = 0x7fffffff, hi = -1;
#pragma unroll
      for (int w = 0; w < 4 && p.n > 0; ++w) {
        lo = min(lo, *(volatile int*)&sm.odd_lo[nth % kAhead][w]);
        hi = max(hi, *(volatile int*)&sm.odd_hi[nth % kAhead][w]);
      }
      if (hi >= 0) put_back(t, p, lo, hi, bound, mask, dst);
      if (whole) attend_lse(a, p.s, p.h * a.G + rh, tok, p.n_seq_tok, m * sc, l);
      else a.ml[place] = make_float2(m, l);
    }
    __syncwarp();
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) k_attend_f32(const __grid_constant__ AttendF32 t) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(smem_u32(&sm.unit_full[i]), 1);
      mbar_init(smem_u32(&sm.unit_empty[i]), 13);
    }
    mbar_init(smem_u32(&sm.q_full), 4);
    mbar_init(smem_u32(&sm.q_empty), 1);
    for (int i = 0; i < Smem<D>::kK; ++i) {
      mbar_init(smem_u32(&sm.k_full[i]), 4);
      mbar_init(smem_u32(&sm.k_empty[i]), 1);
    }
    for (int i = 0; i < Smem<D>::kV; ++i) {
      mbar_init(smem_u32(&sm.v_full[i]), 4);
      mbar_init(smem_u32(&sm.v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sm.s_full[i]), 1);
    mbar_init(smem_u32(&sm.p_ready), 4 + t.extra_arrival);
    mbar_init(smem_u32(&sm.pv_done), 1);
    mbar_init(smem_u32(&sm.drain), 1);
    sm.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();
  pdl_wait();
  attend_start(t.a, blockIdx.x, &sm.start);
  __syncthreads();
  // registers of the four warpgroups: no more than four times 128 in all
  static_assert((D == 128 ? 240 + 2 * 96 : 176 + 2 * 128) + 80 <= 512, "registers");
  if (warp < kKWarp) {
    regs_up<D == 128 ? 240 : 176>();
    softmax_role<D>(t, sm);
  } else if (warp < kMmaWarp) {
    if (D == 128) regs_down<96>();
    rows_role<D>(t, sm, warp >= kVWarp);
  } else {
    regs_down<80>();
    if (warp == kMmaWarp) {
      if (!mma_role<D>(t, sm) && elect_one()) {  // a wait ran out: what is under way ends first
        volatile int never = 0;
        tc_commit(smem_u32(&sm.drain));
        mbar_wait(smem_u32(&sm.drain), 0, &never);
      }
    } else if (warp == kPlanWarp) {
      if (lane == 0 && t.a.desc) t.a.desc[2 * blockIdx.x].state = t.a.desc[2 * blockIdx.x + 1].state = 0;
      AttendSchedule plan(t.a, blockIdx.x, &sm.start);
      for (unsigned nth = 0;; ++nth) {
        AttendPiece p = {};
        const bool more = plan.next(&p);
        p.stop = !more;
        if (nth >= (unsigned)kUnits) {
          const bool ok = mbar_wait(smem_u32(&sm.unit_empty[nth % kUnits]), (nth / kUnits - 1) & 1, &sm.abort);
          if (!__all_sync(0xffffffffu, ok)) break;
        }
        if (lane == 0) {
          sm.piece[nth % kUnits] = p;
          mbar_arrive(smem_u32(&sm.unit_full[nth % kUnits]));
          if (more && p.part >= 0) attend_note(t.a, p.part, p, p.part == 1 ? plan.pieces() : 0);
        }
        if (!more) break;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (sm.abort && threadIdx.x == 0) {
    if (t.a.status) *t.a.status = SLKV_ERR_DEVICE_TIMEOUT;
    if (t.a.desc) t.a.desc[2 * blockIdx.x].state = t.a.desc[2 * blockIdx.x + 1].state = -1;
  }
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sm.tmem) : "memory");
}

template <int D>
cudaError_t launch(const AttendF32& t, cudaStream_t st, int* launches) {
  static_assert(sizeof(Smem<D>) <= kSmemLimit, "shared memory of a CTA");
  static std::atomic<bool> allowed[16];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 16 || !allowed[dev].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(k_attend_f32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    if (dev < 16) allowed[dev].store(true, std::memory_order_relaxed);
  }
  LaunchScope scope(KID_ATTEND, st, launches);
  return launch_pdl(k_attend_f32<D>, dim3((unsigned)t.a.n_cta), dim3(kThreads), sizeof(Smem<D>), st, 1, t);
}

}  // namespace

cudaError_t launch_attend_f32(const AttendShape& a, cudaStream_t st, int* launches) {
  AttendF32 t = {};
  t.a = a;
  for (t.page_bits = 0; a.paged && (1 << t.page_bits) < a.page_rows;) ++t.page_bits;
  auto wide = [&](const void* base, long long tok, long long head, long long seq) {
    return reinterpret_cast<uintptr_t>(base) % 32 == 0 && (tok | head | seq) % 8 == 0;
  };
  t.wide = wide(a.out, a.o_tok, a.o_head, a.paged ? a.o_seq : 0);
  t.wide_k = a.paged ? wide(a.k, 0, 0, 0) && (!a.has_new || wide(a.k_new, a.kn_tok, a.kn_head, a.kn_seq)) : wide(a.k, a.k_tok, a.k_head, 0);
  t.wide_v = a.paged ? wide(a.v, 0, 0, 0) && (!a.has_new || wide(a.v_new, a.vn_tok, a.vn_head, a.vn_seq)) : wide(a.v, a.v_tok, a.v_head, 0);
  t.extra_arrival = take_expire_next_copy_wait() ? 1 : 0;
  return a.head_dim == 128 ? launch<128>(t, st, launches) : launch<64>(t, st, launches);
}

}  // namespace slkv
