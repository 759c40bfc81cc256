// Attention of prompts and of tokens over a paged cache on the tensor cores, bf16.
//
//   out_i = sum_j p_ij v_j,  p_ij = 2^(sc (x_ij - m_i)) / sum_j 2^(sc (x_ij - m_i)),  x_ij = q_i . k_j over the keys row i sees,
//   sc = scale log2(e)
//
// One pass over the keys with a running reference m and sum per row.  A CTA takes pieces of units (AttendSchedule): two blocks of 128
// query rows, tokens times the query heads of one KV head, against tiles of 128 keys.  S = Q K^T of a block goes to TMEM (128
// columns), a warpgroup turns its 128 rows, a row per thread, into P = 2^(sc (x - m)) in bf16 over the same columns, and O += P V takes P from
// TMEM as its left operand; while one block's rows are exponentiated the tensor cores work on the other block.  m is raised, and O
// rescaled in TMEM, only where a tile's maximum lies 2^8 above it.  A unit of one block (few tokens) has its tiles shared by the two
// warpgroups in turn, each with sums of its own, which are merged in the end.
//   warps 0-3, 4-7  softmax of the two blocks, results
//   warp 8  TMA loads of K, V      warp 9  MMAs      warp 10  schedule      warp 11  TMA loads of Q
// P is rounded to bf16 for the product (2^-8 of each term); the sum of a row is taken of what is not rounded, in fp32.
//
// Measured (B200, head_dim 128, 32 query heads on 8 KV heads; in a row, the same inputs): 32000 tokens 7.7 ms, 1090 TFLOP/s, 8000 tokens 459 us,
// 1140 TFLOP/s (other inputs from call to call: 8.1 ms, 480 us); drafted trees of 64 over segments of 8000 to 32000 rows 217 us, 5.8 TB/s.  What bounds prompts is the chain of a block: a tile's softmax takes 2280 cycles (loads
// from TMEM 170, maximum 400, exponentials 1220 to 1320 beside the other block's, the rest conversions, stores and barriers), the products
// before and behind it 1300 more, of which 1024 are the matrix unit's; two blocks in turn keep it busy 57 % of the time, the exponentials'
// unit as long.  There is no TMEM for a third block or a second S.  Tried, 8000 tokens: four warps more, two threads to a row (8.7 ms at
// 32000 tokens); halves of 64 keys with S in two buffers and a softmax each (550 us); two warps that issue products; a part of the exponentials as polynomials
// (beside it in one call, in turn: none 459 us, an eighth of them 467, a quarter 479, half 510; at 32000 tokens 7.71 ms, 7.86, 7.99, 8.42); the maximum beside the
// exponentials of the reference before (506 to 524 us, 479 without in that call).
//
// A key that a row does not see gives it nothing, whatever K and V hold there: scores are replaced, not biased, and since 0 times an
// infinity is not 0, the V rows of a tile that not every row of the block sees are looked through first: rows behind the last key become 0 in
// shared memory, and so do values that are not finite, which the rows that do see them add again at the end.
#include <atomic>

#include "slkv_attend_device.cuh"

namespace slkv {
namespace {

constexpr int kThreads = 384;
constexpr int kLoadWarp = 8, kMmaWarp = 9, kPlanWarp = 10, kQueryWarp = 11;
constexpr int kUnits = 4;                        // pieces the schedule is ahead by: nobody is more than these ahead of a warp that is at one
constexpr int kAhead = 2 * kUnits;
constexpr float kLift = 8.0f;                    // log2 of how far P may exceed 1 before the reference is raised
constexpr int kTmemS = 0, kTmemO = 256;          // columns: S of block b at 128 b, O at 256 + 128 b

template <int D>
struct Smem {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kStages = D == 128 ? 5 : 8;
  alignas(1024) unsigned char q[2][kTileBytes];
  alignas(1024) unsigned char kv[kStages][kTileBytes];
  union {
    float2 ml[2][128];
    AttendStart start;                           // before anything else
  };
  AttendPiece piece[kUnits];
  unsigned long long unit_full[kUnits], unit_empty[kUnits], q_full[2], q_empty[2], kv_full[kStages], kv_empty[kStages], s_full[2],
      p_most[2], p_ready[2], o_full[2], merge_full, merge_done, drain;
  int odd[kAhead];                               // number + 1 of the piece that found V values that are not finite
  int abort;
  uint32_t tmem;
};

struct AttendMaps {
  CUtensorMap q, k, v, kn, vn;
};
struct AttendTc {
  AttendShape a;
  int k_head_inner, v_head_inner, kn_head_inner, vn_head_inner;
  float sc;                                      // scale * log2(e)
  int wide;                                      // rows of out begin at 32-byte boundaries
  int arrivals;                                  // at p_ready: 4, or 5 where a test makes the wait for them run out
};

// What both the MMA warp and the softmax warps derive from a piece.
struct Blocks {
  int alt;                                       // one block: its tiles in turn to the warpgroups
  int n[2];                                      // tiles of each warpgroup
  __device__ __forceinline__ Blocks(const AttendTc& t, const AttendPiece& p) {
    alt = p.n_tok <= t.a.block_tokens;
    if (alt) {
      n[0] = (p.n + 1) >> 1;
      n[1] = p.n >> 1;
    } else {
      n[0] = n[1] = p.n;
      if (!t.a.paged) {                          // tiles that the first block sees
        const int seen = p.tok0 + t.a.block_tokens + p.shift;
        n[0] = max(min(p.n, (seen + kAttendTile - 1) / kAttendTile - p.tile0), 0);
      }
    }
  }
  __device__ __forceinline__ int tile(int g, int i) const { return alt ? 2 * i + g : i; }
  // The order of a piece's loads, which the MMAs follow: K0 V0 K1 V1 .., or K0 K1 V0 K2 V1 K3 ..
  __device__ __forceinline__ int k_load(int t) const { return !alt ? 2 * t : (t < 2 ? t : 2 * t - 1); }
  __device__ __forceinline__ int v_load(int t, int total) const { return !alt ? 2 * t + 1 : t + min(total, t + 2); }
};
// Of a tile, for the block of a warpgroup whose first token is tok and which has n_tok of them: columns below `all` are seen by every
// row, columns from `end` on are no keys, and the product with V needs `used` of them.
struct Columns { int all, end, used; };
__device__ __forceinline__ Columns columns(const AttendTc& t, const AttendPiece& p, int tile, int tok, int n_tok) {
  Columns c;
  if (t.a.paged) {
    const bool drafted = t.a.has_new && tile == p.n_all - 1;
    c.end = drafted ? p.n_seq_tok : min(p.nk - tile * kAttendTile, kAttendTile);
    c.all = drafted ? 0 : c.end;
    c.used = (c.end + 15) & ~15;
  } else {
    c.end = min(p.nk - tile * kAttendTile, kAttendTile);
    c.all = max(min(tok + 1 + p.shift - tile * kAttendTile, c.end), 0);
    c.used = (max(min(tok + n_tok + p.shift - tile * kAttendTile, c.end), 0) + 15) & ~15;
  }
  return c;
}

template <int D>
__device__ __forceinline__ void load_role(const AttendTc& t, const AttendMaps& m, Smem<D>& sm) {
  using S = Smem<D>;
  const AttendShape& a = t.a;
  const int lane = threadIdx.x & 31;
  unsigned loads = 0, issued = 0;                // loads: of earlier pieces
  bool ok = true;
  for (unsigned nth = 0;; ++nth) {
    ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.unit_full[nth % kUnits]), (nth / kUnits) & 1, &sm.abort));
    if (!ok) break;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) break;
    if (p.n == 0) continue;
    const Blocks b(t, p);
    const int total = 2 * p.n;
    int ids = 0, ids_first = -1;                 // lane l: page ids_first + l of the segment
    for (int i = 0; i < total; ++i) {
      // load i of the piece: which operand of which tile
      bool is_v;
      int tl;
      if (!b.alt) {
        is_v = i & 1;
        tl = i >> 1;
      } else if (i < 2 && i < p.n) {
        is_v = false;
        tl = i;
      } else {
        const int j = i - min(2, p.n);           // V0 K2 V1 K3 ..; K runs out first
        const int both = 2 * max(p.n - 2, 0);
        is_v = j >= both || !(j & 1);
        tl = j >= both ? max(p.n - 2, 0) + (j - both) : (j & 1 ? 2 + (j >> 1) : j >> 1);
      }
      const int tile = p.tile0 + tl;
      const unsigned no = loads + i, slot = no % S::kStages;
      const uint32_t bar = smem_u32(&sm.kv_full[slot]), dst = smem_u32(sm.kv[slot]);
      if (no >= (unsigned)S::kStages) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.kv_empty[slot]), (no / S::kStages - 1) & 1, &sm.abort));
        if (!ok) break;
      }
      issued = no + 1;
      if (!a.paged) {
        if (lane == 0) {
          mbar_expect_tx(bar, S::kTileBytes);
          const int row = p.k_row + tile * kAttendTile;
          const int inner = is_v ? t.v_head_inner : t.k_head_inner;
          for (int hf = 0; hf < S::kHalves; ++hf)
            tma_load_3d(dst + hf * kHalfBytes, is_v ? &m.v : &m.k, hf * 64, inner ? p.h : row, inner ? row : p.h, bar);
        }
      } else if (a.has_new && tile == p.n_all - 1) {
        if (lane == 0) {
          mbar_expect_tx(bar, (uint32_t)(S::kHalves * a.n_tokens * 128));
          const int inner = is_v ? t.vn_head_inner : t.kn_head_inner;
          for (int hf = 0; hf < S::kHalves; ++hf)
            tma_load_4d(dst + hf * kHalfBytes, is_v ? &m.vn : &m.kn, hf * 64, inner ? p.h : 0, inner ? 0 : p.h, p.s, bar);
        }
      } else {
        // pages of the tile that hold rows: a lane each
        const int per = kAttendTile / a.page_rows, first = tile * per;
        const int have = (p.nk + a.page_rows - 1) / a.page_rows, n = min(per, have - first);
        if (ids_first < 0 || first < ids_first || first + n > ids_first + 32) {
          ids_first = first;
          const int at = first + lane;
          ids = at < have ? __ldg(a.tables + (long long)(p.s * a.n_kv_heads + p.h) * a.max_pages + at) : 0;
        }
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n * S::kHalves * a.page_rows * 128));
        const int id = __shfl_sync(0xffffffffu, ids, (first - ids_first + lane) & 31);
        __syncwarp();
        if (lane < n) {
          const bool there = (unsigned)id < (unsigned)a.n_pages;
          if (!there && a.status) *a.status = SLKV_ERR_BAD_SHAPE;
          const int row = there ? id * a.page_rows : (int)a.rows_k;      // behind the pool: zeros
          for (int hf = 0; hf < S::kHalves; ++hf)
            tma_load_3d(dst + hf * kHalfBytes + lane * a.page_rows * 128, is_v ? &m.v : &m.k, hf * 64, row, 0, bar);
        }
        __syncwarp();
      }
    }
    if (!ok) break;
    loads += total;
  }
  if (ok) return;
  // a wait ran out: the copies in flight end before the CTA does
  volatile int never = 0;
  for (unsigned no = issued > (unsigned)S::kStages ? issued - S::kStages : 0; no < issued; ++no)
    mbar_wait(smem_u32(&sm.kv_full[no % S::kStages]), (no / S::kStages) & 1, &never);
}

// Blocks of query rows, ahead of the products with them as far as two buffers allow.
template <int D>
__device__ __forceinline__ void query_role(const AttendTc& t, const AttendMaps& m, Smem<D>& sm) {
  using S = Smem<D>;
  const AttendShape& a = t.a;
  unsigned n_q = 0;                              // blocks
  bool ok = true;
  for (unsigned nth = 0;; ++nth) {
    ok = mbar_wait(smem_u32(&sm.unit_full[nth % kUnits]), (nth / kUnits) & 1, &sm.abort);
    if (!ok) break;
    const AttendPiece p = sm.piece[nth % kUnits];
    mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) break;
    if (p.n == 0) continue;
    const int blocks = p.n_tok <= a.block_tokens ? 1 : 2;
    for (int g = 0; g < blocks && ok; ++g) {
      const unsigned slot = n_q & 1;
      if (n_q >= 2) ok = mbar_wait(smem_u32(&sm.q_empty[slot]), ((n_q >> 1) - 1) & 1, &sm.abort);
      if (!ok) break;
      ++n_q;
      const uint32_t bar = smem_u32(&sm.q_full[slot]), dst = smem_u32(sm.q[slot]);
      mbar_expect_tx(bar, (uint32_t)(S::kHalves * a.box_tokens * a.G * 128));
      const int tok = (a.paged ? 0 : p.q_row) + p.tok0 + g * a.block_tokens, head = p.h * a.G;
      for (int hf = 0; hf < S::kHalves; ++hf)
        tma_load_4d(dst + hf * kHalfBytes, &m.q, hf * 64, a.q_head_inner ? head : tok, a.q_head_inner ? tok : head, a.paged ? p.s : 0, bar);
    }
    if (!ok) break;
  }
  if (ok) return;
  volatile int never = 0;                        // a wait ran out: the copies in flight end before the CTA does
  for (unsigned no = n_q > 2 ? n_q - 2 : 0; no < n_q; ++no) mbar_wait(smem_u32(&sm.q_full[no & 1]), (no >> 1) & 1, &never);
}

// The whole warp waits, one lane issues (elect.sync: what it is given then lies in uniform registers; under lane == 0 a product took 70 to
// 110 cycles to issue instead of 48 to 64).  What a step needs beside P is waited for before P is; six of P's eight products go out when three
// quarters of P are there (32000 tokens 7963 -> 7880 us).
template <int D>
__device__ __forceinline__ bool mma_role(const AttendTc& t, Smem<D>& sm) {
  using S = Smem<D>;
  const AttendShape& a = t.a;
  const uint32_t tmem = sm.tmem;
  constexpr uint32_t kIdS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kAttendTile >> 3) << 17) | (8u << 24);
  constexpr uint32_t kIdO = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(D >> 3) << 17) | (8u << 24) | kRowsB;
  unsigned loads = 0, n_q = 0, n_p[2] = {0, 0};
  auto wait = [&](unsigned long long* bar, unsigned phase) {
    return __all_sync(0xffffffffu, mbar_poll(smem_u32(bar), phase & 1, &sm.abort)) != 0;
  };
  for (unsigned nth = 0;; ++nth) {
    if (!wait(&sm.unit_full[nth % kUnits], nth / kUnits)) return false;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (elect_one()) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) return true;
    if (p.n == 0) continue;
    const Blocks b(t, p);
    auto k_there = [&](int g, int i) {
      const unsigned no = loads + b.k_load(b.tile(g, i));
      return wait(&sm.kv_full[no % S::kStages], no / S::kStages);
    };
    auto v_there = [&](int g, int i) {
      const unsigned no = loads + b.v_load(b.tile(g, i), p.n);
      return wait(&sm.kv_full[no % S::kStages], no / S::kStages);
    };
    auto qk = [&](int g, int i) {                // by the issuer
      const unsigned slot = (loads + b.k_load(b.tile(g, i))) % S::kStages, block = (n_q + (b.alt ? 0 : g)) & 1;
      const uint32_t qa = desc_lo(smem_u32(sm.q[block])), ka = desc_lo(smem_u32(sm.kv[slot])), d = tmem + kTmemS + 128 * g;
      #pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
        tc_mma_ss(d, qa + off, ka + off, kIdS, k > 0);
      }
      tc_commit(smem_u32(&sm.s_full[g]));
      if (b.alt || g == 1) tc_commit(smem_u32(&sm.kv_empty[slot]));
      if (b.alt ? 2 * i + g + 1 == p.n : i + 1 == b.n[g]) tc_commit(smem_u32(&sm.q_empty[block]));
    };
    for (int g = 0; g < 2; ++g) {
      if (!b.alt || g == 0) {
        const unsigned block = n_q + g;
        if (!wait(&sm.q_full[block & 1], block >> 1)) return false;
        // a block that sees none of the tiles
        if (b.n[g] == 0 && elect_one()) mbar_arrive(smem_u32(&sm.q_empty[block & 1]));
      }
      if (b.n[g] == 0) continue;
      if (!k_there(g, 0)) return false;
      tc_fence_after();
      if (elect_one()) qk(g, 0);
      __syncwarp();
    }
    const int steps = max(b.n[0], b.n[1]);
    for (int i = 0; i < steps; ++i)
      for (int g = 0; g < 2; ++g) {
        if (i >= b.n[g]) continue;
        const bool more = i + 1 < b.n[g];
        if (b.alt || g == 0 || i >= b.n[0]) {
          if (!v_there(g, i)) return false;
        }
        if (more && (b.alt || g == 0 || i + 1 >= b.n[0])) {
          if (!k_there(g, i + 1)) return false;
        }
        const int tok = p.tok0 + (b.alt ? 0 : g * a.block_tokens);
        const int used = columns(t, p, p.tile0 + b.tile(g, i), tok, min(a.block_tokens, p.n_seq_tok - tok)).used;
        const unsigned slot = (loads + b.v_load(b.tile(g, i), p.n)) % S::kStages;
        const uint32_t va = desc_lo(smem_u32(sm.kv[slot])), d = tmem + kTmemO + 128 * g, pa = tmem + kTmemS + 128 * g;
        constexpr int kMost = 6;                 // products with P's first three quarters
        if (!wait(&sm.p_most[g], n_p[g])) return false;
        if (used == kAttendTile) {
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kMost; ++k) tc_mma_ts(d, pa + 8 * k, va + k * 128, kIdO, k > 0 ? 1 : i > 0);
          }
          __syncwarp();
        }
        if (!wait(&sm.p_ready[g], n_p[g]++)) return false;
        tc_fence_after();
        if (elect_one()) {
          if (used == kAttendTile) {
#pragma unroll
            for (int k = kMost; k < kAttendTile / 16; ++k) tc_mma_ts(d, pa + 8 * k, va + k * 128, kIdO, 1);
          } else {
#pragma unroll 1
            for (int k = 0; k < used / 16; ++k) tc_mma_ts(d, pa + 8 * k, va + k * 128, kIdO, k > 0 || i > 0);
          }
          if (b.alt || g == 1) tc_commit(smem_u32(&sm.kv_empty[slot]));
          if (more) qk(g, i + 1);
          else tc_commit(smem_u32(&sm.o_full[g]));
        }
        __syncwarp();
      }
    loads += 2 * p.n;
    n_q += b.alt ? 1 : 2;
  }
}

// The first n of 32 keys, a bit each.
__device__ __forceinline__ uint32_t seen_below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// V rows all .. used of a tile: those from `end` on become zero, and what is not finite in the others too.  Returns whether there was any.
template <int D>
__device__ __forceinline__ bool clean_rows(unsigned char* v, const Columns& c, int tid) {
  constexpr int kChunks = D / 8;                 // of 16 bytes, of a row
  bool odd = false;
  for (int i = tid; i < (c.used - c.all) * kChunks; i += 128) {
    const int row = c.all + i / kChunks, ch = i % kChunks;
    uint4* at = reinterpret_cast<uint4*>(v + (ch >> 3) * kHalfBytes + row * 128 + (ch & 7) * 16);
    if (row >= c.end) {
      *at = make_uint4(0, 0, 0, 0);
      continue;
    }
    uint32_t w[4];
    *reinterpret_cast<uint4*>(w) = *at;
    bool here = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; here = true; }
      if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; here = true; }
    }
    if (here) {
      odd = true;
      *at = *reinterpret_cast<uint4*>(w);
    }
  }
  return odd;
}

// Values of V that are not finite and were taken out, in the channels ch0 .. ch1 - 1: rows that see them get them back, in the results
// that the thread has written.
template <bool WHOLE>
__device__ __noinline__ void put_back(const AttendTc& t, const AttendPiece& p, int bound, unsigned long long mask, int ch0, int ch1, void* out) {
  const AttendShape& a = t.a;
  int j0, j1;
  const __nv_bfloat16* base;
  long long stride;
  if (a.paged) {
    if (!a.has_new || p.tile0 + p.n != p.n_all) return;
    j0 = 0;
    j1 = p.n_seq_tok;
    base = static_cast<const __nv_bfloat16*>(a.v_new) + p.s * a.vn_seq + p.h * a.vn_head;
    stride = a.vn_tok;
  } else {
    j0 = max(max(p.tok0 + 1 + p.shift, 0), p.tile0 * kAttendTile);
    j1 = min(bound, (p.tile0 + p.n) * kAttendTile);
    base = static_cast<const __nv_bfloat16*>(a.v) + p.k_row * a.v_tok + p.h * a.v_head;
    stride = a.v_tok;
  }
  for (int j = j0; j < j1; ++j) {
    if (a.paged && !(mask >> j & 1)) continue;
    for (int ch = ch0; ch < ch1; ++ch) {
      const float x = __bfloat162float(base[j * stride + ch]);
      if (fabsf(x) < INFINITY) continue;
      if (WHOLE) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out) + ch;
        *o = __float2bfloat16_rn(__bfloat162float(*o) + x);
      } else {
        static_cast<float*>(out)[ch] += x;
      }
    }
  }
}

template <int D>
__device__ __forceinline__ void softmax_role(const AttendTc& t, Smem<D>& sm, int g) {
  using S = Smem<D>;
  const AttendShape& a = t.a;
  const int tid = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t lanes = sm.tmem + ((uint32_t)(tid >> 5) << 21);
  const uint32_t ts = lanes + kTmemS + 128 * g, to = lanes + kTmemO + 128 * g;
  const f32x2 sc2 = pack2(t.sc, t.sc);
  unsigned loads = 0, n_s = 0, n_o = 0, n_merge = 0;
  int rt, rh;                                    // the thread's row: token of the block, query head of the group
  if (!attend_row(a, tid, &rt, &rh)) rt = 1 << 20;
  auto say_most = [&] {
    tc_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.p_most[g]));
  };
  for (unsigned nth = 0;; ++nth) {
    bool ok = mbar_wait(smem_u32(&sm.unit_full[nth % kUnits]), (nth / kUnits) & 1, &sm.abort);
    if (!__all_sync(0xffffffffu, ok)) return;
    const AttendPiece p = sm.piece[nth % kUnits];
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.unit_empty[nth % kUnits]));
    if (p.stop) return;
    const Blocks b(t, p);
    const int tok0 = p.tok0 + (b.alt ? 0 : g * a.block_tokens), n_tok = min(a.block_tokens, p.n_seq_tok - tok0);
    const bool there = rt < n_tok;
    const int tok = tok0 + rt;
    const int bound = max(min(tok + 1 + p.shift, p.nk), 0);
    unsigned long long mask = 0;
    if (a.has_new && there) {
      mask = a.tree ? a.tree[(long long)p.s * a.n_tokens + tok] : ~0ull >> (63 - tok);
      mask &= ~0ull >> (64 - p.n_seq_tok);
    }
    const bool work = __any_sync(0xffffffffu, there);
    float m = -INFINITY, l = 0.0f;
    const int n = b.n[g];
    const int all = a.paged ? p.nk : min(tok0 + 1 + p.shift, p.nk);      // keys that every row sees
#pragma unroll 1
    for (int i = 0; i < n; ++i, ++n_s) {
      const int tl = b.tile(g, i), tile = p.tile0 + tl;
      const bool drafted = a.has_new && tile == p.n_all - 1, edge = drafted || (tile + 1) * kAttendTile > all;
      ok = mbar_wait(smem_u32(&sm.s_full[g]), n_s & 1, &sm.abort);
      if (!__all_sync(0xffffffffu, ok)) return;
      tc_fence_after();
      if (work) {
        uint32_t r[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_ld32(ts + 32 * q, r[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_wait_ld(r[q]);
        if (edge) {
          const int end = (a.paged ? p.nk : bound) - tile * kAttendTile;             // keys that the row sees
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t see = drafted ? (q < 2 ? (uint32_t)(mask >> (32 * q)) : 0u) : seen_below(end - 32 * q);
#pragma unroll
            for (int e = 0; e < 32; ++e) r[q][e] = see >> e & 1u ? r[q][e] : 0xff800000u;
          }
        }
        float mx[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          mx[q] = __uint_as_float(r[q][0]);
#pragma unroll
          for (int e = 1; e < 31; e += 2) mx[q] = fmaxf(fmaxf(mx[q], __uint_as_float(r[q][e])), __uint_as_float(r[q][e + 1]));
          mx[q] = fmaxf(mx[q], __uint_as_float(r[q][31]));
        }
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        if (i == 0) {
          m = top;
        } else {
          const bool lift = (top - m) * t.sc > kLift;      // m = -infinity: any score lifts it
          if (__any_sync(0xffffffffu, lift)) {
            // the product before this one is done: its commit lies in front of this tile's
            const float f = lift ? ex2((m - top) * t.sc) : 1.0f;
            if (lift) { m = top; l *= f; }
#pragma unroll 1
            for (int ch = 0; ch < D; ch += 32) {
              uint32_t o[32];
              tc_ld32(to + ch, o);
              tc_wait_ld(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tc_st32(to + ch, o);
            }
          }
        }
        // 2^(x - m sc) with one rounding of the difference, which is as large as m sc 2^-24: where that is much, differences first.  That
        // changes last bits, so rows that there are not, whose scores are what shared memory held, have no say in it.
        float base = m == -INFINITY ? 0.0f : m;
        if (__any_sync(0xffffffffu, there && fabsf(base) * t.sc > 0x1p20f)) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 32; ++e) r[q][e] = __float_as_uint(__uint_as_float(r[q][e]) - base);
          base = 0.0f;
        }
        const float nm = -base * t.sc;
        const f32x2 nm2 = pack2(nm, nm);
        f32x2 s0 = 0, s1 = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const f32x2 x0 = fma2(pack2(__uint_as_float(r[q][e]), __uint_as_float(r[q][e + 1])), sc2, nm2);
            const f32x2 x1 = fma2(pack2(__uint_as_float(r[q][e + 2]), __uint_as_float(r[q][e + 3])), sc2, nm2);
            const f32x2 p0 = ex2_pair(x0), p1 = ex2_pair(x1);
            s0 = add2(s0, p0);
            s1 = add2(s1, p1);
            w[e / 2] = bf16_pair(p0);
            w[e / 2 + 1] = bf16_pair(p1);
          }
          tc_st16(ts + 16 * q, w);
          if (q == 2 && !edge) say_most();       // three quarters of the product with V can begin
        }
        l += sum2(s0, s1);
      } else if (!edge) {
        say_most();
      }
      // Drafted rows are the first warpgroup's to clean, for both blocks.  Both would look through the same ones, and the one that comes
      // second find nothing, so that nothing orders what the other notes in front of its results; the first one's note lies in front of
      // both blocks' products, which are issued in this order.  In prompts no row of the first block sees what the second one cleans.
      const Columns c = edge && (b.alt || g == 0 || !drafted) ? columns(t, p, tile, tok0, n_tok) : Columns{0, 0, 0};
      if (c.all < c.used) {
        // The only wait on this barrier here, so phases before this one are passed over, and a parity tells this phase from the one before only if
        // that is done: load no - kStages of the ring has to have landed.  S of tile t is there, and its products were issued behind waits for
        // K's loads up to tile t and V's up to t - 1 (tiles in turn: t - 2) of the piece, and for all of earlier pieces.  The latest of which nothing
        // is known are, with tiles in turn, V of t - 1 and K of t + 1, the two loads in front of V of t.
        static_assert(S::kStages >= 3, "a ring shorter than what nobody here has waited for");
        const unsigned no = loads + b.v_load(tl, p.n), slot = no % S::kStages;
        ok = mbar_wait(smem_u32(&sm.kv_full[slot]), (no / S::kStages) & 1, &sm.abort);
        if (!__all_sync(0xffffffffu, ok)) return;
        if (clean_rows<D>(sm.kv[slot], c, tid)) *(volatile int*)&sm.odd[nth % kAhead] = (int)nth + 1;
        fence_async_smem();
      }
      if (edge) say_most();
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.p_ready[g]));
    }
    loads += 2 * p.n;
    // ---- results
    if (n > 0) {
      ok = mbar_wait(smem_u32(&sm.o_full[g]), n_o++ & 1, &sm.abort);
      if (!__all_sync(0xffffffffu, ok)) return;
      tc_fence_after();
    }
    const bool merge = b.alt && b.n[1] > 0;
    float f0 = 1.0f, f1 = 0.0f;                  // weights of the two warpgroups' sums
    int ch0 = 0, ch1 = D;
    uint32_t o_at = to;
    if (merge) {
      sm.ml[g][tid] = make_float2(m, l);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.merge_full));
      ok = mbar_wait(smem_u32(&sm.merge_full), n_merge & 1, &sm.abort);
      if (!__all_sync(0xffffffffu, ok)) return;
      tc_fence_after();
      const float2 x = sm.ml[0][tid], y = sm.ml[1][tid];
      m = fmaxf(x.x, y.x);
      f0 = x.y == 0.0f ? 0.0f : ex2((x.x - m) * t.sc);
      f1 = y.y == 0.0f ? 0.0f : ex2((y.x - m) * t.sc);
      l = x.y * f0 + y.y * f1;
      o_at = lanes + kTmemO;
      ch0 = g * (D / 2);
      ch1 = ch0 + D / 2;
    }
    if (work && !(b.alt && g == 1 && !merge)) {
      const bool whole = p.part < 0;
      const float inv = !whole ? 1.0f : l > 0.0f || l != l ? 1.0f / l : 0.0f;
      const long long place = (long long)(blockIdx.x * 2 + p.part) * a.part_rows + (b.alt ? 0 : g * 128) + tid;
      char* const dst = whole ? reinterpret_cast<char*>(static_cast<__nv_bfloat16*>(a.out) + (a.paged ? p.s * a.o_seq : p.q_row * a.o_tok) +
                                                        tok * a.o_tok + (p.h * a.G + rh) * a.o_head)
                              : reinterpret_cast<char*>(a.part + place * D);
#pragma unroll 1
      for (int ch = ch0; ch < ch1; ch += 32) {
        uint32_t o[32];
        if (n > 0 || merge) {
          tc_ld32(o_at + ch, o);
          tc_wait_ld(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0;
        }
        if (merge) {
          uint32_t r[32];
          tc_ld32(o_at + 128 + ch, r);
          tc_wait_ld(r);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint((__uint_as_float(o[e]) * f0 + __uint_as_float(r[e]) * f1));
        }
        if (there) {
          if (whole) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = bf16_pair(pack2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv));
            if (t.wide) {
              store32(dst + 2 * ch, w);
              store32(dst + 2 * ch + 32, w + 8);
            } else {
#pragma unroll
              for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(dst + 2 * ch + 2 * e * 2) = make_uint4(w[e], w[e + 1], w[e + 2], w[e + 3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 8) store32(dst + 4 * (ch + e), o + e);
          }
        }
        __syncwarp();                            // the next load is the whole warp's
      }
      if (there && *(volatile int*)&sm.odd[nth % kAhead] == (int)nth + 1) {
        if (whole) put_back<true>(t, p, bound, mask, ch0, ch1, dst);
        else put_back<false>(t, p, bound, mask, ch0, ch1, dst);
      }
      if (there && ch0 == 0) {
        if (whole) attend_lse(a, p.s, p.h * a.G + rh, tok, p.n_seq_tok, m * t.sc, l);
        else a.ml[place] = make_float2(m, l);
      }
      __syncwarp();
    }
    if (merge) {                                 // the other warpgroup's accumulator is read
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.merge_done));
      ok = mbar_wait(smem_u32(&sm.merge_done), n_merge++ & 1, &sm.abort);
      if (!__all_sync(0xffffffffu, ok)) return;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(const __grid_constant__ AttendTc t, const __grid_constant__ AttendMaps maps) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(raw);
  using S = Smem<D>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(smem_u32(&sm.unit_full[i]), 1);
      mbar_init(smem_u32(&sm.unit_empty[i]), 11);
    }
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(smem_u32(&sm.kv_full[i]), 1);
      mbar_init(smem_u32(&sm.kv_empty[i]), 1);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(smem_u32(&sm.q_full[g]), 1);
      mbar_init(smem_u32(&sm.q_empty[g]), 1);
      mbar_init(smem_u32(&sm.s_full[g]), 1);
      mbar_init(smem_u32(&sm.p_most[g]), 4);
      mbar_init(smem_u32(&sm.p_ready[g]), t.arrivals);
      mbar_init(smem_u32(&sm.o_full[g]), 1);
    }
    for (int i = 0; i < kAhead; ++i) sm.odd[i] = 0;
    mbar_init(smem_u32(&sm.merge_full), 8);
    mbar_init(smem_u32(&sm.merge_done), 8);
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
  if (warp == kLoadWarp && lane < 5) {
    const CUtensorMap* m = lane == 0 ? &maps.q : lane == 1 ? &maps.k : lane == 2 ? &maps.v : lane == 3 ? &maps.kn : &maps.vn;
    if (lane < 3 || t.a.has_new) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
  }
  pdl_launch_dependents();
  pdl_wait();
  attend_start(t.a, blockIdx.x, &sm.start);
  __syncthreads();
  if (warp >= 8) {
    regs_down<80>();
    if (warp == kLoadWarp) {
      load_role<D>(t, maps, sm);
    } else if (warp == kMmaWarp) {
      if (!mma_role<D>(t, sm) && elect_one()) {  // a wait ran out: what is under way ends first
        volatile int never = 0;
        tc_commit(smem_u32(&sm.drain));
        mbar_wait(smem_u32(&sm.drain), 0, &never);
      }
    } else if (warp == kQueryWarp) {
      if (lane == 0) query_role<D>(t, maps, sm);
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
  } else {
    regs_up<208>();
    softmax_role<D>(t, sm, warp >> 2);
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

// ---- host side --------------------------------------------------------------------------------------------------------
cudaError_t encode(CUtensorMap* m, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  return encode_tiled_bf16(m, base, rank, dims, strides, box) ? cudaSuccess : cudaErrorInvalidValue;
}

// Rows of head_dim by (head, token, sequence); the axis with the smaller stride of head and token comes first.
cudaError_t encode_rows(CUtensorMap* m, const void* base, int head_dim, long long heads, long long tokens, long long seqs, long long s_head,
                        long long s_tok, long long s_seq, int box_heads, int box_tokens, int* head_inner) {
  *head_inner = s_head <= s_tok;
  cuuint64_t dims[4] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)seqs};
  cuuint64_t strides[3] = {(cuuint64_t)s_head * 2, (cuuint64_t)s_tok * 2, (cuuint64_t)s_seq * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens, 1};
  if (!*head_inner) {
    dims[1] = (cuuint64_t)tokens; dims[2] = (cuuint64_t)heads;
    strides[0] = (cuuint64_t)s_tok * 2; strides[1] = (cuuint64_t)s_head * 2;
    box[1] = (cuuint32_t)box_tokens; box[2] = (cuuint32_t)box_heads;
  }
  return encode(m, base, 4, dims, strides, box);
}

template <int D>
cudaError_t launch(const AttendTc& t, const AttendMaps& maps, cudaStream_t st, int* launches) {
  static std::atomic<bool> allowed[16];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 16 || !allowed[dev].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(k_attend_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    if (dev < 16) allowed[dev].store(true, std::memory_order_relaxed);
  }
  LaunchScope scope(KID_ATTEND, st, launches);
  return launch_pdl(k_attend_tc<D>, dim3((unsigned)t.a.n_cta), dim3(kThreads), sizeof(Smem<D>), st, 1, t, maps);
}

}  // namespace

cudaError_t launch_attend_tensor(const AttendShape& a, cudaStream_t st, int* launches) {
  static_assert(sizeof(Smem<128>) <= kSmemLimit && sizeof(Smem<64>) <= kSmemLimit, "shared memory of a CTA");
  AttendTc t = {};
  AttendMaps m = {};
  t.a = a;
  t.sc = a.ml_unit;
  t.wide = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && a.o_tok % 16 == 0 && a.o_head % 16 == 0 && (!a.paged || a.o_seq % 16 == 0);
  t.arrivals = take_expire_next_copy_wait() ? 5 : 4;
  t.a.box_tokens = a.paged && a.n_tokens < a.block_tokens ? a.n_tokens : a.block_tokens;
  cudaError_t e = encode_rows(&m.q, a.q, a.head_dim, a.n_q_heads, a.paged ? a.n_tokens : a.rows_q, a.paged ? a.n_seqs : 1, a.q_head,
                              a.q_tok, a.paged ? a.q_seq : a.q_tok, a.G, a.box_tokens, &t.a.q_head_inner);
  if (e != cudaSuccess) return e;
  if (a.paged) {
    const cuuint64_t dims[3] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.rows_k, 1}, strides[2] = {(cuuint64_t)a.head_dim * 2, 16};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.page_rows, 1};
    e = encode(&m.k, a.k, 3, dims, strides, box);
    if (e == cudaSuccess) e = encode(&m.v, a.v, 3, dims, strides, box);
    if (a.has_new && e == cudaSuccess)
      e = encode_rows(&m.kn, a.k_new, a.head_dim, a.n_kv_heads, a.n_tokens, a.n_seqs, a.kn_head, a.kn_tok, a.kn_seq, 1, a.n_tokens, &t.kn_head_inner);
    if (a.has_new && e == cudaSuccess)
      e = encode_rows(&m.vn, a.v_new, a.head_dim, a.n_kv_heads, a.n_tokens, a.n_seqs, a.vn_head, a.vn_tok, a.vn_seq, 1, a.n_tokens, &t.vn_head_inner);
  } else {
    const struct { CUtensorMap* m; const void* base; long long head, tok; int* inner; } kv[2] = {
        {&m.k, a.k, a.k_head, a.k_tok, &t.k_head_inner}, {&m.v, a.v, a.v_head, a.v_tok, &t.v_head_inner}};
    for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
      const bool inner = *kv[i].inner = kv[i].head <= kv[i].tok;
      const cuuint64_t heads = (cuuint64_t)a.n_kv_heads, rows = (cuuint64_t)a.rows_k, sh = (cuuint64_t)kv[i].head * 2, st_ = (cuuint64_t)kv[i].tok * 2;
      const cuuint64_t dims[3] = {(cuuint64_t)a.head_dim, inner ? heads : rows, inner ? rows : heads}, strides[2] = {inner ? sh : st_, inner ? st_ : sh};
      const cuuint32_t box[3] = {64, inner ? 1u : (cuuint32_t)kAttendTile, inner ? (cuuint32_t)kAttendTile : 1u};
      e = encode(kv[i].m, kv[i].base, 3, dims, strides, box);
    }
  }
  if (e != cudaSuccess) return e;
  return a.head_dim == 128 ? launch<128>(t, m, st, launches) : launch<64>(t, m, st, launches);
}

}  // namespace slkv
