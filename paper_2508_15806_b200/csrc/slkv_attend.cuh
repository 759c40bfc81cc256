// What the attention kernels of prompts and of paged caches share (slkv_attend_tc.cu, slkv_attend_f32.cu, slkv_attend_join.cu, slkv_attend_api.cu).
//
// Both are one problem: a unit is a block of query rows of one KV head -- some tokens times the G query heads that share its keys --
// against tiles of 128 keys.  What differs is where a tile lies and which of its keys a row sees:
//   prompt  keys are rows of the packed sequence; token i of nq sees the first i + 1 + nk - nq
//   paged   the segment's rows lie in pages and all tokens see them; one more tile holds the drafted tokens' own rows, of which
//           token i sees those whose bit is set in its mask
#pragma once

#include "slkv_internal.cuh"

namespace slkv {

constexpr int kAttendTileBits = 7, kAttendTile = 1 << kAttendTileBits;                 // keys of a tile, query rows of a block
constexpr int kF32TileBits = 6;                   // keys of a tile of fp32 rows: 64
constexpr int kMaxDrafted = 64;                  // drafted tokens of a sequence: the bits of a mask
constexpr int kMaxGroup = 64;                    // query heads of a KV head

// What the kernels need to know of a call.
struct AttendShape {
  int n_seqs, n_kv_heads, n_q_heads, G, head_dim;
  int block_tokens, unit_tokens, tile_bits;      // tokens of a block of query rows and of a unit (one or two blocks); log2 of a tile's keys
  int paged;
  // prompt
  const int32_t *cu_q, *cu_k;
  int window;                                    // rows of lse
  // paged
  const int32_t *tables, *lens;                  // of the layer
  int page_rows, max_pages, n_pages;
  int n_tokens;
  int has_new;
  const int32_t* n_new;                          // may be null: n_tokens
  const unsigned long long* tree;                // may be null: token i sees 0 .. i
  // tensors: q, out, drafted rows by (sequence, token, head); a prompt's sequence stride is not used
  const void *q, *k, *v, *k_new, *v_new;         // paged: k, v are the pools
  long long q_seq, q_tok, q_head, o_seq, o_tok, o_head, k_tok, k_head, v_tok, v_head, kn_seq, kn_tok, kn_head, vn_seq, vn_tok, vn_head;
  long long rows_q, rows_k;                      // that exist: of all sequences; paged: of the pool
  void* out;
  float* lse;                                    // may be null
  int32_t* status;                               // may be null
  float scale, lse_unit;                         // lse_unit: log2 units -> the caller's
  // how the units are shared out
  int spread;                                    // 1: whole units in turn, the longest first; 0: equal shares
  int whole;                                     // equal shares of whole units: nothing is joined; 2: all units count alike
  int n_cta;
  int levels;                                    // spread: blocks of the longest sequence
  // partial results of units that several CTAs share
  float* part;                                   // [n_cta][2][rows][head_dim]
  float2* ml;                                    // [n_cta][2][rows]
  float ml_unit;                                 // times a reference in ml: log2 units
  struct AttendPart* desc;                       // [n_cta][2]
  int part_rows, used_rows;                      // rows of a unit there is room for, and at most in use
  int q_head_inner, box_tokens;                  // how a block's rows lie: see attend_row; tokens of a block in shared memory
  int row_inverse;                               // 2^16 / G or 2^16 / box_tokens, rounded up: exact for rows below 128
};

size_t attend_workspace(int n_cta, int part_rows, int head_dim);
void attend_bind(AttendShape* a, void* workspace);
cudaError_t launch_attend_tensor(const AttendShape& a, cudaStream_t st, int* launches);
cudaError_t launch_attend_f32(const AttendShape& a, cudaStream_t st, int* launches);
cudaError_t launch_attend_join(const AttendShape& a, bool f32, cudaStream_t st, int* launches);

constexpr int kUnitCost = 3;                     // see AttendSchedule

#ifdef __CUDACC__
// A piece of a unit: its tiles tile0 .. tile0 + n - 1 of n_all.
struct AttendPiece {
  int s, h;
  int tok0, n_tok;               // the unit's tokens, of the sequence
  int n_seq_tok;                 // tokens of the sequence
  int nk;                        // keys: prompt: of the sequence, paged: rows of the segment
  int shift;                     // prompt: token i sees keys below i + 1 + shift
  int q_row, k_row;              // prompt: first rows of the sequence
  int tile0, n, n_all;
  int part;                      // -1: the unit's only piece; 0: one that does not begin it; 1: its first
  int stop;
};

// Row r of a unit: its token of the unit and its query head of the group; false: no row.  Rows come in blocks of 128; in a block the query heads of a token lie next to each other, or the tokens of a query head (q_head_inner = 0).
__device__ __forceinline__ bool attend_row(const AttendShape& a, int r, int* tok, int* head) {
  const int b = r >> 7, i = r & 127;
  const int quotient = i * a.row_inverse >> 16, rest = i - quotient * (a.q_head_inner ? a.G : a.box_tokens);
  const int rt = a.q_head_inner ? quotient : rest, rh = a.q_head_inner ? rest : quotient;
  *tok = b * a.block_tokens + rt;
  *head = rh;
  return rt < a.block_tokens && rh < a.G;
}
// The row's log-sum-exp m + log2(l), where the caller wants it.
__device__ __forceinline__ void attend_lse(const AttendShape& a, int s, int qh, int tok, int n_seq_tok, float m, float l) {
  if (!a.lse) return;
  const float lse = (l > 0.f || l != l ? m + log2f(l) : -INFINITY) * a.lse_unit;
  const long long row = (long long)s * a.n_q_heads + qh;
  if (a.paged) a.lse[row * a.n_tokens + tok] = lse;
  else if (tok >= n_seq_tok - a.window) a.lse[row * a.window + tok - (n_seq_tok - a.window)] = lse;
}

// Deals out the pieces of a launch; one warp runs it, every lane with the same results.
//   spread       whole units, to the CTAs in turn and back (0 .. n - 1, n - 1 .. 0, ..), the ones with the most tiles of their
//                sequence first: shares differ by about the last units, which are short, and CTAs that run beside each other read the
//                same keys
//   not spread   all units in one row, cut into equal shares: for few units.  A unit is as long as its tiles and kUnitCost more, which is
//                about what beginning and ending it costs beside them (units of one tile, 2000 tokens: a CTA with 15 of them took
//                119 us, one with a unit of 15 tiles 55).  Where shares are long, parts have two tiles or more;
//                with `whole`, through none: the unit is the share's that its middle lies in (whole = 2: no more units than CTAs, one each).
// The first piece is what a launch waits for, and most of that is instructions that come in for the first time: the threads of the CTA
// look for it together (attend_start), a few segments each, in little code.
__device__ __forceinline__ int attend_tokens(const AttendShape& a, int s) {
  if (!a.paged) return max(a.cu_q[s + 1] - a.cu_q[s], 0);
  return a.n_new ? min(max(a.n_new[s], 0), a.n_tokens) : a.n_tokens;
}
__device__ __forceinline__ int attend_blocks(const AttendShape& a, int tokens) {
  return tokens <= a.unit_tokens ? tokens > 0 : (int)((unsigned)(tokens + a.unit_tokens - 1) / (unsigned)a.unit_tokens);
}
__device__ __forceinline__ int attend_rows(const AttendShape& a, int seg) { return min(max(a.lens[seg], 0), a.max_pages * a.page_rows); }
// Tiles of a unit.
__device__ __forceinline__ int attend_prompt_tiles(const AttendShape& a, int nq, int nk, int t) {
  const int seen = min(nq, (t + 1) * a.unit_tokens) + nk - nq;
  return seen <= 0 ? 0 : (seen + (1 << a.tile_bits) - 1) >> a.tile_bits;
}
__device__ __forceinline__ int attend_paged_tiles(const AttendShape& a, int rows) {
  return ((rows + (1 << a.tile_bits) - 1) >> a.tile_bits) + a.has_new;
}
__device__ __forceinline__ int attend_length(const AttendShape& a, int tiles) { return a.whole == 2 ? 1 : tiles + kUnitCost; }
// How long all units of a segment (paged) or a sequence (prompt) are.
__device__ __forceinline__ int attend_weight(const AttendShape& a, int i) {
  if (a.paged)
    return attend_blocks(a, attend_tokens(a, (unsigned)i / (unsigned)a.n_kv_heads)) * attend_length(a, attend_paged_tiles(a, attend_rows(a, i)));
  const int nq = attend_tokens(a, i), nk = max(a.cu_k[i + 1] - a.cu_k[i], 0);
  int sum = 0;
  for (int t = 0; t * a.unit_tokens < nq; ++t) sum += attend_length(a, attend_prompt_tiles(a, nq, nk, t));
  return sum * a.n_kv_heads;
}
// Where a CTA's share begins.
struct AttendStart {
  int warp_sum[32];
  int total;
  int group, before;             // segment or sequence that the share begins in, what lies in front of it
};
// By all threads of a CTA, 32 times n_warps; two barriers inside, one left to the caller.
__device__ __forceinline__ void attend_start(const AttendShape& a, int cta, AttendStart* st) {
  if (a.spread) return;
  const int n = a.paged ? a.n_seqs * a.n_kv_heads : a.n_seqs;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const int per = (unsigned)n <= blockDim.x ? 1 : (int)((unsigned)(n + blockDim.x - 1) / blockDim.x);
  const int first = threadIdx.x * per, last = min(first + per, n);
  int sum = 0;
#pragma unroll 4
  for (int i = first; i < last; ++i) sum += attend_weight(a, i);
  int incl = sum;
#pragma unroll 1
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) st->warp_sum[warp] = incl;
  __syncthreads();
  int before = incl - sum, total = 0;
#pragma unroll 1
  for (int w = 0; w < n_warps; ++w) {
    const int x = st->warp_sum[w];
    if (w < warp) before += x;
    total += x;
  }
  if (threadIdx.x == 0) st->total = total;
  const int each = (unsigned)total / (unsigned)a.n_cta, more = total - each * a.n_cta, pos = each * cta + min(cta, more);
  if (pos >= before && pos < before + sum) {
    int i = first;
    for (;; ++i) {
      const int w = attend_weight(a, i);
      if (pos < before + w || i + 1 >= last) break;
      before += w;
    }
    st->group = i;
    st->before = before;
  }
}

class AttendSchedule {
 public:
  __device__ __forceinline__ AttendSchedule(const AttendShape& a, int cta, const AttendStart* st) : a_(a), cta_(cta), lane_(threadIdx.x & 31) {
    cached_ = !a_.paged && a_.n_seqs <= 32;
    if (cached_ && lane_ < a_.n_seqs) {
      q0_ = a_.cu_q[lane_];
      q1_ = a_.cu_q[lane_ + 1];
      k0_ = a_.cu_k[lane_];
      k1_ = a_.cu_k[lane_ + 1];
    }
    if (a_.spread) {
      item_ = cta;
      round_ = 0;
      level_ = a_.levels - 1;
      base_ = 0;
      count_ = level_count(level_);
      return;
    }
    // the first `more` shares are longer by one; where there is less than one for each CTA the last ones have none
    const int total = st->total;
    share_ = (unsigned)total / (unsigned)a_.n_cta;
    more_ = total - share_ * a_.n_cta;
    pos_ = share_ * cta + min(cta, more_);
    end_ = pos_ + share_ + (cta < more_);
    if (pos_ >= end_) return;
    group_ = st->before;
    s_ = st->group;
    x_ = 0;
    if (a_.paged) {
      const int seg = s_;
      s_ = (unsigned)seg / (unsigned)a_.n_kv_heads;
      x_ = seg - s_ * a_.n_kv_heads;
    }
    load_group();
  }
  __device__ __forceinline__ bool next(AttendPiece* p) { return a_.spread ? next_spread(p) : next_share(p); }
  // Of the piece at hand, one of several: how many pieces its unit has.  One more than there are shares that begin where it is cut.
  __device__ __forceinline__ int pieces() const {
    return 1 + cta_of(unit_ + each_ - least_part()) - cta_of(unit_ + kUnitCost + least_part() - 1);
  }

 private:
  const AttendShape& a_;
  int cta_, lane_;
  bool cached_ = false;          // prompts of up to 32 sequences: lane s has where sequence s lies
  int q0_ = 0, q1_ = 0, k0_ = 0, k1_ = 0;
  // spread
  long long item_, base_, count_;
  int level_, round_;
  int scan_s_ = 0, scan_before_ = 0;       // sequences looked through for this level; those of them that have such a block
  // shares: the group of units with the same tiles (prompt: a block of tokens, all KV heads; paged: a segment, all blocks)
  int pos_, end_, group_;        // group_: first position of the group
  int s_, x_;                    // sequence; prompt: block of tokens, paged: KV head
  int inner_, each_, tiles_, blocks_;      // units of the group, their length and tiles; blocks of the sequence
  int unit_;                     // first position of the unit at hand
  int share_, more_;

  __device__ __forceinline__ int least_part() const { return share_ < 8 ? 1 : 2; }     // tiles of a part
  __device__ __forceinline__ int cta_of(int pos) const {
    const int big = more_ * (share_ + 1);
    return pos < big ? pos / (share_ + 1) : more_ + (pos - big) / max(share_, 1);
  }
  // Of sequence s, the same in all lanes.
  __device__ __forceinline__ int first_query(int s) const { return cached_ ? __shfl_sync(0xffffffffu, q0_, s) : a_.cu_q[s]; }
  __device__ __forceinline__ int first_key(int s) const { return cached_ ? __shfl_sync(0xffffffffu, k0_, s) : a_.cu_k[s]; }
  __device__ __forceinline__ int seq_tokens(int s) const {
    return cached_ ? __shfl_sync(0xffffffffu, max(q1_ - q0_, 0), s) : attend_tokens(a_, s);
  }
  __device__ __forceinline__ int seq_keys(int s) const {
    return cached_ ? __shfl_sync(0xffffffffu, max(k1_ - k0_, 0), s) : max(a_.cu_k[s + 1] - a_.cu_k[s], 0);
  }
  // Of the sequence s0 + lane: its blocks.
  __device__ __forceinline__ int lane_blocks(int s0) const {
    if (s0 + lane_ >= a_.n_seqs) return 0;
    return attend_blocks(a_, cached_ ? max(q1_ - q0_, 0) : attend_tokens(a_, s0 + lane_));
  }

  // ---- spread
  __device__ __forceinline__ long long level_count(int t) const {
    int n = 0;
    for (int s0 = 0; s0 < a_.n_seqs; s0 += 32) {
      n += __popc(__ballot_sync(0xffffffffu, lane_blocks(s0) > t));
    }
    return (long long)n * a_.n_kv_heads;
  }
  __device__ __forceinline__ bool next_spread(AttendPiece* p) {
    while (level_ >= 0 && item_ >= base_ + count_) {
      base_ += count_;
      scan_s_ = scan_before_ = 0;
      if (--level_ >= 0) count_ = level_count(level_);
    }
    if (level_ < 0) return false;
    const unsigned rel = (unsigned)(item_ - base_);            // fewer than 2^31 sequences times heads
    const int nth = (int)(rel / (unsigned)a_.n_kv_heads);      // of the sequences that have such a block
    const int h = (int)(rel - (unsigned)nth * (unsigned)a_.n_kv_heads);
    int s = 0;
    for (; scan_s_ < a_.n_seqs; scan_s_ += 32) {               // on from where the last item was: items come in ascending order
      unsigned m = __ballot_sync(0xffffffffu, lane_blocks(scan_s_) > level_);
      const int n = __popc(m);
      if (nth < scan_before_ + n) {
        for (int skip = nth - scan_before_; skip > 0; --skip) m &= m - 1;
        s = scan_s_ + __ffs(m) - 1;
        break;
      }
      scan_before_ += n;
    }
    fill(p, s, h, level_);
    p->tile0 = 0;
    p->n = p->n_all;
    p->part = -1;
    ++round_;
    item_ = (long long)round_ * a_.n_cta + (round_ & 1 ? a_.n_cta - 1 - cta_ : cta_);
    return true;
  }

  // ---- equal shares
  __device__ __forceinline__ void load_group() {
    const int nq = seq_tokens(s_);
    blocks_ = attend_blocks(a_, nq);
    if (a_.paged) {
      inner_ = blocks_;
      tiles_ = attend_paged_tiles(a_, attend_rows(a_, s_ * a_.n_kv_heads + x_));
    } else {
      inner_ = x_ < blocks_ ? a_.n_kv_heads : 0;
      tiles_ = attend_prompt_tiles(a_, nq, seq_keys(s_), x_);
    }
    each_ = attend_length(a_, tiles_);
  }
  // Tiles of a unit of length each_ that lie in front of a cut at v.
  __device__ __forceinline__ int cut(int v) const {
    const int n = tiles_;
    if (v >= each_) return n;
    if (v <= 0) return 0;
    if (a_.whole) return 2 * v < each_ ? 0 : n;
    const int t = v - kUnitCost, least = least_part();
    return t < least ? 0 : t > n - least ? n : t;
  }
  __device__ __forceinline__ bool next_share(AttendPiece* p) {
    while (pos_ < end_) {
      while (pos_ >= group_ + inner_ * each_) {
        group_ += inner_ * each_;
        if (++x_ >= (a_.paged ? a_.n_kv_heads : blocks_)) { x_ = 0; ++s_; }
        if (s_ >= a_.n_seqs) return false;                     // lengths on the device that are not the host's
        load_group();
      }
      const int rel = pos_ - group_, unit = (unsigned)rel / (unsigned)each_, v0 = rel - unit * each_;
      const int v1 = min(each_, v0 + end_ - pos_), n = tiles_;
      const int tile0 = cut(v0), tile1 = cut(v1);
      unit_ = pos_ - v0;
      pos_ += v1 - v0;
      if (n == 0 ? v0 > 0 : tile0 == tile1) continue;
      if (a_.paged) fill(p, s_, x_, unit);
      else fill(p, s_, unit, x_);
      p->tile0 = tile0;
      p->n = tile1 - tile0;
      p->part = p->n == n ? -1 : (tile0 == 0 ? 1 : 0);
      return true;
    }
    return false;
  }
  __device__ __forceinline__ void fill(AttendPiece* p, int s, int h, int t) const {
    p->s = s;
    p->h = h;
    const int nq = seq_tokens(s);
    p->n_seq_tok = nq;
    p->tok0 = t * a_.unit_tokens;
    p->n_tok = min(a_.unit_tokens, nq - p->tok0);
    if (a_.paged) {
      p->nk = attend_rows(a_, s * a_.n_kv_heads + h);
      p->shift = p->q_row = p->k_row = 0;
      p->n_all = attend_paged_tiles(a_, p->nk);
    } else {
      p->nk = seq_keys(s);
      p->shift = p->nk - nq;
      p->q_row = first_query(s);
      p->k_row = first_key(s);
      p->n_all = attend_prompt_tiles(a_, nq, p->nk, t);
    }
    p->stop = 0;
  }
};
// What the joining launch needs to know of a CTA's pieces: state 0: none, 1: a piece, -1: one that failed; of a unit's first piece
// all the rest.
struct AttendPart {
  int state, pieces, s, h, tok0, n_tok, n_seq_tok, q_row;
};
__device__ __forceinline__ void attend_note(const AttendShape& a, int slot, const AttendPiece& p, int pieces) {
  int4* to = reinterpret_cast<int4*>(a.desc + 2 * blockIdx.x + slot);
  to[0] = make_int4(1, pieces, p.s, p.h);
  to[1] = make_int4(p.tok0, p.n_tok, p.n_seq_tok, p.q_row);
}
#endif

}  // namespace slkv
