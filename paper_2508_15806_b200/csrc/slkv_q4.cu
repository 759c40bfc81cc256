// Rows into and out of the 4-bit cache: whole packed layers, new tokens, and back.
//
// Quantisation of 32 channels x: zero = min x rounded down to bf16, scale = (max x - zero) / 15 rounded up to bf16, code = the
// fp32 quotient (x - zero) / scale rounded to an integer (ties to even).  With both roundings outwards the codes are in 0 .. 15 by
// themselves, and |x - value| <= scale / 2 up to fp32 rounding.  A group whose range is not finite becomes NaN throughout.
// Four lanes share a group, eight channels each: one 16-byte load (two for fp32), two exchanges for the range, one word of
// codes.  What bounds it: DRAM bytes (512 + 160 per row for bf16, head_dim 128) for many rows, one launch for few.
#include "slkv_q4_device.cuh"

namespace slkv {
namespace {

constexpr int kQ4Warps = 8;             // per CTA of the packing kernels

template <int HD>
struct Q4Lane {
  static constexpr int kLanes = HD / 8;                    // lanes per row, eight channels each
  static constexpr int kRows = 16 / kLanes;                // rows (K and V) a warp takes at once
  static constexpr int kGroups = HD / 32;
};

// Eight channels as they lie in memory: fp32, or bf16.
template <bool F32> struct Q4Raw { uint4 w[F32 ? 2 : 1]; };
template <bool F32>
__device__ __forceinline__ Q4Raw<F32> q4_load8(const void* p) {
  Q4Raw<F32> r;
  r.w[0] = __ldcs(static_cast<const uint4*>(p));           // read once
  if constexpr (F32) r.w[1] = __ldcs(static_cast<const uint4*>(p) + 1);
  return r;
}
template <bool F32>
__device__ __forceinline__ void q4_widen(const Q4Raw<F32>& r, float (&x)[8]) {
  const unsigned* w = reinterpret_cast<const unsigned*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = F32 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
}

// The lane's eight codes (nibble e: channel e), and the group's scale and zero as bf16 bits.
__device__ __forceinline__ unsigned q4_quantise(const float (&x)[8], unsigned& scale_bits, unsigned& zero_bits) {
  constexpr float kLargest = 3.4028234663852886e38f;
  float lo = x[0], hi = x[0], odd = 0.0f;                  // odd: NaN if there is an infinity or a NaN
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    odd = __fmaf_rn(x[i], 0.0f, odd);
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const unsigned lane = threadIdx.x & 31, all = __ballot_sync(0xffffffffu, odd == 0.0f);
  const float zero = __bfloat162float(__float2bfloat16_rd(lo)) + 0.0f;       // -0 as 0: which of the two comes out of a minimum is open
  const float span = hi - zero;
  const bool fine = ((all >> (lane & 28)) & 15u) == 15u && span <= kLargest;
  const __nv_bfloat16 sb = __float2bfloat16_ru(__fdiv_rn(span, 15.0f));
  const float scale = __bfloat162float(sb);
  scale_bits = fine ? __bfloat16_as_ushort(sb) : 0x7fffu;
  zero_bits = fine ? __float_as_uint(zero) >> 16 : 0x7fffu;
  // Quotients by the rounded reciprocal and one correction, which gives the correctly rounded quotient as long as nothing
  // leaves fp32's range (P. Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  Under
  // 1.5 * 2^23 a quotient's integer is in the low bits of the sum; eight of them are put together by multiplying with 16.
  const float magic = 12582912.0f;
  unsigned codes = 0;
  if (scale < 0x1p-100f) {                                 // the reciprocal would leave it
#pragma unroll
    for (int i = 7; i >= 0; --i) codes = codes * 16u + (scale > 0.0f ? __float_as_uint(__fdiv_rn(x[i] - zero, scale) + magic) & 15u : 0u);
  } else {
    const float r = __frcp_rn(scale);
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const float a = x[i] - zero, q = a * r;
      const float c = __fadd_rn(__fmaf_rn(__fmaf_rn(-q, scale, a), r, q), magic);
      codes = codes * 16u + __float_as_uint(c);
    }
    codes -= 0x3f400000u;                                  // what the eight 1.5 * 2^23 themselves come to
  }
  return fine ? codes : 0u;
}

// A warp quantises kRows tokens' K and V rows -- lanes 0 .. 15 K, 16 .. 31 V -- and writes their records.  `to` < 0: none.
template <int HD>
__device__ __forceinline__ void q4_store(const float (&x)[8], long long to, unsigned char* records, int lane) {
  using Q = Q4Lane<HD>;
  unsigned scale, zero;
  const unsigned codes = q4_quantise(x, scale, zero);
  const bool is_v = lane >= 16;
  const int l = lane % Q::kLanes, j = l >> 2, t = l & 3;
  // V: a lane's word is two units, of lanes g = 2 t and 2 t + 1; with the lane of the neighbouring group whole words come out
  const unsigned other = __shfl_xor_sync(0xffffffffu, j & 1 ? codes & 0xffffu : codes >> 16, 4);
  const unsigned v_word = j & 1 ? (other | (codes & 0xffff0000u)) : ((codes & 0xffffu) | (other << 16));
  if (to < 0) return;
  unsigned char* rec = records + to * q4_record_bytes(HD);
  const int word = is_v ? HD / 8 + (2 * t + (j & 1)) * (Q::kGroups / 2) + (j >> 1) : t * Q::kGroups + j;
  reinterpret_cast<unsigned*>(rec)[word] = is_v ? v_word : codes;
  if (t < 2)                                               // lane t = 0 of a group its scale, t = 1 its zero
    reinterpret_cast<unsigned short*>(rec + HD)[(is_v ? 2 * Q::kGroups : 0) + t * Q::kGroups + j] = (unsigned short)(t ? zero : scale);
}

struct Q4PackArgs {
  const void *k, *v;
  const int32_t *offsets, *kept_idx;
  Q4CacheView c;
  int32_t* status;
  long long n_rows;
  int chunk;                            // rows that a warp takes one after the other
};

constexpr int kChunkRows = 32;          // consecutive rows of a warp
constexpr int kAhead = 4;               // steps whose rows are loaded before the steps before them are done

template <int HD, bool F32>
__global__ void __launch_bounds__(kQ4Warps * 32) k_q4_pack(const __grid_constant__ Q4PackArgs a) {
  using Q = Q4Lane<HD>;
  constexpr int elem = F32 ? 4 : 2;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_seg = a.c.n_seg;
  // lengths: every segment's, whether it has rows or not
  for (int seg = blockIdx.x * blockDim.x + threadIdx.x; seg < n_seg; seg += gridDim.x * blockDim.x) {
    const int b = max(a.offsets[seg], 0), e = (int)min((long long)a.offsets[seg + 1], a.n_rows);
    const Q4Segment s = q4_segment(a.c.starts, a.c.starts, seg, a.c.capacity);
    const int n = max(e - b, 0);
    a.c.lens[seg] = min(n, s.room);
    if (a.status && (n > s.room || a.offsets[seg + 1] > a.n_rows)) *a.status = SLKV_ERR_CAPACITY;
  }
  const long long rows = min((long long)max(a.offsets[n_seg], 0), a.n_rows);
  const int sub = (lane & 15) / Q::kLanes, l = lane % Q::kLanes;
  const char* src = static_cast<const char*>(lane < 16 ? a.k : a.v) + l * 8 * elem;
  for (long long r0 = ((long long)blockIdx.x * kQ4Warps + warp) * a.chunk; r0 < rows; r0 += (long long)gridDim.x * kQ4Warps * a.chunk) {
    const int steps = (int)min((long long)(a.chunk / Q::kRows), (rows - r0 + Q::kRows - 1) / Q::kRows);
    auto load = [&](int i) { return q4_load8<F32>(src + min(r0 + i * Q::kRows + sub, rows - 1) * (HD * elem)); };
    Q4Raw<F32> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i] = load(min(i, steps - 1));
    // lane i finds row i's slot, and writes what the slot has beside the record
    int slot = -1;
    int seg = q4_find(a.offsets, n_seg, (int)r0, lane);
    if (lane < a.chunk && r0 + lane < rows) {
      const int r = (int)r0 + lane;
      const int pos = a.kept_idx[r];
      while (seg + 1 < n_seg && a.offsets[seg + 1] <= r) ++seg;
      const Q4Segment s = q4_segment(a.c.starts, a.c.starts, seg, a.c.capacity);
      const int at = r - max(a.offsets[seg], 0);
      if (at >= 0 && at < s.room) {
        slot = s.begin + at;
        a.c.pos[slot] = pos;
        if (a.c.weight) a.c.weight[slot] = 0.0f;
      }
    }
    for (int i0 = 0; i0 < steps; i0 += kAhead) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u;
        if (i >= steps) break;
        float x[8];
        q4_widen(raw[u], x);
        if (i + kAhead < steps) raw[u] = load(i + kAhead);
        q4_store<HD>(x, __shfl_sync(0xffffffffu, slot, i * Q::kRows + sub), a.c.records, lane);
      }
    }
  }
}

struct Q4AppendArgs {
  const void *k, *v;
  const int32_t* pos;
  Q4CacheView c;
  int32_t *lens_out, *status;
  long long k_seq, k_tok, k_head, v_seq, v_tok, v_head;     // bytes
  int n_tokens, n_kv_heads;
};

// One CTA per segment: its length is read by all of it before any of it writes the new one.
template <int HD, bool F32>
__global__ void __launch_bounds__(kQ4Warps * 32) k_q4_append(const __grid_constant__ Q4AppendArgs a) {
  using Q = Q4Lane<HD>;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const int seg = blockIdx.x, s = seg / a.n_kv_heads, h = seg - s * a.n_kv_heads;
  const Q4Segment at = q4_segment(a.c.starts, a.c.lens, seg, a.c.capacity);
  const int fit = min(a.n_tokens, at.room - at.len);
  const int sub = (lane & 15) / Q::kLanes, l = lane % Q::kLanes;
  const char* src = static_cast<const char*>(lane < 16 ? a.k : a.v) + s * (lane < 16 ? a.k_seq : a.v_seq) +
                    h * (lane < 16 ? a.k_head : a.v_head) + l * (F32 ? 32 : 16);
  const long long tok = lane < 16 ? a.k_tok : a.v_tok;
  for (int i0 = warp * Q::kRows; i0 < a.n_tokens; i0 += n_warps * Q::kRows) {
    const int i = i0 + sub;
    float x[8];
    q4_widen(q4_load8<F32>(src + min(i, a.n_tokens - 1) * tok), x);
    const long long to = i < fit ? (long long)at.begin + at.len + i : -1;
    q4_store<HD>(x, to, a.c.records, lane);
    if (to >= 0 && l == 0) {
      if (lane < 16) a.c.pos[to] = a.pos[(long long)s * a.n_tokens + i];
      else if (a.c.weight) a.c.weight[to] = 0.0f;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.lens_out[seg] = at.len + fit;
    if (fit < a.n_tokens && a.status) *a.status = SLKV_ERR_CAPACITY;
  }
}

struct Q4UnpackArgs {
  Q4CacheView c;
  const int32_t* slots;                  // null: every filled slot's row at its own place
  void *k_out, *v_out;
  long long n;
};

constexpr int kUnpackRows = 8;          // of a warp at once

template <int HD, bool F32>
__global__ void __launch_bounds__(kQ4Warps * 32, 5) k_q4_unpack(const __grid_constant__ Q4UnpackArgs a) {
  using Q = Q4Lane<HD>;
  constexpr int kSteps = kUnpackRows / Q::kRows;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool is_v = lane >= 16;
  const int sub = (lane & 15) / Q::kLanes, l = lane % Q::kLanes, j = l >> 2, t = l & 3;
  // K: the lane's word.  V: the word that has the lane's channels of its group and the neighbouring one
  const int word = is_v ? HD / 8 + (2 * t + (j & 1)) * (Q::kGroups / 2) + (j >> 1) : t * Q::kGroups + j;
  const int scale_at = HD + ((is_v ? 2 * Q::kGroups : 0) + j) * 2;
  char* dst = static_cast<char*>(is_v ? a.v_out : a.k_out) + l * 8 * (F32 ? 4 : 2);
  for (long long r0 = ((long long)blockIdx.x * kQ4Warps + warp) * kUnpackRows; r0 < a.n;
       r0 += (long long)gridDim.x * kQ4Warps * kUnpackRows) {
    // lane i < 8 finds row i's slot
    int slot = -1;
    if (a.slots) {
      if (lane < kUnpackRows && r0 + lane < a.n) slot = a.slots[r0 + lane];
      if (slot >= a.c.capacity) slot = -1;
    } else {
      int seg = q4_find(a.c.starts, a.c.n_seg, (int)r0, lane);
      const long long r = r0 + lane;
      if (lane < kUnpackRows && r < a.n) {
        while (seg + 1 < a.c.n_seg && a.c.starts[seg + 1] <= r) ++seg;
        const Q4Segment s = q4_segment(a.c.starts, a.c.lens, seg, a.c.capacity);
        if (r >= s.begin && r < (long long)s.begin + s.len) slot = (int)r;
      }
    }
    unsigned codes[kSteps], scale[kSteps], zero[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int from = __shfl_sync(0xffffffffu, slot, i * Q::kRows + sub);
      codes[i] = scale[i] = zero[i] = 0;
      if (from >= 0) {
        const unsigned char* rec = a.c.records + (long long)from * q4_record_bytes(HD);
        codes[i] = reinterpret_cast<const unsigned*>(rec)[word];
        scale[i] = *reinterpret_cast<const unsigned short*>(rec + scale_at);
        zero[i] = *reinterpret_cast<const unsigned short*>(rec + scale_at + 2 * Q::kGroups);
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const unsigned other = __shfl_xor_sync(0xffffffffu, j & 1 ? codes[i] & 0xffffu : codes[i] >> 16, 4);
      const unsigned mine = !is_v ? codes[i] : j & 1 ? (other | (codes[i] & 0xffff0000u)) : ((codes[i] & 0xffffu) | (other << 16));
      if (__shfl_sync(0xffffffffu, slot, i * Q::kRows + sub) < 0) continue;
      const float s = __uint_as_float(scale[i] << 16), z = __uint_as_float(zero[i] << 16);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)                          // a nibble under the exponent of 2^23 is 2^23 + c
        x[e] = __fmaf_rn(__uint_as_float(((mine >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f, s, z);
      char* o = dst + (r0 + i * Q::kRows + sub) * (HD * (F32 ? 4 : 2));
      if (F32) {
        __stcs(reinterpret_cast<float4*>(o), make_float4(x[0], x[1], x[2], x[3]));
        __stcs(reinterpret_cast<float4*>(o) + 1, make_float4(x[4], x[5], x[6], x[7]));
      } else {
        unsigned w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
          w[e] = *reinterpret_cast<const unsigned*>(&b);
        }
        __stcs(reinterpret_cast<uint4*>(o), make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

template <typename Args>
cudaError_t launch_rows(void (*kernel)(Args), long long n, int rows_per_warp, cudaStream_t st, const Args& a) {
  const long long ctas = (n + kQ4Warps * rows_per_warp - 1) / (kQ4Warps * rows_per_warp), most = (long long)sm_count() * 8;
  return launch_pdl(kernel, dim3((unsigned)(ctas < 1 ? 1 : ctas < most ? ctas : most)), dim3(kQ4Warps * 32), 0, st, 1, a);
}

}  // namespace

cudaError_t launch_q4_pack(const Q4CacheView& c, int head_dim, bool f32, const void* k, const void* v, long long n_rows,
                           const int32_t* offsets, const int32_t* kept_idx, int32_t* status, cudaStream_t st, int* launches) {
  // few rows: a warp takes no more than it loads at once, so that more of them share the work
  const int chunk = n_rows > (long long)sm_count() * kQ4Warps * kChunkRows ? kChunkRows : 8;
  const Q4PackArgs a = {k, v, offsets, kept_idx, c, status, n_rows, chunk};
  LaunchScope scope(KID_Q4_ROWS, st, launches);
  if (head_dim == 128) return launch_rows(f32 ? k_q4_pack<128, true> : k_q4_pack<128, false>, n_rows, chunk, st, a);
  return launch_rows(f32 ? k_q4_pack<64, true> : k_q4_pack<64, false>, n_rows, chunk, st, a);
}

cudaError_t launch_q4_append(const Q4CacheView& c, int n_kv_heads, int head_dim, bool f32, const void* k, const void* v, int n_tokens,
                             const int64_t (&stride)[6], const int32_t* pos, int32_t* lens_out, int32_t* status, cudaStream_t st,
                             int* launches) {
  const int e = f32 ? 4 : 2;
  const Q4AppendArgs a = {k, v, pos, c, lens_out, status, stride[0] * e, stride[1] * e, stride[2] * e,
                          stride[3] * e, stride[4] * e, stride[5] * e, n_tokens, n_kv_heads};
  const int rows = 128 / head_dim, warps = (n_tokens + rows - 1) / rows;
  const dim3 grid((unsigned)c.n_seg), block(32u * (unsigned)(warps < kQ4Warps ? warps : kQ4Warps));
  LaunchScope scope(KID_Q4_ROWS, st, launches);
  if (head_dim == 128) return launch_pdl(f32 ? k_q4_append<128, true> : k_q4_append<128, false>, grid, block, 0, st, 1, a);
  return launch_pdl(f32 ? k_q4_append<64, true> : k_q4_append<64, false>, grid, block, 0, st, 1, a);
}

cudaError_t launch_q4_unpack(const Q4CacheView& c, int head_dim, bool f32, const int32_t* slots, long long n, void* k_out,
                             void* v_out, cudaStream_t st, int* launches) {
  const Q4UnpackArgs a = {c, slots, k_out, v_out, n};
  LaunchScope scope(KID_Q4_ROWS, st, launches);
  if (head_dim == 128) return launch_rows(f32 ? k_q4_unpack<128, true> : k_q4_unpack<128, false>, n, kUnpackRows, st, a);
  return launch_rows(f32 ? k_q4_unpack<64, true> : k_q4_unpack<64, false>, n, kUnpackRows, st, a);
}

}  // namespace slkv
