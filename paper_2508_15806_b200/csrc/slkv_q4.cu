// Rows into and out of the 4-bit cache: whole packed layers, new tokens, and back.
//
// Quantisation of 32 channels x: zero = min x rounded down to bf16, scale = (max x - zero) / 15 rounded up to bf16, code = the
// fp32 quotient (x - zero) / scale rounded to an integer (ties to even).  With both roundings outwards the codes are in 0 .. 15 by
// themselves, and |x - value| <= scale / 2 up to fp32 rounding.  A group whose range is not finite becomes NaN throughout.
// A lane takes a whole group when it packs: 64 bytes in (128 for fp32), four words of codes out, which the lanes of a row exchange
// so that each writes 16 bytes of the record.  (With eight channels to a lane, range, scale and reciprocal of a group were
// worked out four times: 171 instructions per row, and 157 us for 744k rows where this takes 92.)
// What bounds it: DRAM bytes (512 + 160 per row for bf16, head_dim 128) for many rows, one launch for few.
#include "slkv_q4_device.cuh"

namespace slkv {
namespace {

constexpr int kQ4Warps = 8;             // per CTA of the packing kernels

// A group of 32 channels as it lies in memory: fp32, or bf16.
template <bool F32> struct Q4Raw { uint4 w[F32 ? 8 : 4]; };
template <bool F32>
__device__ __forceinline__ Q4Raw<F32> q4_load(const void* p) {
  Q4Raw<F32> r;
#pragma unroll
  for (int i = 0; i < (F32 ? 8 : 4); ++i) r.w[i] = static_cast<const uint4*>(p)[i];
  return r;
}
// Channel i.
template <bool F32>
__device__ __forceinline__ float q4_channel(const Q4Raw<F32>& r, int i) {
  const unsigned* w = reinterpret_cast<const unsigned*>(&r);
  return F32 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
}

// Minimum and maximum that a NaN passes through, of numbers or of the numbers' halves.
__device__ __forceinline__ float least(float a, float b) { float y; asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float most(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ unsigned least2(unsigned a, unsigned b) { unsigned y; asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b)); return y; }
__device__ __forceinline__ unsigned most2(unsigned a, unsigned b) { unsigned y; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b)); return y; }

// a / b rounded correctly, from r, the rounded reciprocal of b (P. Markstein, Computation of elementary functions on the IBM RISC
// System/6000 processor, 1990), as long as nothing leaves fp32's range.
__device__ __forceinline__ float quotient(float a, float b, float r) {
  const float q = a * r;
  return __fmaf_rn(__fmaf_rn(-q, b, a), r, q);
}

// The codes of a group, eight channels to a word (nibble e: channel e), and its scale and zero as bf16 bits, zero above.
template <bool F32>
__device__ __forceinline__ void q4_quantise(const Q4Raw<F32>& raw, unsigned (&codes)[4], unsigned& scale_zero) {
  constexpr float kLargest = 3.4028234663852886e38f;
  float lo, hi;
  if constexpr (F32) {
    lo = hi = q4_channel(raw, 0);
#pragma unroll
    for (int i = 1; i < 32; ++i) { lo = least(lo, q4_channel(raw, i)); hi = most(hi, q4_channel(raw, i)); }
  } else {
    const unsigned* w = reinterpret_cast<const unsigned*>(&raw);
    unsigned a = w[0], b = w[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) { a = least2(a, w[i]); b = most2(b, w[i]); }
    lo = least(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    hi = most(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
  }
  const float zero = __bfloat162float(__float2bfloat16_rd(lo)) + 0.0f;       // -0 as 0: which of the two comes out of a minimum is open
  const float span = hi - zero;
  const bool fine = span <= kLargest;                      // not if there is a NaN or an infinity
  // Under 1.5 * 2^23 a quotient's integer is in the low bits of the sum; eight of them are put together by multiplying with 16.
  const float magic = 12582912.0f;
  unsigned scale16;
  if (span >= 0x1p-100f) {
    const __nv_bfloat16 sb = __float2bfloat16_ru(quotient(span, 15.0f, 1.0f / 15.0f));
    const float scale = __bfloat162float(sb), r = __frcp_rn(scale);
    scale16 = __bfloat16_as_ushort(sb);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      unsigned c = 0;
#pragma unroll
      for (int e = 7; e >= 0; --e) c = c * 16u + __float_as_uint(__fadd_rn(quotient(q4_channel(raw, 8 * t + e) - zero, scale, r), magic));
      codes[t] = fine ? c - 0x3f400000u : 0u;              // less what the eight 1.5 * 2^23 themselves come to
    }
  } else {                                                 // quotients and reciprocals would leave it; zeros, and what is not fine
    const __nv_bfloat16 sb = __float2bfloat16_ru(__fdiv_rn(span, 15.0f));
    const float scale = __bfloat162float(sb);
    scale16 = __bfloat16_as_ushort(sb);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      codes[t] = 0;
      if (scale > 0.0f)
#pragma unroll
        for (int e = 7; e >= 0; --e) codes[t] = codes[t] * 16u + (__float_as_uint(__fdiv_rn(q4_channel(raw, 8 * t + e) - zero, scale) + magic) & 15u);
    }
  }
  scale_zero = fine ? scale16 | (__float_as_uint(zero) & 0xffff0000u) : 0x7fff7fffu;
}

// The lanes of a warp take tokens one after the other, a token's K groups first, then its V groups.
template <int HD>
struct Q4Lane {
  static constexpr int kGroups = HD / 32;                  // of a row
  static constexpr int kRows = 32 / (2 * kGroups);         // tokens of a warp
  __device__ static int token(int lane) { return lane / (2 * kGroups); }
  __device__ static bool is_v(int lane) { return lane & kGroups; }
  __device__ static int group(int lane) { return lane & (kGroups - 1); }
};

// A warp quantises kRows tokens' K and V rows and writes their records.  `to`: the slot of the lane's token, < 0: none.
template <int HD, bool F32>
__device__ __forceinline__ void q4_store(const Q4Raw<F32>& raw, int to, unsigned char* records, int lane) {
  using Q = Q4Lane<HD>;
  unsigned w[4], sz;
  q4_quantise(raw, w, sz);
  const int j = Q::group(lane);
  const bool is_v = Q::is_v(lane);
  // words of the lanes j of a row: [lane][word] -> [word][lane], two lanes at a time
  {
    const bool odd = j & 1;
    const unsigned x = __shfl_xor_sync(0xffffffffu, odd ? w[0] : w[1], 1), y = __shfl_xor_sync(0xffffffffu, odd ? w[2] : w[3], 1);
    if (odd) { w[0] = x; w[2] = y; } else { w[1] = x; w[3] = y; }
  }
  if constexpr (Q::kGroups == 4) {
    const bool up = j & 2;
    const unsigned x = __shfl_xor_sync(0xffffffffu, up ? w[0] : w[2], 2), y = __shfl_xor_sync(0xffffffffu, up ? w[1] : w[3], 2);
    if (up) { w[0] = x; w[1] = y; } else { w[2] = x; w[3] = y; }
  }
  // HD 128: lane j has the words j of groups 0 .. 3.  HD 64: lane 0 the words 0 and 2 of both groups, lane 1 words 1 and 3.
  if constexpr (Q::kGroups == 2) {                         // to words 0 and 1, words 2 and 3
    const unsigned x = __shfl_xor_sync(0xffffffffu, j ? w[0] : w[2], 1), y = __shfl_xor_sync(0xffffffffu, j ? w[1] : w[3], 1);
    if (j) { w[0] = x; w[1] = y; } else { w[2] = x; w[3] = y; }
  }
  uint4 out = make_uint4(w[0], w[1], w[2], w[3]);          // K: as it is
  if (is_v) {                                              // V: units of 16 bits, group after group
    if constexpr (Q::kGroups == 4)
      out = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
    else
      out = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[2], w[3], 0x7632));
  }
  // scales and zeros: the even lane of a pair writes both scales, the odd one both zeros
  const unsigned other = __shfl_xor_sync(0xffffffffu, sz, 1);
  const unsigned pair = j & 1 ? __byte_perm(other, sz, 0x7632) : __byte_perm(sz, other, 0x5410);
  if (to < 0) return;
  unsigned char* rec = records + (long long)to * q4_record_bytes(HD);
  *reinterpret_cast<uint4*>(rec + (is_v ? HD / 2 : 0) + 16 * j) = out;
  reinterpret_cast<unsigned*>(rec + HD)[((is_v ? 2 : 0) + (j & 1)) * (Q::kGroups / 2) + (j >> 1)] = pair;
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

template <int HD, bool F32>
__global__ void __launch_bounds__(kQ4Warps * 32) k_q4_pack(const __grid_constant__ Q4PackArgs a) {
  using Q = Q4Lane<HD>;
  constexpr int elem = F32 ? 4 : 2;
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
  const int token = Q::token(lane);
  const char* src = static_cast<const char*>(Q::is_v(lane) ? a.v : a.k) + Q::group(lane) * 32 * elem;
  for (long long r0 = ((long long)blockIdx.x * kQ4Warps + warp) * a.chunk; r0 < rows; r0 += (long long)gridDim.x * kQ4Warps * a.chunk) {
    const int n = (int)min((long long)a.chunk, rows - r0);
    auto load = [&](int i) { return q4_load<F32>(src + (r0 + min(i + token, n - 1)) * (HD * elem)); };
    Q4Raw<F32> next = load(0);
    // lane i finds row i's slot, and writes what the slot has beside the record
    int slot = -1;
    int seg = q4_find(a.offsets, n_seg, (int)r0, lane);
    if (lane < n) {
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
    for (int i = 0; i < n; i += Q::kRows) {
      const Q4Raw<F32> now = next;
      if (i + Q::kRows < n) next = load(i + Q::kRows);
      const int to = __shfl_sync(0xffffffffu, slot, (i + token) & 31);
      q4_store<HD>(now, i + token < n ? to : -1, a.c.records, lane);
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
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const int seg = blockIdx.x, s = seg / a.n_kv_heads, h = seg - s * a.n_kv_heads;
  const Q4Segment at = q4_segment(a.c.starts, a.c.lens, seg, a.c.capacity);
  const int fit = min(a.n_tokens, at.room - at.len);
  const bool is_v = Q::is_v(lane);
  const int token = Q::token(lane);
  const char* src = static_cast<const char*>(is_v ? a.v : a.k) + s * (is_v ? a.v_seq : a.k_seq) + h * (is_v ? a.v_head : a.k_head) +
                    Q::group(lane) * (F32 ? 128 : 64);
  const long long tok = is_v ? a.v_tok : a.k_tok;
  for (int i0 = warp * Q::kRows; i0 < a.n_tokens; i0 += n_warps * Q::kRows) {
    const int i = i0 + token;
    const Q4Raw<F32> x = q4_load<F32>(src + min(i, a.n_tokens - 1) * tok);
    const int to = i < fit ? at.begin + at.len + i : -1;
    q4_store<HD>(x, to, a.c.records, lane);
    if (to >= 0 && Q::group(lane) == 0) {
      if (!is_v) a.c.pos[to] = a.pos[(long long)s * a.n_tokens + i];
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

__device__ __forceinline__ unsigned sub2(unsigned a, unsigned b) {
  const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const unsigned*>(&y);
}
__device__ __forceinline__ unsigned fma2(unsigned a, unsigned b, unsigned c) {
  unsigned y;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(y) : "r"(a), "r"(b), "r"(c));
  return y;
}

template <int HD, bool F32>
__global__ void __launch_bounds__(kQ4Warps * 32, 4) k_q4_unpack(const __grid_constant__ Q4UnpackArgs a) {
  // K in lanes 0 .. 15, V in 16 .. 31, eight channels to a lane
  constexpr int kGroups = HD / 32, kLanes = HD / 8, kRows = 16 / kLanes, kSteps = kUnpackRows / kRows;
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool is_v = lane >= 16;
  const int sub = (lane & 15) / kLanes, l = lane % kLanes, j = l >> 2, t = l & 3;
  // K: the lane's word.  V: the word that has the lane's channels of its group and the neighbouring one
  const int word = is_v ? HD / 8 + (2 * t + (j & 1)) * (kGroups / 2) + (j >> 1) : t * kGroups + j;
  const int scale_at = HD + ((is_v ? 2 * kGroups : 0) + j) * 2;
  char* dst = static_cast<char*>(is_v ? a.v_out : a.k_out) + l * 8 * (F32 ? 4 : 2);
  // lane i < 8 finds row i's slot, a step ahead where slots are given
  const long long step = (long long)gridDim.x * kQ4Warps * kUnpackRows;
  auto given = [&](long long r0) { return a.slots && lane < kUnpackRows && r0 + lane < a.n ? a.slots[r0 + lane] : -1; };
  long long r0 = ((long long)blockIdx.x * kQ4Warps + warp) * kUnpackRows;
  int ahead = given(r0);
  for (; r0 < a.n; r0 += step) {
    int slot = ahead < a.c.capacity ? ahead : -1;
    ahead = given(r0 + step);
    if (!a.slots) {
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
      const int from = __shfl_sync(0xffffffffu, slot, i * kRows + sub);
      // a lane without a slot reads the first one's: loads under a condition are not issued together
      const unsigned char* rec = a.c.records + (long long)max(from, 0) * q4_record_bytes(HD);
      codes[i] = reinterpret_cast<const unsigned*>(rec)[word];
      scale[i] = *reinterpret_cast<const unsigned short*>(rec + scale_at);
      zero[i] = *reinterpret_cast<const unsigned short*>(rec + scale_at + 2 * kGroups);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const unsigned other = __shfl_xor_sync(0xffffffffu, j & 1 ? codes[i] & 0xffffu : codes[i] >> 16, 4);
      const unsigned mine = !is_v ? codes[i] : j & 1 ? (other | (codes[i] & 0xffff0000u)) : ((codes[i] & 0xffffu) | (other << 16));
      if (__shfl_sync(0xffffffffu, slot, i * kRows + sub) < 0) continue;
      char* o = dst + (r0 + i * kRows + sub) * (HD * (F32 ? 4 : 2));
      if constexpr (F32) {
        const float s = __uint_as_float(scale[i] << 16), z = __uint_as_float(zero[i] << 16);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)                        // a nibble under the exponent of 2^23 is 2^23 + c
          x[e] = __fmaf_rn(__uint_as_float(((mine >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f, s, z);
        __stcs(reinterpret_cast<float4*>(o), make_float4(x[0], x[1], x[2], x[3]));
        __stcs(reinterpret_cast<float4*>(o) + 1, make_float4(x[4], x[5], x[6], x[7]));
      } else {
        // two channels at a time: under the exponent of 128 a nibble is 128 + c; one packed multiply-add, rounded once
        const unsigned s = scale[i] * 0x10001u, z = zero[i] * 0x10001u, odd = mine >> 4;
        unsigned w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned u = (__byte_perm(mine, odd, e | (4 + e) << 8) & 0x000f000fu) | 0x43004300u;
          w[e] = fma2(sub2(u, 0x43004300u), s, z);
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
  const int rows = 512 / head_dim, warps = (n_tokens + rows - 1) / rows;
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
