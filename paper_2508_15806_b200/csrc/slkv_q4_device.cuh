// The 4-bit cache: what its kernels share.  A record is one cached token of one KV head, both rows in 4 bits:
//   d/2 bytes K codes | d/2 bytes V codes | d/32 bf16 each of K scales, K zeros, V scales, V zeros
// Channel 32 j + i of a row stands for zero[j] + scale[j] * code.  The codes lie the way the attention kernel's matrix
// fragments want them, so that a lane takes all its codes of a row with one load:
//   K  32-bit word t * (d/32) + j: channels 32 j + 8 t + e in its nibbles e = 0 .. 7                (lane t of four)
//   V  16-bit unit g * (d/32) + j: channels 32 j + 4 g + e in its nibbles e = 0 .. 3                (lane g of eight)
// None of the kernels lets the next launch begin early, which would only wait: its CTAs take the places that come free first, so
// that their SMs have an uneven share of it (packing and unpacking 4636 rows 7.5 us against 5.8, one row in and one out for 128
// segments 12.0 against 10.2, attention to 8 short segments 7.7 against 7.4 and to 64 long ones, two launches, 98 against 92).
#pragma once
#include "slkv_internal.cuh"

namespace slkv {
namespace {

__host__ __device__ constexpr int q4_record_bytes(int head_dim) { return head_dim + head_dim / 4; }

// A segment's slots, whatever the device arrays hold: [begin, begin + room) lies inside the cache, len <= room.
struct Q4Segment { int begin, room, len; };
__device__ __forceinline__ Q4Segment q4_segment(const int32_t* starts, const int32_t* lens, int seg, long long capacity) {
  const long long b = starts[seg], e = starts[seg + 1];
  Q4Segment s;
  s.begin = (int)min(max(b, 0ll), capacity);
  s.room = (int)max(min(e, capacity) - s.begin, 0ll);
  s.len = min(max(lens[seg], 0), s.room);
  return s;
}

// The segment of row `row` in ascending `offsets` [n_seg + 1]: the last one that begins at or before it.  Whole warp.
__device__ __forceinline__ int q4_find(const int32_t* offsets, int n_seg, int row, int lane) {
  int lo = 0, n = n_seg;                                   // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) >> 5;
    const int probe = lo + lane * step;
    const unsigned at = __ballot_sync(0xffffffffu, lane * step < n && offsets[probe] <= row);
    const int k = at ? 31 - __clz(at) : 0;
    n = min(step, n - k * step);
    lo += k * step;
  }
  return lo;
}

}  // namespace
}  // namespace slkv
