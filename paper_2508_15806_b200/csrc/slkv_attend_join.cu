// Joins the pieces of units that several CTAs share, for both kinds of rows, and lays out the workspace.
#include "slkv_attend.cuh"

namespace slkv {
namespace {

__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One CTA's unit that goes on in the next ones: the pieces' outputs by their references.  What bounds it is latency -- what the pieces are,
// then their references, sums and outputs, kAtOnce pieces at a time, then the result -- so nothing else stands between the loads.  A row is
// a warp's; where the rows are few (tokens that decode over long segments, many pieces), the eight warps of a CTA share its pieces: one user
// over 8000 rows 25.9 us without, 17.0 with it.  The launch takes 5 us by itself, 1 to 2 behind the other one, 12 where four chunks of
// 512 tokens leave 256 rows a unit (39 MB of pieces).
constexpr int kJoinWarps = 8, kAtOnce = 4;
constexpr int kFewRows = 16;
template <int D, bool F32, int SHARE>                          // SHARE: warps of a row
__global__ void __launch_bounds__(kJoinWarps * 32) k_attend_join(const __grid_constant__ AttendShape a) {
  pdl_launch_dependents();
  constexpr int V = D / 32, kRows = kJoinWarps / SHARE;
  const int cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.y * kRows + warp / SHARE, first = warp % SHARE;
  int tok, hh;
  const bool row = attend_row(a, r, &tok, &hh);
  pdl_wait();
  const int4* note = reinterpret_cast<const int4*>(a.desc + 2 * cta + 1);
  const int4 x0 = note[0], x1 = note[1];
  if (x0.x != 1) return;
  const int n = x0.y, s = x0.z, h = x0.w, tok0 = x1.x, n_tok = x1.y, n_seq_tok = x1.z, q_row = x1.w;
  float acc[V], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) acc[e] = 0.f;
  bool failed = false;
  if (row && tok < n_tok) {
    for (int i0 = first; i0 < n; i0 += SHARE * kAtOnce) {
      float2 x[kAtOnce];
      float o[kAtOnce][V];
      int state[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int i = min(i0 + SHARE * k, n - 1), slot = i == 0 ? 2 * cta + 1 : 2 * (cta + i);
        const long long at = (long long)slot * a.part_rows + r;
        x[k] = a.ml[at];
        state[k] = a.desc[slot].state;
#pragma unroll
        for (int e = 0; e < V; e += 2) *reinterpret_cast<float2*>(o[k] + e) = *reinterpret_cast<const float2*>(a.part + at * D + V * lane + e);
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, x[k].x);
      const float f0 = m == -INFINITY ? 0.f : exp2_of((m - top) * a.ml_unit);
      m = top;
      l *= f0;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] *= f0;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const bool there = i0 + SHARE * k < n, some = there && x[k].y != 0.f;      // else nothing is seen there; outputs may not be written
        failed |= there && state[k] != 1;
        const float f = some ? exp2_of((x[k].x - m) * a.ml_unit) : 0.f;
        l = some ? fmaf(x[k].y, f, l) : l;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = some ? fmaf(o[k][e], f, acc[e]) : acc[e];
      }
    }
  }
  if (SHARE > 1) {
    __shared__ float2 ml[kJoinWarps];
    __shared__ float out[kJoinWarps][D];
    if (lane == 0) ml[warp] = make_float2(m, failed ? __int_as_float(0x7fffffff) : l);
#pragma unroll
    for (int e = 0; e < V; ++e) out[warp][V * lane + e] = acc[e];
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int w = 0; w < SHARE; ++w) m = fmaxf(m, ml[w].x);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < SHARE; ++w) {
      const float f = ml[w].y == 0.f ? 0.f : exp2_of((ml[w].x - m) * a.ml_unit);
      l = ml[w].y == 0.f ? l : fmaf(ml[w].y, f, l);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = ml[w].y == 0.f ? acc[e] : fmaf(out[w][V * lane + e], f, acc[e]);
    }
  }
  if (!row || tok >= n_tok) return;
  tok += tok0;
  float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (failed) inv = l = __int_as_float(0x7fffffff);
  const int qh = h * a.G + hh;
  const long long at = (a.paged ? s * a.o_seq : q_row * a.o_tok) + tok * a.o_tok + qh * a.o_head + V * lane;
#pragma unroll
  for (int e = 0; e < V; e += 2) {
    if (F32) *reinterpret_cast<float2*>(static_cast<float*>(a.out) + at + e) = make_float2(acc[e] * inv, acc[e + 1] * inv);
    else *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at + e) = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
  }
  if (lane == 0) attend_lse(a, s, qh, tok, n_seq_tok, m * a.ml_unit, l);
}

template <int D, bool F32>
cudaError_t launch_join(const AttendShape& a, cudaStream_t st) {
  const dim3 block(kJoinWarps * 32);
  if (a.used_rows <= kFewRows) return launch_pdl(k_attend_join<D, F32, kJoinWarps>, dim3((unsigned)(a.n_cta - 1), (unsigned)a.used_rows), block, 0, st, 1, a);
  return launch_pdl(k_attend_join<D, F32, 1>, dim3((unsigned)(a.n_cta - 1), (unsigned)((a.used_rows + kJoinWarps - 1) / kJoinWarps)), block, 0, st, 1, a);
}

}  // namespace

cudaError_t launch_attend_join(const AttendShape& a, bool f32, cudaStream_t st, int* launches) {
  if (a.spread || a.whole || a.n_cta < 2) return cudaSuccess;
  LaunchScope scope(KID_ATTEND_JOIN, st, launches);
  if (a.head_dim == 128) return f32 ? launch_join<128, true>(a, st) : launch_join<128, false>(a, st);
  return f32 ? launch_join<64, true>(a, st) : launch_join<64, false>(a, st);
}

// Workspace: outputs of pieces, their references and sums, what they belong to, each from a 256-byte boundary: outputs are written 32 bytes at a
// time.  A caller's workspace begins at any 16-byte boundary, so there is room for the way to the first of them.
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
size_t attend_workspace(int n_cta, int part_rows, int head_dim) {
  const size_t places = 2 * (size_t)n_cta * part_rows;
  return 256 + up256(places * head_dim * sizeof(float)) + up256(places * sizeof(float2)) + up256(2 * n_cta * sizeof(AttendPart));
}
void attend_bind(AttendShape* a, void* workspace) {
  const size_t places = 2 * (size_t)a->n_cta * a->part_rows;
  char* w = reinterpret_cast<char*>(up256(reinterpret_cast<uintptr_t>(workspace)));
  a->part = reinterpret_cast<float*>(w);
  w += up256(places * a->head_dim * sizeof(float));
  a->ml = reinterpret_cast<float2*>(w);
  w += up256(places * sizeof(float2));
  a->desc = reinterpret_cast<AttendPart*>(w);
}

}  // namespace slkv
