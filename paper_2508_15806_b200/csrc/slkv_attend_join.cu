// Joins the pieces of units that several CTAs share, for both kinds of rows, and lays out the workspace.
#include "slkv_attend.cuh"

namespace slkv {
namespace {

__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One CTA's unit that goes on in the next ones: the pieces' outputs by their references, a warp a row.  What bounds it is latency: what
// the pieces are, then their references and outputs, all at once.
constexpr int kJoinWarps = 8, kJoinRows = 16;    // rows of a block
template <int D, bool F32>
__global__ void __launch_bounds__(kJoinWarps * 32) k_attend_join(const __grid_constant__ AttendShape a) {
  pdl_launch_dependents();
  pdl_wait();
  const int cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int4* note = reinterpret_cast<const int4*>(a.desc + 2 * cta + 1);
  const int4 x0 = note[0], x1 = note[1];
  if (x0.x != 1) return;
  const int n = x0.y, s = x0.z, h = x0.w, tok0 = x1.x, n_tok = x1.y, n_seq_tok = x1.z, q_row = x1.w;
  constexpr int V = D / 32;
  for (int r = blockIdx.y * kJoinRows + warp; r < (blockIdx.y + 1) * kJoinRows && r < a.part_rows; r += kJoinWarps) {
    int tok, hh;
    if (!attend_row(a, r, &tok, &hh) || tok >= n_tok) continue;
    tok += tok0;
    auto place = [&](int i) { return (long long)(i == 0 ? 2 * cta + 1 : 2 * (cta + i)) * a.part_rows + r; };
    float m = -INFINITY;
    bool failed = false;
    for (int i = lane; i < n; i += 32) {
      m = fmaxf(m, a.ml[place(i)].x);
      failed |= i > 0 && a.desc[2 * (cta + i)].state != 1;
    }
    failed = __any_sync(0xffffffffu, failed);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float acc[V], l = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const float2 x = a.ml[place(i)];
      float o[V];
#pragma unroll
      for (int e = 0; e < V; e += 2) *reinterpret_cast<float2*>(o + e) = *reinterpret_cast<const float2*>(a.part + place(i) * D + V * lane + e);
      const bool some = x.y != 0.f;              // else nothing is seen there, and outputs may not have been computed
      const float f = some ? exp2_of((x.x - m) * a.ml_unit) : 0.f;
      l = fmaf(x.y, f, l);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = some ? fmaf(o[e], f, acc[e]) : acc[e];
    }
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
}

}  // namespace

cudaError_t launch_attend_join(const AttendShape& a, bool f32, cudaStream_t st, int* launches) {
  if (a.spread || a.whole || a.n_cta < 2) return cudaSuccess;
  LaunchScope scope(KID_ATTEND_JOIN, st, launches);
  const dim3 grid((unsigned)(a.n_cta - 1), (unsigned)((a.used_rows + kJoinRows - 1) / kJoinRows)), block(kJoinWarps * 32);
  if (a.head_dim == 128) return f32 ? launch_pdl(k_attend_join<128, true>, grid, block, 0, st, 1, a) : launch_pdl(k_attend_join<128, false>, grid, block, 0, st, 1, a);
  return f32 ? launch_pdl(k_attend_join<64, true>, grid, block, 0, st, 1, a) : launch_pdl(k_attend_join<64, false>, grid, block, 0, st, 1, a);
}

// Workspace: outputs of pieces, their references and sums, what they belong to.
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
size_t attend_workspace(int n_cta, int part_rows, int head_dim) {
  const size_t places = 2 * (size_t)n_cta * part_rows;
  return up256(places * head_dim * sizeof(float)) + up256(places * sizeof(float2)) + up256(2 * n_cta * sizeof(AttendPart));
}
void attend_bind(AttendShape* a, void* workspace) {
  const size_t places = 2 * (size_t)a->n_cta * a->part_rows;
  char* w = static_cast<char*>(workspace);
  a->part = reinterpret_cast<float*>(w);
  w += up256(places * a->head_dim * sizeof(float));
  a->ml = reinterpret_cast<float2*>(w);
  w += up256(places * sizeof(float2));
  a->desc = reinterpret_cast<AttendPart*>(w);
}

}  // namespace slkv
