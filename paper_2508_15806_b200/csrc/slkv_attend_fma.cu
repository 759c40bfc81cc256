// Attention of prompts and of tokens over a paged cache in fp32, on the FMA pipe, and the kernel that joins the pieces of units which
// several CTAs share, for both paths.
//
// k_attend_fma: a CTA has BM query rows (tokens times the query heads of a KV head) and goes through tiles of 64 keys: S = Q K^T with a
// 4 x 4 (BM = 64) or 1 x 4 (BM = 16) square of a thread, the running reference and sum of a row in the 16 threads that share it, then
// O += P V.  All products and sums in fp32.
#include <atomic>

#include "slkv_attend.cuh"
#include "slkv_fma_device.cuh"

namespace slkv {
namespace {

constexpr int kKeys = 64, kFmaThreads = 256, kFmaPerSm = 2;

__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int BM, int D>
struct FmaSmem {
  static constexpr int kLd = D + 4;
  static constexpr int kLdP = kKeys + 4;
  float q[BM][kLd], v[kKeys][kLd];
  union {
    float k[kKeys][kLd];
    float p[BM][kLdP];                           // once the scores are there; -0: the row does not see the key
  };
  const float* krow[kKeys];                      // of the tile at hand; null: nothing there
  const float* vrow[kKeys];
};

template <int BM, int D>
__global__ void __launch_bounds__(kFmaThreads, kFmaPerSm)
k_attend_fma(const __grid_constant__ AttendShape a) {
  extern __shared__ __align__(16) unsigned char raw[];
  FmaSmem<BM, D>& sm = *reinterpret_cast<FmaSmem<BM, D>*>(raw);
  constexpr int RT = BM / 16, C = D / 64;        // rows of a thread; float4s of a row's channels that it has
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  pdl_launch_dependents();
  pdl_wait();
  if (tid == 0 && !a.spread) a.desc[2 * blockIdx.x].state = a.desc[2 * blockIdx.x + 1].state = 0;
  __shared__ AttendStart start;
  attend_start(a, blockIdx.x, &start);
  __syncthreads();
  AttendSchedule plan(a, blockIdx.x, &start);    // every warp runs it
  const float sc = a.scale * kLog2e;
  for (;;) {
    AttendPiece p = {};
    if (!plan.next(&p)) break;
    if (tid == 0 && p.part >= 0) attend_note(a, p.part, p, p.part == 1 ? plan.pieces() : 0);
    // row r: token r / G of the unit, query head r % G of the group
    const int rows = p.n_tok * a.G;
    const float* qb = static_cast<const float*>(a.q) + (a.paged ? p.s * a.q_seq : p.q_row * a.q_tok);
    __syncthreads();
    for (int i = tid; i < BM * (D / 4); i += kFmaThreads) {
      const int r = i / (D / 4), c = i - r * (D / 4), rt = r / a.G;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) x = *reinterpret_cast<const float4*>(qb + (p.tok0 + rt) * a.q_tok + (p.h * a.G + r - rt * a.G) * a.q_head + 4 * c);
      *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
    }
    int tok[RT], bound[RT];
    unsigned long long mask[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
      tok[i] = p.tok0 + min(r, rows - 1) / a.G;
      bound[i] = max(min(tok[i] + 1 + p.shift, p.nk), 0);
      mask[i] = 0;
      if (a.has_new) {
        mask[i] = a.tree ? a.tree[(long long)p.s * a.n_tokens + tok[i]] : ~0ull >> (63 - tok[i]);
        mask[i] &= ~0ull >> (64 - p.n_seq_tok);
      }
    }
    float m[RT], l[RT];
    float4 o[RT][C];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int t = p.tile0; t < p.tile0 + p.n; ++t) {
      const bool drafted = a.has_new && t == p.n_all - 1;
      const int key0 = t * kKeys, end = drafted ? p.n_seq_tok : min(p.nk - key0, kKeys);
      __syncthreads();
      if (tid < kKeys) {
        const float *kr = nullptr, *vr = nullptr;
        if (tid < end) {
          if (drafted) {
            kr = static_cast<const float*>(a.k_new) + p.s * a.kn_seq + tid * a.kn_tok + p.h * a.kn_head;
            vr = static_cast<const float*>(a.v_new) + p.s * a.vn_seq + tid * a.vn_tok + p.h * a.vn_head;
          } else if (a.paged) {
            const int row = key0 + tid, pg = row / a.page_rows;
            const int id = a.tables[(long long)(p.s * a.n_kv_heads + p.h) * a.max_pages + pg];
            if ((unsigned)id < (unsigned)a.n_pages) {
              const long long at = ((long long)id * a.page_rows + row - pg * a.page_rows) * D;
              kr = static_cast<const float*>(a.k) + at;
              vr = static_cast<const float*>(a.v) + at;
            } else if (a.status) {
              *a.status = SLKV_ERR_BAD_SHAPE;
            }
          } else {
            const long long row = p.k_row + key0 + tid;
            kr = static_cast<const float*>(a.k) + row * a.k_tok + p.h * a.k_head;
            vr = static_cast<const float*>(a.v) + row * a.v_tok + p.h * a.v_head;
          }
        }
        sm.krow[tid] = kr;
        sm.vrow[tid] = vr;
      }
      __syncthreads();
#pragma unroll 4
      for (int i = tid; i < kKeys * (D / 4); i += kFmaThreads) {
        const int r = i / (D / 4), c = i - r * (D / 4);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (sm.krow[r]) x = *reinterpret_cast<const float4*>(sm.krow[r] + 4 * c);
        if (sm.vrow[r]) y = *reinterpret_cast<const float4*>(sm.vrow[r] + 4 * c);
        *reinterpret_cast<float4*>(&sm.k[r][4 * c]) = x;
        *reinterpret_cast<float4*>(&sm.v[r][4 * c]) = y;
      }
      __syncthreads();
      float s[RT][4];
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        float4 kk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][c]);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const float4 qq = *reinterpret_cast<const float4*>(&sm.q[ty * RT + i][c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(qq.x, kk[j].x, s[i][j]);
            s[i][j] = fmaf(qq.y, kk[j].y, s[i][j]);
            s[i][j] = fmaf(qq.z, kk[j].z, s[i][j]);
            s[i][j] = fmaf(qq.w, kk[j].w, s[i][j]);
          }
        }
      }
      __syncthreads();                           // K gives way to P
      // the first row sees the fewest keys of a prompt's tile
      const bool edge = drafted || end < kKeys || (!a.paged && p.tok0 + 1 + p.shift < key0 + kKeys);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        bool see[4];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = tx + 16 * j;
          see[j] = drafted ? (mask[i] >> key & 1) != 0 : (a.paged ? key < end : key0 + key < bound[i]);
          s[i][j] = see[j] ? s[i][j] * sc : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float mn = fmaxf(m[i], top), base = mn == -INFINITY ? 0.f : mn;
        const float f = m[i] == -INFINITY ? 0.f : exp2_of(m[i] - base);
        m[i] = mn;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = exp2_of(s[i][j] - base);
          sum += e;
          sm.p[ty * RT + i][tx + 16 * j] = see[j] ? e : -0.f;
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l[i] = l[i] * f + sum;
#pragma unroll
        for (int c = 0; c < C; ++c) { o[i][c].x *= f; o[i][c].y *= f; o[i][c].z *= f; o[i][c].w *= f; }
      }
      __syncwarp();                              // a row's 16 threads are in one warp
      auto product = [&](auto masked) {
#pragma unroll 2
        for (int k = 0; k < kKeys; k += 4) {
          float4 pp[RT];
#pragma unroll
          for (int i = 0; i < RT; ++i) pp[i] = *reinterpret_cast<const float4*>(&sm.p[ty * RT + i][k]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < C; ++c) {
              const float4 vv = *reinterpret_cast<const float4*>(&sm.v[k + e][4 * tx + 64 * c]);
#pragma unroll
              for (int i = 0; i < RT; ++i) {
                const float w = e == 0 ? pp[i].x : e == 1 ? pp[i].y : e == 2 ? pp[i].z : pp[i].w;
                if (decltype(masked)::value && (__float_as_uint(w) >> 31)) continue;     // whatever V holds there
                o[i][c].x = fmaf(w, vv.x, o[i][c].x);
                o[i][c].y = fmaf(w, vv.y, o[i][c].y);
                o[i][c].z = fmaf(w, vv.z, o[i][c].z);
                o[i][c].w = fmaf(w, vv.w, o[i][c].w);
              }
            }
        }
      };
      if (edge) product(std::true_type());
      else product(std::false_type());
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int r = ty * RT + i;
      if (r >= rows) continue;
      const int qh = p.h * a.G + r - (r / a.G) * a.G;
      const bool some = l[i] > 0.f || l[i] != l[i];
      const long long place = p.part < 0 ? 0 : (long long)(blockIdx.x * 2 + p.part) * a.part_rows + r;
      const float inv = p.part >= 0 ? 1.f : (some ? 1.f / l[i] : 0.f);
      float* dst = p.part >= 0 ? a.part + place * D
                               : static_cast<float*>(a.out) + (a.paged ? p.s * a.o_seq : p.q_row * a.o_tok) + tok[i] * a.o_tok + qh * a.o_head;
#pragma unroll
      for (int c = 0; c < C; ++c)
        *reinterpret_cast<float4*>(dst + 4 * tx + 64 * c) = make_float4(o[i][c].x * inv, o[i][c].y * inv, o[i][c].z * inv, o[i][c].w * inv);
      if (tx == 0) {
        if (p.part >= 0) a.ml[place] = make_float2(m[i], l[i]);
        else attend_lse(a, p.s, qh, tok[i], p.n_seq_tok, m[i], l[i]);
      }
    }
  }
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

template <int BM, int D>
cudaError_t launch(const AttendShape& a, cudaStream_t st, int* launches) {
  static std::atomic<bool> allowed[16];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 16 || !allowed[dev].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(k_attend_fma<BM, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(FmaSmem<BM, D>));
    if (e != cudaSuccess) return e;
    if (dev < 16) allowed[dev].store(true, std::memory_order_relaxed);
  }
  LaunchScope scope(KID_ATTEND, st, launches);
  return launch_pdl(k_attend_fma<BM, D>, dim3((unsigned)a.n_cta), dim3(kFmaThreads), sizeof(FmaSmem<BM, D>), st, 1, a);
}

}  // namespace

cudaError_t launch_attend_fma(const AttendShape& a, cudaStream_t st, int* launches) {
  if (a.part_rows == 64) return a.head_dim == 128 ? launch<64, 128>(a, st, launches) : launch<64, 64>(a, st, launches);
  return a.head_dim == 128 ? launch<16, 128>(a, st, launches) : launch<16, 64>(a, st, launches);
}

cudaError_t launch_attend_join(const AttendShape& a, bool f32, cudaStream_t st, int* launches) {
  if (a.spread || a.n_cta < 2) return cudaSuccess;
  LaunchScope scope(KID_ATTEND_JOIN, st, launches);
  const dim3 grid((unsigned)(a.n_cta - 1), (unsigned)((a.used_rows + kJoinRows - 1) / kJoinRows)), block(kJoinWarps * 32);
  if (a.head_dim == 128) return f32 ? launch_pdl(k_attend_join<128, true>, grid, block, 0, st, 1, a) : launch_pdl(k_attend_join<128, false>, grid, block, 0, st, 1, a);
  return f32 ? launch_pdl(k_attend_join<64, true>, grid, block, 0, st, 1, a) : launch_pdl(k_attend_join<64, false>, grid, block, 0, st, 1, a);
}

int attend_fma_ctas() { return kFmaPerSm * sm_count(); }

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
