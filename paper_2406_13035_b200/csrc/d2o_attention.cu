// Attention of a prompt (Eq. 2-3 over all positions at once), causal, over a window and the first tokens: fp32 on CUDA cores.
//
// One CTA per 64 queries of a head; keys and values in tiles of 64.  A thread owns 8 queries x 4 keys of a tile's logits and 8
// queries x d / 16 elements of the output; the weights of a tile travel through shared memory.  Running maximum and sum per
// query, everything in fp32.
#include <math.h>

#include <algorithm>

#include "d2o_attention.cuh"
#include "d2o_common.cuh"
#include "d2o_decode.cuh"

namespace d2o {

constexpr int kAttThreads = 128;
constexpr int kAttTile = 64;
constexpr int kAttLd = kAttTile + 4;         // row of a transposed tile in shared memory

template <typename T, int D>
__global__ void __launch_bounds__(kAttThreads)
prompt_attention_kernel(PromptAttentionArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int EPV = Elem<T>::kPerVec, CD = D / 16;         // elements of the output per thread and query
  extern __shared__ __align__(16) float att_smem[];
  float* sQ = att_smem;                                      // [D][kAttLd] transposed, scaled
  float* sK = sQ + D * kAttLd;                               // [D][kAttLd] transposed
  float* sV = sK + D * kAttLd;                               // [64][D]
  float* sP = sV + kAttTile * D;                             // [64 keys][kAttLd] transposed weights
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4; // queries ty * 8 .., keys tx * 4 ..
  const int bh = blockIdx.x, b = bh / a.Hq, hk = b * a.Hkv + bh % a.Hq / (a.Hq / a.Hkv);
  const int P = a.length(b);
  const int q0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * kAttTile;      // the last queries see the most keys: first
  if (q0 >= P) return;
  const T* Q = (const T*)a.Q + (size_t)bh * a.P * D;
  const T* K = (const T*)a.K + (size_t)hk * a.P * D;
  const T* V = (const T*)a.V + (size_t)hk * a.P * D;
  const float scale = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  // a thread reads 16-byte pieces of one row: neighbouring lanes write neighbouring rows of the transposed tile
  auto load_t = [&](float* to, const T* from, int row0, float mul) {
    for (int i = tid; i < kAttTile * (D / EPV); i += kAttThreads) {
      const int r = i % kAttTile, piece = i / kAttTile;
      float f[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) f[e] = 0.f;
      if (row0 + r < P) Elem<T>::unpack(ld_global_v4(from + (size_t)(row0 + r) * D + piece * EPV), f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) to[(piece * EPV + e) * kAttLd + r] = f[e] * mul;
    }
  };
  load_t(sQ, Q, q0, scale);
  float m[8], l[8], acc[8][CD];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < CD; ++e) acc[i][e] = 0.f;
  }
  const PromptSpan span(q0, kAttTile, P, kAttTile, a.window, a.n_sink);
  for (int t = 0; t < span.tiles; ++t) {
    const int k0 = span.tile(t) * kAttTile;
    __syncthreads();                                         // the tile before has been read
    load_t(sK, K, k0, 1.f);
    for (int i = tid; i < kAttTile * (D / EPV); i += kAttThreads) {
      const int r = i / (D / EPV), piece = i % (D / EPV);
      float f[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) f[e] = 0.f;
      if (k0 + r < P) Elem<T>::unpack(ld_global_v4(V + (size_t)(k0 + r) * D + piece * EPV), f);
#pragma unroll
      for (int e = 0; e < EPV; e += 4) *reinterpret_cast<float4*>(sV + r * D + piece * EPV + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
    }
    __syncthreads();
    float2 s2[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) s2[i][0] = s2[i][1] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int kk = 0; kk < D; ++kk) {
      const float4 kv = *reinterpret_cast<const float4*>(sK + kk * kAttLd + tx * 4);
      const float4 qa = *reinterpret_cast<const float4*>(sQ + kk * kAttLd + ty * 8);
      const float4 qb = *reinterpret_cast<const float4*>(sQ + kk * kAttLd + ty * 8 + 4);
      const float qv[8] = {qa.x, qa.y, qa.z, qa.w, qb.x, qb.y, qb.z, qb.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s2[i][0] = ffma2(make_float2(qv[i], qv[i]), make_float2(kv.x, kv.y), s2[i][0]);
        s2[i][1] = ffma2(make_float2(qv[i], qv[i]), make_float2(kv.z, kv.w), s2[i][1]);
      }
    }
    const bool masked = !span.full(t);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s[4] = {s2[i][0].x, s2[i][0].y, s2[i][1].x, s2[i][1].y};
      if (masked) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!a.sees(q0 + ty * 8 + i, k0 + tx * 4 + j)) s[j] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float mn = fmaxf(m[i], mx), base = mn > -INFINITY ? mn : 0.f;
      const float old = mn > -INFINITY ? exp2f(m[i] - mn) : 0.f;
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = exp2f(s[j] - base);
        sum += w;
        sP[(tx * 4 + j) * kAttLd + ty * 8 + i] = w;
      }
      l[i] = fmaf(l[i], old, sum);                           // this thread's keys: summed over the 16 threads at the end
#pragma unroll
      for (int e = 0; e < CD; ++e) acc[i][e] *= old;
    }
    __syncwarp();                                            // a query's 16 threads are in one warp
#pragma unroll 2
    for (int j = 0; j < kAttTile; ++j) {
      const float4 pa = *reinterpret_cast<const float4*>(sP + j * kAttLd + ty * 8);
      const float4 pb = *reinterpret_cast<const float4*>(sP + j * kAttLd + ty * 8 + 4);
      const float pv[8] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
      for (int e = 0; e < CD; e += 4) {
        const float4 v = *reinterpret_cast<const float4*>(sV + j * D + e * 16 + tx * 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 lo = ffma2(make_float2(pv[i], pv[i]), make_float2(v.x, v.y), make_float2(acc[i][e], acc[i][e + 1]));
          const float2 hi = ffma2(make_float2(pv[i], pv[i]), make_float2(v.z, v.w), make_float2(acc[i][e + 2], acc[i][e + 3]));
          acc[i][e] = lo.x; acc[i][e + 1] = lo.y; acc[i][e + 2] = hi.x; acc[i][e + 3] = hi.y;
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float t = l[i];
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    const int q = q0 + ty * 8 + i;
    if (q >= P) continue;
    T* out = (T*)a.out + ((size_t)bh * a.P + q) * D;
#pragma unroll
    for (int e = 0; e < CD; e += 4)
#pragma unroll
      for (int j = 0; j < 4; ++j) out[e * 16 + tx * 4 + j] = Elem<T>::from_float(acc[i][e + j] / t);
    if (a.lse && tx == 0) a.lse[(size_t)bh * a.P + q] = (m[i] + log2f(t)) * 0.6931471805599453f;
  }
}

template <typename T, int D>
static cudaError_t launch_one(const PromptAttentionArgs& a, cudaStream_t st) {
  const size_t smem = (size_t)(2 * D * kAttLd + kAttTile * D + kAttTile * kAttLd) * 4;
  cudaError_t e = cudaFuncSetAttribute(prompt_attention_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_behind(prompt_attention_kernel<T, D>, dim3((unsigned)(a.B * a.Hq), (unsigned)((a.P + kAttTile - 1) / kAttTile)),
                       kAttThreads, smem, st, a);
}

cudaError_t launch_prompt_attention(int dtype, int D, const PromptAttentionArgs& a, cudaStream_t st) {
  if (dtype == D2O_F32) return D == 64 ? launch_one<float, 64>(a, st) : launch_one<float, 128>(a, st);
  return launch_prompt_attention_tc(dtype, D, a, st);
}

}  // namespace d2o
