// Attention of a prompt (Eq. 2-3 over all positions at once), causal, over a window and the first tokens: fp32 on CUDA cores.
//
// One CTA per 64 queries of a head; keys and values in tiles of 64, which two groups of 256 threads take in turns, each with a running
// maximum, sum and output of its own, joined at the end: twice the warps where a prompt has few CTAs (8 heads of 1024 tokens, d = 64,
// window 256: 46 us with one group, 30.8 with two, 35 with four of 128 threads and 8 queries each).  A thread owns 4 queries x 4 keys of a tile's logits and 4 queries x d / 16 elements of the
// output (packed FMAs); keys come through registers (transposed), values by asynchronous copies beside the logits, the weights go
// through shared memory.  Everything in fp32.  Bound by shared memory (L1 81 % busy, FMA 25 % of its issue): two loads of 16 bytes feed 16
// FMAs per thread.  8 heads of 2000 tokens: d = 64 145 us, d = 128 259 (28 and 32 TFLOP/s).
#include <math.h>

#include <algorithm>

#include "d2o_attention.cuh"
#include "d2o_common.cuh"
#include "d2o_decode.cuh"

namespace d2o {

constexpr int kAttGroup = 256;
constexpr int kAttThreads = 2 * kAttGroup;
constexpr int kAttTile = 64;
constexpr int kAttLd = kAttTile + 4;         // row of 64 floats in shared memory

__host__ __device__ constexpr int att_group_floats(int D) { return D * kAttLd + kAttTile * D + kAttTile * kAttLd; }

template <int D>
__global__ void __launch_bounds__(kAttThreads, 1)
prompt_attention_kernel(PromptAttentionArgs a) {
  wait_for_prior_grid();
  constexpr int CD = D / 16, V4 = D / 16;                    // output elements per thread and query; 16-byte pieces per thread and tile
  extern __shared__ __align__(16) float att_smem[];
  float* sQ = att_smem;                                      // [D][kAttLd] transposed, scaled
  const int grp = threadIdx.x / kAttGroup, tid = threadIdx.x % kAttGroup;
  float* sK = sQ + D * kAttLd + grp * att_group_floats(D);   // [D][kAttLd] transposed
  float* sV = sK + D * kAttLd;                               // [64][D]
  float* sP = sV + kAttTile * D;                             // [64 queries][kAttLd]
  auto sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + grp), "n"(kAttGroup) : "memory"); };      // of the group
  const int tx = tid & 15, ty = tid >> 4; // queries ty * 4 .., keys tx * 4 ..
  const int bh = blockIdx.x, b = bh / a.Hq, hk = b * a.Hkv + bh % a.Hq / (a.Hq / a.Hkv);
  const int P = a.length(b);
  const int q0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * kAttTile;      // the last queries see the most keys: first
  if (q0 >= P) return;
  const float* Q = (const float*)a.Q + (size_t)bh * a.P * D;
  const float* K = (const float*)a.K + (size_t)hk * a.P * D;
  const float* V = (const float*)a.V + (size_t)hk * a.P * D;
  const float scale = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  // Transposed tiles: a thread takes 16-byte pieces of one row, so that neighbouring lanes write neighbouring rows.  Rows behind the
  // sequence's end are zero.
  auto fetch_t = [&](float4 (&f)[V4], const float* from, int row0) {
    const int r = row0 + tid % kAttTile;
#pragma unroll
    for (int i = 0; i < V4; ++i)
      f[i] = r < P ? *reinterpret_cast<const float4*>(from + (size_t)r * D + (tid / kAttTile + 4 * i) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  auto store_t = [&](float* to, const float4 (&f)[V4], float mul) {
    float* at = to + tid / kAttTile * 4 * kAttLd + tid % kAttTile;
#pragma unroll
    for (int i = 0; i < V4; ++i) {
      at[(16 * i + 0) * kAttLd] = f[i].x * mul; at[(16 * i + 1) * kAttLd] = f[i].y * mul;
      at[(16 * i + 2) * kAttLd] = f[i].z * mul; at[(16 * i + 3) * kAttLd] = f[i].w * mul;
    }
  };
  auto copy_v = [&](int row0) {
#pragma unroll
    for (int i = 0; i < V4; ++i) {
      const int x = tid + i * kAttGroup, r = row0 + x / (D / 4);
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(sV + x * 4);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(V + (size_t)min(r, P - 1) * D + x % (D / 4) * 4), "r"(r < P ? 16 : 0) : "memory");
    }
  };
  const PromptSpan span(q0, kAttTile, P, kAttTile, a.window, a.n_sink);
  float4 kf[V4];
  if (grp == 0) {
    fetch_t(kf, Q, q0);
    store_t(sQ, kf, scale);
  }
  if (grp < span.tiles) fetch_t(kf, K, span.tile(grp) * kAttTile);
  __syncthreads();
  float m[4], l[4], acc[4][CD];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < CD; ++e) acc[i][e] = 0.f;
  }
  for (int t = grp; t < span.tiles; t += 2) {
    const int k0 = span.tile(t) * kAttTile;
    sync();                                                  // the tile before has been read
    copy_v(k0);
    store_t(sK, kf, 1.f);
    sync();
    if (t + 2 < span.tiles) fetch_t(kf, K, span.tile(t + 2) * kAttTile);
    float2 s2[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) s2[i][0] = s2[i][1] = make_float2(0.f, 0.f);
#pragma unroll 8
    for (int kk = 0; kk < D; ++kk) {
      const float4 kv = *reinterpret_cast<const float4*>(sK + kk * kAttLd + tx * 4);
      const float4 q = *reinterpret_cast<const float4*>(sQ + kk * kAttLd + ty * 4);
      const float qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s2[i][0] = ffma2(make_float2(qv[i], qv[i]), make_float2(kv.x, kv.y), s2[i][0]);
        s2[i][1] = ffma2(make_float2(qv[i], qv[i]), make_float2(kv.z, kv.w), s2[i][1]);
      }
    }
    const bool masked = !span.full(t);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float s[4] = {s2[i][0].x, s2[i][0].y, s2[i][1].x, s2[i][1].y};
      if (masked) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!a.sees(q0 + ty * 4 + i, k0 + tx * 4 + j)) s[j] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float mn = fmaxf(m[i], mx), base = mn > -INFINITY ? mn : 0.f;
      const float old = mn > -INFINITY ? exp2f(m[i] - mn) : 0.f;
      m[i] = mn;
      const float4 w = make_float4(exp2f(s[0] - base), exp2f(s[1] - base), exp2f(s[2] - base), exp2f(s[3] - base));
      *reinterpret_cast<float4*>(sP + (ty * 4 + i) * kAttLd + tx * 4) = w;
      l[i] = fmaf(l[i], old, (w.x + w.y) + (w.z + w.w));     // this thread's keys: summed over the 16 threads at the end
#pragma unroll
      for (int e = 0; e < CD; ++e) acc[i][e] *= old;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (k0 < span.lo) {      // values between the sinks and the first query's window, which no query of the tile sees, may be anything, and 0 * NaN is NaN
#pragma unroll
      for (int i = 0; i < V4; ++i) {
        const int x = tid + i * kAttGroup, r = k0 + x / (D / 4);
        if (r >= a.n_sink && r < span.lo) *reinterpret_cast<float4*>(sV + x * 4) = make_float4(0.f, 0.f, 0.f, 0.f);      // this thread's copy
      }
    }
    sync();
#pragma unroll 2
    for (int j = 0; j < kAttTile; j += 4) {
      float p[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(p[i]) = *reinterpret_cast<const float4*>(sP + (ty * 4 + i) * kAttLd + j);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
#pragma unroll
        for (int e = 0; e < CD; e += 4) {
          const float4 v = *reinterpret_cast<const float4*>(sV + (j + jj) * D + e * 16 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 w = make_float2(p[i][jj], p[i][jj]);
            const float2 lo = ffma2(w, make_float2(v.x, v.y), make_float2(acc[i][e], acc[i][e + 1]));
            const float2 hi = ffma2(w, make_float2(v.z, v.w), make_float2(acc[i][e + 2], acc[i][e + 3]));
            acc[i][e] = lo.x; acc[i][e + 1] = lo.y; acc[i][e + 2] = hi.x; acc[i][e + 3] = hi.y;
          }
        }
    }
  }
  // Not earlier: the CTAs of the next kernel would take places beside these and then lie unevenly over the SMs (back-to-back calls of
  // 8 heads of 1024 tokens 87 us each instead of 63 with the first form of this kernel).
  start_dependents();
  // ---- join the groups: the second hands over through the first one's tiles
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
  __syncthreads();
  float* swap = sQ + D * kAttLd;
  if (grp == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < CD; e += 4)
        *reinterpret_cast<float4*>(swap + (ty * 4 + i) * D + e * 16 + tx * 4) = make_float4(acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]);
      if (tx == 0) { swap[kAttTile * D + (ty * 4 + i) * 2] = m[i]; swap[kAttTile * D + (ty * 4 + i) * 2 + 1] = l[i]; }
    }
  }
  __syncthreads();
  if (grp == 1) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int q = q0 + ty * 4 + i;
    if (q >= P) continue;
    const float m1 = swap[kAttTile * D + (ty * 4 + i) * 2], l1 = swap[kAttTile * D + (ty * 4 + i) * 2 + 1];
    const float mn = fmaxf(m[i], m1), base = mn > -INFINITY ? mn : 0.f;
    const float f0 = exp2f(m[i] - base), f1 = exp2f(m1 - base);          // nothing seen by a group: 0
    const float t = l[i] * f0 + l1 * f1, f = 1.f / t;
    float* out = (float*)a.out + ((size_t)bh * a.P + q) * D;
#pragma unroll
    for (int e = 0; e < CD; e += 4) {
      const float4 o = *reinterpret_cast<const float4*>(swap + (ty * 4 + i) * D + e * 16 + tx * 4);
      *reinterpret_cast<float4*>(out + e * 16 + tx * 4) =
          make_float4((acc[i][e] * f0 + o.x * f1) * f, (acc[i][e + 1] * f0 + o.y * f1) * f, (acc[i][e + 2] * f0 + o.z * f1) * f, (acc[i][e + 3] * f0 + o.w * f1) * f);
    }
    if (a.lse && tx == 0) a.lse[(size_t)bh * a.P + q] = (mn + log2f(t)) * 0.6931471805599453f;
  }
}

template <int D>
static cudaError_t launch_one(const PromptAttentionArgs& a, cudaStream_t st) {
  const size_t smem = (size_t)(D * kAttLd + 2 * att_group_floats(D)) * 4;
  cudaError_t e = cudaFuncSetAttribute(prompt_attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_behind(prompt_attention_kernel<D>, dim3((unsigned)(a.B * a.Hq), (unsigned)((a.P + kAttTile - 1) / kAttTile)),
                       kAttThreads, smem, st, a);
}

cudaError_t launch_prompt_attention(int dtype, int D, const PromptAttentionArgs& a, cudaStream_t st) {
  if (dtype == D2O_F32) return D == 64 ? launch_one<64>(a, st) : launch_one<128>(a, st);
  return launch_prompt_attention_tc(dtype, D, a, st);
}

}  // namespace d2o
