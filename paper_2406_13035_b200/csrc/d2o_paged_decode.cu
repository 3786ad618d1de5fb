// Decode attention over a cache in pages (Eq. 2-3), with the accumulation of Eq. 6 (case 2).
//
// The rows that the new tokens see are counted in tiles of 16, slice after slice (slice = sequence and KV head), and every
// CTA takes an equal share of all tiles: a batch of any lengths, or one long sequence, fills the GPU evenly without the host
// knowing a length.  A share covers parts of one or several slices.  For each part a CTA forms a running softmax (maximum,
// sum, un-normalised output) per query head; a slice that lies in one share is finished there, the parts of the others are
// joined by join_kernel, in the order of the shares.  With scores, the logits go to scratch on the way and join_kernel, which
// knows the normalisers, adds the weights to the rows' scores.
#include <math.h>

#include <algorithm>

#include "d2o_common.cuh"
#include "d2o_decode.cuh"
#include "d2o_paged.cuh"

namespace d2o {

constexpr int kPagedThreads = 256;
constexpr int kPagedWarps = kPagedThreads / 32;
constexpr int kPagedMinTiles = 4;            // least share of a CTA

struct PagedDecodeArgs {
  PagedView p;
  const void *q, *k, *v;                     // [B, Hq, d], [B, Hkv, d] x 2
  void* out;                                 // [B, Hq, d]
  const int32_t* positions;                  // [B], or NULL
  int window, n_sink;
  int ctas;                                  // CTAs of the first kernel
  int4* desc;                                // per slice: first share, last share, which part of the first share; -1: finished there
  float* lse2;                               // [slices][G] normalisers in the log2 domain of slices finished in one share
  float* parts;                              // [ctas][2][G][D + 2]: output, maximum, sum; 0: the share's first part, 1: its last
  float* logits;                             // per row of the pools, G logits in the log2 domain (with scores)
};

// The shares.  `share` CTAs of `tot` tiles: share c holds the tiles [tot * c / share, tot * (c + 1) / share).
__device__ __forceinline__ int shares_of(long long tot, int ctas) {
  return (int)min((long long)ctas, (tot + kPagedMinTiles - 1) / kPagedMinTiles);
}
__device__ __forceinline__ long long share_begin(long long tot, int share, int c) { return tot * c / share; }
__device__ __forceinline__ int share_of_tile(long long tot, int share, long long tile) {
  int c = (int)(tile * share / tot);
  while (share_begin(tot, share, c + 1) <= tile) ++c;
  return c;
}

// Where this CTA begins: tiles before its first slice, and that slice.  Every CTA adds up the tiles of all slices: a thread
// those of consecutive slices, then a scan over the block.
struct PagedStart {
  long long tot;                             // tiles in all
  long long before;                          // tiles ahead of `slice`
  int slice, share;
};
__device__ __forceinline__ PagedStart paged_start(const PagedDecodeArgs& a, int c, long long* s_scan /* [threads + 1] */, int* s_found) {
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_slices = p.B * p.Hkv, per = (n_slices + kPagedThreads - 1) / kPagedThreads;
  const int s0 = min(n_slices, tid * per), s1 = min(n_slices, s0 + per);
  long long mine = 0;
  for (int s = s0; s < s1; ++s) mine += PagedSpan(p.len[s], p.reach(), a.window, a.n_sink).tiles;
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += t; }
  if (lane == 31) s_scan[warp] = inc;
  __syncthreads();
  long long base = 0, tot = 0;
#pragma unroll
  for (int w = 0; w < kPagedWarps; ++w) { if (w < warp) base += s_scan[w]; tot += s_scan[w]; }
  PagedStart r;
  r.tot = tot; r.share = shares_of(tot, a.ctas); r.slice = -1; r.before = 0;
  const long long first = c < r.share ? share_begin(tot, r.share, c) : tot;
  long long at = base + inc - mine;
  if (first >= at && first < at + mine) {                    // one thread
    int s = s0;
    for (;; ++s) {
      const int tiles = PagedSpan(p.len[s], p.reach(), a.window, a.n_sink).tiles;
      if (first < at + tiles) break;
      at += tiles;
    }
    *s_found = s; s_scan[kPagedWarps] = at;
  }
  __syncthreads();
  if (c < r.share) { r.slice = *s_found; r.before = s_scan[kPagedWarps]; }
  return r;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kPagedThreads, 1)
paged_decode_kernel(PagedDecodeArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPW = 32 / LPR, U = kPagedTile / RPW, QL = LPR / 4;
  extern __shared__ __align__(16) float red[];               // [warps][G][D]
  __shared__ float s_m[kPagedWarps][G], s_l[kPagedWarps][G];
  __shared__ long long s_scan[kPagedWarps + 1];
  __shared__ int s_found;
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int grp = lane / LPR, lig = lane % LPR, c = blockIdx.x;
  const PagedStart start = paged_start(a, c, s_scan, &s_found);
  if (start.slice < 0) return;
  const long long first = share_begin(start.tot, start.share, c), last = share_begin(start.tot, start.share, c + 1);
  long long before = start.before;
  int sl = start.slice;
  for (long long at = first; at < last; ++sl) {
    const PagedSpan span(p.len[sl], p.reach(), a.window, a.n_sink);
    if (span.tiles == 0) continue;
    const int b = sl / p.Hkv, h = sl % p.Hkv;
    const int i0 = (int)(at - before), i1 = (int)min((long long)span.tiles, last - before);      // this part: tiles i0 .. i1 of the slice
    const T* q_in = (const T*)a.q + ((size_t)b * p.Hq + (size_t)h * G) * D;
    const T* k_new = (const T*)a.k + (size_t)sl * D;
    const T* v_new = (const T*)a.v + (size_t)sl * D;
    const T *kp = (const T*)p.k, *vp = (const T*)p.v;
    float qf[G][EPV], m[G], l[G], acc[G][EPV];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      Elem<T>::unpack(ld_global_v4(q_in + g * D + lig * EPV), qf[g]);
      m[g] = -INFINITY; l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < EPV; ++e) { qf[g][e] *= (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e; acc[g][e] = 0.f; }
    }
    for (int i = i0 + warp; i < i1; i += kPagedWarps) {
      const int row0 = span.row0(i);
      const int page0 = p.page_row0(b, h, row0);
      const size_t prow = (size_t)(page0 < 0 ? 0 : page0) + p.in_page(row0);
      if (page0 < 0) {
        if (lane == 0) p.report(kPagedBadPage);
#pragma unroll
        for (int g = 0; g < G; ++g) l[g] = NAN;
        continue;
      }
      uint4 kv[U], vv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = u * RPW + grp;
        kv[u] = make_uint4(0, 0, 0, 0);
        if (span.sees(row0 + r)) kv[u] = ld_stream_v4((row0 + r < span.t ? kp + (prow + r) * D : k_new) + lig * EPV);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = u * RPW + grp;
        vv[u] = make_uint4(0, 0, 0, 0);
        if (span.sees(row0 + r)) vv[u] = ld_stream_v4((row0 + r < span.t ? vp + (prow + r) * D : v_new) + lig * EPV);
      }
      float x[G][U / 4];                                     // logit of this lane's row of every four
#pragma unroll
      for (int j = 0; j < U / 4; ++j) {
        float dot[G][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float f[EPV];
          Elem<T>::unpack(kv[j * 4 + u], f);
#pragma unroll
          for (int g = 0; g < G; ++g) dot[g][u] = dot_pairs<EPV>(qf[g], f);
        }
        const int r = (j * 4 + lig / QL) * RPW + grp;
        const bool in = span.sees(row0 + r);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float t = reduce4<LPR>(dot[g][0], dot[g][1], dot[g][2], dot[g][3], lig);
          x[g][j] = in ? t : -INFINITY;
          if (a.logits && lig % QL == 0 && in) a.logits[(prow + r) * G + g] = t;
        }
      }
      float f[U][EPV];
#pragma unroll
      for (int u = 0; u < U; ++u) Elem<T>::unpack(vv[u], f[u]);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float mx = x[g][0];
#pragma unroll
        for (int j = 1; j < U / 4; ++j) mx = fmaxf(mx, x[g][j]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, QL));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2 * QL));
        const float mn = fmaxf(m[g], mx);
        const float old = mn > -INFINITY ? exp2f(m[g] - mn) : 0.f;
        m[g] = mn;
        const float base = mn > -INFINITY ? mn : 0.f;        // rows not seen, and logits of -inf: 0; a NaN stays one
        float w[U / 4], s = 0.f;
#pragma unroll
        for (int j = 0; j < U / 4; ++j) { w[j] = exp2f(x[g][j] - base); s += w[j]; }
        l[g] = fmaf(l[g], old, s);                           // this lane's rows only: summed over the group at the end
#pragma unroll
        for (int e = 0; e < EPV; ++e) acc[g][e] *= old;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float pw = __shfl_sync(0xffffffffu, w[u / 4], (u & 3) * QL, LPR);
#pragma unroll
          for (int e = 0; e < EPV; e += 2) {
            const float2 t = ffma2(make_float2(pw, pw), make_float2(f[u][e], f[u][e + 1]), make_float2(acc[g][e], acc[g][e + 1]));
            acc[g][e] = t.x; acc[g][e + 1] = t.y;
          }
        }
      }
      // the new token's row
      const int rt = span.t - row0;
      if (rt >= 0 && rt < kPagedTile && grp == 0) {
        *reinterpret_cast<uint4*>((T*)p.k + (prow + rt) * D + lig * EPV) = ld_global_v4(k_new + lig * EPV);
        *reinterpret_cast<uint4*>((T*)p.v + (prow + rt) * D + lig * EPV) = ld_global_v4(v_new + lig * EPV);
        if (p.pos && lig == 0) p.pos[prow + rt] = a.positions ? a.positions[b] : span.t;
      }
    }
    // ---- combine the row groups of a warp, then the warps
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float ls = l[g];                                       // QL lanes hold the same rows
      ls += __shfl_xor_sync(0xffffffffu, ls, QL);
      ls += __shfl_xor_sync(0xffffffffu, ls, 2 * QL);
      float mw = m[g];
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) mw = fmaxf(mw, __shfl_xor_sync(0xffffffffu, mw, o));
      const float w = mw > -INFINITY ? exp2f(m[g] - mw) : 1.f;           // 1: a NaN sum of a bad page stays
      ls *= w;
#pragma unroll
      for (int e = 0; e < EPV; ++e) acc[g][e] *= w;
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) {
        ls += __shfl_xor_sync(0xffffffffu, ls, o);
#pragma unroll
        for (int e = 0; e < EPV; ++e) acc[g][e] += __shfl_xor_sync(0xffffffffu, acc[g][e], o);
      }
      if (lane == 0) { s_m[warp][g] = mw; s_l[warp][g] = ls; }
      if (lane < LPR) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) red[(warp * G + g) * D + lane * EPV + e] = acc[g][e];
      }
    }
    __syncthreads();
    const bool whole = i0 == 0 && i1 == span.tiles;
    const int part = at == first ? 0 : 1;
    float* to = a.parts + ((size_t)c * 2 + part) * G * (D + 2);
    for (int i = tid; i < G * D; i += kPagedThreads) {
      const int g = i / D;
      float mc = s_m[0][g];
#pragma unroll
      for (int w = 1; w < kPagedWarps; ++w) mc = fmaxf(mc, s_m[w][g]);
      float t = 0.f, lc = 0.f;
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) {
        const float f = s_m[w][g] > -INFINITY ? exp2f(s_m[w][g] - mc) : mc > -INFINITY ? 0.f : 1.f;
        t = fmaf(red[w * G * D + i], f, t);
        lc = s_l[w][g] != s_l[w][g] ? NAN : fmaf(s_l[w][g], f, lc);
      }
      if (whole) {
        ((T*)a.out)[((size_t)b * p.Hq + (size_t)h * G) * D + i] = Elem<T>::from_float(t / lc);
        if (i % D == 0) a.lse2[sl * G + g] = mc + log2f(lc);
      } else {
        to[g * (D + 2) + i % D] = t;
        if (i % D == 0) { to[g * (D + 2) + D] = mc; to[g * (D + 2) + D + 1] = lc; }
      }
    }
    if (i0 == 0 && tid == 0)
      a.desc[sl] = whole ? make_int4(c, -1, 0, 0) : make_int4(c, share_of_tile(start.tot, start.share, before + span.tiles - 1), part, 0);
    __syncthreads();                                         // before the exchange area is written again
    at = before + i1;
    before += span.tiles;
  }
}

// Joins the parts of a slice (blockIdx.x) and adds the weights to the scores of its rows (divided over blockIdx.y).
template <typename T, int D, int G>
__global__ void __launch_bounds__(kPagedThreads)
join_kernel(PagedDecodeArgs a) {
  start_dependents();
  wait_for_prior_grid();
  __shared__ float s_m[G], s_lse[G];
  const PagedView& p = a.p;
  const int sl = blockIdx.x, b = sl / p.Hkv, h = sl % p.Hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = p.len[sl];
  if (n < 0) return;
  T* out = (T*)a.out + ((size_t)b * p.Hq + (size_t)h * G) * D;
  const PagedSpan span(n, p.reach(), a.window, a.n_sink);
  if (span.t < 0) {                                          // the table has no row for the new token
    if (blockIdx.y == 0) {
      if (tid == 0) p.report(kPagedShortTable);
      for (int i = tid; i < G * D; i += kPagedThreads) out[i] = Elem<T>::from_float(NAN);
    }
    return;
  }
  const int4 desc = a.desc[sl];
  auto part = [&](int c) { return a.parts + ((size_t)c * 2 + (c == desc.x ? desc.z : 0)) * G * (D + 2); };
  if (desc.y < 0) {
    if (tid < G) s_lse[tid] = a.lse2[sl * G + tid];
    __syncthreads();
  } else {
    if (warp < G) {                                          // a warp per head: largest maximum, then the sum
      float mc = -INFINITY;
      for (int c = desc.x + lane; c <= desc.y; c += 32) mc = fmaxf(mc, part(c)[warp * (D + 2) + D]);
      mc = warp_max(mc);
      float lc = 0.f;
      for (int c = desc.x + lane; c <= desc.y; c += 32) {
        const float* x = part(c) + warp * (D + 2) + D;
        lc += x[0] > -INFINITY ? x[1] * exp2f(x[0] - mc) : x[1];     // nothing finite: 0 or NaN
      }
      lc = warp_sum(lc);
      if (lane == 0) { s_m[warp] = mc; s_lse[warp] = mc + log2f(lc); }
    }
    __syncthreads();
    if (blockIdx.y == 0) {
      for (int i = tid; i < G * D; i += kPagedThreads) {
        const int g = i / D;
        float t = 0.f;
        for (int c = desc.x; c <= desc.y; ++c) {
          const float* x = part(c) + g * (D + 2);
          t = fmaf(x[i % D], x[D] > -INFINITY ? exp2f(x[D] - s_m[g]) : 0.f, t);
        }
        out[i] = Elem<T>::from_float(t * exp2f(s_m[g] - s_lse[g]));
      }
    }
  }
  if (!a.logits) return;
  for (int i = blockIdx.y * kPagedThreads + tid; i < span.tiles * kPagedTile; i += gridDim.y * kPagedThreads) {
    const int r = span.row0(i / kPagedTile) + i % kPagedTile;
    if (!span.sees(r)) continue;
    const int page0 = p.page_row0(b, h, r);
    if (page0 < 0) continue;
    const size_t at = (size_t)page0 + p.in_page(r);
    float w = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) w += exp2f(a.logits[at * G + g] - s_lse[g]);
    p.score[at] = r == span.t ? w : p.score[at] + w;
  }
}

// ------------------------------------------------------------------------------------ launch
template <typename T, int D, int G>
static cudaError_t launch_one(const PagedDecodeArgs& a, cudaStream_t st) {
  const size_t smem = (size_t)kPagedWarps * G * D * 4;
  cudaError_t e = cudaFuncSetAttribute(paged_decode_kernel<T, D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  e = launch_behind(paged_decode_kernel<T, D, G>, dim3((unsigned)a.ctas), kPagedThreads, smem, st, a);
  if (e != cudaSuccess) return e;
  const int n_slices = a.p.B * a.p.Hkv;
  int y = 1;                                                 // CTAs per slice that share the scores: what fills the GPU twice, 1024 rows each at least
  if (a.logits) {
    const long long reach = (long long)a.p.max_pages << a.p.page_shift;
    y = (int)std::max<long long>(1, std::min<long long>((4 * a.ctas + n_slices - 1) / n_slices, reach / 1024));
  }
  return launch_behind(join_kernel<T, D, G>, dim3((unsigned)n_slices, (unsigned)y), kPagedThreads, 0, st, a);
}

template <typename T, int D>
static cudaError_t launch_g(const PagedDecodeArgs& a, cudaStream_t st) {
  switch (a.p.Hq / a.p.Hkv) {
    case 1: return launch_one<T, D, 1>(a, st);
    case 2: return launch_one<T, D, 2>(a, st);
    case 4: return launch_one<T, D, 4>(a, st);
    default: return launch_one<T, D, 8>(a, st);
  }
}

cudaError_t launch_paged_decode(const PagedView& p, int dtype, int D, int window, int n_sink, const void* q, const void* k,
                                const void* v, const int32_t* positions, void* out, char* scratch, cudaStream_t st) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaGetLastError();
  const int G = p.Hq / p.Hkv;
  const PagedScratch s(p.B * p.Hkv, G, D, (size_t)p.n_pages * p.Hkv << p.page_shift, p.score != nullptr);
  PagedDecodeArgs a;
  a.p = p;
  a.q = q; a.k = k; a.v = v; a.out = out; a.positions = positions; a.window = window; a.n_sink = n_sink;
  a.ctas = std::min(sms, kPagedCtas);
  a.desc = reinterpret_cast<int4*>(scratch + s.desc);
  a.lse2 = reinterpret_cast<float*>(scratch + s.lse2);
  a.parts = reinterpret_cast<float*>(scratch + s.parts);
  a.logits = p.score ? reinterpret_cast<float*>(scratch + s.rows) : nullptr;
  if (dtype == D2O_F32) return D == 64 ? launch_g<float, 64>(a, st) : launch_g<float, 128>(a, st);
  if (dtype == D2O_F16) return D == 64 ? launch_g<__half, 64>(a, st) : launch_g<__half, 128>(a, st);
  return D == 64 ? launch_g<__nv_bfloat16, 64>(a, st) : launch_g<__nv_bfloat16, 128>(a, st);
}

}  // namespace d2o
