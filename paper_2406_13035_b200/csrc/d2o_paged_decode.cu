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
#include "d2o_tc.cuh"

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
  float* parts;                              // [ctas][2][G][D + 4]: output, maximum, sum, -; 0: the share's first part, 1: its last
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

// The warps' results of one part (tiles i0 .. i1 of slice `sl`) become the slice's output, or a part for join_kernel.
template <typename T, int D, int G, int LD>
__device__ __forceinline__ void finish_part(const PagedDecodeArgs& a, const PagedStart& start, int part, int sl, int i0, int i1, const PagedSpan& span,
                                            long long before, const float* red, const float* s_m, const float* s_l, int ld) {
  const PagedView& p = a.p;
  const int c = blockIdx.x, b = sl / p.Hkv, h = sl % p.Hkv;
  const bool whole = i0 == 0 && i1 == span.tiles;
  float* to = a.parts + ((size_t)c * 2 + part) * G * (D + 4);
  for (int i = threadIdx.x; i < G * D; i += kPagedThreads) {
    const int g = i / D;
    float mc = s_m[g];
#pragma unroll
    for (int w = 1; w < kPagedWarps; ++w) mc = fmaxf(mc, s_m[w * ld + g]);
    float t = 0.f, lc = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWarps; ++w) {
      const float m = s_m[w * ld + g], l = s_l[w * ld + g], f = m > -INFINITY ? exp2f(m - mc) : mc > -INFINITY ? 0.f : 1.f;
      t = fmaf(red[(w * G + g) * LD + i % D], f, t);
      lc = l != l ? NAN : fmaf(l, f, lc);
    }
    if (whole) {
      ((T*)a.out)[((size_t)b * p.Hq + (size_t)h * G) * D + i] = Elem<T>::from_float(t / lc);
      if (i % D == 0) a.lse2[sl * G + g] = mc + log2f(lc);
    } else {
      to[g * (D + 4) + i % D] = t;
      if (i % D == 0) { to[g * (D + 4) + D] = mc; to[g * (D + 4) + D + 1] = lc; }
    }
  }
  if (i0 == 0 && threadIdx.x == 0)
    a.desc[sl] = whole ? make_int4(c, -1, 0, 0) : make_int4(c, share_of_tile(start.tot, start.share, before + span.tiles - 1), part, 0);
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
    finish_part<T, D, G, D>(a, start, at == first ? 0 : 1, sl, i0, i1, span, before, red, &s_m[0][0], &s_l[0][0], G);
    __syncthreads();                                         // before the exchange area is written again
    at = before + i1;
    before += span.tiles;
  }
}

// ------------------------------------------------------------------------------------ 16-bit caches: mma.sync
// Every warp takes every eighth tile of its CTA's share, through a ring of its own in shared memory that tiled tensor maps fill (128-
// byte swizzle; one lane asks for the tile three ahead, across slices): nothing waits for another warp but the end of a part.  Logits:
// rows x heads = K q^T on m16n8k16 (the up to eight heads are the columns); outputs: d x heads = V^T P with the weights as two 16-bit
// terms, so that they keep 16 (bf16) or 22 (fp16) bits.  Tiles at the edge of what is seen have their unseen value rows zeroed in shared
// memory (0 * NaN), and the new token's row put in its place.
constexpr int kPagedStages = 3;

struct PagedMaps { CUtensorMap k, v; };

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A warp's place in the tiles of its CTA: tile `at` of all, in slice `sl`, which begins at tile `before`.
struct PagedCursor {
  long long at, before;
  int sl;
  PagedSpan span;
  __device__ __forceinline__ PagedCursor(const PagedDecodeArgs& a, long long at_, long long last, long long before_, int sl_)
      : at(at_), before(before_), sl(sl_), span(a.p.len[sl_], a.p.reach(), a.window, a.n_sink) { settle(a, last); }
  __device__ __forceinline__ void settle(const PagedDecodeArgs& a, long long last) {
    while (at < last && at >= before + span.tiles) {
      before += span.tiles;
      ++sl;
      span = PagedSpan(a.p.len[sl], a.p.reach(), a.window, a.n_sink);
    }
  }
  __device__ __forceinline__ int row0() const { return span.row0((int)(at - before)); }
};

template <typename T, int D, int G>
__global__ void __launch_bounds__(kPagedThreads, 1)
paged_decode_tc_kernel(PagedDecodeArgs a, const __grid_constant__ PagedMaps maps) {
  start_dependents();
  constexpr int HALVES = D / 64, TILE = kPagedTile * D * 2, LD = D + 8;
  extern __shared__ __align__(1024) unsigned char paged_smem[];
  unsigned char* ring = paged_smem;                          // [warps][stages][K, V][D / 64][16 rows][128 B]
  float* red = reinterpret_cast<float*>(paged_smem + (size_t)kPagedWarps * kPagedStages * 2 * TILE);       // [warps][G][LD]
  __shared__ unsigned long long s_full[kPagedWarps][kPagedStages];
  __shared__ int s_row[kPagedWarps][kPagedStages];           // pool row of the stage's tile; -1: bad page
  __shared__ float s_m[kPagedWarps][8], s_l[kPagedWarps][8];
  __shared__ long long s_scan[kPagedWarps + 1];
  __shared__ int s_found;
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3, c = blockIdx.x;
  if (lane == 0)
    for (int s = 0; s < kPagedStages; ++s) tc::mbar_init(&s_full[warp][s], 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  wait_for_prior_grid();
  asm volatile("fence.proxy.async.global;" ::: "memory");    // rows that kernels ahead wrote with ordinary stores are read by copies
  const PagedStart start = paged_start(a, c, s_scan, &s_found);
  if (start.slice < 0) return;
  const long long first = share_begin(start.tot, start.share, c), last = share_begin(start.tot, start.share, c + 1);
  unsigned char* my_ring = ring + (size_t)warp * kPagedStages * 2 * TILE;

  // ---- requests: the cursor is one tile ahead of them, its page number on the way
  PagedCursor ask(a, first + warp, last, start.before, start.slice);
  auto page_row = [&](const PagedCursor& x) {
    if (x.at >= last) return -1;
    const int r = x.row0(), row0 = p.page_row0(x.sl / p.Hkv, x.sl % p.Hkv, r);
    return row0 < 0 ? -1 : row0 + p.in_page(r);
  };
  int asked = 0, ask_row = page_row(ask);
  auto request = [&]() {
    if (ask.at >= last) return;
    const int s = asked % kPagedStages;
    if (lane == 0) {
      s_row[warp][s] = ask_row;
      unsigned char* to = my_ring + s * 2 * TILE;
      if (ask_row >= 0) {
        tc::mbar_expect_tx(&s_full[warp][s], 2 * TILE);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          tc::tma_load_2d(to + h * kPagedTile * 128, &maps.k, h * 64, ask_row, &s_full[warp][s]);
          tc::tma_load_2d(to + TILE + h * kPagedTile * 128, &maps.v, h * 64, ask_row, &s_full[warp][s]);
        }
      } else {
        tc::mbar_arrive(&s_full[warp][s]);
      }
    }
    ++asked;
    ask.at += kPagedWarps;
    ask.settle(a, last);
    ask_row = page_row(ask);
  };
#pragma unroll 1
  for (int s = 0; s < kPagedStages; ++s) request();

  // ---- the parts of the share
  const float scale = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  const int krow = (lane & 7) + ((lane >> 4) & 1) * 8;       // this lane's row of the 16 x 16 tile for ldmatrix
  uint32_t v_off[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) v_off[mt] = (uint32_t)(krow * 128 + (((mt * 2 + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
  PagedCursor cur(a, first, last, start.before, start.slice);            // at: first tile of the part
  long long mine = first + warp;                             // this warp's next tile
  int taken = 0;
  bool lost = false;                                         // a wait ran out: NaN from here on
  while (cur.at < last) {
    const PagedSpan& span = cur.span;
    const int sl = cur.sl, b = sl / p.Hkv, h = sl % p.Hkv;
    const long long end = min(last, cur.before + span.tiles);
    const T* k_new = (const T*)a.k + (size_t)sl * D;
    const T* v_new = (const T*)a.v + (size_t)sl * D;
    uint4 qb[D / 32];                                        // the heads' fragments; columns without a head are zero
    {
      const T* q = (const T*)a.q + ((size_t)b * p.Hq + (size_t)h * G + gid) * D + tig * 16;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) qb[j] = gid < G ? ld_global_v4(q + (j >> 1) * 64 + (j & 1) * 8) : make_uint4(0, 0, 0, 0);
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, acc[D / 16][4];      // of heads 2 tig, 2 tig + 1
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    for (; mine < end; mine += kPagedWarps) {
      const int s = taken % kPagedStages;
      if (!lost && !tc::mbar_wait(&s_full[warp][s], (uint32_t)((taken / kPagedStages) & 1))) {
        lost = true;
        if (lane == 0 && p.status) report_error(p.status, D2O_ERR_TIMEOUT, 0x9A6E3000u);
      }
      lost = __any_sync(0xffffffffu, lost);
      ++taken;
      const int row0 = span.row0((int)(mine - cur.before)), prow = s_row[warp][s];
      unsigned char* stage = my_ring + s * 2 * TILE;
      if (prow < 0 || lost) {
        if (lane == 0 && prow < 0) p.report(kPagedBadPage);
        l[0] = l[1] = NAN;
        __syncwarp();
        if (!lost) request();
        continue;
      }
      const bool edge = !(row0 + kPagedTile <= span.t && (row0 >= span.lo || row0 + kPagedTile <= span.sinks));
      if (edge) {
        for (int x = lane; x < kPagedTile * HALVES * 8; x += 32) {           // 16-byte pieces of value rows
          const int r = x / (HALVES * 8), piece = x % (HALVES * 8);
          if (!span.sees(row0 + r)) *reinterpret_cast<uint4*>(stage + TILE + piece / 8 * kPagedTile * 128 + r * 128 + piece % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        const int rt = span.t - row0;                        // the new token
        if (rt < kPagedTile && lane < HALVES * 8) {
          const uint4 kn = ld_global_v4(k_new + lane * 8), vn = ld_global_v4(v_new + lane * 8);
          const uint32_t to = (uint32_t)(lane / 8 * kPagedTile * 128 + rt * 128 + ((lane % 8 ^ (rt & 7)) << 4));
          *reinterpret_cast<uint4*>(stage + to) = kn;
          *reinterpret_cast<uint4*>(stage + TILE + to) = vn;
          *reinterpret_cast<uint4*>((T*)p.k + ((size_t)prow + rt) * D + lane * 8) = kn;
          *reinterpret_cast<uint4*>((T*)p.v + ((size_t)prow + rt) * D + lane * 8) = vn;
          if (p.pos && lane == 0) p.pos[prow + rt] = a.positions ? a.positions[b] : span.t;
        }
        __syncwarp();
      }
      float x[4];                                            // rows gid (0, 1) and gid + 8 (2, 3), heads 2 tig and 2 tig + 1
      tile_dots<T, D, kPagedTile>(stage, 0, qb, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= scale;
      const bool in0 = !edge || span.sees(row0 + gid), in1 = !edge || span.sees(row0 + gid + 8);
      if (a.logits && 2 * tig < G) {
        float* to = a.logits + ((size_t)prow + gid) * G + 2 * tig;
        if (G == 1) {
          if (in0) to[0] = x[0];
          if (in1) to[8] = x[2];
        } else {
          if (in0) *reinterpret_cast<float2*>(to) = make_float2(x[0], x[1]);
          if (in1) *reinterpret_cast<float2*>(to + 8 * G) = make_float2(x[2], x[3]);
        }
      }
      if (!in0) x[0] = x[1] = -INFINITY;
      if (!in1) x[2] = x[3] = -INFINITY;
      float mx[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])}, f[2];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], o));
        mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], o));
      }
      float w[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float mn = fmaxf(m[e], mx[e]), base = mn > -INFINITY ? mn : 0.f;
        f[e] = exp2f(m[e] - base);                           // nothing so far: 0
        m[e] = mn;
        w[e] = exp2f(x[e] - base); w[e + 2] = exp2f(x[e + 2] - base);
        l[e] = fmaf(l[e], f[e], w[e] + w[e + 2]);            // this thread's rows
      }
      if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) { acc[i][0] *= f[0]; acc[i][1] *= f[1]; acc[i][2] *= f[0]; acc[i][3] *= f[1]; }
      }
      uint32_t h0, l0, h1, l1;
      split_pair<T>(w[0], w[1], h0, l0);
      split_pair<T>(w[2], w[3], h1, l1);
      h0 = transpose_8x8(h0); h1 = transpose_8x8(h1); l0 = transpose_8x8(l0); l1 = transpose_8x8(l1);
      const uint32_t v_u32 = smem_u32(stage + TILE);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t v0, v1, v2, v3;
        ldmatrix_x4_trans(v_u32 + (uint32_t)(i / 4 * kPagedTile * 128) + v_off[i % 4], v0, v1, v2, v3);
        mma_16x8x16<T>(acc[i], v0, v1, v2, v3, h0, h1);
        mma_16x8x16<T>(acc[i], v0, v1, v2, v3, l0, l1);
      }
      if (edge) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // ordinary stores ahead of the next copy
      __syncwarp();
      request();
    }
    // ---- join the warps
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) { l[0] += __shfl_xor_sync(0xffffffffu, l[0], o); l[1] += __shfl_xor_sync(0xffffffffu, l[1], o); }
    if (gid == 0) { s_m[warp][2 * tig] = m[0]; s_m[warp][2 * tig + 1] = m[1]; s_l[warp][2 * tig] = l[0]; s_l[warp][2 * tig + 1] = l[1]; }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      float* to = red + (warp * G + 2 * tig) * LD + i * 16 + gid;
      if (2 * tig < G) { to[0] = acc[i][0]; to[8] = acc[i][2]; }
      if (2 * tig + 1 < G) { to[LD] = acc[i][1]; to[LD + 8] = acc[i][3]; }
    }
    __syncthreads();
    finish_part<T, D, G, LD>(a, start, cur.at == first ? 0 : 1, sl, (int)(cur.at - cur.before), (int)(end - cur.before), span, cur.before, red, &s_m[0][0], &s_l[0][0], 8);
    __syncthreads();                                         // before the exchange area is written again
    cur.at = end;
    cur.settle(a, last);
  }
  if (lost)                                                  // see the copies on their way land before the CTA may end
    for (int i = max(0, asked - kPagedStages); i < asked; ++i)
      if (!tc::mbar_wait(&s_full[warp][i % kPagedStages], (uint32_t)((i / kPagedStages) & 1))) break;
}

// Joins the parts of a slice (blockIdx.x): blockIdx.y < G one head of its output, a warp every eighth part; the others add the
// weights to the scores of the slice's rows, divided over them.  (One CTA and one thread per element for all of a slice's parts, one
// after another, took 21 us for 20 parts.)
template <typename T, int D, int G>
__global__ void __launch_bounds__(kPagedThreads)
join_kernel(PagedDecodeArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int LPR = D / 4, GRPS = kPagedThreads / LPR, GPW = 32 / LPR;      // lanes per row of D floats, row groups, of a warp
  __shared__ float s_lse[G];
  __shared__ float4 s_acc[GRPS][LPR];
  const PagedView& p = a.p;
  const int sl = blockIdx.x, b = sl / p.Hkv, h = sl % p.Hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = p.len[sl];
  if (n < 0) return;
  const PagedSpan span(n, p.reach(), a.window, a.n_sink);
  if (span.t < 0) {                                          // the table has no row for the new token
    if (blockIdx.y == 0 && tid == 0) p.report(kPagedShortTable);
    if (blockIdx.y < G && tid < D) ((T*)a.out)[((size_t)b * p.Hq + (size_t)h * G + blockIdx.y) * D + tid] = Elem<T>::from_float(NAN);
    return;
  }
  const int4 desc = a.desc[sl];
  const bool whole = desc.y < 0;
  auto part = [&](int c, int g) { return a.parts + (((size_t)c * 2 + (c == desc.x ? desc.z : 0)) * G + g) * (D + 4); };
  // largest maximum and sum of a head's parts, by a warp
  auto total = [&](int g, float& m, float& l) {
    m = -INFINITY; l = 0.f;
    for (int c = desc.x + lane; c <= desc.y; c += 32) {
      const float2 x = *reinterpret_cast<const float2*>(part(c, g) + D);
      const float mn = fmaxf(m, x.x);
      l = (m > -INFINITY ? l * exp2f(m - mn) : l) + (x.x > -INFINITY ? x.y * exp2f(x.x - mn) : x.y);      // nothing finite: 0 or NaN
      m = mn;
    }
    const float mc = warp_max(m);
    l = warp_sum(m > -INFINITY ? l * exp2f(m - mc) : l);
    m = mc;
  };
  if (blockIdx.y < G) {
    if (whole) return;
    const int g = blockIdx.y, grp = tid / LPR, lig = tid % LPR;
    float m, l;
    total(g, m, l);                                          // by every warp: the same
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = desc.x + grp; c <= desc.y; c += GRPS) {
      const float* x = part(c, g);
      const float4 v = *reinterpret_cast<const float4*>(x + lig * 4);
      const float f = x[D] > -INFINITY ? exp2f(x[D] - m) : 0.f;
      t.x = fmaf(v.x, f, t.x); t.y = fmaf(v.y, f, t.y); t.z = fmaf(v.z, f, t.z); t.w = fmaf(v.w, f, t.w);
    }
    s_acc[grp][lig] = t;
    __syncthreads();
    if (tid < LPR) {
      t = s_acc[0][tid];
#pragma unroll
      for (int i = 1; i < GRPS; ++i) { t.x += s_acc[i][tid].x; t.y += s_acc[i][tid].y; t.z += s_acc[i][tid].z; t.w += s_acc[i][tid].w; }
      T* out = (T*)a.out + ((size_t)b * p.Hq + (size_t)h * G + g) * D + tid * 4;
      out[0] = Elem<T>::from_float(t.x / l); out[1] = Elem<T>::from_float(t.y / l);
      out[2] = Elem<T>::from_float(t.z / l); out[3] = Elem<T>::from_float(t.w / l);
    }
    return;
  }
  if (whole) {
    if (tid < G) s_lse[tid] = a.lse2[sl * G + tid];
  } else if (warp < G) {
    float m, l;
    total(warp, m, l);
    if (lane == 0) s_lse[warp] = m + log2f(l);
  }
  __syncthreads();
  float lse[G];
#pragma unroll
  for (int g = 0; g < G; ++g) lse[g] = s_lse[g];
  const int stride = (int)(gridDim.y - G) * kPagedThreads;
#pragma unroll 2
  for (int i = (int)(blockIdx.y - G) * kPagedThreads + tid; i < span.tiles * kPagedTile; i += stride) {
    const int r = span.row0(i / kPagedTile) + i % kPagedTile;
    if (!span.sees(r)) continue;
    const int page0 = p.page_row0(b, h, r);
    if (page0 < 0) continue;
    const size_t at = (size_t)page0 + p.in_page(r);
    const float was = r == span.t ? 0.f : p.score[at];
    float x[G];
    if constexpr (G == 1) x[0] = a.logits[at];
    else if constexpr (G == 2) *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(a.logits + at * 2);
    else
#pragma unroll
      for (int g = 0; g < G; g += 4) *reinterpret_cast<float4*>(x + g) = *reinterpret_cast<const float4*>(a.logits + at * G + g);
    float w = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) w += exp2f(x[g] - lse[g]);
    p.score[at] = was + w;
  }
}

// ------------------------------------------------------------------------------------ launch
template <typename T, int D, int G>
static cudaError_t launch_one(const PagedDecodeArgs& a, cudaStream_t st) {
  const int n_slices = a.p.B * a.p.Hkv;
  cudaError_t e;
  if constexpr (sizeof(T) == 4) {
    const size_t smem = (size_t)kPagedWarps * G * D * 4;
    e = cudaFuncSetAttribute(paged_decode_kernel<T, D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = launch_behind(paged_decode_kernel<T, D, G>, dim3((unsigned)a.ctas), kPagedThreads, smem, st, a);
  } else {
    const size_t smem = (size_t)kPagedWarps * (kPagedStages * 2 * kPagedTile * D * 2 + G * (D + 8) * 4);
    PagedMaps maps;
    const int dtype = cuda::std::is_same<T, __half>::value ? D2O_F16 : D2O_BF16;
    const uint64_t rows = (uint64_t)a.p.n_pages * a.p.Hkv << a.p.page_shift;
    if (!encode_rows_2d(&maps.k, dtype, a.p.k, rows, D, kPagedTile) || !encode_rows_2d(&maps.v, dtype, a.p.v, rows, D, kPagedTile))
      return cudaErrorNotSupported;
    e = cudaFuncSetAttribute(paged_decode_tc_kernel<T, D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = launch_behind(paged_decode_tc_kernel<T, D, G>, dim3((unsigned)a.ctas), kPagedThreads, smem, st, a, maps);
  }
  if (e != cudaSuccess) return e;
  int y = 0;                                                 // CTAs per slice that share the scores: up to four per SM, 1024 rows each at least
  if (a.logits) {
    const long long reach = (long long)a.p.max_pages << a.p.page_shift;
    y = (int)std::max<long long>(1, std::min<long long>((4 * a.ctas + n_slices - 1) / n_slices, reach / 1024));
  }
  return launch_behind(join_kernel<T, D, G>, dim3((unsigned)n_slices, (unsigned)(G + y)), kPagedThreads, 0, st, a);
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
