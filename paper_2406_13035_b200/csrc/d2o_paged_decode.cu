// Decode attention over a cache in pages (Eq. 2-3), with the accumulation of Eq. 6 (case 2).
//
// The rows that the new tokens see are counted in tiles of 16, slice after slice (slice = sequence and KV head), and every
// CTA takes an equal share of all tiles: a batch of any lengths, or one long sequence, fills the GPU evenly without the host
// knowing a length.  A share covers parts of one or several slices.  For each part a CTA forms a running softmax (maximum,
// sum, un-normalised output) per query head; a slice that lies in one share is finished there, the parts of the others are
// joined, in the order of the shares, by the CTA that is done with its part last (a counter per slice says so): one launch, which
// matters to a host that launches step by step (4 us each).  Few short slices get a cluster each instead (paged_cluster).  With scores
// the logits go to scratch on the way, and score_kernel, which knows the normalisers, adds the weights to the rows' scores.
//
// Bound by HBM where there is enough to read, by a chain of dependent steps elsewhere (lengths, page numbers, rows, softmax, join).
// us: one sequence of 131072 rows (8 KV heads of four query heads, bf16, d = 128: 537 MB) 89 - 94 (5.7 - 6.0 TB/s; the slowest SMs take 15 %
// longer than the mean), heads of one or two 87, of eight 95; d = 64 with heads of one 49 (5.5 TB/s), four 52, eight 69 (3.9); fp32 211 (5.1), d = 64
// 99 (5.4); 32 sequences of up to 16384 rows under a window of 2048 (270 MB) 54; 8 of up to 4096 rows, 32 heads, with scores (255 MB) 54; in a graph
// one of 1640 rows 8.6, 25 of up to 8 rows 9.0.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "d2o_common.cuh"
#include "d2o_decode.cuh"
#include "d2o_paged.cuh"
#include "d2o_tc.cuh"

namespace cg = cooperative_groups;

namespace d2o {

constexpr int kPagedThreads = 256;           // of score_kernel
constexpr int kPagedWarpsF32 = 8;            // of a CTA
// 16-bit caches: a warp's time per tile is latency (two instructions of ten issued), so that as many warps as shared memory has
// rings of two tiles for, beside their results; eight heads leave room for eight warps, with three.
__host__ __device__ constexpr int paged_warps(int G) { return G <= 4 ? 12 : 8; }
__host__ __device__ constexpr int paged_stages(int G) { return G <= 4 ? 2 : 3; }
constexpr int kPagedClusters = 4;            // cluster sizes 1 (none), 2, 4, 8
constexpr int kPagedMinTiles = 8;            // least share of a CTA where slices are long: a tile for most of its warps
constexpr int kPagedSnap = 8;

struct PagedDecodeArgs {
  PagedView p;
  const void *q, *k, *v;                     // [B, Hq, d], [B, Hkv, d] x 2
  void* out;                                 // [B, Hq, d]
  const int32_t* positions;                  // [B], or NULL
  int window, n_sink;
  int ctas;                                  // CTAs of the first kernel
  uint32_t* done;                            // per slice: parts that are written; zero between launches
  float* lse2;                               // [slices][G] normalisers in the log2 domain (with scores)
  float* parts;                              // [ctas][2][G][D + 4]: output, maximum, sum, -; 0: of a slice that ends in the share, 1: that goes on
  float* logits;                             // per row of the pools, G logits in the log2 domain (with scores)
  unsigned long long wait_ns;                // limit of every wait (16-bit kernel)
  int stop_stage;                            // failure-detection tests: the tile of this number of every CTA's share is not copied; -1: none
};

// a / b; nearly always both fit 32 bits, and a division of 64 bits is a hundred instructions
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
// The shares of all tiles: the first `more` CTAs take size + 1 of them, the others, up to `share`, size.  A border fewer than kPagedSnap
// tiles from a border between slices moves there: a part costs more than that many tiles (a CTA has a warp for each), and slices of fewer
// than twice as many tiles stay whole.
struct PagedShares {
  long long tot, size;
  int share, more;
  __device__ __forceinline__ PagedShares() {}
  __device__ __forceinline__ PagedShares(long long tot_, int ctas, int n_slices) : tot(tot_) {
    share = (int)min((long long)ctas, max(quotient(tot + kPagedMinTiles - 1, kPagedMinTiles), min((long long)n_slices, tot)));
    size = share ? quotient(tot, share) : 0;
    more = (int)(tot - size * share);
  }
  __device__ __forceinline__ long long border(int c) const { return c * size + min(c, more); }       // before it moves
  __device__ __forceinline__ int of_tile(long long tile) const {
    const long long head = more * (size + 1);
    return tile < head ? (int)quotient(tile, size + 1) : more + (int)quotient(tile - head, size);
  }
  static __device__ __forceinline__ long long snap(long long x, long long before, int tiles) {         // a border in that slice
    return x - before < kPagedSnap ? before : before + tiles - x < kPagedSnap ? before + tiles : x;
  }
  // first and last share with tiles of a slice that more than one has: those that end or begin at its unmoved borders
  __device__ __forceinline__ int first_of(long long before) const { return of_tile(before + kPagedSnap - 1); }
  __device__ __forceinline__ int last_of(long long before, int tiles) const { return of_tile(before + tiles - kPagedSnap); }
};

// A CTA's share: tiles first .. last, and the slice in which it begins.  Every CTA adds up the tiles of all slices: a thread
// those of consecutive slices, then a scan over the block.
struct PagedStart {
  PagedShares shares;
  long long first, last;
  long long before;                          // tiles ahead of `slice`
  int slice;                                 // -1: no share
  int n;                                     // rows that it holds
};
struct PagedStartShared {
  long long sum[16], border[2], before;
  int slice, n;
};
template <int NW, typename F>
__device__ __forceinline__ PagedStart paged_start(const PagedDecodeArgs& a, int c, PagedStartShared& sh, F&& short_table) {
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_slices = p.B * p.Hkv, per = (n_slices + (NW * 32) - 1) / (NW * 32);
  const int s0 = min(n_slices, tid * per), s1 = min(n_slices, s0 + per);
  long long mine = 0;
  for (int s = s0; s < s1; ++s) {
    const int n = p.len[s];
    mine += PagedSpan(n, p.reach(), a.window, a.n_sink).tiles;
    if (c == 0 && n >= p.reach()) short_table(s);            // no row for the new token
  }
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += t; }
  if (lane == 31) sh.sum[warp] = inc;
  __syncthreads();
  long long base = 0, tot = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) { if (w < warp) base += sh.sum[w]; tot += sh.sum[w]; }
  PagedStart r;
  r.shares = PagedShares(tot, a.ctas, n_slices); r.slice = -1;
  if (c >= r.shares.share) return r;
  const long long at0 = base + inc - mine;
  for (int e = 0; e < 2; ++e) {                              // its two borders
    const long long x = r.shares.border(c + e);
    if (x >= at0 && x < at0 + mine) {                        // one thread
      long long at = at0;
      int s = s0, n, tiles;
      for (;; ++s) {
        n = p.len[s];
        tiles = PagedSpan(n, p.reach(), a.window, a.n_sink).tiles;
        if (x < at + tiles) break;
        at += tiles;
      }
      sh.border[e] = PagedShares::snap(x, at, tiles);
      if (e == 0) { sh.slice = s; sh.n = n; sh.before = at; }
    }
    if (x == tot && tid == 0) sh.border[e] = tot;
  }
  __syncthreads();
  r.first = sh.border[0]; r.last = sh.border[1]; r.before = sh.before; r.n = sh.n;
  if (r.first < r.last) r.slice = sh.slice;
  return r;
}

// The share of a CTA in a cluster per slice: its first tile, and behind its last one, of the slice's.  -1: nothing to do.
template <typename F>
__device__ __forceinline__ PagedStart cluster_start(const PagedDecodeArgs& a, F&& short_table) {
  const cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), r = (int)cluster.block_rank(), sl = (int)blockIdx.x / C, n = a.p.len[sl];
  const PagedSpan span(n, a.p.reach(), a.window, a.n_sink);
  if (n >= a.p.reach() && r == 0 && threadIdx.x == 0) short_table(sl);
  PagedStart s;
  s.first = span.tiles * r / C; s.last = span.tiles * (r + 1) / C;
  s.slice = span.t < 0 ? -1 : sl; s.before = 0; s.n = n;
  return s;
}

// A slice whose table has no row for the new token: NaN, by one thread.
template <typename T, int D, int G>
__device__ __forceinline__ void short_table_output(const PagedDecodeArgs& a, int sl) {
  a.p.report(kPagedShortTable);
  T* out = (T*)a.out + ((size_t)(sl / a.p.Hkv) * a.p.Hq + (size_t)(sl % a.p.Hkv) * G) * D;
  for (int i = 0; i < G * D; ++i) out[i] = Elem<T>::from_float(NAN);
}

// Joins the parts that the shares c0 .. c1 have of a slice (in c1, where it ends, place 0; in those that it goes on behind, place 1).  NW / G warps per head,
// each every so many parts, whose results are added in shared memory: the order is that of the shares whatever CTA does it.
template <typename T, int D, int G, int NW>
__device__ __forceinline__ void join_parts(const PagedDecodeArgs& a, int sl, int c0, int c1, float4* s_acc /* [warps][D / 4] */) {
  constexpr int LPR = D / 4, RPW = 32 / LPR, W = NW / G, STEP = W * RPW;        // lanes per row of D floats, rows of a warp, warps per head
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = min(warp / W, G - 1), sub = warp % W, lig = lane % LPR;
  const bool spare = warp >= W * G;                          // more warps than heads take
  auto part = [&](int c) { return a.parts + (((size_t)c * 2 + (c < c1 ? 1 : 0)) * G + g) * (D + 4); };
  // the first outputs on their way beside the maxima
  constexpr int AHEAD = 2;
  float4 ahead[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int k = i * STEP + sub * RPW + lane / LPR;
    ahead[i] = c0 + k <= c1 && k < 32 ? __ldcg(reinterpret_cast<const float4*>(part(c0 + k) + lig * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // the largest maximum and the sum; the first 32 parts' maxima stay in registers
  float m = -INFINITY, l = 0.f, m0 = -INFINITY;
  for (int c = c0 + lane; c <= c1; c += 32) {
    const float2 x = __ldcg(reinterpret_cast<const float2*>(part(c) + D));
    const float mn = fmaxf(m, x.x);
    l = (m > -INFINITY ? l * exp2f(m - mn) : l) + (x.x > -INFINITY ? x.y * exp2f(x.x - mn) : x.y);        // nothing finite: 0 or NaN
    m = mn;
    if (c < c0 + 32) m0 = x.x;
  }
  const float mc = warp_max(m);
  l = warp_sum(m > -INFINITY ? l * exp2f(m - mc) : l);
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int base = c0; base <= c1; base += 32) {
    const float mx = base == c0 ? m0 : base + lane <= c1 ? __ldcg(part(base + lane) + D) : -INFINITY;
    const float f = mx > -INFINITY ? exp2f(mx - mc) : 0.f;   // of part base + lane
    const int n = min(32, c1 - base + 1);
    if (base == c0) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int k = i * STEP + sub * RPW + lane / LPR;
        const float w = __shfl_sync(0xffffffffu, f, k & 31);
        if (k < n) { t.x = fmaf(ahead[i].x, w, t.x); t.y = fmaf(ahead[i].y, w, t.y); t.z = fmaf(ahead[i].z, w, t.z); t.w = fmaf(ahead[i].w, w, t.w); }
      }
    }
#pragma unroll 2
    for (int i = base == c0 ? AHEAD * STEP : 0; i < n; i += STEP) {
      const int k = i + sub * RPW + lane / LPR;
      const float w = __shfl_sync(0xffffffffu, f, k & 31);
      if (k < n) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(part(base + k) + lig * 4));
        t.x = fmaf(v.x, w, t.x); t.y = fmaf(v.y, w, t.y); t.z = fmaf(v.z, w, t.z); t.w = fmaf(v.w, w, t.w);
      }
    }
  }
  if (RPW == 2) {
    t.x += __shfl_xor_sync(0xffffffffu, t.x, 16); t.y += __shfl_xor_sync(0xffffffffu, t.y, 16);
    t.z += __shfl_xor_sync(0xffffffffu, t.z, 16); t.w += __shfl_xor_sync(0xffffffffu, t.w, 16);
  }
  if (lane < LPR) s_acc[warp * LPR + lane] = t;
  if (a.logits && sub == 0 && lane == 0 && !spare) a.lse2[sl * G + g] = mc + log2f(l);
  __syncthreads();
  if (sub == 0 && lane < LPR && !spare) {
#pragma unroll
    for (int i = 1; i < W; ++i) {
      const float4 u = s_acc[(warp + i) * LPR + lane];
      t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
    }
    T* out = (T*)a.out + ((size_t)(sl / a.p.Hkv) * a.p.Hq + (size_t)(sl % a.p.Hkv) * G + g) * D + lane * 4;
    out[0] = Elem<T>::from_float(t.x / l); out[1] = Elem<T>::from_float(t.y / l);
    out[2] = Elem<T>::from_float(t.z / l); out[3] = Elem<T>::from_float(t.w / l);
  }
}

// Parts of slices that other shares continue: at most the share's first and its last.
struct PagedOpen {
  int n = 0, sl[2], tiles[2];
  long long before[2];
  __device__ __forceinline__ void add(int sl_, long long before_, int tiles_) {
    // two constant places, not an indexed one: registers
    if (n == 0) { sl[0] = sl_; before[0] = before_; tiles[0] = tiles_; }
    else { sl[1] = sl_; before[1] = before_; tiles[1] = tiles_; }
    ++n;
  }
};

// The warps' results of one part (tiles i0 .. i1 of slice `sl`) become the slice's output, or one of the parts to be joined.  s_m, s_l:
// maxima and sums [warps][ld]; the maxima become the warps' factors.  CL: a part for join_cluster, in shared memory.  Begins and ends behind a barrier of the caller's.
template <typename T, int D, int G, int LD, bool CL>
__device__ __forceinline__ void finish_part(const PagedDecodeArgs& a, PagedOpen& open, float* swap, int part, int sl, int i0, int i1,
                                            const PagedSpan& span, long long before, const float* red, float* s_m, float* s_l, int ld) {
  const PagedView& p = a.p;
  const int tid = threadIdx.x, c = blockIdx.x, b = sl / p.Hkv, h = sl % p.Hkv;
  const bool whole = !CL && i0 == 0 && i1 == span.tiles;
  float* to = CL ? swap : a.parts + ((size_t)c * 2 + part) * G * (D + 4);
  if (tid < G) {
    float m[kPagedWarpsF32], mc = -INFINITY, lc = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWarpsF32; ++w) { m[w] = s_m[w * ld + tid]; mc = fmaxf(mc, m[w]); }
#pragma unroll
    for (int w = 0; w < kPagedWarpsF32; ++w) {
      const float l = s_l[w * ld + tid], f = m[w] > -INFINITY ? exp2f(m[w] - mc) : mc > -INFINITY ? 0.f : 1.f;
      s_m[w * ld + tid] = f;
      lc = l != l ? NAN : fmaf(l, f, lc);
    }
    s_l[tid] = lc;
    if (!whole) *reinterpret_cast<float2*>(to + tid * (D + 4) + D) = make_float2(mc, lc);
    else if (a.logits) a.lse2[sl * G + tid] = mc + log2f(lc);
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < (G * D + (kPagedWarpsF32 * 32) - 1) / (kPagedWarpsF32 * 32); ++x) {
    const int i = x * (kPagedWarpsF32 * 32) + tid, g = i / D;
    if (G * D < (kPagedWarpsF32 * 32) && i >= G * D) break;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWarpsF32; ++w) t = fmaf(red[(w * G + g) * LD + i % D], s_m[w * ld + g], t);
    if (whole) ((T*)a.out)[((size_t)b * p.Hq + (size_t)h * G) * D + i] = Elem<T>::from_float(t / s_l[g]);
    else to[g * (D + 4) + i % D] = t;
  }
  if (!CL && !whole) open.add(sl, before, span.tiles);
}

// Joins the parts of a cluster's CTAs, which lie in their shared memory at `swap` ([G][D + 4]; `empty`: this CTA had no tiles).
template <typename T, int D, int G, int NW>
__device__ __forceinline__ void join_cluster(const PagedDecodeArgs& a, int sl, float* swap, bool empty) {
  constexpr int MAX = 1 << (kPagedClusters - 1);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), tid = threadIdx.x;
  if (empty)
    for (int i = tid; i < G * (D + 4); i += (NW * 32)) swap[i] = i % (D + 4) == D ? -INFINITY : 0.f;
  cluster.sync();
  if (cluster.block_rank() == 0) {
#pragma unroll
    for (int x = 0; x < (G * D + (NW * 32) - 1) / (NW * 32); ++x) {
      const int i = x * (NW * 32) + tid, g = i / D;
      if (i >= G * D) break;
      float2 ml[MAX];
      float v[MAX], mc = -INFINITY, t = 0.f, l = 0.f;
#pragma unroll
      for (int r = 0; r < MAX; ++r) {
        const float* y = cluster.map_shared_rank(swap, r < C ? r : 0) + g * (D + 4);
        ml[r] = *reinterpret_cast<const float2*>(y + D);
        v[r] = y[i % D];
      }
#pragma unroll
      for (int r = 0; r < MAX; ++r)
        if (r < C) mc = fmaxf(mc, ml[r].x);
#pragma unroll
      for (int r = 0; r < MAX; ++r) {
        const float f = r < C ? (ml[r].x > -INFINITY ? exp2f(ml[r].x - mc) : mc > -INFINITY ? 0.f : 1.f) : 0.f;
        t = r < C ? fmaf(v[r], f, t) : t;
        l = r < C ? (ml[r].y != ml[r].y ? NAN : fmaf(ml[r].y, f, l)) : l;
      }
      ((T*)a.out)[((size_t)(sl / a.p.Hkv) * a.p.Hq + (size_t)(sl % a.p.Hkv) * G) * D + i] = Elem<T>::from_float(t / l);
      if (a.logits && i % D == 0) a.lse2[sl * G + g] = mc + log2f(l);
    }
  }
  cluster.sync();                                            // the others' parts have been read
}

// Counts the CTA's open parts, and joins the slices of which they were the last.
template <typename T, int D, int G, int NW>
__device__ __forceinline__ void close_parts(const PagedDecodeArgs& a, const PagedStart& start, const PagedOpen& open, float* red, int4* s_join /* [2] */) {
  if (open.n == 0) return;                                   // the caller's barrier lies behind the last part
  // thread x looks after part x
  if (threadIdx.x < open.n) {
    const int x = threadIdx.x, sl = x ? open.sl[1] : open.sl[0], tiles = x ? open.tiles[1] : open.tiles[0];
    const long long first = x ? open.before[1] : open.before[0];
    const int c0 = start.shares.first_of(first), c1 = start.shares.last_of(first, tiles);
    uint32_t before;
    // the CTA's stores, ordered ahead of this thread by the barrier, become visible with the count; with the last count the others' are
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.done + sl) : "memory");
    const bool all = before == (uint32_t)(c1 - c0);
    if (all) a.done[sl] = 0u;                                // for the next launch
    s_join[x] = make_int4(all ? sl : -1, c0, c1, 0);
  }
  __syncthreads();
#pragma unroll 1                                             // code that is run once comes from far: half of it
  for (int x = 0; x < open.n; ++x) {
    const int4 j = s_join[x];
    if (j.x < 0) continue;
    join_parts<T, D, G, NW>(a, j.x, j.y, j.z, reinterpret_cast<float4*>(red));
    __syncthreads();                                         // before the exchange area is written again
  }
}

template <typename T, int D, int G, bool CL>
__global__ void __launch_bounds__(kPagedWarpsF32 * 32, 1)
paged_decode_kernel(PagedDecodeArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPW = 32 / LPR, U = kPagedTile / RPW, QL = LPR / 4;
  extern __shared__ __align__(16) float red[];               // [warps][G][D]
  __shared__ float s_m[kPagedWarpsF32][G], s_l[kPagedWarpsF32][G];
  __shared__ PagedStartShared s_start;
  __shared__ int4 s_join[2];
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int grp = lane / LPR, lig = lane % LPR, c = blockIdx.x;
  auto short_table = [&](int sl) { short_table_output<T, D, G>(a, sl); };
  const PagedStart start = CL ? cluster_start(a, short_table) : paged_start<kPagedWarpsF32>(a, c, s_start, short_table);
  if (start.slice < 0) return;
  const long long first = start.first, last = start.last;
  float* swap = red + kPagedWarpsF32 * G * D;                   // [G][D + 4], clusters
  long long before = start.before;
  int sl = start.slice;
  PagedOpen open;
  for (long long at = first; at < last; ++sl) {
    const PagedSpan span(p.len[sl], p.reach(), a.window, a.n_sink);
    if (at >= before + span.tiles) { before += span.tiles; continue; }       // absent, or the share begins behind it
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
    for (int i = i0 + warp; i < i1; i += kPagedWarpsF32) {
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
    finish_part<T, D, G, D, CL>(a, open, swap, i1 < span.tiles ? 1 : 0, sl, i0, i1, span, before, red, &s_m[0][0], &s_l[0][0], G);
    __syncthreads();                                         // before the exchange area is written again
    at = before + i1;
    before += span.tiles;
  }
  if (CL) join_cluster<T, D, G, kPagedWarpsF32>(a, start.slice, swap, first == last);
  else close_parts<T, D, G, kPagedWarpsF32>(a, start, open, red, s_join);
}

// ------------------------------------------------------------------------------------ 16-bit caches: mma.sync
// Every warp takes every twelfth (eighth) tile of its CTA's share, through a ring of its own in shared memory that tiled tensor maps fill (128-
// byte swizzle; one lane asks for the tiles ahead, across slices): nothing waits for another warp but the end of a part.  Logits:
// rows x heads = K q^T on m16n8k16 (the up to eight heads are the columns); outputs: d x heads = V^T P with the weights as two 16-bit
// terms, so that they keep 16 (bf16) or 22 (fp16) bits.  The references m of fp16 weights 2^(x - m) lie 14 below the maximum: the largest
// weight is 2^14, and those below 2^-16 of it, whose second term is subnormal, are off by up to 2^-39 of it (2^-25 with the
// reference at the maximum, half a percent of a weight of 2^-17).  Tiles at the edge of what is seen have their unseen value rows zeroed in shared
// memory (0 * NaN), and the new token's row put in its place.
struct PagedMaps { CUtensorMap k, v; };

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Two weights as 16-bit terms, hi strictly below a weight that is not zero and lo the rest, rounded: both positive, so that an infinite value gives
// infinity (0 * inf would be NaN, and so would the sum with a negative second term).  fp16: down to weights of 2^-13, below which lo may round to zero.
template <typename T>
__device__ __forceinline__ void split_below(float x, float y, uint32_t& hi, uint32_t& lo) {
  const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y), xd = xb - min(xb, 1u), yd = yb - min(yb, 1u);
  if constexpr (cuda::std::is_same<T, __nv_bfloat16>::value) {
    hi = __byte_perm(xd, yd, 0x7632);                        // the upper halves
    const __nv_bfloat162 l = __floats2bfloat162_rn(x - __uint_as_float(xd & 0xffff0000u), y - __uint_as_float(yd & 0xffff0000u));
    lo = *reinterpret_cast<const uint32_t*>(&l);
  } else {
    const __half xh = __float2half_rz(__uint_as_float(xd)), yh = __float2half_rz(__uint_as_float(yd));
    const __half2 h = __halves2half2(xh, yh), l = __floats2half2_rn(x - __half2float(xh), y - __half2float(yh));
    hi = *reinterpret_cast<const uint32_t*>(&h); lo = *reinterpret_cast<const uint32_t*>(&l);
  }
}

// A warp's place in the tiles of its CTA: tile `at` of all, in slice `sl`, which begins at tile `before`.
struct PagedCursor {
  long long at, before;
  int sl, b, h;
  PagedSpan span;
  __device__ __forceinline__ PagedCursor(const PagedDecodeArgs& a, const PagedStart& start, long long at_, long long last)
      : at(at_), before(start.before), sl(start.slice), b(start.slice / a.p.Hkv), h(start.slice % a.p.Hkv), span(start.n, a.p.reach(), a.window, a.n_sink) {
    settle(a, last);
  }
  __device__ __forceinline__ void settle(const PagedDecodeArgs& a, long long last) {
    while (at < last && at >= before + span.tiles) {
      before += span.tiles;
      ++sl;
      if (++h == a.p.Hkv) { h = 0; ++b; }
      span = PagedSpan(a.p.len[sl], a.p.reach(), a.window, a.n_sink);
    }
  }
  __device__ __forceinline__ int row0() const { return span.row0((int)(at - before)); }
};

// Buffers for the warps' results: two where shared memory has the room
__host__ __device__ constexpr int paged_buffers(int G) { return G <= 2 ? 2 : 1; }

// One warp adds the results of all warps for one part ([warps][G][LD] outputs, [warps][G, even] maxima and sums): the slice's output, or a part
// for the joins in `to` ([G][D + 4]).  `lost`: not all results are there, NaN.
template <typename T, int D, int G, int LD>
__device__ __forceinline__ void combine_warps(const PagedDecodeArgs& a, int sl, int b, int h, bool whole, bool lost, float* to, const float* red, const float* s_m, const float* s_l) {
  constexpr int WARPS = paged_warps(G);
  static_assert(WARPS <= 16, "sixteen lanes per head");
  constexpr int LPR = D / 4, HEADS = 32 / LPR, N = (G + 1) / 2;          // lanes per row of D floats, heads at a time; factors per lane
  const int lane = threadIdx.x & 31, lig = lane % LPR;
  // lane w + 16 (g % 2), entry g / 2: factor of warp w for head g, and the sum
  float f[N], lc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int w = lane & 15, g = 2 * e + lane / 16;
    const bool in = w < WARPS && g < G;
    const float m = in ? s_m[w * (G + G % 2) + g] : -INFINITY;
    float l = in ? s_l[w * (G + G % 2) + g] : 0.f, mc = m;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) mc = fmaxf(mc, __shfl_xor_sync(0xffffffffu, mc, o));
    f[e] = m > -INFINITY ? exp2f(m - mc) : mc > -INFINITY ? 0.f : 1.f;
    l = lost || l != l ? NAN : l * f[e];                     // a NaN sum of a bad page stays
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    lc[e] = l;
    if (w == 0 && g < G) {
      if (!whole) *reinterpret_cast<float2*>(to + g * (D + 4) + D) = make_float2(mc, l);
      else if (a.logits) a.lse2[sl * G + g] = mc + log2f(l);
    }
  }
#pragma unroll
  for (int g0 = 0; g0 < G; g0 += HEADS) {
    const int g = g0 + lane / LPR;                           // of this lane
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    const int from = (g & 1) * 16;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float x = __shfl_sync(0xffffffffu, f[g0 / 2], from + w);
      if (g < G) {
        const float4 v = *reinterpret_cast<const float4*>(red + (w * G + g) * LD + lig * 4);
        t.x = fmaf(v.x, x, t.x); t.y = fmaf(v.y, x, t.y); t.z = fmaf(v.z, x, t.z); t.w = fmaf(v.w, x, t.w);
      }
    }
    const float l = __shfl_sync(0xffffffffu, lc[g0 / 2], from);
    if (g < G) {
      if (whole) {
        T* out = (T*)a.out + ((size_t)b * a.p.Hq + (size_t)h * G + g) * D + lig * 4;
        out[0] = Elem<T>::from_float(t.x / l); out[1] = Elem<T>::from_float(t.y / l);
        out[2] = Elem<T>::from_float(t.z / l); out[3] = Elem<T>::from_float(t.w / l);
      } else {
        *reinterpret_cast<float4*>(to + g * (D + 4) + lig * 4) = t;
      }
    }
  }
}

template <typename T, int D, int G, bool CL>
__global__ void __launch_bounds__(paged_warps(G) * 32, 1)
paged_decode_tc_kernel(PagedDecodeArgs a, const __grid_constant__ PagedMaps maps) {
  start_dependents();
  constexpr int WARPS = paged_warps(G), STAGES = paged_stages(G), HALVES = D / 64, TILE = kPagedTile * D * 2, LD = D + 8;
  extern __shared__ __align__(1024) unsigned char paged_smem[];
  unsigned char* ring = paged_smem;                          // [warps][stages][K, V][D / 64][16 rows][128 B]
  constexpr int BUFS = paged_buffers(G);
  float* red = reinterpret_cast<float*>(paged_smem + (size_t)WARPS * STAGES * 2 * TILE);       // [BUFS][warps][G][LD]
  __shared__ unsigned long long s_full[WARPS][STAGES], s_written[BUFS], s_free[BUFS];
  __shared__ int s_row[WARPS][STAGES];           // pool row of the stage's tile; -1: bad page
  __shared__ float s_m[BUFS][WARPS][G + G % 2], s_l[BUFS][WARPS][G + G % 2];
  __shared__ PagedStartShared s_start;
  __shared__ int4 s_join[2];
  const PagedView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3, c = blockIdx.x;
  if (lane == 0)
    for (int s = 0; s < STAGES; ++s) tc::mbar_init(&s_full[warp][s], 1);
  if (tid == 0)
    for (int i = 0; i < BUFS; ++i) { tc::mbar_init(&s_written[i], WARPS); tc::mbar_init(&s_free[i], 1); }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  // A warp without a tile arrives at the shared mbarriers after one load: their initialisation comes first.  (The shares have a barrier of the
  // CTA in paged_start.)
  if (CL) __syncthreads();
  wait_for_prior_grid();
  __syncwarp();
  asm volatile("fence.proxy.async.global;" ::: "memory");    // rows that kernels ahead wrote with ordinary stores are read by copies
  auto short_table = [&](int sl) { short_table_output<T, D, G>(a, sl); };
  const PagedStart start = CL ? cluster_start(a, short_table) : paged_start<WARPS>(a, c, s_start, short_table);
  if (start.slice < 0) return;
  const long long first = start.first, last = start.last;
  unsigned char* my_ring = ring + (size_t)warp * STAGES * 2 * TILE;

  // ---- requests: the cursor is one tile ahead of them, its page number on the way
  PagedCursor ask(a, start, first + warp, last);
  auto page_row = [&](const PagedCursor& x) {
    if (x.at >= last) return -1;
    const int r = x.row0(), row0 = p.page_row0(x.b, x.h, r);
    return row0 < 0 ? -1 : row0 + p.in_page(r);
  };
  int asked = 0, ask_row = -1, missing = -1;                 // lane 0: the copy that a test left out
  unsigned long long drop;                                   // read once
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(drop));
  auto copy = [&](long long at, int row) {                   // of the tile at pool row `row`
    if (at >= last) return;
    const int s = asked % STAGES;
    if (lane == 0) {
      s_row[warp][s] = row;
      unsigned char* to = my_ring + s * 2 * TILE;
      if (a.stop_stage >= 0 && at - first == a.stop_stage) {             // never arrives
        missing = asked;
      } else if (row >= 0) {
        tc::mbar_expect_tx(&s_full[warp][s], 2 * TILE);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          tma_load_2d_hint(to + h * kPagedTile * 128, &maps.k, h * 64, row, &s_full[warp][s], drop);
          tma_load_2d_hint(to + TILE + h * kPagedTile * 128, &maps.v, h * 64, row, &s_full[warp][s], drop);
        }
      } else {
        tc::mbar_arrive(&s_full[warp][s]);
      }
    }
    ++asked;
  };
  auto request = [&]() {
    if (ask.at >= last) return;
    copy(ask.at, ask_row);
    ask.at += WARPS;
    ask.settle(a, last);
    ask_row = page_row(ask);
  };
  {
    int rows[STAGES];                                  // the first page numbers, side by side
    long long at[STAGES];
#pragma unroll
    for (int s = 0; s < STAGES; ++s) { rows[s] = page_row(ask); at[s] = ask.at; ask.at += WARPS; ask.settle(a, last); }
    ask_row = page_row(ask);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) copy(at[s], rows[s]);
  }

  // ---- the parts of the share
  const float scale = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  const int krow = (lane & 7) + ((lane >> 4) & 1) * 8;       // this lane's row of the 16 x 16 tile for ldmatrix
  uint32_t v_off[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) v_off[mt] = (uint32_t)(krow * 128 + (((mt * 2 + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
  PagedCursor cur(a, start, first, last);            // at: first tile of the part
  long long mine = first + warp;                             // this warp's next tile
  int taken = 0, parts = 0;
  PagedOpen open;
  bool lost = false;                                         // a wait of this warp ran out: NaN from here on
  auto wait = [&](unsigned long long* bar, uint32_t phase) {             // of the whole warp
    lost = __any_sync(0xffffffffu, lost || !tc::mbar_wait(bar, phase, a.wait_ns));
  };
  while (cur.at < last) {
    const PagedSpan& span = cur.span;
    const int sl = cur.sl, b = cur.b, h = cur.h;
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
    for (; mine < end; mine += WARPS) {
      const int s = taken % STAGES;
      if (!lost) wait(&s_full[warp][s], (uint32_t)((taken / STAGES) & 1));
      ++taken;
      const int row0 = span.row0((int)(mine - cur.before)), prow = s_row[warp][s];
      unsigned char* stage = my_ring + s * 2 * TILE;
      if (prow < 0 || lost) {
        if (lane == 0 && !lost) p.report(kPagedBadPage);
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
        // rounded up: with huge logits the difference is not there, and must not be more
        const float mn = fmaxf(m[e], cuda::std::is_same<T, __half>::value ? __fsub_ru(mx[e], 14.f) : mx[e]), base = mn > -INFINITY ? mn : 0.f;
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
      split_below<T>(w[0], w[1], h0, l0);
      split_below<T>(w[2], w[3], h1, l1);
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
    // ---- the warp's result goes to a buffer; the warp whose turn it is waits for all of them, the others go on
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) { l[0] += __shfl_xor_sync(0xffffffffu, l[0], o); l[1] += __shfl_xor_sync(0xffffffffu, l[1], o); }
    const int buf = parts % BUFS;
    const uint32_t phase = (uint32_t)((parts / BUFS) & 1);
    if (parts >= BUFS && !lost) wait(&s_free[buf], phase ^ 1);
    float* mine_red = red + (size_t)buf * WARPS * G * LD + warp * G * LD;
    if (gid == 0 && 2 * tig < G) {
      // without the buffer, which may be read for the part before: a NaN sum alone, which makes either part NaN
      if (!lost) { s_m[buf][warp][2 * tig] = m[0]; s_m[buf][warp][2 * tig + 1] = m[1]; }
      s_l[buf][warp][2 * tig] = lost ? NAN : l[0]; s_l[buf][warp][2 * tig + 1] = lost ? NAN : l[1];
    }
    if (!lost)
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      float* to = mine_red + 2 * tig * LD + i * 16 + gid;
      if (2 * tig < G) { to[0] = acc[i][0]; to[8] = acc[i][2]; }
      if (2 * tig + 1 < G) { to[LD] = acc[i][1]; to[LD + 8] = acc[i][3]; }
    }
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&s_written[buf]);
    const int i0 = (int)(cur.at - cur.before), i1 = (int)(end - cur.before);
    const bool whole = !CL && i0 == 0 && i1 == span.tiles;
    if (warp == parts % WARPS) {
      if (!lost) wait(&s_written[buf], phase);
      float* to = CL ? reinterpret_cast<float*>(paged_smem) : a.parts + ((size_t)c * 2 + (end < cur.before + span.tiles ? 1 : 0)) * G * (D + 4);
      combine_warps<T, D, G, LD>(a, sl, b, h, whole, lost, to, red + (size_t)buf * WARPS * G * LD, &s_m[buf][0][0], &s_l[buf][0][0]);
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&s_free[buf]);
    }
    if (!CL && !whole) open.add(sl, cur.before, span.tiles);
    ++parts;
    cur.at = end;
    cur.settle(a, last);
  }
  if (__syncthreads_or(lost)) {                              // the last parts are combined
    if (tid == 0 && p.status) report_error(p.status, D2O_ERR_TIMEOUT, 0x9A6E3000u);
    // see the copies on their way land before the CTA may end, and before a cluster's part, which lies in the ring's place, is read
    for (int i = max(0, asked - STAGES); lane == 0 && i < asked; ++i)
      if (i != missing) (void)tc::mbar_wait(&s_full[warp][i % STAGES], (uint32_t)((i / STAGES) & 1));
    __syncthreads();
    if (CL && tid < G) reinterpret_cast<float*>(paged_smem)[tid * (D + 4) + D + 1] = NAN;
  }
  if (CL) join_cluster<T, D, G, WARPS>(a, start.slice, reinterpret_cast<float*>(paged_smem), first == last);
  else close_parts<T, D, G, WARPS>(a, start, open, red, s_join);
}

// Adds the weights to the scores of a slice's rows (blockIdx.x), divided over blockIdx.y.
template <int G>
__global__ void __launch_bounds__(kPagedThreads)
score_kernel(PagedDecodeArgs a) {
  start_dependents();
  wait_for_prior_grid();
  const PagedView& p = a.p;
  const int sl = blockIdx.x, b = sl / p.Hkv, h = sl % p.Hkv;
  const PagedSpan span(p.len[sl], p.reach(), a.window, a.n_sink);
  if (span.t < 0) return;
  float lse[G];
#pragma unroll
  for (int g = 0; g < G; ++g) lse[g] = a.lse2[sl * G + g];
#pragma unroll 4
  for (int i = (int)(blockIdx.y * kPagedThreads + threadIdx.x); i < span.tiles * kPagedTile; i += (int)gridDim.y * kPagedThreads) {
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
// CTAs per slice of a call whose slices get a cluster each, 1: shares of all tiles.  A cluster joins its parts through distributed shared
// memory, in about a microsecond where counters and parts in global memory take five; but it knows no other slice, and one that is much
// longer than the rest is left with its own CTAs.  So: calls whose slices get at least two CTAs each with one CTA per SM, up to eight
// (the portable size; for up to three quarters of the SMs, because sixteen clusters of eight are not resident at once), as long as what
// the table can hold gives a CTA at most 64 tiles (16-bit rows of d = 128: 512 KB, 10 us).  us, shares / clusters, 8 KV heads, d = 128, bf16: one
// sequence of 3000 rows 11.7 / 9.0, of 7000 17.0 / 12.6, two of 3000 15.1 / 11.1 (16.9 with eight CTAs each), four of 3000 16.8 / 11.6; nine
// ragged ones of up to 3500 (beyond the bound) 16.5 / 18.2.  The lengths are not known here: one sequence in a table with room for sixteen times its
// rows gets shares, and their times.
static int paged_cluster(const PagedView& p, int n_slices, int sms) {
  int C = 1;
  while (2 * C <= 1 << (kPagedClusters - 1) && (long)n_slices * 2 * C <= (2 * C < 8 ? sms : sms * 3 / 4)) C *= 2;
  return ((long long)p.max_pages << p.page_shift) <= 64ll * kPagedTile * C ? C : 1;
}

template <typename K, typename... A>
static cudaError_t launch_shares(K kernel, const PagedDecodeArgs& a, int n_slices, int C, int warps, size_t smem, cudaStream_t st, const A&... args) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(C > 1 ? n_slices * C : a.ctas)); cfg.blockDim = dim3((unsigned)warps * 32); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, args...);
}

template <typename T, int D, int G>
static cudaError_t launch_one(const PagedDecodeArgs& a, cudaStream_t st) {
  const int n_slices = a.p.B * a.p.Hkv, C = paged_cluster(a.p, n_slices, a.ctas);
  cudaError_t e;
  if constexpr (sizeof(T) == 4) {
    const size_t smem = (size_t)(kPagedWarpsF32 * G * D + G * (D + 4)) * 4;
    e = C > 1 ? launch_shares(paged_decode_kernel<T, D, G, true>, a, n_slices, C, kPagedWarpsF32, smem, st)
              : launch_shares(paged_decode_kernel<T, D, G, false>, a, n_slices, C, kPagedWarpsF32, smem, st);
  } else {
    const size_t smem = (size_t)paged_warps(G) * (paged_stages(G) * 2 * kPagedTile * D * 2 + paged_buffers(G) * G * (D + 8) * 4);
    PagedMaps maps;
    const int dtype = cuda::std::is_same<T, __half>::value ? D2O_F16 : D2O_BF16;
    const uint64_t rows = (uint64_t)a.p.n_pages * a.p.Hkv << a.p.page_shift;
    if (!encode_rows_2d(&maps.k, dtype, a.p.k, rows, D, kPagedTile) || !encode_rows_2d(&maps.v, dtype, a.p.v, rows, D, kPagedTile))
      return cudaErrorNotSupported;
    e = C > 1 ? launch_shares(paged_decode_tc_kernel<T, D, G, true>, a, n_slices, C, paged_warps(G), smem, st, maps)
              : launch_shares(paged_decode_tc_kernel<T, D, G, false>, a, n_slices, C, paged_warps(G), smem, st, maps);
  }
  if (e != cudaSuccess) return e;
  if (!a.logits) return cudaSuccess;
  // CTAs per slice: up to eight per SM, a row per thread at least
  const long long reach = (long long)a.p.max_pages << a.p.page_shift;
  const int y = (int)std::max<long long>(1, std::min<long long>((8 * a.ctas + n_slices - 1) / n_slices, reach / kPagedThreads));
  return launch_behind(score_kernel<G>, dim3((unsigned)n_slices, (unsigned)y), kPagedThreads, 0, st, a);
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
                                const void* v, const int32_t* positions, void* out, char* scratch, cudaStream_t st, unsigned long long wait_ns,
                                int stop_stage) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaGetLastError();
  const int G = p.Hq / p.Hkv;
  const PagedScratch s(p.B * p.Hkv, G, D, (size_t)p.n_pages * p.Hkv << p.page_shift, p.score != nullptr);
  PagedDecodeArgs a;
  a.p = p;
  a.q = q; a.k = k; a.v = v; a.out = out; a.positions = positions; a.window = window; a.n_sink = n_sink;
  a.wait_ns = wait_ns; a.stop_stage = stop_stage;
  a.ctas = std::min(sms, kPagedCtas);
  a.done = reinterpret_cast<uint32_t*>(scratch + s.done);
  a.lse2 = reinterpret_cast<float*>(scratch + s.lse2);
  a.parts = reinterpret_cast<float*>(scratch + s.parts);
  a.logits = p.score ? reinterpret_cast<float*>(scratch + s.rows) : nullptr;
  if (dtype == D2O_F32) return D == 64 ? launch_g<float, 64>(a, st) : launch_g<float, 128>(a, st);
  if (dtype == D2O_F16) return D == 64 ? launch_g<__half, 64>(a, st) : launch_g<__half, 128>(a, st);
  return D == 64 ? launch_g<__nv_bfloat16, 64>(a, st) : launch_g<__nv_bfloat16, 128>(a, st);
}

}  // namespace d2o
