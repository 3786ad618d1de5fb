// A key-value cache in pages: filling it, and evicting from it by accumulated attention weight (Eq. 6-8).
//
//   append_kernel   rows of a prompt or a turn -> pages, with positions and scores
//   evict_kernel    which rows stay (radix select over the cluster of a slice), and the moves that close the gaps
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "d2o_common.cuh"
#include "d2o_paged.cuh"

namespace cg = cooperative_groups;

namespace d2o {

// ------------------------------------------------------------------------------------ append
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 64;              // rows per CTA

struct AppendArgs {
  PagedView p;
  const char *K, *V;                         // [B, Hkv, n_rows, row bytes]
  const int32_t *lens, *first_pos;
  const float* colsum;                       // [B, Hq, n_rows]
  int n_rows;
};

// A copy: bound by HBM, each byte read and written once (four prompts of 4096 tokens, 32 heads, fp16, with scores: 543 MB in 85 us, 6.4 TB/s).
// A group of lanes takes one row's 16-byte pieces of K and V, four rows in flight.
template <int ROWB>
__global__ void __launch_bounds__(kAppendThreads)
append_kernel(AppendArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int LPR = ROWB / 16, GRPS = kAppendThreads / LPR, U = kAppendRows / GRPS < 4 ? kAppendRows / GRPS : 4;
  const PagedView& p = a.p;
  const int sl = blockIdx.y, b = sl / p.Hkv, h = sl % p.Hkv;
  const int held = p.len[sl];
  if (held < 0) return;
  const int n = a.lens ? min(a.lens[b], a.n_rows) : a.n_rows;
  const int i0 = blockIdx.x * kAppendRows, grp = threadIdx.x / LPR, lig = threadIdx.x % LPR;
  const long long reach = p.reach();
  auto place = [&](int i) {                                  // pool row of row i; -1: none
    const long long r = (long long)held + i;
    if (r >= reach) { p.report(kPagedShortTable); return -1; }
    const int row0 = p.page_row0(b, h, (int)r);
    if (row0 < 0) { p.report(kPagedBadPage); return -1; }
    return row0 + p.in_page((int)r);
  };
  const size_t src = ((size_t)sl * a.n_rows + i0) * ROWB + lig * 16;
#pragma unroll
  for (int base = 0; base < kAppendRows; base += U * GRPS) {
    uint4 kv[U], vv[U];
    int to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * GRPS + grp;
      to[u] = -1;
      if (i0 + i < n) {
        kv[u] = ld_stream_v4(a.K + src + (size_t)i * ROWB);
        vv[u] = ld_stream_v4(a.V + src + (size_t)i * ROWB);
        to[u] = place(i0 + i);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u] >= 0) {
        *reinterpret_cast<uint4*>((char*)p.k + (size_t)to[u] * ROWB + lig * 16) = kv[u];
        *reinterpret_cast<uint4*>((char*)p.v + (size_t)to[u] * ROWB + lig * 16) = vv[u];
      }
  }
  const int i = i0 + threadIdx.x;
  if (p.pos && threadIdx.x < kAppendRows && i < n) {
    const int to = place(i);
    if (to >= 0) {
      p.pos[to] = (a.first_pos ? a.first_pos[b] : 0) + i;
      float s = 0.f;
      if (a.colsum) {
        const int G = p.Hq / p.Hkv;
        const float* c = a.colsum + ((size_t)b * p.Hq + (size_t)h * G) * a.n_rows + i;
        s = c[0];
        for (int g = 1; g < G; ++g) s += c[(size_t)g * a.n_rows];
      }
      p.score[to] = s;
    }
  }
}

cudaError_t launch_paged_append(const PagedView& p, int dtype, int D, int n_rows, const void* K, const void* V, const int32_t* lens,
                                const int32_t* first_pos, const float* colsum, cudaStream_t st) {
  AppendArgs a = {p, (const char*)K, (const char*)V, lens, first_pos, colsum, n_rows};
  const int rowb = D * (dtype == D2O_F32 ? 4 : 2);
  // x: chunks of rows (up to 2^31), y: slices, at most 65535 of them per launch (checked by the caller)
  const dim3 grid((unsigned)((n_rows + kAppendRows - 1) / kAppendRows), (unsigned)(p.B * p.Hkv));
  return rowb == 128 ? launch_behind(append_kernel<128>, grid, kAppendThreads, 0, st, a)
       : rowb == 256 ? launch_behind(append_kernel<256>, grid, kAppendThreads, 0, st, a)
                     : launch_behind(append_kernel<512>, grid, kAppendThreads, 0, st, a);
}

// ------------------------------------------------------------------------------------ evict
constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictKeys = 12288;            // rows of a CTA whose keys stay in shared memory
constexpr int kEvictMaxCluster = 16;
constexpr int kEvictMinRows = 1024;          // rows of a full table per CTA of a cluster
constexpr int kEvictMoves = 4;               // moves of a group of lanes in flight
constexpr int kEvictFew = kEvictThreads;     // rows in question that are ranked one by one instead of by further rounds

struct EvictArgs {
  PagedView p;
  const int32_t *budgets, *next_pos;         // [B, Hkv], [B]
  int2* moves;                               // per row of the pools: (from, to) of the move with that number, as pool rows
  int n_sink, window;
};

// A row's rank among the rows of its slice is decided by a key, then by the position (earlier is higher).  Keys: protected rows
// above all, then NaN, then the scores in their order.
__device__ __forceinline__ uint32_t evict_key(float score, int pos, int n_sink, long long first_recent) {
  if (pos < n_sink || pos >= first_recent) return 0xffffffffu;
  if (score != score) return 0xfffffffeu;
  return float_ord(score + 0.f);                             // -0 + 0 = +0
}

struct EvictExchange {                       // read by the other CTAs of the cluster
  int hist[2][256];
  int holes, movers, bad, few;
  unsigned long long last;                   // the lowest (key, position) that stays, of the first CTA
  unsigned long long list[kEvictFew];        // rows in question, of the first CTA
};

// One CTA or one cluster (CL) per slice, its rows divided evenly over the CTAs.  (1) Keys.  (2) Radix select, 8 bits per round, of the
// lowest key that stays: each CTA counts its rows, all add up the counts of all.  The scores of a slice share their leading bits, so that
// most lanes of a warp count in the same bin: they count together.  As soon as the border lies among a few hundred rows, those are
// gathered with their positions and ranked one by one (nearly always behind the second round); where more than that are equal to the last
// bit, rounds over their positions follow.  (3) The rows below the budget that go and the rows behind it that stay, each numbered in ascending order
// (every warp counts its own consecutive rows, one scan, every warp numbers them), form the moves; as many of one as of the other, and
// sources and targets do not overlap, so that all moves run at once.  (4) The moves, divided over the cluster, several rows of a
// group of lanes in flight.  What costs are the dependent steps.  us, counting lane by lane, numbering by block scans twice, one row in
// flight, clusters of at most eight / so (with the copy that restores the scores): 8 slices of 32768 rows to 6554 63 / 34 (selection 15, moves
// 9 at 5 TB/s), 256 slices of 2064 rows to 2048 31 / 16.  Stalls: loads, then the barriers; DRAM 9 % busy.
template <int ROWB, bool CL>
__global__ void __launch_bounds__(kEvictThreads, 2)
evict_kernel(EvictArgs a) {
  start_dependents();
  wait_for_prior_grid();
  constexpr int LPR = ROWB / 16, GRPS = kEvictThreads / LPR;
  extern __shared__ __align__(16) uint32_t s_keys[];
  __shared__ EvictExchange x;
  __shared__ int s_warp[kEvictWarps], s_holes[kEvictWarps], s_movers[kEvictWarps], s_bin, s_need, s_count;
  cg::cluster_group cluster = cg::this_cluster();
  const PagedView& p = a.p;
  const int C = CL ? (int)cluster.num_blocks() : 1, rank = CL ? (int)cluster.block_rank() : 0;
  const int sl = blockIdx.x / C, b = sl / p.Hkv, h = sl % p.Hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto sync_all = [&]() { if (CL) cluster.sync(); else __syncthreads(); };
  auto of_rank = [&](int r) { return CL ? (const EvictExchange*)cluster.map_shared_rank(&x, r) : &x; };
  const int n = p.len[sl], budget = a.budgets[sl];
  // the same for all CTAs of the cluster
  if (n < 0) return;
  if (n > p.reach()) { if (tid == 0) p.report(kPagedShortTable); return; }
  if (budget < 0) { if (tid == 0) p.report(kPagedBadBudget); return; }
  if (n <= budget || budget == 0) return;
  const long long first_recent = (long long)a.next_pos[b] - a.window;
  const int chunk = (n + C - 1) / C, r0 = min(n, rank * chunk), m = min(n, r0 + chunk) - r0;      // this CTA's rows r0 .. r0 + m
  if (tid < 256) { x.hist[0][tid] = 0; x.hist[1][tid] = 0; }
  if (tid == 0) { x.holes = x.movers = x.bad = x.few = 0; x.last = 0; }
  __syncthreads();
  auto pool_row = [&](int r) { const int row0 = p.page_row0(b, h, r); return row0 < 0 ? -1 : row0 + p.in_page(r); };
  auto load_key = [&](int r) {
    const int at = pool_row(r);
    if (at < 0) { x.bad = 1; return 0u; }
    return evict_key(p.score[at], p.pos[at], a.n_sink, first_recent);
  };
  auto key = [&](int i) { return i < kEvictKeys ? s_keys[i] : load_key(r0 + i); };
  for (int i0 = tid; i0 < m; i0 += 8 * kEvictThreads) {       // eight rows of a thread side by side: three dependent loads each
    int at[8], ps[8];
    float sc[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) at[u] = i0 + u * kEvictThreads < m ? pool_row(r0 + i0 + u * kEvictThreads) : -2;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (at[u] >= 0) { sc[u] = p.score[at[u]]; ps[u] = p.pos[at[u]]; }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u * kEvictThreads;
      if (at[u] == -1) x.bad = 1;
      if (at[u] >= 0 && i < kEvictKeys) s_keys[i] = evict_key(sc[u], ps[u], a.n_sink, first_recent);
    }
  }
  __syncthreads();
  // ---- the lowest (key, position) that stays, from the top eight bits down
  uint32_t kth = 0, inv_pos = 0;                             // rows above (kth, inv_pos), or equal, stay
  int need = budget, in_bin = n;                             // rows of the bin in question that stay, and in all
  int round = 0;
  // 32 bits of the rows in question (value(i, v): is row i one, and its bits); true: the border is found
  auto select = [&](auto&& value, uint32_t& prefix, uint32_t& mask) {
    prefix = mask = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      int* hist = x.hist[round & 1];
      for (int i0 = tid; i0 - lane < m; i0 += 4 * kEvictThreads) {           // whole warps, four rows of a thread side by side
        uint32_t v[4];
        bool in[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = i0 + u * kEvictThreads;
          v[u] = 0;
          in[u] = i < m && value(i, v[u]) && (v[u] & mask) == prefix;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int bin = (v[u] >> shift) & 255;
          const unsigned who = __ballot_sync(0xffffffffu, in[u]);
          const int lead = who ? __ffs(who) - 1 : 0, first = __shfl_sync(0xffffffffu, bin, lead);
          const unsigned same = __ballot_sync(0xffffffffu, in[u] && bin == first);
          if (in[u] && (lane == lead || bin != first)) atomicAdd(&hist[bin], lane == lead ? __popc(same) : 1);
        }
      }
      sync_all();
      int c = 0;
      if (tid < 256) {
        if (CL) {
#pragma unroll 16
          for (int r = 0; r < C; ++r) c += of_rank(r)->hist[round & 1][255 - tid];        // highest bin first
        } else {
          c = hist[255 - tid];
        }
      }
      // inclusive prefix over the 256 bins: eight warps
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += t; }
      if (lane == 31 && warp < 8) s_warp[warp] = inc;
      if (tid >= 256) x.hist[(round + 1) & 1][tid - 256] = 0;            // read by all before the barrier above
      __syncthreads();
      if (tid < 256) {
#pragma unroll
        for (int w = 0; w < 7; ++w) inc += w < warp ? s_warp[w] : 0;
        if (inc >= need && inc - c < need) { s_bin = 255 - tid; s_need = need - (inc - c); s_count = c; }
      }
      __syncthreads();
      prefix |= (uint32_t)s_bin << shift; mask |= 255u << shift;
      need = s_need; in_bin = s_count;
      ++round;
      if (need == in_bin) return true;                       // all rows of this bin stay: the lower bits do not matter
      if (in_bin <= kEvictFew) return false;
    }
    return false;
  };
  uint32_t mask = 0;
  bool exact = select([&](int i, uint32_t& v) { v = key(i); return true; }, kth, mask), by_pos = !exact;
  bool bad = false;
  for (int r = 0; r < C; ++r) bad |= of_rank(r)->bad != 0;
  if (bad) {                                                 // the same for all
    if (tid == 0 && rank == 0) p.report(kPagedBadPage);
    sync_all();                                              // our exchange area may still be read
    return;
  }
  auto inverse_pos = [&](int i) { return (uint32_t)p.pos[pool_row(r0 + i)] ^ 0x7fffffffu; };      // falls as the position, of either sign, grows
  EvictExchange* const lead_x = CL ? cluster.map_shared_rank(&x, 0) : &x;
  auto gather = [&](unsigned long long v) {                  // to the first CTA's list: in_bin rows
    const int at = atomicAdd(&lead_x->few, 1);
    if (at < kEvictFew) lead_x->list[at] = v;
  };
  if (!exact && in_bin > kEvictFew) {                        // equal to the last bit: by their positions
    uint32_t pos_mask;
    exact = select([&](int i, uint32_t& v) {
      if (key(i) != kth) return false;
      v = inverse_pos(i);
      return true;
    }, inv_pos, pos_mask);
    if (in_bin > kEvictFew) exact = true;                    // positions that stand many times over
    if (!exact)
      for (int i = tid; i < m; i += kEvictThreads)
        if (key(i) == kth) {
          const uint32_t v = inverse_pos(i);
          if ((v & pos_mask) == inv_pos) gather((unsigned long long)kth << 32 | v);
        }
  } else if (!exact) {
    for (int i = tid; i < m; i += kEvictThreads) {
      const uint32_t k = key(i);
      if ((k & mask) == kth) gather((unsigned long long)k << 32 | inverse_pos(i));
    }
  }
  if (!exact) {                                              // the border among the rows of the list
    sync_all();
    if (rank == 0 && tid < in_bin) {
      const unsigned long long mine = x.list[tid];
      int above = 0, equal = 0;
#pragma unroll 8
      for (int i = 0; i < in_bin; ++i) { above += x.list[i] > mine; equal += x.list[i] == mine; }
      if (above < need && need <= above + equal) x.last = mine;
    }
    sync_all();
    const unsigned long long last = of_rank(0)->last;
    kth = (uint32_t)(last >> 32); inv_pos = (uint32_t)last;
  }
  auto stays = [&](int i) {
    const uint32_t k = key(i);
    if (!by_pos || k != kth) return k >= kth;
    return inverse_pos(i) >= inv_pos;
  };
  // ---- number the rows below the budget that go (holes) and those behind it that stay (movers): each warp its own consecutive rows
  const int per = (m + kEvictWarps - 1) / kEvictWarps, w0 = min(m, warp * per), w1 = min(m, w0 + per);
  auto each = [&](auto&& f) {                                // f(row, its hole, its mover bits among the warp's 32)
    for (int base = w0; base < w1; base += 32) {
      const int i = base + lane;
      const bool in = i < w1, s = in && stays(i), low = r0 + i < budget;
      f(r0 + i, __ballot_sync(0xffffffffu, in && low && !s), __ballot_sync(0xffffffffu, s && !low));
    }
  };
  int holes = 0, movers = 0;
  each([&](int, unsigned hb, unsigned mb) { holes += __popc(hb); movers += __popc(mb); });
  if (lane == 0) { s_holes[warp] = holes; s_movers[warp] = movers; }
  __syncthreads();
  int h0 = 0, m0 = 0, nh = 0, nm = 0;                        // before this warp's; all
#pragma unroll
  for (int w = 0; w < kEvictWarps; ++w) {
    if (w < warp) { h0 += s_holes[w]; m0 += s_movers[w]; }
    nh += s_holes[w]; nm += s_movers[w];
  }
  if (CL) {
    if (tid == 0) { x.holes = nh; x.movers = nm; }
    cluster.sync();
    nh = nm = 0;
    for (int r = 0; r < C; ++r) {
      const EvictExchange* y = of_rank(r);
      const int yh = y->holes, ym = y->movers;
      if (r < rank) { h0 += yh; m0 += ym; }
      nh += yh; nm += ym;
    }
  }
  const int moves = min(nh, nm);                             // equal, unless positions stand twice
  const unsigned below = (1u << lane) - 1u;
  each([&](int r, unsigned hb, unsigned mb) {
    const int hk = h0 + __popc(hb & below), mk = m0 + __popc(mb & below);
    if ((hb >> lane & 1) && hk < moves) a.moves[pool_row(hk)].y = pool_row(r);
    if ((mb >> lane & 1) && mk < moves) a.moves[pool_row(mk)].x = pool_row(r);
    h0 += __popc(hb); m0 += __popc(mb);
  });
  sync_all();
  // ---- the moves
  // Where two sequences' tables name the same page the numberings may disagree, and an entry may be old: nothing outside the pools.
  const unsigned pool_rows = (unsigned)(p.n_pages * p.Hkv) << p.page_shift;
  const int grp = tid / LPR, lig = tid % LPR;
  int2 next[kEvictMoves];                                    // the following moves, read beside the rows of these
  auto look = [&](int k0) {
#pragma unroll
    for (int u = 0; u < kEvictMoves; ++u) {
      const int k = k0 + u * C * GRPS;
      next[u] = k < moves ? a.moves[pool_row(k)] : make_int2(-1, -1);
      if ((unsigned)next[u].x >= pool_rows || (unsigned)next[u].y >= pool_rows) next[u].x = -1;
    }
  };
  look(rank * GRPS + grp);
  for (int k0 = rank * GRPS + grp; k0 < moves; k0 += kEvictMoves * C * GRPS) {
    int2 mv[kEvictMoves];
    uint4 kv[kEvictMoves], vv[kEvictMoves];
    int ps[kEvictMoves];
    float sc[kEvictMoves];
#pragma unroll
    for (int u = 0; u < kEvictMoves; ++u) mv[u] = next[u];
#pragma unroll
    for (int u = 0; u < kEvictMoves; ++u)
      if (mv[u].x >= 0) {
        const size_t from = (size_t)mv[u].x * ROWB + lig * 16;
        kv[u] = ld_stream_v4((const char*)p.k + from);
        vv[u] = ld_stream_v4((const char*)p.v + from);
        if (lig == 0) { ps[u] = p.pos[mv[u].x]; sc[u] = p.score[mv[u].x]; }
      }
    look(k0 + kEvictMoves * C * GRPS);
#pragma unroll
    for (int u = 0; u < kEvictMoves; ++u)
      if (mv[u].x >= 0) {
        const size_t to = (size_t)mv[u].y * ROWB + lig * 16;
        *reinterpret_cast<uint4*>((char*)p.k + to) = kv[u];
        *reinterpret_cast<uint4*>((char*)p.v + to) = vv[u];
        if (lig == 0) { p.pos[mv[u].y] = ps[u]; p.score[mv[u].y] = sc[u]; }
      }
  }
}

template <int ROWB, bool CL>
static cudaError_t launch_evict(const EvictArgs& a, int n_slices, int C, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(evict_kernel<ROWB, CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvictKeys * 4);
  if (e == cudaSuccess && C > 8) e = cudaFuncSetAttribute(evict_kernel<ROWB, CL>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_slices * C)); cfg.blockDim = dim3(kEvictThreads); cfg.dynamicSmemBytes = kEvictKeys * 4; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = CL ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, evict_kernel<ROWB, CL>, a);
}

template <int ROWB>
static cudaError_t launch_evict(const EvictArgs& a, int n_slices, int C, cudaStream_t st) {
  return C > 1 ? launch_evict<ROWB, true>(a, n_slices, C, st) : launch_evict<ROWB, false>(a, n_slices, 1, st);
}

cudaError_t launch_paged_evict(const PagedView& p, int dtype, int D, const int32_t* budgets, const int32_t* next_pos, int n_sink,
                               int window, char* scratch, cudaStream_t st) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return cudaGetLastError();
  const int n_slices = p.B * p.Hkv;
  const PagedScratch s(n_slices, p.Hq / p.Hkv, D, (size_t)p.n_pages * p.Hkv << p.page_shift, true);
  const EvictArgs a = {p, budgets, next_pos, reinterpret_cast<int2*>(scratch + s.rows), n_sink, window};
  // One CTA per SM, as long as the table could hold 1024 rows for each of a cluster (the rows are known on the device only).  us with the
  // restoring copy, 8 slices: of 100 rows to 50 7.2 (one CTA) against 15.7 (sixteen), of 1100 to 1000 10.4 / 16.4, of 5300 to 4300 18.4 (four)
  // against 29.0 (one) and 19.3 (sixteen), of 9000 to 2000 19.6 (eight) / 32.9 / 22.0.  So few rows in a table with room for many pay for the
  // cluster that they do not need.
  int C = 1;
  const long long reach = (long long)p.max_pages << p.page_shift;
  while (2 * C <= kEvictMaxCluster && (long)n_slices * 2 * C <= sms && reach >= (long long)kEvictMinRows * 2 * C) C *= 2;
  const int rowb = D * (dtype == D2O_F32 ? 4 : 2);
  return rowb == 128 ? launch_evict<128>(a, n_slices, C, st) : rowb == 256 ? launch_evict<256>(a, n_slices, C, st)
                                                                           : launch_evict<512>(a, n_slices, C, st);
}

}  // namespace d2o
