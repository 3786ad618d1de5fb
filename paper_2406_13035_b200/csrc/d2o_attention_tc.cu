// Attention of a prompt (Eq. 2-3 over all positions at once), causal, over a window and the first tokens: 16-bit inputs on the
// 5th-generation tensor cores.
//
// One item = 256 queries of a head, as two tiles of 128; keys and values stream in tiles of 128.  Per tile of keys and tile of
// queries: S = Q K^T (128 x 128 x d) into tensor memory; a thread of the softmax warps owns one query = one tensor-memory lane,
// so that maximum and sum run over its registers; the weights go back, rounded to 16 bits, into the columns that held S, from
// where they are the A operand of O += P V (128 x d x 128, V read as it lies, MN-major).  The two query tiles take turns: while
// one's weights are formed the tensor cores work for the other.
//   warps 0-3, 4-7  softmax of the first / second query tile, and its output at the end
//   warp 8          TMA producer: Q once per item, K and V through one ring (128-byte swizzle)
//   warps 9, 10     MMA issue, one per query tile, in turns; the first allocates the tensor memory
//   (warp 11 only completes its warpgroup)
// The weights are 2^(c s - m) with a reference m per query that moves only when the maximum has grown by more than 8 (in the log2
// domain): O in tensor memory is then rescaled by the softmax warps themselves.  The product before it has finished by then: the
// commit that announces a new S covers every product issued ahead of it.
//
// What bounds it: neither the tensor cores (57 % busy) nor the exponentials (57 %) but a query tile's chain from S to the next S, 3000 - 3200
// cycles against 2050 of products for both tiles; under load the power cap.  us: 32 / 8 heads of 32768 tokens under a window of 4096, bf16, 1860 cool and
// 2150 warm (1.11 and 0.96 PFLOP/s); four ragged prompts of up to 6001 tokens 340 - 620 (0.93 - 1.06 PFLOP/s); 32 heads of 1200 tokens 27 - 28; 32 / 8 heads of
// 8192 tokens, d = 64, 389 (0.71).
//
// Rounding: weights to the input type for their product (relative half step 2^-8 bf16, 2^-11 fp16; the errors of many keys average out.
// fp16 weights below 2^-21 of the row's largest are subnormal: off by up to 2^-32 of that, the most keys, 2^20, together by 2^-12);
// their sum and lse from the unrounded ones; S, O and all sums are fp32.
#include <math.h>

#include <cuda/std/type_traits>

#include "d2o_attention.cuh"
#include "d2o_common.cuh"
#include "d2o_decode.cuh"
#include "d2o_tc.cuh"

namespace d2o {

constexpr int kPaTile = 128;
constexpr int kPaSoftWarps = 8;
constexpr int kPaThreads = (kPaSoftWarps + 4) * 32;          // three warpgroups: registers move between whole ones
constexpr float kPaSlack = 8.f;              // growth of the maximum (log2 domain) that the reference leaves standing
// How far below the maximum that it is set to the reference lies: the largest fp16 weight of a row is 2^7 to 2^15, so that nearly all of the
// format's range lies below it.  (Four or two more, with as much less slack: 27.5 -> 28.2, 27.9 us for 32 heads of 1200 tokens, 57.0 -> 60.0, 58.9 for
// two prompts of 2100.)
template <int FMT> __host__ __device__ constexpr float pa_bias() { return FMT == 0 ? 7.f : 0.f; }
constexpr float kPaFar = 1048576.f;          // references (log2 domain) beyond which their rounding is more than 1/16

__host__ __device__ constexpr int pa_stages(int D) { return D == 128 ? 4 : 8; }

struct PaMaps { CUtensorMap q, k, v; };

// One item: 256 queries of one (sequence, head).  The last queries see the most keys: items are numbered with those of all heads
// first, neighbouring heads (which share keys and values) next to one another.  One CTA of the grid is one item; a CTA that is done takes
// the place of one that has not started (clusterlaunchcontrol).
struct PaItem {
  int bh, b, P, q0;
  __device__ __forceinline__ PaItem(const PromptAttentionArgs& a, int i) {
    const int heads = a.B * a.Hq, blocks = (a.P + 2 * kPaTile - 1) / (2 * kPaTile);
    bh = i % heads; b = bh / a.Hq;
    P = a.length(b);
    q0 = (blocks - 1 - i / heads) * 2 * kPaTile;
  }
  __device__ __forceinline__ bool empty() const { return q0 >= P; }
  __device__ __forceinline__ bool exists(int t) const { return q0 + t * kPaTile < P; }
};

// Does query tile t (first query w) see anything of the key tile at k0?
__device__ __forceinline__ bool pa_valid(const PromptAttentionArgs& a, int w, int P, int k0) {
  return w < P && k0 <= w && (k0 + kPaTile - 1 > w - a.window || k0 < a.n_sink);
}

// bits 0 .. n
__device__ __forceinline__ uint32_t pa_bits(int n) { return n < 0 ? 0u : n >= 31 ? 0xffffffffu : (2u << n) - 1u; }
// 32 logits of a row: those not seen become -inf.  Column i is seen if i <= last and (i > low or i < sink): one word of bits for all of
// them.  (A comparison per column and condition took 1300 cycles per tile more, a branch 8000.)
__device__ __forceinline__ void pa_mask(uint32_t (&s)[32], int last, int low, int sink) {
  const uint32_t seen = pa_bits(last) & (~pa_bits(low) | pa_bits(sink - 1));
#pragma unroll
  for (int i = 0; i < 32; ++i) s[i] = seen >> i & 1u ? s[i] : 0xff800000u;
}
// 32 logits of a row: 2^(c s + b), in 16 bits in p[AT ..], and their sum.
template <int FMT, int AT>
__device__ __forceinline__ void pa_block(const uint32_t (&s)[32], uint32_t (&p)[32], float c, float b, tc::f32x2 (&sum)[2]) {
  const tc::f32x2 c2 = tc::pack2(c, c), b2 = tc::pack2(b, b);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const tc::f32x2 y = tc::fma2(tc::pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, b2);
    float y0, y1;
    tc::unpack2(y, y0, y1);
    y0 = tc::ex2(y0); y1 = tc::ex2(y1);
    sum[i & 1] = tc::add2(sum[i & 1], tc::pack2(y0, y1));
    if (FMT == 0) { const __half2 h = __floats2half2_rn(y0, y1); p[AT + i] = *reinterpret_cast<const uint32_t*>(&h); }
    else { const __nv_bfloat162 h = __floats2bfloat162_rn(y0, y1); p[AT + i] = *reinterpret_cast<const uint32_t*>(&h); }
  }
}

// The rows r0 + (bits of `rows`) once more, by one warp, in fp32.  The weights 2^(c s - m) of the tensor-core path have the product c s unrounded
// and m rounded: with logits in the millions their difference would be anything, from 0 to infinity.  Here c s is rounded before m is taken
// from it.  For inputs that no trained model has: 8192 keys take 13 ms per 256 rows (ordinary ones 0.14), and with more than half a million the other
// warps' waits run out.  A function, and behind the item, because any code for such rows in the loop over the tiles costs every prompt 2 - 8 %; this
// one 0.5 %.
template <typename T, int D>
__device__ __noinline__ void pa_far_rows(const T* Q, const T* K, const T* V, T* out, float* lse, unsigned rows, int r0, int window, int n_sink) {
  constexpr int LPR = D / 8, RPW = 32 / LPR, U = 8, QL = LPR / 4;        // lanes per row of 8 elements each, rows of a warp, in flight
  const float c = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
  const int lane = threadIdx.x & 31, grp = lane / LPR, lig = lane % LPR;
  for (; rows; rows &= rows - 1) {
    const int r = r0 + __ffs(rows) - 1, lo = max(0, r - window + 1), sinks = min(n_sink, lo), n = sinks + r + 1 - lo;
    auto at = [&](int i) { return (size_t)(i < sinks ? i : lo + i - sinks) * D + lig * 8; };       // of the i-th key that the row sees
    float q[8], m = -INFINITY, l = 0.f, acc[8];
    Elem<T>::unpack(ld_global_v4(Q + (size_t)r * D + lig * 8), q);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    for (int i0 = 0; i0 < n; i0 += U * RPW) {
      uint4 kv[U], vv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * RPW + grp;
        kv[u] = vv[u] = make_uint4(0, 0, 0, 0);
        if (i < n) { kv[u] = ld_global_v4(K + at(i)); vv[u] = ld_global_v4(V + at(i)); }
      }
      float x[U / 4], mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < U / 4; ++j) {
        float dot[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float k[8];
          Elem<T>::unpack(kv[j * 4 + u], k);
          dot[u] = dot_pairs<8>(q, k);
        }
        const float t = reduce4<LPR>(dot[0], dot[1], dot[2], dot[3], lig) * c;
        x[j] = i0 + (j * 4 + lig / QL) * RPW + grp < n ? t : -INFINITY;
        mx = fmaxf(mx, x[j]);
      }
      const float mn = fmaxf(m, warp_max(mx)), base = mn > -INFINITY ? mn : 0.f, f = exp2f(m - base);
      m = mn;
      l *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= f;
#pragma unroll
      for (int j = 0; j < U / 4; ++j) { x[j] = exp2f(x[j] - base); l += x[j]; }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = __shfl_sync(0xffffffffu, x[u / 4], (u & 3) * QL, LPR);
        float v[8];
        Elem<T>::unpack(vv[u], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, v[e], acc[e]);
      }
    }
    l = warp_sum(l) * (1.f / QL);                            // QL lanes had the same keys
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], o);
      acc[e] /= l;
    }
    if (lane < LPR) *reinterpret_cast<uint4*>(out + (size_t)r * D + lig * 8) = Elem<T>::pack(acc);
    if (lse && lane == 0) lse[r] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(kPaThreads, 1)
prompt_attention_tc_kernel(PromptAttentionArgs a, const __grid_constant__ PaMaps maps) {
  constexpr int KB = D / 64, BLOCK = kPaTile * 128, TILE = KB * BLOCK, STAGES = pa_stages(D);
  constexpr uint32_t IDESC_QK = make_idesc(FMT, kPaTile, kPaTile), IDESC_PV = make_idesc(FMT, kPaTile, D) | kIdescBMn;
  using T = typename cuda::std::conditional<FMT == 0, __half, __nv_bfloat16>::type;
  const float c = (D == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;

  extern __shared__ __align__(1024) unsigned char pa_smem[];
  unsigned char* sQ = pa_smem;                               // [2 tiles][KB][128 rows][128 B]
  unsigned char* sKV = pa_smem + 2 * TILE;                   // [stages][KB][128 rows][128 B]
  __shared__ unsigned long long q_full, q_empty, kv_full[STAGES], kv_empty[STAGES], s_full[2], p_ready[2][2], o_full[2], o_empty[2], turn[2], all_done[2], it_full[2], it_empty[2], answered;
  __shared__ alignas(16) uint4 s_answer;
  // This CTA's items: the one that the slowest warp has taken, the next, and the one that is announced while that warp is at the first; the
  // item that it was given after a wait had run out.  -1: none.
  __shared__ volatile int s_item[3], s_lost;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_fail;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    s_item[0] = s_item[1] = s_item[2] = s_lost = -1;
    s_fail = (tc::smem_u32(pa_smem) & 1023u) != 0u;          // swizzled tiles need 1024-byte aligned shared memory
    tc::mbar_init(&q_full, 1); tc::mbar_init(&q_empty, 2); tc::mbar_init(&answered, 1);
    for (int s = 0; s < STAGES; ++s) { tc::mbar_init(&kv_full[s], 1); tc::mbar_init(&kv_empty[s], 2); }
    for (int t = 0; t < 2; ++t) { tc::mbar_init(&it_full[t], 1); tc::mbar_init(&it_empty[t], kPaSoftWarps + 2); tc::mbar_init(&s_full[t], 1); tc::mbar_init(&p_ready[t][0], 4); tc::mbar_init(&p_ready[t][1], 4); tc::mbar_init(&o_full[t], 1); tc::mbar_init(&o_empty[t], 4); tc::mbar_init(&turn[t], 1); tc::mbar_init(&all_done[t], 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kPaSoftWarps + 1) {
    tc::tmem_alloc(&s_tmem, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tm_s = s_tmem, tm_o = s_tmem + 256;         // S (and P) of tile t at + 128 t, O at + 128 t
  auto wait = [&](unsigned long long* bar, uint32_t parity) {
    if (tc::mbar_try_wait(bar, parity)) return true;
    if (!s_fail && tc::mbar_wait(bar, parity, a.wait_ns)) return true;
    s_fail = 1;
    return false;
  };
  // Of a warp that walks together: its threads may run out of time apart, and those that stayed would wait for the others, at the next
  // instruction of the whole warp, for good.
  auto wait_warp = [&](unsigned long long* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  start_dependents();
  wait_for_prior_grid();
  int loads_q = 0, loads_kv = 0, unanswered = -1;            // of the producer; the request whose answer was not there in time
  // The k-th item of this CTA as a warp sees it; -1: no more.
  auto next_item = [&](int k) {
    if (!wait_warp(&it_full[k & 1], (uint32_t)((k >> 1) & 1)) || __any_sync(0xffffffffu, s_fail != 0)) return -1;
    const int i = s_item[k % 3];
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&it_empty[k & 1]);
    return i;
  };

  if (warp >= kPaSoftWarps) {
    // 384 threads of 168 registers at launch: 256 of 208 and 128 of 88 from here on
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kPaSoftWarps) {
    // ======================================================================= TMA producer
    if (lane == 0) {
      int i = (int)blockIdx.x;
      for (int k = 0;; ++k) {
        if (k >= 2) (void)wait(&it_empty[k & 1], (uint32_t)(((k >> 1) - 1) & 1));
        if (s_fail) { s_lost = i; break; }                   // the others run out of time, too
        s_item[k % 3] = i;
        tc::mbar_arrive(&it_full[k & 1]);
        if (i < 0) break;
        const PaItem it(a, i);
        const PromptSpan span(it.q0, 2 * kPaTile, max(it.P, it.q0 + 1), kPaTile, a.window, a.n_sink);
        const int q_row = it.bh * a.P + it.q0, k_base = (it.b * a.Hkv + it.bh % a.Hq / (a.Hq / a.Hkv)) * a.P;
        for (int j = 0; j < (it.empty() ? 0 : 2 * span.tiles); ++j) {      // K, V, K, V ..
          const int s = loads_kv % STAGES;
          if (loads_kv == a.stop_stage) goto stopped;
          if (loads_kv >= STAGES && !wait(&kv_empty[s], (uint32_t)((loads_kv / STAGES - 1) & 1))) break;
          tc::mbar_expect_tx(&kv_full[s], TILE);
          for (int kb = 0; kb < KB; ++kb)
            tc::tma_load_2d(sKV + s * TILE + kb * BLOCK, j & 1 ? &maps.v : &maps.k, kb * 64, k_base + span.tile(j >> 1) * kPaTile, &kv_full[s]);
          ++loads_kv;
          if (j == 0) {
            if (loads_q >= 1 && !wait(&q_empty, (uint32_t)((loads_q - 1) & 1))) break;
            tc::mbar_expect_tx(&q_full, 2 * TILE);
            for (int t = 0; t < 2; ++t)
              for (int kb = 0; kb < KB; ++kb) tc::tma_load_2d(sQ + t * TILE + kb * BLOCK, &maps.q, kb * 64, q_row + t * kPaTile, &q_full);
            ++loads_q;
          }
        }
        // Not earlier: the loads are two tiles of keys ahead of the products, which covers the answer's way, and an item asked for at the
        // beginning of a long one would wait while other CTAs have nothing to do (1200 tokens of 32 heads: 36 us instead of 30).
        tc::ask_for_cta(&s_answer, &answered);
        if ((a.late_answers == 0 || k + 1 < a.late_answers) && wait(&answered, (uint32_t)(k & 1))) {
          i = tc::cta_answered(&s_answer);
        } else {                                             // the CTA that it may name will not start: looked at again below
          s_fail = 1; unanswered = k; i = -1;
        }
      }
      stopped:;
    }
    __syncwarp();
  } else if (warp < kPaSoftWarps + 3) {
    // ======================================================================= MMA issue: a warp per query tile
    const int t = warp - kPaSoftWarps - 1;
    const uint32_t ts = tm_s + t * 128, to = tm_o + t * 128;
    int ring = 0, items = 0, turns = 0, np = 0, no = 0;      // tiles of keys or values, items, turns, weights taken, outputs begun
    auto full = [&](int slot) { return wait_warp(&kv_full[slot % STAGES], (uint32_t)((slot / STAGES) & 1)); };
    for (int x = 0, i; (i = next_item(x)) >= 0; ++x) {
      const PaItem it(a, i);
      if (it.empty()) continue;
      const PromptSpan span(it.q0, 2 * kPaTile, it.P, kPaTile, a.window, a.n_sink);
      const int n = span.tiles, w0 = it.q0 + t * kPaTile;
      auto qk = [&](int slot) {
        const uint64_t ad = tc::smem_desc_sw128(tc::smem_u32(sQ + t * TILE)), bd = tc::smem_desc_sw128(tc::smem_u32(sKV + slot % STAGES * TILE));
#pragma unroll
        for (int k = 0; k < D / 16; ++k)                     // 16 elements = 32 bytes along d per instruction
          tc::mma_f16_one(ts, ad + (uint64_t)(k / 4 * (BLOCK >> 4) + k % 4 * 2), bd + (uint64_t)(k / 4 * (BLOCK >> 4) + k % 4 * 2), IDESC_QK, k != 0 ? 1u : 0u);
        tc::mma_commit_one(&s_full[t]);
      };
      uint32_t begun = 0;
      if (!wait_warp(&q_full, (uint32_t)(items & 1)) || !full(ring)) break;
      ++items;
      tc::fence_after_sync();
      bool now = pa_valid(a, w0, it.P, span.tile(0) * kPaTile);      // does the tile see anything of job j?
      if (now) qk(ring);
      tc::mma_commit_one(&kv_empty[ring % STAGES]);
      if (n == 1) tc::mma_commit_one(&q_empty);
      ++ring;
      for (int j = 0; j < n; ++j) {
        const int k0 = span.tile(j) * kPaTile;
        const bool next = j + 1 < n && pa_valid(a, w0, it.P, span.tile(j + 1) * kPaTile);
        if (!full(ring)) break;
        // Values that no query of the item sees may be anything, and 0 * NaN is NaN: those behind the sequence's end, and between the sinks and
        // the first query's window, are zeroed.  The former by both warps (the same zeros), the latter by the first, which sees those tiles,
        // ahead of its turn and so of the second's.
        const bool end = k0 + kPaTile > it.P;
        if (now && (end || (t == 0 && k0 < span.lo))) {
          const int z0 = end ? it.P - k0 : max(0, a.n_sink - k0), z1 = end ? kPaTile : min(kPaTile, span.lo - k0), piece = lane % (KB * 8);
          unsigned char* row = sKV + ring % STAGES * TILE + piece / 8 * BLOCK + piece % 8 * 16;
#pragma unroll 4
          for (int r = z0 + lane / (KB * 8); r < z1; r += 32 / (KB * 8)) *reinterpret_cast<uint4*>(row + r * 128) = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        if (j + 1 < n && !full(ring + 1)) break;
        if (now && !begun && no++ > 0 && !wait_warp(&o_empty[t], (uint32_t)(no & 1))) break;
        if (!wait_warp(&turn[t], (uint32_t)((turns++ & 1) ^ (t ^ 1)))) break;
        if (now) {
          const uint64_t bd = tc::smem_desc_sw128_mn(tc::smem_u32(sKV + ring % STAGES * TILE), BLOCK);
#pragma unroll
          for (int h = 0; h < 2; ++h) {                      // the weights of 64 keys at a time
            (void)wait_warp(&p_ready[t][h], (uint32_t)(np & 1));
            tc::fence_after_sync();
#pragma unroll
            for (int k = h * kPaTile / 32; k < (h + 1) * kPaTile / 32; ++k)      // 16 keys: 8 columns of weights, 16 rows of 128 bytes of V
              tc::mma_f16_ts_one(to, ts + k * 8, bd + (uint64_t)(k * (2048 >> 4)), IDESC_PV, k != 0 ? 1u : begun);
          }
          ++np;
          begun = 1;
        }
        // S again: its columns held the weights of the product just issued, and the products of one thread run in the order of
        // their issue
        if (next) qk(ring + 1);
        if (lane == 0) tc::mbar_arrive(&turn[t ^ 1]);
        if (now && k0 == w0) tc::mma_commit_one(&o_full[t]);  // the diagonal: the tile's last keys
        tc::mma_commit_one(&kv_empty[ring % STAGES]);
        if (j + 1 < n) tc::mma_commit_one(&kv_empty[(ring + 1) % STAGES]);
        if (j + 2 == n) tc::mma_commit_one(&q_empty);         // the last product with Q has been issued
        ring += j + 1 < n ? 2 : 1;
        now = next;
      }
    }
    // Tensor memory is freed behind the last products, also where the softmax warps run out of time after this one has left the loop.
    tc::mma_commit_one(&all_done[t]);
    if (lane == 0) (void)tc::mbar_wait(&all_done[t], 0);
    __syncwarp();
  }
  } else {
    // ======================================================================= softmax, output
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int t = warp >> 2, quarter = warp & 3;             // query tile; tensor-memory lanes 32 * quarter ..
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t ts = tm_s + t * 128 + lanes, to = tm_o + t * 128 + lanes;
    int ns = 0, items = 0;
    for (int x = 0, i; (i = next_item(x)) >= 0; ++x) {
      const PaItem it(a, i);
      if (it.empty() || !it.exists(t)) continue;
      const PromptSpan span(it.q0, 2 * kPaTile, it.P, kPaTile, a.window, a.n_sink);
      const int w0 = it.q0 + t * kPaTile, r0 = w0 + quarter * 32, row = r0 + lane;      // first query of tile and warp, this thread's
      float m = -INFINITY, l = 0.f, peak = 0.f;              // reference (log2 domain), sum; largest magnitude of a reference
      for (int j = 0; j < span.tiles; ++j) {
        const int k0 = span.tile(j) * kPaTile;
        if (!pa_valid(a, w0, it.P, k0)) continue;
        if (!wait_warp(&s_full[t], (uint32_t)(ns++ & 1))) break;
        tc::fence_after_sync();
        uint32_t s0[32], s1[32], s2[32], s3[32];
        tc::tmem_ld32_issue(ts, s0); tc::tmem_ld32_issue(ts + 32, s1);
        tc::tmem_ld32_issue(ts + 64, s2); tc::tmem_ld32_issue(ts + 96, s3);
        tc::tmem_ld_wait(s0); tc::tmem_ld_wait(s1); tc::tmem_ld_wait(s2); tc::tmem_ld_wait(s3);
        // does the whole warp see the whole tile?
        if (!(k0 + kPaTile - 1 <= r0 && (k0 > r0 + 31 - a.window || k0 + kPaTile <= a.n_sink))) {
          const int last = row - k0, low = row - a.window - k0, sink = a.n_sink - k0;
          pa_mask(s0, last, low, sink); pa_mask(s1, last - 32, low - 32, sink - 32);
          pa_mask(s2, last - 64, low - 64, sink - 64); pa_mask(s3, last - 96, low - 96, sink - 96);
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          mx[0] = tc::max3(mx[0], __uint_as_float(s0[e]), __uint_as_float(s0[e + 1]));
          mx[1] = tc::max3(mx[1], __uint_as_float(s1[e]), __uint_as_float(s1[e + 1]));
          mx[2] = tc::max3(mx[2], __uint_as_float(s2[e]), __uint_as_float(s2[e + 1]));
          mx[3] = tc::max3(mx[3], __uint_as_float(s3[e]), __uint_as_float(s3[e + 1]));
        }
        const float top = fmaf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), c, -pa_bias<FMT>());
        const bool first = m == -INFINITY, move = !first && top > m + kPaSlack;       // first: O (if any) and l are zero
        if (__any_sync(0xffffffffu, move)) {
          const float f = move ? tc::ex2(m - top) : 1.f;
          l *= f;
#pragma unroll 1
          for (int x = 0; x < D; x += 16) {
            uint32_t o[16];
            tc::tmem_ld16_issue(to + x, o);
            tc::tmem_ld_wait(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tc::tmem_st16(to + x, o);
          }
        }
        if (first || move) m = top;
        const float b = m > -INFINITY ? -m : 0.f;
        peak = fmaxf(peak, fabsf(b));
        tc::f32x2 sum[2] = {0ull, 0ull};
        {
          uint32_t p[32];
          pa_block<FMT, 0>(s0, p, c, b, sum);
          pa_block<FMT, 16>(s1, p, c, b, sum);
          tc::tmem_st32(ts, p);
        }
        tc::tmem_st_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&p_ready[t][0]);
        {
          uint32_t p[32];
          pa_block<FMT, 0>(s2, p, c, b, sum);
          pa_block<FMT, 16>(s3, p, c, b, sum);
          tc::tmem_st32(ts + 32, p);
        }
        tc::tmem_st_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&p_ready[t][1]);
        float lo, hi;
        tc::unpack2(tc::add2(sum[0], sum[1]), lo, hi);
        l += lo + hi;
      }
      if (!wait_warp(&o_full[t], (uint32_t)(items++ & 1))) break;
      tc::fence_after_sync();
      const float f = 1.f / l;
      T* out = (T*)a.out + ((size_t)it.bh * a.P + row) * D;
      uint32_t o[D / 32][32];
#pragma unroll
      for (int x = 0; x < D / 32; ++x) tc::tmem_ld32_issue(to + x * 32, o[x]);
#pragma unroll
      for (int x = 0; x < D / 32; ++x) tc::tmem_ld_wait(o[x]);
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&o_empty[t]);
      if (row < it.P) {
#pragma unroll
        for (int e = 0; e < D; e += 8) {
          float y[8];
#pragma unroll
          for (int z = 0; z < 8; ++z) y[z] = __uint_as_float(o[e / 32][e % 32 + z]) * f;
          *reinterpret_cast<uint4*>(out + e) = Elem<T>::pack(y);
        }
      }
      if (a.lse && row < it.P) a.lse[(size_t)it.bh * a.P + row] = (m + log2f(l)) * 0.6931471805599453f;
      const unsigned far = __ballot_sync(0xffffffffu, row < it.P && peak > kPaFar);
      if (far) {
        const size_t hk = (size_t)(it.b * a.Hkv + it.bh % a.Hq / (a.Hq / a.Hkv)) * a.P, hq = (size_t)it.bh * a.P;
        __syncwarp();                                        // the rows' first outputs are written
        pa_far_rows<T, D>((const T*)a.Q + hq * D, (const T*)a.K + hk * D, (const T*)a.V + hk * D, (T*)a.out + hq * D, a.lse ? a.lse + hq : nullptr, far, r0,
                          a.window, a.n_sink);
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kPaSoftWarps + 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc(s_tmem, 512);
  }
  if (s_fail) {
    if (tid == kPaSoftWarps * 32) {                          // see the copies on their way land before the CTA may end
      for (int i = max(0, loads_kv - STAGES); i < loads_kv; ++i)
        if (!tc::mbar_wait(&kv_full[i % STAGES], (uint32_t)((i / STAGES) & 1))) break;
      if (loads_q > 0) (void)tc::mbar_wait(&q_full, (uint32_t)((loads_q - 1) & 1));
      if (unanswered >= 0 && tc::mbar_wait(&answered, (uint32_t)(unanswered & 1))) s_lost = tc::cta_answered(&s_answer);
      if (a.status) report_error(a.status, D2O_ERR_TIMEOUT, 0xA7710000u | (uint32_t)(blockIdx.x & 0xffff));
    }
    __syncthreads();
    for (int x = 0; x < 4; ++x) {                            // NaN for the items in hand
      const int i = x < 3 ? s_item[x] : s_lost;
      if (i < 0) continue;
      const PaItem it(a, i);
      for (int r = it.q0 + tid; r < min(it.P, it.q0 + 2 * kPaTile); r += kPaThreads) {
        for (int e = 0; e < D; ++e) ((T*)a.out)[((size_t)it.bh * a.P + r) * D + e] = Elem<T>::from_float(NAN);
        if (a.lse) a.lse[(size_t)it.bh * a.P + r] = NAN;
      }
    }
  }
}

template <int D, int FMT>
static cudaError_t launch_one(const PromptAttentionArgs& a, const PaMaps& maps, cudaStream_t st) {
  const size_t smem = (size_t)(2 + pa_stages(D)) * (D / 64) * kPaTile * 128;
  cudaError_t e = cudaFuncSetAttribute(prompt_attention_tc_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  const int n_items = a.B * a.Hq * ((a.P + 2 * kPaTile - 1) / (2 * kPaTile));
  return launch_behind(prompt_attention_tc_kernel<D, FMT>, dim3((unsigned)n_items), kPaThreads, smem, st, a, maps);
}

cudaError_t launch_prompt_attention_tc(int dtype, int D, const PromptAttentionArgs& a, cudaStream_t st) {
  PaMaps maps;
  if (!encode_rows_2d(&maps.q, dtype, a.Q, (uint64_t)a.B * a.Hq * a.P, D, kPaTile) ||
      !encode_rows_2d(&maps.k, dtype, a.K, (uint64_t)a.B * a.Hkv * a.P, D, kPaTile) ||
      !encode_rows_2d(&maps.v, dtype, a.V, (uint64_t)a.B * a.Hkv * a.P, D, kPaTile))
    return cudaErrorNotSupported;
  if (dtype == D2O_F16) return D == 64 ? launch_one<64, 0>(a, maps, st) : launch_one<128, 0>(a, maps, st);
  return D == 64 ? launch_one<64, 1>(a, maps, st) : launch_one<128, 1>(a, maps, st);
}

}  // namespace d2o
