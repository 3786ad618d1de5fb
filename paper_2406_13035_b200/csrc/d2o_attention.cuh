// Shared by the kernels of the prompt attention: arguments, the mask, and the tiles of keys that a tile of queries sees.
#pragma once

#include "d2o_common.cuh"

namespace d2o {

struct PromptAttentionArgs {
  const void *Q, *K, *V;                     // [B, Hq, P, d], [B, Hkv, P, d] x 2
  const int32_t* lens;                       // [B] or NULL
  void* out;                                 // [B, Hq, P, d]
  float* lse;                                // [B, Hq, P] or NULL
  uint32_t* status;                          // may be NULL
  int B, Hq, Hkv, P, window, n_sink;         // window: P where there is none
  unsigned long long wait_ns;                // limit of every wait (16-bit kernel)
  int stop_stage;                            // failure-detection tests: no copy of keys or values from this one of a CTA on; -1: never
  int late_answers;                          // failure-detection tests: a CTA's answers to requests for work count as late from this one on; 0: none

  __device__ __forceinline__ int length(int b) const { return lens ? max(0, min(lens[b], P)) : P; }
  // does query i see key j (of a sequence that has both)?
  __device__ __forceinline__ bool sees(int i, int j) const { return j <= i && (i - j < window || j < n_sink); }
};

// The key tiles (of TK keys) that `rows` queries from q0 on see: those of the sinks, then those from the first window's first
// key to the last query (all up to there where the two meet).
struct PromptSpan {
  int q0, last, lo, hi, sinks;               // last query; first keys of the first and of the last query's window; sinks
  int head, skip, tiles, TK;
  __device__ __forceinline__ PromptSpan(int first, int rows, int P, int tk, int window, int n_sink)
      : q0(first), last(min(first + rows, P) - 1), TK(tk) {
    lo = max(0, q0 - window + 1);
    hi = max(0, last - window + 1);
    sinks = min(n_sink, hi);                 // sinks that some query sees by that rule alone
    head = (min(sinks, lo) + tk - 1) / tk;
    skip = max(0, lo / tk - head);
    tiles = last / tk + 1 - skip;
  }
  __device__ __forceinline__ int tile(int t) const { return t < head ? t : t + skip; }
  // do all queries see all keys of the tile?
  __device__ __forceinline__ bool full(int t) const {
    const int k0 = tile(t) * TK, k1 = k0 + TK - 1;
    return k1 <= q0 && (k0 >= hi || k1 < sinks);
  }
};

cudaError_t launch_prompt_attention(int dtype, int D, const PromptAttentionArgs& a, cudaStream_t st);
cudaError_t launch_prompt_attention_tc(int dtype, int D, const PromptAttentionArgs& a, cudaStream_t st);      // fp16, bf16

}  // namespace d2o
