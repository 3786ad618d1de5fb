// Shared by the kernels on a cache in pages: where a row lies, and how the rows that a token sees are counted in tiles.
#pragma once

#include "d2o_common.cuh"

namespace d2o {

constexpr int kPagedTile = 16;               // rows per tile: the smallest page, and the row count of one mma.sync step
constexpr int kPagedCtas = 320;              // most CTAs that divide the rows of a decode step (partial results in scratch)

// detail words of the error reports
enum { kPagedShortTable = 0x9A6E0000u, kPagedBadPage = 0x9A6E1000u, kPagedBadBudget = 0x9A6E2000u };

struct PagedView {
  void* k; void* v;                          // [n_pages, Hkv, page_size, d]
  int32_t* pos; float* score;                // [n_pages, Hkv, page_size], or NULL
  const int32_t* table;                      // [B, max_pages]
  const int32_t* len;                        // [B, Hkv]
  uint32_t* status;                          // may be NULL
  int B, Hq, Hkv, page_shift, n_pages, max_pages;

  __device__ __forceinline__ long long reach() const { return (long long)max_pages << page_shift; }     // rows of a full table
  // The pool row of the page that holds row `r` of (sequence b, head h), at the page's first row; -1: bad page number.
  // r < reach().
  __device__ __forceinline__ int page_row0(int b, int h, int r) const {
    const int page = table[(size_t)b * max_pages + (r >> page_shift)];
    return (unsigned)page < (unsigned)n_pages ? (page * Hkv + h) << page_shift : -1;
  }
  __device__ __forceinline__ int in_page(int r) const { return r & ((1 << page_shift) - 1); }
  __device__ __forceinline__ void report(uint32_t detail) const { if (status) report_error(status, D2O_ERR_STATE, detail); }
};

// The rows that the new token of a slice sees, in tiles of 16: those of the sinks, then those from the window's first row
// on (all of them where the two meet).
struct PagedSpan {
  int t;                                     // row of the new token; -1: nothing to do
  int lo, sinks;                             // seen: r <= t and (r >= lo or r < sinks)
  int head, skip, tiles;                     // tiles of the sinks, tiles left out behind them, tiles in all
  __device__ __forceinline__ PagedSpan(int n, long long reach, int window, int n_sink) {
    t = n < 0 || n >= reach ? -1 : n;
    lo = window > 0 ? max(0, t - window + 1) : 0;
    sinks = min(n_sink, lo);
    head = (sinks + kPagedTile - 1) / kPagedTile;
    skip = max(0, lo / kPagedTile - head);
    tiles = t < 0 ? 0 : t / kPagedTile + 1 - skip;
  }
  __device__ __forceinline__ int row0(int i) const { return (i < head ? i : i + skip) * kPagedTile; }       // of the i-th tile
  __device__ __forceinline__ bool sees(int r) const { return r <= t && (r >= lo || r < sinks); }
};

// launchers
cudaError_t launch_paged_append(const PagedView& p, int dtype, int D, int n_rows, const void* K, const void* V, const int32_t* lens,
                                const int32_t* first_pos, const float* colsum, cudaStream_t st);
cudaError_t launch_paged_decode(const PagedView& p, int dtype, int D, int window, int n_sink, const void* q, const void* k,
                                const void* v, const int32_t* positions, void* out, char* scratch, cudaStream_t st, unsigned long long wait_ns,
                                int stop_stage);
cudaError_t launch_paged_evict(const PagedView& p, int dtype, int D, const int32_t* budgets, const int32_t* next_pos, int n_sink,
                               int window, char* scratch, cudaStream_t st);

// Layout of the scratch (bytes): counters that are zero between calls, first and always of the same size; what the decode step's CTAs
// hand over; and per row of the pools the logits of its query
// heads, or an entry of the eviction's lists.
struct PagedScratch {
  size_t done, lse2, parts, rows, end;
  PagedScratch(int n_slices, int group, int D, size_t pool_rows, bool scored) {
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    done = take((size_t)D2O_PAGED_ZERO_BYTES);
    lse2 = take((size_t)n_slices * group * 4);
    parts = take((size_t)kPagedCtas * 2 * group * (D + 4) * 4);
    rows = take(scored ? pool_rows * (size_t)(group > 2 ? group * 4 : 8) : 0);
    end = o;
  }
};

}  // namespace d2o
