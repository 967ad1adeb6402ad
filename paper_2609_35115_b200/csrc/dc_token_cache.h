// What the kernels over a token cache share (include/dc.h, dc_cache_open): the cache's geometry, the batch a call brings, and the
// map from positions to rows.
#pragma once
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "dc.h"

namespace dc {

// Keys and values lie as [session][kv_head][n_sink + ring][head_dim]: the rows that one CTA streams are contiguous.
struct CacheDims {
  int n_sessions, n_heads, n_kv_heads, n_sink, window, ring;
};

struct TokenBatch {
  int            n_seqs, n_tokens, max_tokens;
  const int32_t *sessions, *cu_tokens, *start;
};

struct TokenSeq {
  int session, start, first, count;   // count 0: the sequence has no tokens, or its values are outside of what the cache holds
};

// The device-side admission of a sequence: what the host cannot see without waiting for the device.  A sequence that fails
// it is left alone: none of its rows is read or written.
__device__ __forceinline__ TokenSeq load_seq(const TokenBatch& b, const CacheDims& d, int i) {
  TokenSeq s;
  s.session = b.sessions ? b.sessions[i] : i;
  s.start = b.start[i];
  s.first = i;
  int last = i + 1;
  if (b.cu_tokens) {
    s.first = b.cu_tokens[i];
    last = b.cu_tokens[i + 1];
  }
  // (last - first cannot overflow once both are known to lie in [0, n_tokens])
  const bool in = s.first >= 0 && last <= b.n_tokens && s.first < last;
  s.count = in ? last - s.first : 0;
  if (s.count > b.max_tokens || s.count > d.ring - d.window + 1 || s.session < 0 || s.session >= d.n_sessions || s.start < 0 ||
      s.start > INT_MAX - 1 - s.count)
    s.count = 0;
  return s;
}

__host__ __device__ __forceinline__ int cache_row(const CacheDims& d, int pos) {
  return pos < d.n_sink ? pos : d.n_sink + (pos - d.n_sink) % d.ring;
}

// The rows that hold a range of positions which some queries see, as at most three intervals [lo, hi) of rows: the first tokens,
// and the ring's part of the window, in two pieces where it runs over the ring's end.
struct RowSet {
  int s_hi, a_lo, a_hi, b_hi;   // [0, s_hi), [a_lo, a_hi), [n_sink, b_hi)
};
// Positions p <= newest that are first tokens, or >= oldest (newest - oldest < ring).
__host__ __device__ __forceinline__ RowSet row_set(const CacheDims& d, int oldest, int newest) {
  RowSet r;
  r.s_hi = newest + 1 < d.n_sink ? newest + 1 : d.n_sink;
  const int lo = oldest > d.n_sink ? oldest : d.n_sink;
  r.a_lo = r.a_hi = r.b_hi = d.n_sink;
  if (newest >= lo) {
    const int x = (lo - d.n_sink) % d.ring, end = x + (newest - lo + 1);
    r.a_lo = d.n_sink + x;
    r.a_hi = d.n_sink + (end < d.ring ? end : d.ring);
    r.b_hi = d.n_sink + (end > d.ring ? end - d.ring : 0);
  }
  return r;
}

// What the tokens at positions q_lo .. q_hi see: some of them, and all of them.
__host__ __device__ __forceinline__ RowSet seen_by_any(const CacheDims& d, int q_lo, int q_hi) { return row_set(d, q_lo >= d.window ? q_lo - d.window + 1 : 0, q_hi); }
__host__ __device__ __forceinline__ RowSet seen_by_all(const CacheDims& d, int q_lo, int q_hi) { return row_set(d, q_hi >= d.window ? q_hi - d.window + 1 : 0, q_lo); }

// The same for one token as two runs of rows, [0, n_first) and [lo_second, lo_second + n_second): where the window runs over the
// ring's end its second piece follows the first tokens' rows, and so does a window that begins at the first ring row.
struct RowRuns {
  int n_first, lo_second, n_second;
};
__host__ __device__ __forceinline__ RowRuns row_runs(const CacheDims& d, int pos) {
  const RowSet s = seen_by_any(d, pos, pos);
  RowRuns r{s.s_hi, s.a_lo, s.a_hi - s.a_lo};
  if (s.b_hi > d.n_sink) {
    r.n_first = s.b_hi;
  } else if (s.a_lo == r.n_first) {
    r.n_first += r.n_second;
    r.n_second = 0;
  }
  return r;
}

constexpr int STEP_N = 64;   // rows of a step of the chunk kernel
__host__ __device__ __forceinline__ uint64_t low_bits(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__host__ __device__ __forceinline__ uint64_t rows64(int r0, int lo, int hi) { return low_bits(hi - r0) & ~low_bits(lo - r0); }
// Which of the rows r0 .. r0 + 63 are in the set.
__host__ __device__ __forceinline__ uint64_t mask64(const RowSet& s, int n_sink, int r0) {
  return rows64(r0, 0, s.s_hi) | rows64(r0, s.a_lo, s.a_hi) | rows64(r0, n_sink, s.b_hi);
}

// The steps over a set of rows: step j covers rows 64 t .. 64 t + 63.  At most three runs of t, in ascending order; one CTA of a
// cluster takes `build`'s return value of them, from `first` on.
struct StepList {
  int lo[3], n[3], first;
  __host__ __device__ __forceinline__ int build(const RowSet& s, int n_sink, int rank, int splits) {
    const int from[3] = {0, n_sink, s.a_lo}, to[3] = {s.s_hi, s.b_hi, s.a_hi};
    int end = 0, all = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int t0 = from[i] / STEP_N > end ? from[i] / STEP_N : end, t1 = to[i] > from[i] ? (to[i] + STEP_N - 1) / STEP_N : 0;
      lo[i] = t0;
      n[i] = t1 > t0 ? t1 - t0 : 0;
      end = t1 > end ? t1 : end;
      all += n[i];
    }
    first = (int)((long long)rank * all / splits);
    return (int)((long long)(rank + 1) * all / splits) - first;
  }
  __host__ __device__ __forceinline__ int tile(int j) const {
    j += first;
    if (j < n[0]) return lo[0] + j;
    j -= n[0];
    return j < n[1] ? lo[1] + j : lo[2] + (j - n[1]);
  }
};


}  // namespace dc
