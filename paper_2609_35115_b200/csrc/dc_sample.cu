// Choice of the next token from rows of logits (include/dc.h, dc_sample_tokens): temperature, top-k, top-p, min-p, from given random numbers.
//
// A cluster of CTAs keeps a row in shared memory, each CTA a contiguous slice of the vocabulary, and everything after the load happens
// there; rows enough for every SM are streamed from memory instead, pass by pass, by one or two CTAs each.  The rules cut a prefix of the order "descending logit, ties by lowest index", so the kept set is
// a cut key and a number of its ties; cuts are found by selection through histograms, by counts (top-k) or by mass (top-p).
//
// The result is a whole number that has to be the right one, so masses are exact: a weight exp((l - max) / T) is evaluated in fp64
// (2^(j/256) from a table times a polynomial; about 2^-50) and held as an integer multiple of 2^-45.  Integer sums do not depend on their order: atomics, splits
// and replays give the same token.  Against sums in real arithmetic a border is off by at most 2^-46 for every token of the row; a
// border that close to a row's random number is met once in millions of rows.
//
// Bound by the latency of the passes and of the cluster's barriers between them (few rows), by the passes' instructions, fp64 and shared-memory adds
// among them (many; the streamed form, two CTAs of 512 threads an SM, has 64 registers a thread and spills 16 to 72 bytes).  Measured, 256 rows of 131,072 fp32 logits: greedy 37 us, no rule 106 us, top-k 50 85 us, top-p 0.9 247 us; 48 rows of 32,001: 10, 12, 15, 27 us; one
// of 4,097: 8 to 10 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "dc_internal.h"
#include "dc_ptx.cuh"

namespace dc {
namespace {

constexpr int SMP_THREADS = 256, SMP_WIDE = 512;      // threads of a CTA: rows in shared memory, rows that are streamed
constexpr int SMP_WARPS = SMP_WIDE / 32;                // at most
constexpr int SMP_BINS = 1024;
constexpr int SMP_FEW = SMP_THREADS;       // candidates that one CTA finishes at most, one a thread (they lie where a histogram does)
constexpr int SMP_SLICE = 8192;           // logits of a CTA, while 16 CTAs are enough (then up to twice as many)
constexpr int SMP_MAX_CLUSTER = 16;
static_assert(2 * SMP_WIDE <= SMP_BINS, "a bin's logits and their masses lie where a histogram does");
constexpr uint32_t KEY_NONE = 0x007fffffu;   // key of -infinity: such logits, and NaN, take no part
constexpr unsigned long long ONE = 1ull << 45;
constexpr float LOWEST = -3.402823466e38f;

struct SampleArgs {
  const void*    logits;
  long long      stride;
  int            vocab, slice, splits;    // slice: logits of a CTA
  const float *  temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t*       tokens;
  float*         probs;
};

constexpr int SMP_GROUPS = SMP_BINS / 32;

struct SampleShared {
  unsigned long long hist[2][SMP_BINS];
  unsigned long long group[2][SMP_GROUPS];   // sums of 32 neighbouring bins
  double             table[256];             // 2^(j / 256): one a thread
  unsigned long long best;                   // the slice's maximum: key and inverted index
  unsigned long long range[2];               // smallest and inverted largest key of a selection's last bin
  unsigned long long kept;                   // mass of the slice's kept tokens
  unsigned long long warp_sum[SMP_WARPS];
  unsigned long long above, inside, target;  // of the found bin
  float              at_least;               // by mass: the logits in it and above are no fewer
  uint32_t           warp_ties[SMP_WARPS];
  uint32_t           ties;                   // of the slice
  uint32_t           few[2];                 // collected logits of the slice: candidates of the whole draw, and of a selection's last bin
  uint32_t           found;                  // key of a selection among few, and what lies above it
  unsigned long long found_above;
  int                bin;
};

// Bits in the logits' order (the two zeros are one logit).
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ unsigned long long ld_cluster64(uint32_t addr) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_cluster32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
// Sum of a word over the cluster's CTAs.
__device__ __forceinline__ unsigned long long cluster_sum(const unsigned long long* word, int splits) {
  const uint32_t at = ptx::smem_u32(word);
  unsigned long long s = 0;
#pragma unroll 16
  for (int c = 0; c < splits; ++c) s += ld_cluster64(ptx::map_to_cta(at, c));
  return s;
}
__device__ __forceinline__ void cluster_or_block_sync(int splits) {
  if (splits > 1) {
    __syncwarp();      // (the cluster's barrier is met by whole warps)
    ptx::cluster_arrive();
    ptx::cluster_wait();
  } else {
    __syncthreads();
  }
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int m = 16; m; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
__device__ __forceinline__ unsigned long long warp_scan(unsigned long long v, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += x;
  }
  return v;
}

// 2^(j / 256), j = 0 .. 255, by the series of exp(j ln 2 / 256), which 24 terms take below the last bit.
struct Exp2Table {
  double v[256];
  constexpr Exp2Table() : v() {
    for (int j = 0; j < 256; ++j) {
      const double x = j * (0.69314718055994530942 / 256.0);
      double sum = 0.0;
      for (int k = 24; k >= 1; --k) sum = (sum + 1.0) * x / k;      // x + x^2 / 2 + ..., smallest terms first
      v[j] = 1.0 + sum;
    }
  }
};
__device__ constexpr Exp2Table exp2_table;

// Weights of a row: 2^((l - top) scale).
struct Weigh {
  double scale, top;     // scale: log2(e) / T
  const double* table;
  // y = k / 256 + f with |f| <= 2^-9; 2^f by the first terms of its series (the rest is below 2^-54).  Of finite l whose y is -64 or more.
  __device__ __forceinline__ double value(float l) const {
    const double y = ((double)l - top) * scale;
    const double magic = 6755399441055744.0 / 256.0;      // 1.5 * 2^52 / 256
    const double t = y + magic, f = y - (t - magic);
    const int k = __double2loint(t);
    const double r = table[k & 255];
    const double p = fma(fma(fma(9.618129107628477e-3, f, 5.550410866482158e-2), f, 2.402265069591007e-1), f, 6.931471805599453e-1) * f;
    const double v = fma(r, p, r);
    return __hiloint2double(__double2hiint(v) + (k >> 8) * (1 << 20), __double2loint(v));
  }
  // in units of 2^-45: the lowest bit of a number just above 2^7 is that
  static __device__ __forceinline__ unsigned long long fix(double w) { return (unsigned long long)__double_as_longlong(w + 128.0) - 0x4060000000000000ull; }
  __device__ __forceinline__ unsigned long long fixed(float l) const { return fix(value(l)); }
};

// The kept tokens: logits from `low` up, and the first `ties` (in the vocabulary's order) of those equal to `tie`, just below.
struct Cut {
  float              low, tie;
  unsigned long long ties;
};

template <typename T>
__device__ __forceinline__ float as_float(T x) { return (float)x; }

// A CTA's slice of a row, as places: logit i of the slice is at place shift + i, where 16-byte vectors of the caller's memory begin at
// multiples of their size.  Either the slice lies in shared memory, as fp32, or (STREAM) every pass reads the caller's memory, which the L2
// cache holds behind the first.  NaN is left: it compares as false, like -infinity it is never kept.
template <typename T, bool STREAM, int NT>
struct Row {
  const T* src;       // place 0
  int      shift, end, places;      // the slice is [shift, end); places: whole steps of all warps
  float*   l;
  bool     infinite;  // +infinity is the largest: it counts as 0, everything finite as -infinity

  // STREAM: four places from the caller's memory
  __device__ __forceinline__ float4 from_memory(int i) const {
    float4 y;
    if (i >= shift && i + 4 <= end) {
      if (sizeof(T) == 4) {
        y = *reinterpret_cast<const float4*>(src + i);
      } else {
        alignas(8) T x[4];
        *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(src + i);
        y = make_float4(as_float(x[0]), as_float(x[1]), as_float(x[2]), as_float(x[3]));
      }
    } else {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = i + e >= shift && i + e < end ? as_float(src[i + e]) : -INFINITY;
      y = make_float4(x[0], x[1], x[2], x[3]);
    }
    return y;
  }
  static __device__ __forceinline__ float against_infinity(float x) { return x == INFINITY ? 0.f : -INFINITY; }
  __device__ __forceinline__ float4 quad(int i) const {
    if (!STREAM) return *reinterpret_cast<const float4*>(l + i);
    float4 y = from_memory(i);
    if (infinite) y = make_float4(against_infinity(y.x), against_infinity(y.y), against_infinity(y.z), against_infinity(y.w));
    return y;
  }
  // Calls f(place, four logits) for this thread's share of the slice; several loads are under way at once.
  template <typename F>
  __device__ __forceinline__ void each_quad(F f) const {
    constexpr int U = STREAM ? 4 : 2;
    for (int i0 = threadIdx.x * 4; i0 < places; i0 += U * NT * 4) {
      float4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * NT * 4 < places) v[u] = quad(i0 + u * NT * 4);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * NT * 4 < places) f(i0 + u * NT * 4, v[u]);
    }
  }
  template <typename F>
  __device__ __forceinline__ void each_logit(F f) const {
    each_quad([&](int, const float4& v) {
      f(v.x);
      f(v.y);
      f(v.z);
      f(v.w);
    });
  }
  // This thread's maximum; fills shared memory.
  __device__ __forceinline__ float load() const {
    float top = -INFINITY;
    if constexpr (STREAM) {
      each_quad([&](int, const float4& y) { top = fmaxf(fmaxf(top, fmaxf(y.x, y.y)), fmaxf(y.z, y.w)); });
    } else {
      constexpr int VE = 16 / sizeof(T);
#pragma unroll 4
      for (int at = threadIdx.x * VE; at < end; at += NT * VE) {
        alignas(16) T x[VE];
        if (at >= shift && at + VE <= end) {
          *reinterpret_cast<uint4*>(x) = __ldcs(reinterpret_cast<const uint4*>(src + at));
        } else {
#pragma unroll
          for (int i = 0; i < VE; ++i) x[i] = at + i >= shift && at + i < end ? src[at + i] : (T)-INFINITY;
        }
#pragma unroll
        for (int i = 0; i < VE; i += 4) {
          const float4 y = make_float4(as_float(x[i]), as_float(x[i + 1]), as_float(x[i + 2]), as_float(x[i + 3]));
          top = fmaxf(fmaxf(top, fmaxf(y.x, y.y)), fmaxf(y.z, y.w));
          *reinterpret_cast<float4*>(l + at + i) = y;
        }
      }
      for (int i = (end + VE - 1) / VE * VE + threadIdx.x; i < places; i += NT) l[i] = -INFINITY;
    }
    return top;
  }
};

// Bins of a row.  Selection needs bins that fall with the logit and spread the row's logits, so that few of a warp's lanes meet in one:
// 22 to a factor of two of weight, then 1024 in each of those, by fp32 arithmetic (each operation is monotone, and the
// second bin is exact in what the first one left; products and differences are spelt out, joined into one operation they would not be what
// the bins were cut by).
struct Binned {
  float half_top, scale;      // scale: 44 log2(e) / T, of half a difference (a whole one may pass fp32's range)
  static constexpr float END = 46.f * 22.f;      // 2^-46: what lies behind rounds to nothing
  __device__ __forceinline__ float place(float l) const { return __fmul_rn(fmaf(l, -0.5f, half_top), scale); }
  __device__ __forceinline__ float logit(float t) const { return 2.f * (half_top - t / scale); }
  static __device__ __forceinline__ int inner(float t, int bin) { return (int)__fmul_rn(__fsub_rn(t, (float)bin), (float)SMP_BINS); }
};

// What a selection sums: one for every logit, or its mass.
template <bool BY_MASS>
__device__ __forceinline__ void add_to_bin(unsigned long long* bin, const Weigh& w, float l) {
  uint32_t* half = reinterpret_cast<uint32_t*>(bin);
  if (!BY_MASS) {
    atomicAdd(half, 1u);
    return;
  }
  // 32-bit adds, with the carry: shared memory adds those in place, 64-bit ones in a loop
  const unsigned long long m = w.fixed(l);
  const uint32_t lo = (uint32_t)m, old = atomicAdd(half, lo), hi = (uint32_t)(m >> 32) + (old + lo < lo);
  if (hi) atomicAdd(half + 1, hi);
}

// Finds the bin of the cluster's histograms in which `over` plus the running sum, from bin 0 up (DOWN: from the last bin down), reaches
// target(total): groups of bins first, then the group's bins, so that little is read from the other CTAs.
template <bool DOWN, int NT, typename F>
__device__ __forceinline__ bool find_bin(SampleShared& sh, int buf, unsigned long long over, F target_of, int splits) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
#pragma unroll
  for (int g = warp; g < SMP_GROUPS; g += NT / 32) {
    const unsigned long long s = warp_sum(sh.hist[buf][g * 32 + lane]);
    if (lane == 0) sh.group[buf][g] = s;
  }
  cluster_or_block_sync(splits);
  if (warp == 0) {
    unsigned long long s[SMP_GROUPS / 32], sum = 0;
#pragma unroll
    for (int i = 0; i < SMP_GROUPS / 32; ++i) {
      const int g = lane * (SMP_GROUPS / 32) + i;
      s[i] = cluster_sum(&sh.group[buf][DOWN ? SMP_GROUPS - 1 - g : g], splits);
      sum += s[i];
    }
    unsigned long long upto = warp_scan(sum, lane);
    const unsigned long long target = target_of(__shfl_sync(0xffffffffu, upto, 31));
    upto += over - sum;
    int group = -1;
    unsigned long long base = 0;
#pragma unroll
    for (int i = 0; i < SMP_GROUPS / 32; ++i) {
      if (upto < target && upto + s[i] >= target) {
        group = lane * (SMP_GROUPS / 32) + i;
        base = upto;
      }
      upto += s[i];
    }
    const unsigned who = __ballot_sync(0xffffffffu, group >= 0);
    if (lane == 0) sh.bin = -1;
    // no logit of a group weighs more than the group's first bin allows
    float weighed = 0.f;
#pragma unroll
    for (int i = 0; i < SMP_GROUPS / 32; ++i) weighed += lane * (SMP_GROUPS / 32) + i < (who ? __ffs(who) - 1 : 0) * (SMP_GROUPS / 32) ? (float)s[i] * exp2f((lane * (SMP_GROUPS / 32) + i) * (32.f / 22.f) - 45.f) : 0.f;
#pragma unroll
    for (int m = 16; m; m >>= 1) weighed += __shfl_xor_sync(0xffffffffu, weighed, m);
    if (lane == 0) sh.at_least = weighed;
    if (who) {
      group = __shfl_sync(0xffffffffu, group, __ffs(who) - 1);
      base = __shfl_sync(0xffffffffu, base, __ffs(who) - 1);
      const int at = group * 32 + lane, bin = DOWN ? SMP_BINS - 1 - at : at;
      const unsigned long long own = cluster_sum(&sh.hist[buf][bin], splits), before = warp_scan(own, lane) + base - own;
      if (before < target && before + own >= target) {
        sh.bin = bin;
        sh.above = before;
        sh.inside = own;
        sh.target = target;
      }
    }
  }
  __syncthreads();
  return sh.bin >= 0;      // (all of this is written anew behind a barrier that everyone passes)
}

// The words that the cluster's CTAs have collected, one CTA's behind the other's.  `count`: CTA `lane`'s number of them; n in all.
// (A read from another CTA takes a thousand cycles: all are under way at once.)
template <int NT>
__device__ __forceinline__ void pull_few(unsigned long long* to, const unsigned long long* collected, uint32_t count, int n, int splits) {
  const int lane = threadIdx.x & 31;
  uint32_t upto = count;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  for (int i0 = 0; i0 < n; i0 += NT) {
    const int i = i0 + (int)threadIdx.x;
    int k = 0, before = 0;
    for (int x = 0; x < splits - 1; ++x) {
      const int end = (int)__shfl_sync(0xffffffffu, upto, x);
      if (i >= end) {
        k = x + 1;
        before = end;
      }
    }
    if (i < n) to[i] = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(collected + (i - before)), k));
  }
}

// Selection over the cluster: the key at which the running count (BY_MASS: mass) of the descending order reaches the target, among the
// logits from `low` up; what lies above it, what it holds itself, and the target are left in `sh`.  False if the whole of it does not
// reach the target.  `buf` alternates: a buffer is cleared two rounds after it was filled, when every CTA has read it.
enum Selected { SELECT_NONE, SELECT_KEY, SELECT_FEW };
template <bool BY_MASS, typename T, bool STREAM, int NT, typename F>
__device__ __forceinline__ Selected select(SampleShared& sh, const Row<T, STREAM, NT>& row, const Weigh& w, const Binned& bins, float low, F target_of, int splits, int& buf, bool may_few,
                                           int index0, uint32_t* key, int* few) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto clear = [&] {
    for (int i = tid; i < SMP_BINS; i += NT) sh.hist[buf][i] = 0;
    __syncthreads();
  };
  clear();
  row.each_quad([&](int, const float4& v) {
    const float x[4] = {v.x, v.y, v.z, v.w};
    if (!BY_MASS) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x[e] >= low) add_to_bin<BY_MASS>(&sh.hist[buf][(int)bins.place(x[e])], w, x[e]);
    } else if (x[0] >= low || x[1] >= low || x[2] >= low || x[3] >= low) {      // (add_to_bin four times over, its steps side by side)
      unsigned long long m[4];
      uint32_t* bin[4];
      uint32_t old[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = w.fixed(x[e]);
        bin[e] = reinterpret_cast<uint32_t*>(&sh.hist[buf][x[e] >= low ? (int)bins.place(x[e]) : 0]);
        if (!(x[e] >= low)) m[e] = 0;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) old[e] = (uint32_t)m[e] ? atomicAdd(bin[e], (uint32_t)m[e]) : 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t hi = (uint32_t)(m[e] >> 32) + (old[e] + (uint32_t)m[e] < old[e]);
        if (hi) atomicAdd(bin[e] + 1, hi);
      }
    }
  });
  const bool found = find_bin<false, NT>(sh, buf, 0, target_of, splits);
  buf ^= 1;
  if (!found) return SELECT_NONE;
  const int b0 = sh.bin;
  const unsigned long long target = sh.target;
  auto known = [&](unsigned long long) { return target; };
  unsigned long long above = sh.above;
  // the bin's logits lie in this range (half a bin and two steps wider than that on both sides), which is cheaper to ask for
  const float x_top = 2.f * bins.half_top;
  float x_lo = fmaxf(low, bins.logit(b0 + 1.5f)), x_hi = fminf(x_top, bins.logit(b0 - 0.5f));
  if (x_lo > low) x_lo = logit_of(key_of(x_lo) - 2);
  if (x_hi < x_top) x_hi = logit_of(key_of(x_hi) + 2);
  // All that reaches the target lies in this bin and above.  If that is few logits, one CTA finishes with them: each collects its own in
  // the histogram that is free, as keys with inverted indices.  (By mass their number is not known, only that it is no less than at_least.)
  const bool try_few = may_few && (BY_MASS ? sh.at_least <= (float)SMP_FEW : above + sh.inside <= SMP_FEW);
  if (try_few) {
    if (tid == 0) sh.few[0] = 0;
    __syncthreads();
    row.each_quad([&](int i, const float4& v) {
      const float x[4] = {v.x, v.y, v.z, v.w};
      if (!(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= x_lo)) return;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x[e] >= low && (int)bins.place(x[e]) <= b0) {
          const uint32_t at = atomicAdd(&sh.few[0], 1u);
          if (at < SMP_FEW) sh.hist[buf][at] = (unsigned long long)key_of(x[e]) << 32 | (uint32_t)~(index0 + i + e);
        }
    });
    cluster_or_block_sync(splits);
    const uint32_t n = __reduce_add_sync(0xffffffffu, lane < splits ? ld_cluster32(ptx::map_to_cta(ptx::smem_u32(&sh.few[0]), lane)) : 0u);
    if (n <= SMP_FEW) {
      *few = (int)n;
      return SELECT_FEW;
    }
  }
  // A bin with a logit for every thread at most is resolved as it is (by mass, no logit of it weighs less than its end allows), another one by bins of its own.
  const bool small = BY_MASS ? (float)sh.inside * exp2f((float)(b0 + 1) * (1.f / 22.f) - 45.f) <= (float)NT : sh.inside <= NT;
  int b1 = -1;
  if (!small) {
    clear();
    row.each_logit([&](float x) {
      if (!(x >= x_lo && x <= x_hi)) return;
      const float t = bins.place(x);
      if (x >= low && (int)t == b0) add_to_bin<BY_MASS>(&sh.hist[buf][Binned::inner(t, b0)], w, x);
    });
    find_bin<false, NT>(sh, buf, above, known, splits);
    buf ^= 1;
    b1 = sh.bin;
  }
  auto in_bin = [&](float x) {
    if (!(x >= x_lo && x <= x_hi)) return false;
    const float t = bins.place(x);
    return x >= low && (int)t == b0 && (b1 < 0 || Binned::inner(t, b0) == b1);
  };
  // one logit, as a rule, or equal ones, or a few: each CTA collects its own, with the bin's smallest and largest key (the latter inverted)
  uint32_t lo = 0xffffffffu, hi = 0xffffffffu;
  if (tid == 0) sh.few[1] = 0;
  __syncthreads();
  row.each_logit([&](float x) {
    if (in_bin(x)) {
      lo = min(lo, key_of(x));
      hi = min(hi, ~key_of(x));
      const uint32_t at = atomicAdd(&sh.few[1], 1u);
      if (at < NT) sh.hist[buf][at] = key_of(x);
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_min_sync(0xffffffffu, hi);
  if (lane == 0) sh.warp_sum[warp] = (unsigned long long)hi << 32 | lo;
  __syncthreads();
  for (int i = 0; i < NT / 32; ++i) {
    lo = min(lo, (uint32_t)sh.warp_sum[i]);
    hi = min(hi, (uint32_t)(sh.warp_sum[i] >> 32));
  }
  uint32_t count = sh.few[1], n = count;
  if (splits > 1) {
    if (tid == 0) sh.range[BY_MASS] = (unsigned long long)hi << 32 | lo;
    cluster_or_block_sync(splits);
    count = 0;
    if (lane < splits) {
      const unsigned long long x = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.range[BY_MASS]), lane));
      count = ld_cluster32(ptx::map_to_cta(ptx::smem_u32(&sh.few[1]), lane));
      lo = min(lo, (uint32_t)x);
      hi = min(hi, (uint32_t)(x >> 32));
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_min_sync(0xffffffffu, hi);
    n = __reduce_add_sync(0xffffffffu, count);
  }
  *key = lo;
  if (lo == ~hi) return SELECT_KEY;
  if (n <= NT) {      // every CTA takes them all and finds the same
    unsigned long long *c = sh.hist[buf ^ 1], *mass = sh.hist[buf ^ 1] + NT;
    pull_few<NT>(c, sh.hist[buf], splits > 1 ? count : lane == 0 ? n : 0, (int)n, splits);
    buf ^= 1;              // (the collected ones stay as they are until the next histogram's barrier)
    __syncthreads();
    const uint32_t me = tid < (int)n ? (uint32_t)c[tid] : 0;
    if (tid < (int)n) mass[tid] = BY_MASS ? w.fixed(logit_of(me)) : 1ull;
    __syncthreads();
    if (tid < (int)n) {
      unsigned long long over = sh.above, same = 0;
      for (uint32_t i = 0; i < n; ++i) {
        const uint32_t k = (uint32_t)c[i];
        if (k > me) over += mass[i];
        if (k == me) same += mass[i];
      }
      if (over < target && over + same >= target) {      // (equal logits write the same)
        sh.found = me;
        sh.found_above = over;
        sh.inside = same;
      }
    }
    __syncthreads();
    *key = sh.found;
    if (tid == 0) sh.above = sh.found_above;
    __syncthreads();
    return SELECT_KEY;
  }
  // several logits share the bin (scores far closer to each other than weights can tell): by the bits of their keys
  uint32_t prefix = 0;
#pragma unroll 1
  for (int level = 0; level < 4; ++level) {
    const int shift = 22 - 10 * level > 0 ? 22 - 10 * level : 0, bits = level == 3 ? 2 : 10;
    above = sh.above;
    clear();
    row.each_logit([&](float x) {
      const uint32_t k = key_of(x);
      if (in_bin(x) && (level == 0 || k >> (shift + bits) == prefix)) add_to_bin<BY_MASS>(&sh.hist[buf][k >> shift & ((1u << bits) - 1)], w, x);
    });
    find_bin<true, NT>(sh, buf, above, known, splits);
    buf ^= 1;
    prefix = prefix << bits | (uint32_t)sh.bin;
  }
  *key = prefix;
  return SELECT_KEY;
}

// The place of the draw in `mass`: u >= 1 is the last unit, NaN the first.
__device__ __forceinline__ unsigned long long place_of(float u, unsigned long long mass) {
  const double at = (double)u * (double)mass;
  const unsigned long long target = at > 0.0 ? (unsigned long long)at : 0ull;
  return at >= (double)mass || target >= mass ? mass - 1 : target;
}

template <typename T, bool STREAM>
__global__ void __launch_bounds__(STREAM ? SMP_WIDE : SMP_THREADS, STREAM ? 2 : 4) sample_kernel(const SampleArgs a) {
  constexpr int NT = STREAM ? SMP_WIDE : SMP_THREADS, WARPS = NT / 32;
  extern __shared__ __align__(16) float l[];
  __shared__ SampleShared sh;
  ptx::pdl_wait();
  ptx::pdl_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x, row_i = blockIdx.y;
  const int from = min(a.vocab, rank * a.slice), n = min(a.vocab, from + a.slice) - from;
  const T* first = static_cast<const T*>(a.logits) + (long long)row_i * a.stride + from;
  Row<T, STREAM, NT> row;
  row.shift = (int)((reinterpret_cast<uintptr_t>(first) & 15) / sizeof(T));
  row.src = first - row.shift;
  row.end = row.shift + n;
  row.l = l;
  row.infinite = false;
  // a warp's part of the slice is contiguous: what is summed in the vocabulary's order is summed by warps, in steps of 128
  constexpr int STEP = 128;
  const int part = (row.end + WARPS * STEP - 1) / (WARPS * STEP) * STEP, index0 = from - row.shift;
  row.places = part * WARPS;
  const float temperature = a.temperature ? a.temperature[row_i] : 1.f, top_p = a.top_p ? a.top_p[row_i] : 1.f, min_p = a.min_p ? a.min_p[row_i] : 0.f, u = a.u[row_i];
  const int top_k = a.top_k ? a.top_k[row_i] : 0;
  const bool greedy = !(temperature > 0.f) || top_k == 1;
  float top = row.load();
  if (tid < 256) sh.table[tid] = exp2_table.v[tid];

  // ---- the largest logit -----------------------------------------------------------------------------------------------------
#pragma unroll
  for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
  if (lane == 0) sh.warp_sum[warp] = __float_as_uint(top);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WARPS; ++i) top = fmaxf(top, __uint_as_float((uint32_t)sh.warp_sum[i]));
  unsigned long long best = (unsigned long long)key_of(top) << 32;
  if (greedy) {      // and its first place
    uint32_t at = 0xffffffffu;
    row.each_quad([&](int i, const float4& v) {
      const uint32_t e = v.x == top ? 0 : v.y == top ? 1 : v.z == top ? 2 : v.w == top ? 3 : 4;
      if (e < 4) at = min(at, (uint32_t)(index0 + i) + e);
    });
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) sh.warp_ties[warp] = at;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) at = min(at, sh.warp_ties[i]);
    best |= (uint32_t)~at;
  }
  if (a.splits > 1) {
    if (tid == 0) sh.best = best;
    cluster_or_block_sync(a.splits);
    if (lane < a.splits) best = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.best), lane));
#pragma unroll
    for (int m = 16; m; m >>= 1) {
      const unsigned long long x = __shfl_xor_sync(0xffffffffu, best, m);
      best = x > best ? x : best;
    }
  }
  const uint32_t best_key = (uint32_t)(best >> 32);
  if (greedy || best_key <= KEY_NONE) {
    if (rank == 0 && tid == 0) {
      a.tokens[row_i] = best_key <= KEY_NONE ? -1 : (int)~(uint32_t)best;
      if (a.probs) a.probs[row_i] = best_key <= KEY_NONE ? 0.f : 1.f;
    }
    if (a.splits > 1) cluster_or_block_sync(a.splits);      // no CTA's shared memory goes while another reads it
    return;
  }
  top = logit_of(best_key);
  if (isinf(top)) {      // +infinity outweighs everything finite: as zeros against nothing
    row.infinite = true;
    if (!STREAM)
      for (int i = tid; i < row.places; i += NT) l[i] = row.against_infinity(l[i]);
    top = 0.f;
    __syncthreads();
  }

  // ---- the cut ---------------------------------------------------------------------------------------------------------------
  const double scale = 1.4426950408889634074 / (double)temperature;
  const Weigh w{scale, (double)top, sh.table};
  const Binned bins{0.5f * top, fminf((float)(44.0 * scale), 1e30f)};
  // the logits that weigh anything: nearly as far down as the bins go (two bins short of it: place() is off by less, but where one step of the
  // logits passes a bin, and there a few steps up are enough)
  Cut cut{fmaxf((float)((double)top - 45.9 / scale), LOWEST), 0.f, 0};
  while (cut.low < top && !(bins.place(cut.low) < Binned::END)) cut.low = logit_of(key_of(cut.low) + 1);
  auto cut_at = [&](uint32_t key, unsigned long long ties, bool all) {
    cut.ties = all ? 0 : ties;
    cut.tie = logit_of(key);
    cut.low = all ? cut.tie : logit_of(key + 1);
  };
  uint32_t least_key = 0;      // of the smallest logit whose weight is min_p or more (1 and more: of the largest logit)
  if (min_p > 0.f) {           // a step or two from where it should be, else by halves
    const double least = min_p < 1.f ? log2((double)min_p) : 0.0;
    const auto enough = [&](uint32_t k) { return ((double)logit_of(k) - (double)top) * scale >= least; };
    uint32_t hi = key_of(top), lo = key_of(LOWEST);
    const uint32_t near = key_of(fmaxf(fminf((float)((double)top + least / scale), top), LOWEST));
    if (near < hi - 2 && enough(near + 2)) hi = near + 2;
    if (near > lo + 2 && !enough(near - 2)) lo = near - 2;
    if (enough(lo)) hi = lo;
    while (hi - lo > 1) {      // (lo: not enough, hi: enough)
      const uint32_t mid = lo + (hi - lo) / 2;
      if (enough(mid)) hi = mid;
      else lo = mid;
    }
    least_key = hi;
  }
  auto share_of = [&](unsigned long long mass) {      // what top-p wants of a mass, one unit at least
    const double want = ceil((double)top_p * (double)mass);
    const unsigned long long target = want >= 1.0 ? (unsigned long long)want : 1ull;
    return target < mass ? target : mass;
  };
  int buf = 0, few = 0;
  uint32_t key;
  unsigned long long too_many = 0;      // ties that top-k leaves out
  Selected got = SELECT_NONE;
  bool by_count = false;
  if (top_k > 0 && top_k < a.vocab) {
    got = select<false>(sh, row, w, bins, cut.low, [&](unsigned long long) { return (unsigned long long)top_k; }, a.splits, buf, true, index0, &key, &few);
    by_count = got == SELECT_FEW;
    if (got == SELECT_KEY) {
      too_many = sh.inside - (top_k - sh.above);
      cut_at(key, top_k - sh.above, too_many == 0);
    }
  }
  if (top_p < 1.f && got != SELECT_FEW) {
    // of the mass that top-k left: the logits above the cut and the cut's ties (the bins hold all of those)
    if (too_many) too_many *= w.fixed(cut.tie);
    const bool whole = cut.ties == 0;      // (the candidates are those from the cut up)
    got = select<true>(sh, row, w, bins, cut.ties ? cut.tie : cut.low, [&](unsigned long long total) { return share_of(total - too_many); }, a.splits, buf, whole, index0, &key, &few);
    if (got == SELECT_KEY) {
      const unsigned long long each = w.fixed(logit_of(key)), ties = (sh.target - sh.above + each - 1) / each;
      cut_at(key, ties, ties * each == sh.inside);
    }
  }

  // ---- few candidates: the first CTA takes them all, in their order, and finishes alone ------------------------------------------------
  if (got == SELECT_FEW) {
    unsigned long long *c = sh.hist[buf ^ 1], *sums = sh.hist[buf];      // (the first was read by everyone before the candidates' barrier; the second has the slice's own)
    if (rank == 0) {
      const uint32_t count = lane < a.splits ? ld_cluster32(ptx::map_to_cta(ptx::smem_u32(&sh.few[0]), lane)) : 0;
      pull_few<NT>(c, sh.hist[buf], count, few, a.splits);
    }
    if (a.splits > 1) {
      __syncwarp();
      ptx::cluster_arrive();
      if (rank != 0) {
        ptx::cluster_wait();
        return;
      }
    }
    // in their order: a candidate's place is the number of those before it, and what it adds to the mass comes behind theirs
    const bool on = tid < few;
    __syncthreads();
    const unsigned long long me = on ? c[tid] : 0, weight = on ? w.fixed(logit_of((uint32_t)(me >> 32))) : 0;
    sums[tid] = weight;      // (NT >= SMP_FEW)
    __syncthreads();
    int place = 0;
    unsigned long long before = 0;
    if (on) {
#pragma unroll 4
      for (int i = 0; i < few; ++i) {
        if (c[i] > me) {
          ++place;
          before += sums[i];
        }
      }
    }
    // how many of them each rule keeps, and their mass
    const int counted = by_count ? min(top_k, few) : few;
    if (tid == 0) {
      sh.bin = counted;
      sh.kept = 0;
    }
    __syncthreads();
    if (on && place == counted - 1) sh.kept = before + weight;
    __syncthreads();
    const unsigned long long target = !(top_p < 1.f) ? 0 : by_count ? share_of(sh.kept) : sh.target;
    if (on && place < counted && target && before + weight >= target) atomicMin(&sh.bin, place + 1);
    if (on && (uint32_t)(me >> 32) < least_key) atomicMin(&sh.bin, place);
    __syncthreads();
    const int kept = sh.bin;
    if (on && place == kept - 1) sh.above = before + weight;
    sums[tid] = place < kept ? weight : 0;
    __syncthreads();
    // ... and the draw among those in the vocabulary's order (the inverted index falls with it)
    const unsigned long long draw = place_of(u, sh.above);
    if (on && place < kept) {
      before = 0;
#pragma unroll 4
      for (int i = 0; i < few; ++i)
        if ((uint32_t)c[i] > (uint32_t)me) before += sums[i];
      if (draw >= before && draw < before + weight) {
        a.tokens[row_i] = (int)~(uint32_t)me;
        if (a.probs) a.probs[row_i] = (float)(w.value(logit_of((uint32_t)(me >> 32))) / ((double)sh.above / (double)ONE));
      }
    }
    __syncwarp();
    if (a.splits > 1) ptx::cluster_wait();      // the others read this CTA's count of candidates: its memory stays until all of them have arrived (they have, long ago)
    return;
  }
  if (least_key) {
    const float x = logit_of(least_key);
    if (x > cut.tie) cut.ties = 0;
    cut.low = fmaxf(cut.low, x);
  }

  // ---- ties: those of the slices before this one, and of the warps before this one -----------------------------------------------
  unsigned long long ties_before = 0;
  if (cut.ties) {
    uint32_t mine = 0;
    for (int i = warp * part + lane * 4; i < (warp + 1) * part; i += STEP) {
      const float4 v = row.quad(i);
      mine += (v.x == cut.tie) + (v.y == cut.tie) + (v.z == cut.tie) + (v.w == cut.tie);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) sh.warp_ties[warp] = mine;
    __syncthreads();
    if (tid == 0) {
      uint32_t all = 0;
      for (int i = 0; i < WARPS; ++i) all += sh.warp_ties[i];
      sh.ties = all;
    }
    if (a.splits > 1) {
      cluster_or_block_sync(a.splits);
      for (int c = 0; c < rank; ++c) ties_before += ld_cluster32(ptx::map_to_cta(ptx::smem_u32(&sh.ties), c));
    }
    for (int i = 0; i < warp; ++i) ties_before += sh.warp_ties[i];
  }
  // The weights of four neighbouring places, of kept tokens only; `seen`: the cut's ties in front of this step.
  auto weights = [&](const float4& v, unsigned long long& seen, unsigned long long* m) {
    const float x[4] = {v.x, v.y, v.z, v.w};
    bool on[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) on[e] = x[e] >= cut.low;
    if (cut.ties) {
      uint32_t eq = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) eq += x[e] == cut.tie;
      uint32_t upto = eq;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      unsigned long long rank4 = seen + upto - eq;
      seen += __shfl_sync(0xffffffffu, upto, 31);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x[e] == cut.tie) on[e] = rank4++ < cut.ties;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = 0;
    if (on[0] || on[1] || on[2] || on[3]) {      // (no branch for each: four chains run side by side)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned long long f = w.fixed(x[e]);
        m[e] = on[e] ? f : 0;
      }
    }
  };

  // ---- the draw: running mass in the vocabulary's order ------------------------------------------------------------------------------
  unsigned long long seen = ties_before, sum = 0;
  constexpr int U = STREAM ? 4 : 2;      // steps whose loads are under way at once
  double whole = 0.0;
  for (int i0 = warp * part + lane * 4; i0 < (warp + 1) * part; i0 += U * STEP) {
    float4 v[U];
#pragma unroll
    for (int x = 0; x < U; ++x) v[x] = i0 + x * STEP < (warp + 1) * part ? row.quad(i0 + x * STEP) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
#pragma unroll
    for (int x = 0; x < U; ++x) {
      if (cut.ties) {
        unsigned long long m[4];
        weights(v[x], seen, m);
        sum += (m[0] + m[1]) + (m[2] + m[3]);
      } else if (fmaxf(fmaxf(v[x].x, v[x].y), fmaxf(v[x].z, v[x].w)) >= cut.low) {
        // (multiples of 2^-45, whose sum is exact in fp64 up to 256: fewer integer operations)
        const float y[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
        double r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __dadd_rn(__dadd_rn(w.value(y[e]), 128.0), -128.0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (y[e] >= cut.low) whole += r[e];
      }
    }
    if (whole >= 128.0) {      // (4 U more weights stay far below 256)
      sum += (unsigned long long)(whole * (double)ONE);
      whole = 0.0;
    }
  }
  sum += (unsigned long long)(whole * (double)ONE);
  sum = warp_sum(sum);
  __syncthreads();
  if (lane == 0) sh.warp_sum[warp] = sum;
  __syncthreads();
  unsigned long long start = 0, mass = 0;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    if (i < warp) start += sh.warp_sum[i];
    mass += sh.warp_sum[i];
  }
  if (a.splits > 1) {
    if (tid == 0) sh.kept = mass;
    cluster_or_block_sync(a.splits);
    const unsigned long long x = lane < a.splits ? ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.kept), lane)) : 0;
    start += warp_sum(lane < rank ? x : 0);
    mass = warp_sum(x);
  }
  const unsigned long long target = place_of(u, mass);
  if (target >= start && target < start + sum) {                             // this warp's part
    unsigned long long run = start;
    seen = ties_before;
    for (int i = warp * part + lane * 4; i < (warp + 1) * part; i += STEP) {
      const float4 v = row.quad(i);
      unsigned long long m[4];
      weights(v, seen, m);
      const unsigned long long four = m[0] + m[1] + m[2] + m[3], upto = warp_scan(four, lane) + run, before = upto - four;
      if (target >= before && target < upto) {
        const unsigned long long in = target - before;
        const int e = in < m[0] ? 0 : in < m[0] + m[1] ? 1 : in < m[0] + m[1] + m[2] ? 2 : 3;
        a.tokens[row_i] = index0 + i + e;
        if (a.probs) a.probs[row_i] = (float)(w.value(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w) / ((double)mass / (double)ONE));
      }
      run = __shfl_sync(0xffffffffu, upto, 31);
      if (target < run) break;
    }
  }
  if (a.splits > 1) cluster_or_block_sync(a.splits);
}

template <typename T, bool STREAM>
cudaError_t launch_sample(const SampleArgs& a, int rows, size_t smem, cudaStream_t st) {
  static thread_local int ready = -1;      // device that has the kernel's attributes
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && ready != dev && !STREAM) {
    e = cudaFuncSetAttribute(sample_kernel<T, STREAM>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (SMP_SLICE + SMP_THREADS * 4) * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<T, STREAM>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) ready = dev;
  }
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(a.splits, rows);
  cfg.blockDim = dim3(STREAM ? SMP_WIDE : SMP_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, STREAM>, a);
}
template <typename T>
cudaError_t launch_rows(const SampleArgs& a, int rows, size_t smem, bool stream, cudaStream_t st) {
  return stream ? launch_sample<T, true>(a, rows, 0, st) : launch_sample<T, false>(a, rows, smem, st);
}

}  // namespace
}  // namespace dc

extern "C" dc_status dc_sample_tokens(const void* logits_dev, int dtype, int n_rows, int vocab, long long row_stride, const dc_sample_rules* rules, const float* u_dev,
                                      int32_t* tokens_dev, float* probs_dev, void* cuda_stream) {
  using namespace dc;
  if (!logits_dev || !rules || !u_dev || !tokens_dev) {
    set_error("dc_sample_tokens: null pointer argument");
    return DC_ERR_ARG;
  }
  if (rules->size != sizeof(dc_sample_rules)) {
    set_error("dc_sample_tokens: dc_sample_rules.size is %u, this library's is %zu", rules->size, sizeof(dc_sample_rules));
    return DC_ERR_ARG;
  }
  if ((dtype != DC_F32 && dtype != DC_BF16 && dtype != DC_F16) || n_rows < 1 || n_rows > 65535 || vocab < 1 || vocab > DC_SAMPLE_MAX_VOCAB || row_stride < vocab) {
    set_error("dc_sample_tokens: need a dtype of DC_F32, DC_BF16 or DC_F16, 1 <= n_rows <= 65535, 1 <= vocab <= %d, row_stride >= vocab", DC_SAMPLE_MAX_VOCAB);
    return DC_ERR_ARG;
  }
  if (reinterpret_cast<uintptr_t>(logits_dev) & 15) {
    set_error("dc_sample_tokens: logits_dev must be 16-byte aligned");
    return DC_ERR_ARG;
  }
  int dev = 0, n_sm = 0, major = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (e != cudaSuccess || major != 10) {
    set_error("dc_sample_tokens: %s", e != cudaSuccess ? cudaGetErrorString(e) : "this library is built for sm_100a only");
    return DC_ERR_CUDA;
  }
  SampleArgs a{logits_dev, row_stride, vocab, 0, 1, rules->temperature_dev, rules->top_p_dev, rules->min_p_dev, u_dev, rules->top_k_dev, tokens_dev, probs_dev};
  // Rows enough for every SM: a CTA streams its row, of a long row two, so that the rows under way stay in the L2 cache from one pass to the next (256 rows
  // of 131,072, top-k of 50: 107 us in one, 84 us in two, 100 us in four, 139 us in shared memory).  Else the row lies in the shared memory of a cluster: as many CTAs as its logits need, and while SMs are
  // idle twice as many as long as one has more than 4,096 logits (4,097 become 2 x 2,049; one CTA against two at that border has not been measured).
  const bool stream = n_rows >= n_sm && vocab > SMP_SLICE;
  if (stream) {
    a.splits = vocab > 4 * SMP_SLICE ? 2 : 1;
  } else {
    while (a.splits < SMP_MAX_CLUSTER && (long long)a.splits * SMP_SLICE < vocab) a.splits *= 2;
    while (a.splits < SMP_MAX_CLUSTER && (long long)n_rows * a.splits * 2 <= n_sm && vocab / a.splits > 4096) a.splits *= 2;
  }
  a.slice = ((vocab + a.splits - 1) / a.splits + 7) & ~7;
  const int part = (a.slice + 7 + SMP_THREADS * 4 - 1) / (SMP_THREADS * 4) * (SMP_THREADS * 4);
  const size_t smem = (size_t)part * 4;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  e = dtype == DC_F32 ? launch_rows<float>(a, n_rows, smem, stream, st)
                      : dtype == DC_BF16 ? launch_rows<__nv_bfloat16>(a, n_rows, smem, stream, st) : launch_rows<__half>(a, n_rows, smem, stream, st);
  if (e != cudaSuccess) {
    cudaGetLastError();      // (a refused launch leaves its code behind)
    set_error("dc_sample_tokens: launch failed: %s", cudaGetErrorString(e));
    return DC_ERR_CUDA;
  }
  return DC_OK;
}
