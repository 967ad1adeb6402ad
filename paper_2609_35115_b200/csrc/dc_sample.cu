// Choice of the next token from rows of logits (include/dc.h, dc_sample_tokens): temperature, top-k, top-p, min-p, from given random numbers.
//
// One pass over the logits: a cluster of CTAs keeps a row in shared memory, each CTA a contiguous slice of the vocabulary, and
// everything after the load happens there.  The rules cut a prefix of the order "descending logit, ties by lowest index", so the kept set is
// a cut key and a number of its ties; cuts are found by selection through histograms, by counts (top-k) or by mass (top-p).
//
// The result is a whole number that has to be the right one, so masses are exact: a weight exp((l - max) / T) is evaluated in fp64
// (2^(j/256) from a table times a polynomial; about 2^-50) and held as an integer multiple of 2^-45.  Integer sums do not depend on their order: atomics, splits
// and replays give the same token.  Against sums in real arithmetic a border is off by at most 2^-46 for every token of the row; a
// border that close to a row's random number is met once in millions of rows.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "dc_internal.h"
#include "dc_ptx.cuh"

namespace dc {
namespace {

constexpr int SMP_THREADS = 512, SMP_WARPS = SMP_THREADS / 32;
constexpr int SMP_BINS = 2048, SMP_PER = SMP_BINS / SMP_THREADS;
constexpr int SMP_SLICE = 16384;          // logits of a CTA at most
constexpr int SMP_MAX_CLUSTER = 16;
constexpr uint32_t KEY_NONE = 0x007fffffu;   // key of -infinity: such logits, and NaN, take no part
constexpr unsigned long long ONE = 1ull << 45;

struct SampleArgs {
  const void*    logits;
  long long      stride;
  int            vocab, slice, splits;    // slice: logits of a CTA
  const float *  temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t*       tokens;
  float*         probs;
};

struct SampleShared {
  unsigned long long hist[2][SMP_BINS];
  double             table[256];           // 2^(j / 256)
  unsigned long long best;                 // key and inverted index of the slice's maximum
  unsigned long long range[2];             // smallest and largest key of a selection's last bin
  unsigned long long kept;                 // mass of the slice's kept tokens
  unsigned long long warp_sum[SMP_WARPS];
  unsigned long long above;                // count or mass above the found bin, and of it
  unsigned long long inside;
  uint32_t           warp_ties[SMP_WARPS];
  uint32_t           ties;                 // of the slice
  int                bin;
};

__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l);
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

// Weights of a row.
struct Weigh {
  double scale, top;   // log2(e) / T, the largest logit
  bool   infinite;     // the largest logit is +infinity: it alone has weight
  const double* table;
  // 2^y for -46 <= y <= 0: y = k / 256 + f with |f| <= 2^-9, 2^f by the first terms of its series (the rest is below 2^-54)
  __device__ __forceinline__ double value(float l) const {
    if (infinite) return l == INFINITY ? 1.0 : 0.0;
    const double y = ((double)l - top) * scale;
    if (!(y >= -46.0)) return 0.0;
    const double magic = 6755399441055744.0 / 256.0;      // 1.5 * 2^52 / 256
    const double t = y + magic, f = y - (t - magic);
    const int k = __double2loint(t);
    const double r = table[k & 255];
    const double p = fma(fma(fma(9.618129107628477e-3, f, 5.550410866482158e-2), f, 2.402265069591007e-1), f, 6.931471805599453e-1) * f;
    const double v = fma(r, p, r);
    return __hiloint2double(__double2hiint(v) + (k >> 8) * (1 << 20), __double2loint(v));
  }
  // in units of 2^-45: the lowest bit of a number just above 2^7 is that
  static __device__ __forceinline__ unsigned long long fix(double w) { return (unsigned long long)(__double_as_longlong(w + 128.0) - __double_as_longlong(128.0)); }
  __device__ __forceinline__ unsigned long long fixed(float l) const { return fix(value(l)); }
};

// The kept tokens: keys above `key`, and the first `ties` (in the vocabulary's order) of those equal to it.
struct Cut {
  uint32_t           key;
  unsigned long long ties;
};

// Loads the slice: 16-byte vectors on their own alignment, so that the first `shift` places of shared memory lie before the slice.
template <typename T>
__device__ __forceinline__ float as_float(T x) { return (float)x; }

template <typename T>
__device__ __forceinline__ void load_slice(const T* src, int n, int shift, float* l) {
  constexpr int VE = 16 / sizeof(T);
  const int vectors = (shift + n + VE - 1) / VE;
#pragma unroll 4
  for (int v = threadIdx.x; v < vectors; v += SMP_THREADS) {
    const int at = v * VE - shift;
    alignas(16) T x[VE];
    if (at >= 0 && at + VE <= n) {
      *reinterpret_cast<uint4*>(x) = __ldcs(reinterpret_cast<const uint4*>(src + at));
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = at + i >= 0 && at + i < n ? src[at + i] : (T)-INFINITY;
    }
#pragma unroll
    for (int i = 0; i < VE; i += 4) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f = as_float(x[i + e]) + 0.0f;      // (-0 becomes 0: the two are one logit)
        y[e] = f == f ? f : -INFINITY;
      }
      *reinterpret_cast<float4*>(l + v * VE + i) = make_float4(y[0], y[1], y[2], y[3]);
    }
  }
}

__device__ __forceinline__ void cluster_or_block_sync(int splits) {
  if (splits > 1) {
    ptx::cluster_arrive();
    ptx::cluster_wait();
  } else {
    __syncthreads();
  }
}

// Bins of a row.  Selection needs bins that fall with the logit and spread the row's logits, so that few of a warp's lanes meet in one:
// 32 to a factor of two of weight, then 2048 in each of those, by fp32 arithmetic (each operation is monotone, and the
// second bin is exact in what the first one left).
struct Binned {
  float top, scale;      // scale: 64 log2(e) / T, of half a difference (a whole one may pass fp32's range)
  static __device__ __forceinline__ bool is_weighed(float t) { return t < 46.f * 32.f; }    // behind that a weight is below half of 2^-45
  // (rounded products and differences, spelt out: joined into one operation they would not be what the bins were cut by)
  __device__ __forceinline__ float place(float l) const { return l == top ? 0.f : __fmul_rn(fmaf(l, -0.5f, 0.5f * top), scale); }
  static __device__ __forceinline__ int inner(float t, int bin) { return (int)__fmul_rn(__fsub_rn(t, (float)bin), 2048.f); }
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

// Sums the cluster's histograms from bin 0 up (DOWN: from the last bin down) and finds the bin in which `over` plus the running sum reaches
// target(total).
template <bool DOWN, typename F>
__device__ __forceinline__ bool find_bin(SampleShared& sh, int buf, unsigned long long over, F target_of, int splits, int* bin, unsigned long long* above, unsigned long long* inside) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) sh.bin = -1;
  cluster_or_block_sync(splits);
  unsigned long long own[SMP_PER], sum = 0;
#pragma unroll
  for (int i = 0; i < SMP_PER; ++i) own[i] = 0;
  const int b0 = DOWN ? SMP_BINS - SMP_PER - tid * SMP_PER : tid * SMP_PER;
  for (int c = 0; c < splits; ++c) {
    const uint32_t at = ptx::map_to_cta(ptx::smem_u32(&sh.hist[buf][b0]), c);
#pragma unroll
    for (int i = 0; i < SMP_PER; ++i) own[i] += ld_cluster64(at + (DOWN ? SMP_PER - 1 - i : i) * 8);
  }
#pragma unroll
  for (int i = 0; i < SMP_PER; ++i) sum += own[i];
  unsigned long long upto = warp_scan(sum, lane);
  if (lane == 31) sh.warp_sum[warp] = upto;
  __syncthreads();
  upto += over - sum;
  unsigned long long total = 0;
#pragma unroll
  for (int i = 0; i < SMP_WARPS; ++i) {
    if (i < warp) upto += sh.warp_sum[i];
    total += sh.warp_sum[i];
  }
  const unsigned long long target = target_of(total);
#pragma unroll
  for (int i = 0; i < SMP_PER; ++i) {
    if (upto < target && upto + own[i] >= target) {
      sh.bin = DOWN ? b0 + SMP_PER - 1 - i : b0 + i;
      sh.above = upto;
      sh.inside = own[i];
    }
    upto += own[i];
  }
  __syncthreads();
  *bin = sh.bin;
  *above = sh.above;
  *inside = sh.inside;
  __syncthreads();      // (the next search begins by resetting them)
  return *bin >= 0;
}

// Calls f(logit) for every logit of this thread's share of the slice.
template <typename F>
__device__ __forceinline__ void each_logit(const float* l, int places, F f) {
  for (int i = threadIdx.x * 4; i < places; i += SMP_THREADS * 4) {
    const float4 v = *reinterpret_cast<const float4*>(l + i);
    f(v.x);
    f(v.y);
    f(v.z);
    f(v.w);
  }
}

// Selection over the cluster: the key at which the running count (BY_MASS: mass) of the descending order reaches the target, among the
// keys above `floor_key`; what lies above it; and what it holds itself.  False if the whole of it does not reach the target.  `buf` alternates: a buffer is cleared
// two rounds after it was filled, when every CTA has read it.
template <bool BY_MASS, typename F>
__device__ __forceinline__ bool select(SampleShared& sh, const float* l, int places, const Weigh& w, const Binned& bins, uint32_t floor_key, F target_of, int splits, int& buf, uint32_t* key,
                                       unsigned long long* above, unsigned long long* inside) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int b0, b1;
  auto clear = [&] {
    for (int i = tid; i < SMP_BINS; i += SMP_THREADS) sh.hist[buf][i] = 0;
    __syncthreads();
  };
  clear();
  each_logit(l, places, [&](float x) {
    const float t = bins.place(x);
    if (Binned::is_weighed(t) && key_of(x) > floor_key) add_to_bin<BY_MASS>(&sh.hist[buf][(int)t], w, x);
  });
  unsigned long long target = 0;
  const bool found = find_bin<false>(sh, buf, 0, [&](unsigned long long total) { return target = target_of(total); }, splits, &b0, above, inside);
  buf ^= 1;
  if (!found) return false;
  auto known = [&](unsigned long long) { return target; };
  clear();
  each_logit(l, places, [&](float x) {
    const float t = bins.place(x);
    if (Binned::is_weighed(t) && (int)t == b0 && key_of(x) > floor_key) add_to_bin<BY_MASS>(&sh.hist[buf][Binned::inner(t, b0)], w, x);
  });
  find_bin<false>(sh, buf, *above, known, splits, &b1, above, inside);
  buf ^= 1;
  auto in_bin = [&](float x) {
    const float t = bins.place(x);
    return Binned::is_weighed(t) && (int)t == b0 && Binned::inner(t, b0) == b1 && key_of(x) > floor_key;
  };
  // one logit, as a rule, or equal ones: the bin's smallest and largest key (the latter inverted)
  uint32_t lo = 0xffffffffu, hi = 0xffffffffu;
  each_logit(l, places, [&](float x) {
    if (in_bin(x)) {
      lo = min(lo, key_of(x));
      hi = min(hi, ~key_of(x));
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_min_sync(0xffffffffu, hi);
  if (lane == 0) sh.warp_sum[warp] = (unsigned long long)hi << 32 | lo;
  __syncthreads();
  for (int i = 0; i < SMP_WARPS; ++i) {
    lo = min(lo, (uint32_t)sh.warp_sum[i]);
    hi = min(hi, (uint32_t)(sh.warp_sum[i] >> 32));
  }
  if (splits > 1) {
    if (tid == 0) sh.range[BY_MASS] = (unsigned long long)hi << 32 | lo;
    cluster_or_block_sync(splits);
    for (int c = 0; c < splits; ++c) {
      const unsigned long long x = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.range[BY_MASS]), c));
      lo = min(lo, (uint32_t)x);
      hi = min(hi, (uint32_t)(x >> 32));
    }
  }
  *key = lo;
  if (lo == ~hi) return true;
  // several logits share the bin (scores far closer to each other than a weight can tell): by the bits of their keys
  uint32_t prefix = 0;
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    clear();
    each_logit(l, places, [&](float x) {
      const uint32_t k = key_of(x);
      if (in_bin(x) && (level == 0 || k >> (shift + bits) == prefix)) add_to_bin<BY_MASS>(&sh.hist[buf][k >> shift & ((1u << bits) - 1)], w, x);
    });
    int digit;
    find_bin<true>(sh, buf, *above, known, splits, &digit, above, inside);
    buf ^= 1;
    prefix = prefix << bits | (uint32_t)digit;
  }
  *key = prefix;
  return true;
}

template <typename T>
__global__ void __launch_bounds__(SMP_THREADS, 2) sample_kernel(const SampleArgs a) {
  extern __shared__ __align__(16) float l[];
  __shared__ SampleShared sh;
  ptx::pdl_wait();
  ptx::pdl_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x, row = blockIdx.y;
  const int from = min(a.vocab, rank * a.slice), n = min(a.vocab, from + a.slice) - from;
  const T* src = static_cast<const T*>(a.logits) + (long long)row * a.stride + from;
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
  const float temperature = a.temperature ? a.temperature[row] : 1.f, top_p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f, u = a.u[row];
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const bool greedy = !(temperature > 0.f) || top_k == 1;

  load_slice(src, n, shift, l);
  if (!greedy && tid < 256) sh.table[tid] = exp2(tid * (1.0 / 256.0));
  // a warp's part of the slice is contiguous: what is summed in the vocabulary's order is summed by warps, in steps of 128
  constexpr int STEP = 128;
  const int filled = (shift + n + 7) & ~7;                                  // (vectors of 16 bytes fill up to 8 places)
  const int part = (filled + SMP_WARPS * STEP - 1) / (SMP_WARPS * STEP) * STEP, places = part * SMP_WARPS;
  for (int i = ((shift + n + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T))) * (16 / (int)sizeof(T)) + tid; i < places; i += SMP_THREADS) l[i] = -INFINITY;
  __syncthreads();

  // ---- the largest logit and its first place ------------------------------------------------------------------------------
  unsigned long long best = 0;
  for (int i = tid * 4; i < places; i += SMP_THREADS * 4) {
    const float4 v = *reinterpret_cast<const float4*>(l + i);
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned long long k = (unsigned long long)key_of(x[e]) << 32 | (uint32_t)~(from - shift + i + e);
      best = k > best ? k : best;
    }
  }
#pragma unroll
  for (int m = 16; m; m >>= 1) {
    const unsigned long long x = __shfl_xor_sync(0xffffffffu, best, m);
    best = x > best ? x : best;
  }
  if (lane == 0) sh.warp_sum[warp] = best;
  __syncthreads();
  for (int i = 0; i < SMP_WARPS; ++i) best = sh.warp_sum[i] > best ? sh.warp_sum[i] : best;
  if (a.splits > 1) {
    if (tid == 0) sh.best = best;
    ptx::cluster_arrive();
    ptx::cluster_wait();
    for (int c = 0; c < a.splits; ++c) {
      const unsigned long long x = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.best), c));
      best = x > best ? x : best;
    }
  }
  const uint32_t best_key = (uint32_t)(best >> 32);
  if (greedy || best_key <= KEY_NONE) {
    if (rank == 0 && tid == 0) {
      a.tokens[row] = best_key <= KEY_NONE ? -1 : (int)~(uint32_t)best;
      if (a.probs) a.probs[row] = best_key <= KEY_NONE ? 0.f : 1.f;
    }
    if (a.splits > 1) {      // no CTA's shared memory goes while another reads it
      ptx::cluster_arrive();
      ptx::cluster_wait();
    }
    return;
  }

  // ---- the cut ---------------------------------------------------------------------------------------------------------------
  const float top = logit_of(best_key);
  const Weigh w{1.4426950408889634074 / (double)temperature, (double)top, isinf(top) != 0, sh.table};
  const Binned bins{top, isinf(top) ? 1e30f : fminf((float)(64.0 * w.scale), 1e30f)};
  Cut cut{KEY_NONE, 0};
  int buf = 0;
  uint32_t key;
  unsigned long long above, inside;
  if (top_k > 0 && top_k < a.vocab && select<false>(sh, l, places, w, bins, KEY_NONE, [&](unsigned long long) { return (unsigned long long)top_k; }, a.splits, buf, &key, &above, &inside)) {
    cut.key = key;
    cut.ties = top_k - above;
    if (cut.ties == inside) cut = Cut{key - 1, 0};      // (all of them)
  }
  if (top_p < 1.f) {
    // of the mass that top-k left: the keys above the cut and the cut's ties (the bins hold all of those)
    const uint32_t floor_key = cut.ties ? cut.key - 1 : cut.key;
    const unsigned long long too_many = cut.ties ? (inside - cut.ties) * w.fixed(logit_of(cut.key)) : 0;
    unsigned long long target = 0;
    auto part_of = [&](unsigned long long total) {
      const unsigned long long mass = total - too_many;
      const double want = ceil((double)top_p * (double)mass);
      target = want >= 1.0 ? (unsigned long long)want : 1ull;
      return target = target < mass ? target : mass;
    };
    if (select<true>(sh, l, places, w, bins, floor_key, part_of, a.splits, buf, &key, &above, &inside)) {
      const unsigned long long each = w.fixed(logit_of(key)), need = target - above;
      cut.key = key;
      cut.ties = (need + each - 1) / each;
      if (cut.ties * each == inside) cut = Cut{key - 1, 0};
    }
  }

  // ---- ties: those of the slices before this one, and of the warps before this one -----------------------------------------------
  unsigned long long ties_before = 0;
  if (cut.ties) {
    uint32_t mine = 0;
    for (int i = warp * part + lane * 4; i < (warp + 1) * part; i += STEP) {
      const float4 v = *reinterpret_cast<const float4*>(l + i);
      mine += (key_of(v.x) == cut.key) + (key_of(v.y) == cut.key) + (key_of(v.z) == cut.key) + (key_of(v.w) == cut.key);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) sh.warp_ties[warp] = mine;
    __syncthreads();
    if (tid == 0) {
      uint32_t all = 0;
      for (int i = 0; i < SMP_WARPS; ++i) all += sh.warp_ties[i];
      sh.ties = all;
    }
    if (a.splits > 1) {
      ptx::cluster_arrive();
      ptx::cluster_wait();
      for (int c = 0; c < rank; ++c) ties_before += ld_cluster32(ptx::map_to_cta(ptx::smem_u32(&sh.ties), c));
    }
    for (int i = 0; i < warp; ++i) ties_before += sh.warp_ties[i];
  }
  // The fixed weights of four neighbouring places, of kept tokens only; `seen`: the cut's ties in front of this step.
  auto weights = [&](int i, unsigned long long& seen, unsigned long long* m) {
    const float4 v = *reinterpret_cast<const float4*>(l + i);
    const float x[4] = {v.x, v.y, v.z, v.w};
    unsigned long long rank4 = 0;
    if (cut.ties) {
      uint32_t eq = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) eq += key_of(x[e]) == cut.key;
      uint32_t upto = eq;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      rank4 = seen + upto - eq;
      seen += __shfl_sync(0xffffffffu, upto, 31);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = key_of(x[e]);
      bool on = k > cut.key;
      if (k == cut.key && cut.ties) on = rank4++ < cut.ties;
      const double wd = on ? w.value(x[e]) : 0.0;
      m[e] = on && wd >= (double)min_p ? Weigh::fix(wd) : 0;
    }
  };

  // ---- the draw: running mass in the vocabulary's order ------------------------------------------------------------------------------
  unsigned long long seen = ties_before, sum = 0;
  for (int i = warp * part + lane * 4; i < (warp + 1) * part; i += STEP) {
    unsigned long long m[4];
    weights(i, seen, m);
    sum += m[0] + m[1] + m[2] + m[3];
  }
  sum = warp_sum(sum);
  __syncthreads();
  if (lane == 0) sh.warp_sum[warp] = sum;
  __syncthreads();
  unsigned long long start = 0, total = 0;
  for (int i = 0; i < SMP_WARPS; ++i) {
    if (i < warp) start += sh.warp_sum[i];
    total += sh.warp_sum[i];
  }
  unsigned long long mass = total;
  if (a.splits > 1) {
    if (tid == 0) sh.kept = total;
    ptx::cluster_arrive();
    ptx::cluster_wait();
    mass = 0;
    for (int c = 0; c < a.splits; ++c) {
      const unsigned long long x = ld_cluster64(ptx::map_to_cta(ptx::smem_u32(&sh.kept), c));
      if (c < rank) start += x;
      mass += x;
    }
  }
  const double at = (double)u * (double)mass;
  unsigned long long target = at > 0.0 ? (unsigned long long)at : 0ull;      // (NaN: 0)
  if (at >= (double)mass || target >= mass) target = mass - 1;               // u >= 1: the last kept token
  if (target >= start && target < start + sum) {                             // this warp's part
    unsigned long long run = start;
    seen = ties_before;
    for (int i = warp * part + lane * 4; i < (warp + 1) * part; i += STEP) {
      unsigned long long m[4];
      weights(i, seen, m);
      const unsigned long long four = m[0] + m[1] + m[2] + m[3], upto = warp_scan(four, lane) + run;
      unsigned long long before = upto - four;
      if (target >= before && target < upto) {
        int e = 0;
        while (target >= before + m[e]) before += m[e++];
        a.tokens[row] = from - shift + i + e;
        if (a.probs) a.probs[row] = (float)(w.value(l[i + e]) / ((double)mass / (double)ONE));
      }
      run = __shfl_sync(0xffffffffu, upto, 31);
      if (target < run) break;
    }
  }
  if (a.splits > 1) {
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
}

template <typename T>
cudaError_t launch_sample(const SampleArgs& a, int rows, size_t smem, cudaStream_t st) {
  static thread_local int ready = -1;      // device that has the kernel's attributes
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && ready != dev) {
    e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (SMP_SLICE + SMP_WARPS * 128 + 64) * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) ready = dev;
  }
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(a.splits, rows);
  cfg.blockDim = dim3(SMP_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a);
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
  // CTAs of a row: as many as its logits need, and while SMs are idle more, down to 4096 logits each.
  while ((long long)a.splits * SMP_SLICE < vocab) a.splits *= 2;
  while (a.splits < SMP_MAX_CLUSTER && (long long)n_rows * a.splits * 2 <= n_sm && vocab / a.splits > 4096) a.splits *= 2;
  a.slice = ((vocab + a.splits - 1) / a.splits + 7) & ~7;
  const int filled = (a.slice + 7 + 7) & ~7, part = (filled + SMP_WARPS * 128 - 1) / (SMP_WARPS * 128) * 128;
  const size_t smem = (size_t)part * SMP_WARPS * 4;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  e = dtype == DC_F32 ? launch_sample<float>(a, n_rows, smem, st) : dtype == DC_BF16 ? launch_sample<__nv_bfloat16>(a, n_rows, smem, st) : launch_sample<__half>(a, n_rows, smem, st);
  if (e != cudaSuccess) {
    cudaGetLastError();      // (a refused launch leaves its code behind)
    set_error("dc_sample_tokens: launch failed: %s", cudaGetErrorString(e));
    return DC_ERR_CUDA;
  }
  return DC_OK;
}
