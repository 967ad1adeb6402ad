// The operators over a token cache (include/dc.h): norms and rotation of queries and keys with the append of keys and values,
// and attention with a sliding window and first tokens that stay visible.  This file holds the boundary, the append and the
// attention of single tokens; dc_token_attn.cuh the attention of chunks.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <mutex>
#include <new>

#include "dc_internal.h"
#include "dc_ptx.cuh"
#include "dc_token_cache.h"

namespace dc {
namespace {

using bf16 = __nv_bfloat16;

template <typename T> struct Num;
template <> struct Num<bf16> {
  static constexpr bool is_bf16 = true;
  // whether one of the two values is an infinity or a NaN
  static __device__ __forceinline__ bool odd(uint32_t v) { return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u; }
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  // A weighted mean, its weights' sum off by their rounding: finite values have no mean beyond the type's largest.  (In bf16 the sums pass fp32's range before.)
  static __device__ __forceinline__ float mean(float x) { return x; }
};
template <> struct Num<__half> {
  static constexpr bool is_bf16 = false;
  static __device__ __forceinline__ bool odd(uint32_t v) { return (v & 0x7c00u) == 0x7c00u || (v & 0x7c000000u) == 0x7c000000u; }
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ float mean(float x) { return fabsf(x) < INFINITY ? fminf(fmaxf(x, -65504.f), 65504.f) : x; }
};

// 16 bytes global -> shared, asynchronously; off: zeros, and the source is not read.
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}

// ---------------------------------------------------------------------------------------------
// Append: y = x / sqrt(mean x^2 + eps) * g for each head of q and k, rotated by position * inv_freq; k and v to their rows.
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
  CacheDims   d;
  TokenBatch  b;
  const void* qkv;
  long long   qkv_stride, q_stride;
  void *      q, *k, *v;
  const float *q_gain, *k_gain, *inv_freq;
  int         rot;
  float       eps;
  int         share;     // warps that a token's row is dealt out over
};

constexpr int APPEND_WARPS = 8;
constexpr int APPEND_DEPTH = 8;    // 16-byte pieces that a lane has in flight

// Bound by the reads and writes of the rows.  Warps work alone, `share` of them on a token: all of a CTA's for single tokens, where the
// latency of one row counts, one for prompts, where the look-up of the token's sequence and its angles are paid once for the whole row.
// A head is D / 8 neighbouring lanes of 16 bytes each, so the sum of squares and the partner of a
// rotated pair come from shuffles, every value is read once and written once, and a lane's gains and angles are the same for
// all heads; two values go through each operation.  The angle is position * inv_freq in 64 bits, in turns, whose fraction is exact enough in 32 for sincospi.
// Measured: 6,162 tokens of 48 heads of 128, 28.7 us, 5.3 TB/s (43 us with four pieces a lane in registers in flight instead of eight in shared memory).
template <typename T, int D, bool INTER>
__global__ void __launch_bounds__(APPEND_WARPS * 32, 3) append_kernel(const AppendArgs a) {
  constexpr int LPH = D / 8;
  __shared__ uint4 rings[APPEND_WARPS][APPEND_DEPTH * 32];
  __shared__ __align__(16) float2 turns[APPEND_WARPS][D / 2];
  ptx::pdl_wait();
  ptx::pdl_launch();
  const int lane = threadIdx.x & 31, id = blockIdx.x * APPEND_WARPS + (threadIdx.x >> 5), half = a.rot / 2, l = lane % LPH;
  const int token = id / a.share, part = id % a.share;
  if (token >= a.b.n_tokens) return;
  const int q_end = a.d.n_heads * LPH, k_end = q_end + a.d.n_kv_heads * LPH, chunks = k_end + a.d.n_kv_heads * LPH, step = 32 * a.share;
  const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.qkv) + (long long)token * a.qkv_stride);
  // the row's pieces come through a ring of shared memory, each lane's its own: nobody waits for another's (a row behind the last sequence
  // is read for nothing)
  uint4* ring = rings[threadIdx.x >> 5] + lane;
  auto fetch = [&](int c, int slot) {
    if (c < chunks) cp16(ptx::smem_u32(ring + slot * 32), src + c, true);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int u = 0; u < APPEND_DEPTH; ++u) fetch(part * 32 + u * step + lane, u);
  // the token's sequence: the boundaries at or below it, counted 32 at a time
  int seq = token;
  if (a.b.cu_tokens) {
    seq = -1;
    for (int i0 = 0; i0 <= a.b.n_seqs; i0 += 32) {
      const int c = i0 + lane <= a.b.n_seqs ? a.b.cu_tokens[i0 + lane] : INT_MAX;
      const unsigned le = __ballot_sync(0xffffffffu, c <= token);
      seq += __popc(le);
      if (le != 0xffffffffu) break;
    }
  }
  TokenSeq s{};
  if (seq >= 0 && seq < a.b.n_seqs) s = load_seq(a.b, a.d, seq);
  if (token - s.first >= s.count || token < s.first) {      // no sequence's row, or one that does not fit
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    return;
  }
  const int pos = s.start + (token - s.first);
  float2* turn = turns[threadIdx.x >> 5];
  for (int j = lane; j < half; j += 32) {
    const double t = (double)pos * (double)a.inv_freq[j] * 0.15915494309189533577;
    float sn, cs;
    sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
    turn[j] = make_float2(cs, sn);
  }
  __syncwarp();
  // This lane's part of gain and rotation, for q and for k: y = (x c + other s) / rms, where `other` is the other value of the pair (its
  // neighbour, or the same place of the lane half a rotated head away), c the value's gain times the cosine, s the other's gain times the sine.
  const int hl = half / 8;
  const bool lower = l < hl, turned = INTER ? 8 * l < a.rot : l < 2 * hl;
  const int partner = INTER || !turned ? lane : lane + (lower ? hl : -hl), lp = partner % LPH;
  float2 mc[2][4], ms[2][4];
  {
    float cs[8], sn[8];      // (16 bytes a load: there are many of these values for a row of few heads)
    const float4* t4 = reinterpret_cast<const float4*>(turn + (turned ? (INTER ? 4 * l : 8 * (lower ? l : l - hl)) : 0));
#pragma unroll
    for (int i = 0; i < (INTER ? 2 : 4); ++i) {
      const float4 t = turned ? t4[i] : make_float4(1.f, 0.f, 1.f, 0.f);
      if (INTER) {
        cs[4 * i] = cs[4 * i + 1] = t.x;
        cs[4 * i + 2] = cs[4 * i + 3] = t.z;
        sn[4 * i] = -t.y;
        sn[4 * i + 1] = t.y;
        sn[4 * i + 2] = -t.w;
        sn[4 * i + 3] = t.w;
      } else {
        cs[2 * i] = t.x;
        cs[2 * i + 1] = t.z;
        sn[2 * i] = lower ? -t.y : t.y;
        sn[2 * i + 1] = lower ? -t.w : t.w;
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float4* g = reinterpret_cast<const float4*>(w ? a.k_gain : a.q_gain);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 mine = __ldg(g + 2 * l + i), far = INTER ? make_float4(mine.y, mine.x, mine.w, mine.z) : __ldg(g + 2 * lp + i);
        mc[w][2 * i] = make_float2(mine.x * cs[4 * i], mine.y * cs[4 * i + 1]);
        mc[w][2 * i + 1] = make_float2(mine.z * cs[4 * i + 2], mine.w * cs[4 * i + 3]);
        ms[w][2 * i] = make_float2(far.x * sn[4 * i], far.y * sn[4 * i + 1]);
        ms[w][2 * i + 1] = make_float2(far.z * sn[4 * i + 2], far.w * sn[4 * i + 3]);
      }
    }
  }
  auto normed = [&](const uint4& v, const float2 (&c)[4], const float2 (&n)[4]) {
    const uint32_t own[4] = {v.x, v.y, v.z, v.w};
    uint32_t far[4];
    float2 x[4], sq = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = Num<T>::unpack(own[i]);
      sq = fma2(x[i], x[i], sq);
      if (!INTER) far[i] = __shfl_sync(0xffffffffu, own[i], partner);
    }
    float ss = sq.x + sq.y;
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    const float r = rsqrtf(ss * (1.0f / D) + a.eps);
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 z = mul2(x[i], c[i]);
      if (turned) z = fma2(INTER ? make_float2(x[i].y, x[i].x) : Num<T>::unpack(far[i]), n[i], z);
      z = mul2(z, make_float2(r, r));
      y[i] = Num<T>::pack(z.x, z.y);
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
  };
  uint4* q_row = reinterpret_cast<uint4*>(static_cast<T*>(a.q) + (long long)token * a.q_stride);
  const long long plane = ((long long)a.d.n_sink + a.d.ring) * LPH, at = (long long)s.session * a.d.n_kv_heads * plane + (long long)cache_row(a.d, pos) * LPH + l;
  uint4 *k_row = static_cast<uint4*>(a.k) + at, *v_row = static_cast<uint4*>(a.v) + at;
  int slot = 0;
  for (int first = part * 32; first < chunks; first += step) {
    const int c = first + lane;
    asm volatile("cp.async.wait_group %0;" ::"n"(APPEND_DEPTH - 1) : "memory");
    const uint4 v = ring[slot * 32];
    fetch(c + APPEND_DEPTH * step, slot);
    slot = slot + 1 == APPEND_DEPTH ? 0 : slot + 1;
    // heads of q only, of k only, of v only, or (where they meet inside of a warp's 32 pieces) of several kinds: each lane its own
    if (first + 32 <= q_end) {
      q_row[c] = normed(v, mc[0], ms[0]);
    } else if (first >= q_end && first + 32 <= k_end) {
      k_row[(c - q_end) / LPH * plane] = normed(v, mc[1], ms[1]);
    } else if (first >= k_end) {
      if (c < chunks) v_row[(c - k_end) / LPH * plane] = v;
    } else {
      const uint4 yq = normed(v, mc[0], ms[0]), yk = normed(v, mc[1], ms[1]);
      if (c < q_end) q_row[c] = yq;
      else if (c < k_end) k_row[(c - q_end) / LPH * plane] = yk;
      else if (c < chunks) v_row[(c - k_end) / LPH * plane] = v;
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// Attention of single tokens: one query row per head against the rows of its window and the first tokens.
// ---------------------------------------------------------------------------------------------
struct AttendArgs {
  CacheDims   d;
  TokenBatch  b;
  const void *q, *k, *v;
  void*       out;
  long long   q_stride, out_stride;
  float       scale_log2e;
  int         group;     // query heads of a key/value head
  int         splits;    // CTAs of a cluster
  int*        err;       // where a bounded wait that gives up writes err_id
  int         err_id;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<bf16>(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

constexpr int STEP_STAGES = 3;
constexpr int STEP_HALF = 4096;                         // bytes of K, and of V, in a unit
constexpr int STEP_UNIT = 2 * STEP_HALF;
constexpr int STEP_HEADS = 16;                          // query heads that one CTA serves at most
constexpr int step_smem(int warps) { return warps * STEP_STAGES * STEP_UNIT; }

// Bound by the reads of K and V, so the work is laid out for loads: a unit is 4 KB of K rows and the same V rows (16 rows of 128
// values, 32 of 64), every warp streams units of its own through three stages of asynchronous 16-byte copies and keeps its own
// running maximum, sum and output in registers; no warp waits for another before the end.  The products (m16n8k16) have the rows of K, or the
// columns of V, as their 16 rows and the query heads that share a K/V head as their 8 columns (NH = 2: twice 8): a row is read once for
// all of them, and a group of up to 8 heads takes 8 + 16 products a unit.  (With the heads as the 16 rows it took 48, and
// those, at about 35 cycles each, bounded the kernel: 36 us against 20 for one session of 32,768 rows.)  Measured: 48 sessions of up to 4,100 rows, 8 x 128 values of K and of V each,
// 98 us in short bursts, 6.4 TB/s, 103 us among other calls; one session of 32,768 rows, 4 heads, 20 us, 3.3 TB/s: its four clusters sit in four of the device's eight GPCs.  The units of a
// (sequence, head) are dealt out over the warps of a cluster of CTAs, which joins the partial results through distributed shared
// memory: no workspace, no second launch.  The numerators enter the second product as two values of the cache's type (their rounding and what
// that leaves: 16 bits in bf16, 22 in fp16 down to 2^-25), so that the rounding of the result is the one that counts.
template <typename T, int D, int NH, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) attend_step_kernel(const AttendArgs a) {
  constexpr int UN = STEP_HALF / (2 * D);    // rows of a unit
  constexpr int CPR = D / 8;                 // 16-byte chunks of a row
  constexpr int MT = UN / 16, KS = D / 16, DT = D / 16;
  constexpr int PD = D + 8;                  // floats between two heads of a partial output
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ float wm[WARPS][STEP_HEADS], wl[WARPS][STEP_HEADS];
  __shared__ float cm[STEP_HEADS], cl[STEP_HEADS];
  ptx::pdl_wait();
  ptx::pdl_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x;   // in the cluster: gridDim.x == splits
  const int groups = (a.group + 8 * NH - 1) / (8 * NH);
  const int kvh = blockIdx.y / groups, h0 = (blockIdx.y % groups) * (8 * NH), nh = min(8 * NH, a.group - h0);
  const TokenSeq s = load_seq(a.b, a.d, blockIdx.z);
  if (s.count != 1) return;      // (the whole cluster)
  const int pos = s.start, rows = a.d.n_sink + a.d.ring;
  const RowRuns run = row_runs(a.d, pos);
  const int n_first = run.n_first, lo2 = run.lo_second, n_second = run.n_second;
  const int u_first = (n_first + UN - 1) / UN, units = u_first + (n_second + UN - 1) / UN;
  const long long plane = ((long long)s.session * a.d.n_kv_heads + kvh) * rows;
  const T* K = static_cast<const T*>(a.k) + plane * D;
  const T* V = static_cast<const T*>(a.v) + plane * D;

  uint8_t* ring = smem + warp * STEP_STAGES * STEP_UNIT;
  const uint32_t ring_s = ptx::smem_u32(ring);
  const int step = a.splits * WARPS;
  auto unit_rows = [&](int u, int& row0) {
    row0 = u < u_first ? u * UN : lo2 + (u - u_first) * UN;
    return u < u_first ? n_first - row0 : n_second - (u - u_first) * UN;   // (may exceed UN)
  };
  auto fetch = [&](int u, int stage) {
    if (u < units) {
      int row0;
      const int n = unit_rows(u, row0);
      const uint32_t dst = ring_s + stage * STEP_UNIT;
#pragma unroll
      for (int i = 0; i < UN * CPR / 32; ++i) {
        const int ch = i * 32 + lane, r = ch / CPR, c = ch % CPR;
        const bool on = r < n;     // rows behind the run read as zeros: whatever they hold must not meet a weight of zero
        const long long off = on ? (long long)(row0 + r) * D + c * 8 : 0;
        const uint32_t at = dst + r * (2 * D) + ((c ^ (r & 7)) << 4);
        cp16(at, K + off, on);
        cp16(at + STEP_HALF, V + off, on);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int u = rank * WARPS + warp;
#pragma unroll
  for (int i = 0; i < STEP_STAGES - 1; ++i) fetch(u + i * step, i);

  // the queries as the second operand: head g of each eight
  uint32_t qf[NH][KS][2];
  {
    const T* q = static_cast<const T*>(a.q) + (long long)s.first * a.q_stride + (long long)(kvh * a.group + h0) * D;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i) qf[h][ks][i] = h * 8 + g < nh ? *reinterpret_cast<const uint32_t*>(q + (h * 8 + g) * D + ks * 16 + t * 2 + i * 8) : 0u;
  }
  // of heads 2 t and 2 t + 1 of each eight; output columns g and g + 8 of each sixteen
  float o[NH][DT][4], m[NH][2], l[NH][2];
#pragma unroll
  for (int h = 0; h < NH; ++h) {
#pragma unroll
    for (int j = 0; j < DT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[h][j][i] = 0.f;
    m[h][0] = m[h][1] = -INFINITY;
    l[h][0] = l[h][1] = 0.f;
  }

  int stage = 0;
  for (; u < units; u += step) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STEP_STAGES - 2) : "memory");
    __syncwarp();    // the other lanes' copies of this unit have landed, and all have read the stage that is filled next
    fetch(u + (STEP_STAGES - 1) * step, stage == 0 ? STEP_STAGES - 1 : stage - 1);
    const uint32_t ks_ = ring_s + stage * STEP_UNIT, vs_ = ks_ + STEP_HALF;
    stage = stage + 1 == STEP_STAGES ? 0 : stage + 1;
    int row0;
    const int n = unit_rows(u, row0);
    // all of the unit's rows of K go to registers first, the products of a sixteen run as two chains
    uint32_t kf[MT][KS][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int r = mt * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), c = 2 * ks + (lane >> 4);
        ldsm4(ks_ + r * (2 * D) + ((c ^ (r & 7)) << 4), kf[mt][ks]);
      }
    float sc[NH][MT][4];     // keys g (0, 1) and g + 8 (2, 3) of each sixteen, heads 2 t and 2 t + 1
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        float odd[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[h][mt][i] = odd[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ks += 2) {
          mma16816<T>(sc[h][mt], kf[mt][ks], qf[h][ks][0], qf[h][ks][1]);
          mma16816<T>(odd, kf[mt][ks + 1], qf[h][ks + 1][0], qf[h][ks + 1][1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[h][mt][i] += odd[i];
      }
    // ... and so do the columns of V, under the softmax
    uint32_t vf[MT][DT][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const int r = mt * 16 + (lane >> 4) * 8 + (lane & 7), c = 2 * j + ((lane >> 3) & 1);
        ldsm4t(vs_ + r * (2 * D) + ((c ^ (r & 7)) << 4), vf[mt][j]);
      }
    float top[NH][2];
    bool move = false;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = -INFINITY;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float& y = sc[h][mt][2 * k + i];
            y = mt * 16 + 8 * k + g < n ? __fmul_rn(y, a.scale_log2e) : -INFINITY;      // (rounded here, whatever is taken off below)
            x = fmaxf(x, y);
          }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
        top[h][i] = x;
        move |= x > m[h][i] + 8.f;      // (m = -infinity: at the first row)
      }
    }
    // the running maximum moves when it is passed by 2^8: numerators stay within the types' range, the output is rescaled seldom
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float mn = fmaxf(m[h][i], top[h][i]), f = mn > m[h][i] ? ex2(m[h][i] - mn) : 1.f;
          m[h][i] = mn;
          l[h][i] *= f;
#pragma unroll
          for (int j = 0; j < DT; ++j) {
            o[h][j][i] *= f;
            o[h][j][2 + i] *= f;
          }
        }
    }
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const float base[2] = {m[h][0] == -INFINITY ? 0.f : m[h][0], m[h][1] == -INFINITY ? 0.f : m[h][1]};
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[h][mt][i] = ex2(sc[h][mt][i] - base[i & 1]);
          l[h][i & 1] += sc[h][mt][i];
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      uint32_t hi[NH][2], lo[NH][2];      // keys 0 .. 7 and 8 .. 15 of the sixteen, as the second operand
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float x = sc[h][mt][2 * k], y = sc[h][mt][2 * k + 1];
          const uint32_t p = Num<T>::pack(x, y);
          const float2 r = Num<T>::unpack(p);
          hi[h][k] = transpose8x8(p);
          lo[h][k] = transpose8x8(Num<T>::pack(x - r.x, y - r.y));
        }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
#pragma unroll
        for (int j = 0; j < DT; ++j) mma16816<T>(o[h][j], vf[mt][j], hi[h][0], hi[h][1]);
#pragma unroll
        for (int j = 0; j < DT; ++j) mma16816<T>(o[h][j], vf[mt][j], lo[h][0], lo[h][1]);
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncwarp();

  // ---- join: the warps of the CTA, then the CTAs of the cluster -----------------------------------------------------------
  float* part = reinterpret_cast<float*>(ring);     // [heads][PD] of this warp (at most 9 KB of its 24)
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[h][i] += __shfl_xor_sync(0xffffffffu, l[h][i], d);
      const int head = h * 8 + 2 * t + i;
      if (g == 0) {
        wm[warp][head] = m[h][i];
        wl[warp][head] = l[h][i];
      }
      if (head < nh) {
#pragma unroll
        for (int j = 0; j < DT; ++j) {
          part[head * PD + j * 16 + g] = o[h][j][i];
          part[head * PD + j * 16 + 8 + g] = o[h][j][2 + i];
        }
      }
    }
  __syncthreads();
  constexpr int WSTRIDE = STEP_STAGES * STEP_UNIT / 4;   // floats between two warps' parts
  float* all = reinterpret_cast<float*>(smem);
  T* out = static_cast<T*>(a.out) + (long long)s.first * a.out_stride + (long long)(kvh * a.group + h0) * D;
  for (int e = threadIdx.x * 2; e < nh * D; e += WARPS * 64) {
    const int r = e / D, at = r * PD + e % D;
    float M = wm[0][r];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) M = fmaxf(M, wm[w][r]);
    const float base = M == -INFINITY ? 0.f : M;
    float x = 0.f, y = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = ex2(wm[w][r] - base);
      const float2 v = *reinterpret_cast<const float2*>(all + w * WSTRIDE + at);
      x = fmaf(f, v.x, x);
      y = fmaf(f, v.y, y);
      L = fmaf(f, wl[w][r], L);
    }
    if (a.splits == 1) {
      const float inv = 1.0f / L;
      *reinterpret_cast<uint32_t*>(out + e) = Num<T>::pack(x * inv, y * inv);
    } else {
      *reinterpret_cast<float2*>(all + at) = make_float2(x, y);     // (each element is read and written by one thread)
      if (e % D == 0) {
        cm[r] = M;
        cl[r] = L;
      }
    }
  }
  if (a.splits == 1) return;
  __syncwarp();      // (the cluster's barrier is met by whole warps)
  ptx::cluster_arrive();
  ptx::cluster_wait();
  const uint32_t all_s = ptx::smem_u32(all), cm_s = ptx::smem_u32(cm), cl_s = ptx::smem_u32(cl);
  for (int e = (rank * WARPS * 32 + (int)threadIdx.x) * 2; e < nh * D; e += a.splits * WARPS * 64) {
    const int r = e / D, at = r * PD + e % D;
    float M = -INFINITY;
#pragma unroll 4
    for (int c = 0; c < a.splits; ++c) M = fmaxf(M, ld_cluster(ptx::map_to_cta(cm_s + r * 4, c)));
    const float base = M == -INFINITY ? 0.f : M;
    float x = 0.f, y = 0.f, L = 0.f;
#pragma unroll 4
    for (int c = 0; c < a.splits; ++c) {
      const float f = ex2(ld_cluster(ptx::map_to_cta(cm_s + r * 4, c)) - base);
      const uint32_t from = ptx::map_to_cta(all_s + at * 4, c);
      x = fmaf(f, ld_cluster(from), x);
      y = fmaf(f, ld_cluster(from + 4), y);
      L = fmaf(f, ld_cluster(ptx::map_to_cta(cl_s + r * 4, c)), L);
    }
    const float inv = 1.0f / L;
    *reinterpret_cast<uint32_t*>(out + e) = Num<T>::pack(x * inv, y * inv);
  }
  __syncwarp();
  ptx::cluster_arrive();      // no CTA's shared memory goes while another reads it
  ptx::cluster_wait();
}

#include "dc_token_attn.cuh"

template <typename K>
cudaError_t launch(K kernel, dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const void* arg) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  cfg.attrs = attr;
  void* args[] = {const_cast<void*>(arg)};
  return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), args);
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace
}  // namespace dc

// Words that a bounded device-side wait sets when it gives up: part of the library image, so that opening and closing a cache allocates
// nothing on the device, waits for nothing and may happen while a stream is being captured.
static __device__ int g_cache_err[4096];

namespace {
constexpr int kErrWords = 4096;
bool       g_err_used[kErrWords];
std::mutex g_err_mu;

// A free word (the last one is shared by all caches behind the 4095th).
int take_err_word(int* id) {
  static int opened = 0;
  std::lock_guard<std::mutex> lk(g_err_mu);
  *id = opened = opened == INT_MAX ? 1 : opened + 1;
  for (int i = 0; i < kErrWords - 1; ++i)
    if (!g_err_used[i]) {
      g_err_used[i] = true;
      return i;
    }
  return kErrWords - 1;
}
void give_err_word(int i) {
  std::lock_guard<std::mutex> lk(g_err_mu);
  g_err_used[i] = false;
}
}  // namespace

struct dc_cache {
  dc::CacheDims d;
  int   head_dim, dtype, device, n_sm;
  void *k, *v;
  int   err_word, err_id;   // this cache's number: what another one has left in the word is not taken for its own
  int*  err;                // the word's address
  CUtensorMap kmap, vmap;
};

#define DC_REFUSE(code, ...)    \
  do {                          \
    dc::set_error(__VA_ARGS__); \
    return code;                \
  } while (0)

namespace {

// Everything that can be told about a batch without the device's values.
dc_status admit_batch(const dc_cache* c, const dc_token_batch* b, const char* who) {
  if (!c || !b) DC_REFUSE(DC_ERR_ARG, "%s: null pointer argument", who);
  if (b->size != sizeof(dc_token_batch)) DC_REFUSE(DC_ERR_ARG, "%s: dc_token_batch.size is %u, this library's is %zu", who, b->size, sizeof(dc_token_batch));
  if (b->n_seqs < 1 || b->n_seqs > 65535 || b->n_tokens < 1 || b->max_tokens < 1)
    DC_REFUSE(DC_ERR_ARG, "%s: need 1 <= n_seqs <= 65535, n_tokens >= 1, max_tokens >= 1", who);
  if (!b->start_dev) DC_REFUSE(DC_ERR_ARG, "%s: start_dev is null", who);
  if (!b->cu_tokens_dev && (b->max_tokens != 1 || b->n_tokens != b->n_seqs))
    DC_REFUSE(DC_ERR_ARG, "%s: without cu_tokens_dev every sequence brings one token (n_tokens == n_seqs, max_tokens == 1)", who);
  if (!b->sessions_dev && b->n_seqs > c->d.n_sessions)
    DC_REFUSE(DC_ERR_ARG, "%s: %d sequences without sessions_dev, the cache has %d sessions", who, b->n_seqs, c->d.n_sessions);
  if ((long long)b->max_tokens > (long long)c->d.ring - c->d.window + 1)
    DC_REFUSE(DC_ERR_FRAMES, "%s: %d tokens of a sequence in one call, a ring of %d rows with a window of %d takes %d", who, b->max_tokens, c->d.ring,
              c->d.window, c->d.ring - c->d.window + 1);
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) DC_REFUSE(DC_ERR_CUDA, "%s: cudaGetDevice failed: %s", who, cudaGetErrorString(e));
  if (dev != c->device) DC_REFUSE(DC_ERR_ARG, "%s: the cache is on device %d, the current device is %d", who, c->device, dev);
  return DC_OK;
}

bool bad_rows(const void* p, long long stride, long long width) { return !p || dc::misaligned(p) || stride < width || stride % 8; }

dc_status launched(cudaError_t e, const char* who) {
  if (e != cudaSuccess) {
    cudaGetLastError();   // (a refused launch leaves its code behind)
    DC_REFUSE(DC_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
  }
  return DC_OK;
}

dc::TokenBatch kernel_batch(const dc_token_batch* b) {
  return dc::TokenBatch{b->n_seqs, b->n_tokens, b->max_tokens, b->sessions_dev, b->cu_tokens_dev, b->start_dev};
}

using AppendFn = void (*)(const dc::AppendArgs);
using StepFn = void (*)(const dc::AttendArgs);
AppendFn append_fn(int dtype, int D, bool inter) {
  using namespace dc;
  if (dtype == DC_BF16) return D == 128 ? (inter ? append_kernel<bf16, 128, true> : append_kernel<bf16, 128, false>)
                                        : (inter ? append_kernel<bf16, 64, true> : append_kernel<bf16, 64, false>);
  return D == 128 ? (inter ? append_kernel<__half, 128, true> : append_kernel<__half, 128, false>)
                  : (inter ? append_kernel<__half, 64, true> : append_kernel<__half, 64, false>);
}
template <typename T, int D>
StepFn step_of(bool two, bool wide) {
  using namespace dc;
  return two ? (wide ? attend_step_kernel<T, D, 2, 8> : attend_step_kernel<T, D, 2, 4>) : (wide ? attend_step_kernel<T, D, 1, 8> : attend_step_kernel<T, D, 1, 4>);
}
// two: groups of more than 8 query heads; wide: CTAs of 8 warps
StepFn step_fn(int dtype, int D, bool two, bool wide) {
  if (dtype == DC_BF16) return D == 128 ? step_of<dc::bf16, 128>(two, wide) : step_of<dc::bf16, 64>(two, wide);
  return D == 128 ? step_of<__half, 128>(two, wide) : step_of<__half, 64>(two, wide);
}

using ChunkFn = void (*)(const dc::ChunkArgs);
template <typename T, int D>
ChunkFn chunk_of(bool split) { return split ? dc::attend_chunk_kernel<T, D, true> : dc::attend_chunk_kernel<T, D, false>; }
// split: tiles that a cluster of CTAs shares
ChunkFn chunk_fn(int dtype, int D, bool split) {
  if (dtype == DC_BF16) return D == 128 ? chunk_of<dc::bf16, 128>(split) : chunk_of<dc::bf16, 64>(split);
  return D == 128 ? chunk_of<__half, 128>(split) : chunk_of<__half, 64>(split);
}
size_t chunk_smem_bytes(int D) { return D == 128 ? dc::chunk_smem<128>() : dc::chunk_smem<64>(); }

// The cache as one matrix of rows, fetched in boxes of 64 rows and 64 values in the 128-byte swizzle.
bool cache_map(CUtensorMap* m, const dc_cache* c, void* base) {
  using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return false;
  const cuuint64_t dim[2] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->d.n_sessions * c->d.n_kv_heads * (c->d.n_sink + c->d.ring)}, stride[1] = {(cuuint64_t)c->head_dim * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)dc::CH_N}, one[2] = {1, 1};
  return reinterpret_cast<EncodeFn>(fn)(m, c->dtype == DC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dim, stride, box, one,
                                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" dc_status dc_cache_open(const dc_cache_config* cfg, void* k_dev, void* v_dev, dc_cache** out) {
  if (!out) DC_REFUSE(DC_ERR_ARG, "dc_cache_open: null pointer argument");
  *out = nullptr;
  if (!cfg || !k_dev || !v_dev) DC_REFUSE(DC_ERR_ARG, "dc_cache_open: null pointer argument");
  if (cfg->size != sizeof(dc_cache_config)) DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: dc_cache_config.size is %u, this library's is %zu", cfg->size, sizeof(dc_cache_config));
  if (cfg->dtype != DC_BF16 && cfg->dtype != DC_F16) DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: a cache holds DC_BF16 or DC_F16");
  if (cfg->head_dim != 64 && cfg->head_dim != 128) DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: head_dim is %d, 64 and 128 are served", cfg->head_dim);
  if (cfg->n_kv_heads < 1 || cfg->n_heads < cfg->n_kv_heads || cfg->n_heads % cfg->n_kv_heads || cfg->n_heads / cfg->n_kv_heads > 64 || cfg->n_heads > 1024)
    DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: %d query heads over %d key/value heads: need a whole ratio of 1 to 64, at most 1024 heads", cfg->n_heads, cfg->n_kv_heads);
  if (cfg->n_sessions < 1 || cfg->n_sink < 0 || cfg->window < 1 || cfg->ring_rows < cfg->window || cfg->ring_rows > INT_MAX - 4096 - cfg->n_sink)
    DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: need n_sessions >= 1, n_sink >= 0, 1 <= window <= ring_rows");
  if (((double)cfg->n_sink + cfg->ring_rows) * cfg->n_kv_heads * cfg->n_sessions >= 2147483648.0)
    DC_REFUSE(DC_ERR_CONFIG, "dc_cache_open: the cache has 2^31 rows or more (sessions x key/value heads x rows)");
  if (dc::misaligned(k_dev) || dc::misaligned(v_dev)) DC_REFUSE(DC_ERR_ARG, "dc_cache_open: k_dev and v_dev must be 16-byte aligned");
  const uintptr_t bytes = ((uintptr_t)cfg->n_sink + cfg->ring_rows) * cfg->n_kv_heads * cfg->n_sessions * cfg->head_dim * 2, kp = (uintptr_t)k_dev, vp = (uintptr_t)v_dev;
  if (kp < vp + bytes && vp < kp + bytes) DC_REFUSE(DC_ERR_ARG, "dc_cache_open: k_dev and v_dev overlap");
  dc_cache* c = new (std::nothrow) dc_cache();
  if (!c) DC_REFUSE(DC_ERR_OOM, "dc_cache_open: out of host memory");
  c->d = dc::CacheDims{cfg->n_sessions, cfg->n_heads, cfg->n_kv_heads, cfg->n_sink, cfg->window, cfg->ring_rows};
  c->head_dim = cfg->head_dim;
  c->dtype = cfg->dtype;
  c->k = k_dev;
  c->v = v_dev;
  int major = 0;
  cudaError_t e = cudaGetDevice(&c->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, c->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->n_sm, cudaDevAttrMultiProcessorCount, c->device);
  if (e == cudaSuccess && major != 10) {
    delete c;
    DC_REFUSE(DC_ERR_CUDA, "dc_cache_open: this library is built for sm_100a only");
  }
  const bool two = cfg->n_heads / cfg->n_kv_heads > 8;
  for (int wide = 0; wide < 2; ++wide) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(step_fn(c->dtype, c->head_dim, two, wide), cudaFuncAttributeMaxDynamicSharedMemorySize, dc::step_smem(wide ? 8 : 4));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(step_fn(c->dtype, c->head_dim, two, wide), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  }
  for (int split = 0; split < 2; ++split)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(chunk_fn(c->dtype, c->head_dim, split), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)chunk_smem_bytes(c->head_dim));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(chunk_fn(c->dtype, c->head_dim, true), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess && !(cache_map(&c->kmap, c, k_dev) && cache_map(&c->vmap, c, v_dev))) {
    delete c;
    DC_REFUSE(DC_ERR_CUDA, "dc_cache_open: cuTensorMapEncodeTiled failed or is unavailable");
  }
  void* words = nullptr;
  if (e == cudaSuccess) e = cudaGetSymbolAddress(&words, g_cache_err);
  if (e != cudaSuccess) {
    delete c;
    DC_REFUSE(DC_ERR_CUDA, "dc_cache_open: %s", cudaGetErrorString(e));
  }
  c->err_word = take_err_word(&c->err_id);
  c->err = static_cast<int*>(words) + c->err_word;
  *out = c;
  return DC_OK;
}

extern "C" dc_status dc_cache_close(dc_cache* c) {
  if (!c) DC_REFUSE(DC_ERR_ARG, "dc_cache_close: null pointer argument");
  give_err_word(c->err_word);
  delete c;                 // (calls in flight have all they need as arguments)
  return DC_OK;
}

extern "C" dc_status dc_cache_check(dc_cache* c) {
  if (!c) DC_REFUSE(DC_ERR_ARG, "dc_cache_check: null pointer argument");
  int word = 0, dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev != c->device) DC_REFUSE(DC_ERR_ARG, "dc_cache_check: the cache is on device %d, the current device is %d", c->device, dev);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(&word, c->err, sizeof(int), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && word == c->err_id) e = cudaMemset(c->err, 0, sizeof(int));
  if (e != cudaSuccess) DC_REFUSE(DC_ERR_CUDA, "dc_cache_check: %s", cudaGetErrorString(e));
  if (word == c->err_id) DC_REFUSE(DC_ERR_TIMEOUT, "dc_cache_check: a bounded device-side wait of an attention call gave up; its outputs are not valid");
  return DC_OK;
}

extern "C" dc_status dc_cache_append(dc_cache* c, const dc_token_batch* b, const dc_qk_norm* nm, const void* qkv_dev, long long qkv_stride, void* q_dev,
                                     long long q_stride, void* cuda_stream) {
  const char* who = "dc_cache_append";
  dc_status st = admit_batch(c, b, who);
  if (st != DC_OK) return st;
  if (!nm) DC_REFUSE(DC_ERR_ARG, "%s: null pointer argument", who);
  if (nm->size != sizeof(dc_qk_norm)) DC_REFUSE(DC_ERR_ARG, "%s: dc_qk_norm.size is %u, this library's is %zu", who, nm->size, sizeof(dc_qk_norm));
  if (!nm->q_gain_dev || !nm->k_gain_dev || dc::misaligned(nm->q_gain_dev) || dc::misaligned(nm->k_gain_dev))
    DC_REFUSE(DC_ERR_ARG, "%s: q_gain_dev and k_gain_dev must be 16-byte aligned device pointers", who);
  if (nm->rot_dim < 0 || nm->rot_dim > c->head_dim || nm->rot_dim % 16 || (nm->rot_dim && !nm->inv_freq_dev))
    DC_REFUSE(DC_ERR_ARG, "%s: rot_dim is %d: a multiple of 16 up to head_dim, with inv_freq_dev", who, nm->rot_dim);
  if (!(nm->eps >= 0.f)) DC_REFUSE(DC_ERR_ARG, "%s: eps must not be negative", who);
  const int D = c->head_dim;
  if (bad_rows(qkv_dev, qkv_stride, (long long)(c->d.n_heads + 2 * c->d.n_kv_heads) * D) || bad_rows(q_dev, q_stride, (long long)c->d.n_heads * D))
    DC_REFUSE(DC_ERR_ARG, "%s: qkv_dev and q_dev must be 16-byte aligned, their row strides multiples of 8 values and no shorter than a row", who);
  if (q_dev == qkv_dev && q_stride != qkv_stride) DC_REFUSE(DC_ERR_ARG, "%s: queries written in place keep the rows' stride", who);
  dc::AppendArgs a{c->d, kernel_batch(b), qkv_dev, qkv_stride, q_stride, q_dev, c->k, c->v, nm->q_gain_dev, nm->k_gain_dev, nm->inv_freq_dev, nm->rot_dim, nm->eps, dc::APPEND_WARPS};
  // A token's row is dealt out over a whole CTA's warps while that gives an SM no more than 32 warps to run, and over fewer behind that (6,162 tokens: 43, 33,
  // 30 and 29 us in 8, 4, 2 and 1 warps a row; 64 tokens: 2.6 us in 8).
  while (a.share > 1 && (long long)b->n_tokens * a.share > 32ll * c->n_sm) a.share /= 2;
  const long long warps = (long long)b->n_tokens * a.share;
  return launched(dc::launch(append_fn(c->dtype, D, nm->interleaved != 0), dim3((unsigned)((warps + dc::APPEND_WARPS - 1) / dc::APPEND_WARPS)), dc::APPEND_WARPS * 32, 0, 1,
                             (cudaStream_t)cuda_stream, &a), who);
}

extern "C" dc_status dc_cache_attend(dc_cache* c, const dc_token_batch* b, const void* q_dev, long long q_stride, float scale, void* out_dev,
                                     long long out_stride, void* cuda_stream) {
  const char* who = "dc_cache_attend";
  dc_status st = admit_batch(c, b, who);
  if (st != DC_OK) return st;
  if (!(scale > 0.f) || scale > 1e30f) DC_REFUSE(DC_ERR_ARG, "%s: scale must be positive, 1e30 at most", who);
  const int D = c->head_dim;
  const long long width = (long long)c->d.n_heads * D;
  if (bad_rows(q_dev, q_stride, width) || bad_rows(out_dev, out_stride, width))
    DC_REFUSE(DC_ERR_ARG, "%s: q_dev and out_dev must be 16-byte aligned, their row strides multiples of 8 values and no shorter than a row", who);
  dc::AttendArgs a{c->d, kernel_batch(b), q_dev, c->k, c->v, out_dev, q_stride, out_stride, scale * 1.4426950408889634f, c->d.n_heads / c->d.n_kv_heads, 1, c->err, c->err_id};
  const long long seen = (long long)c->d.n_sink + c->d.window;     // most rows that a token sees
  if (b->max_tokens > 1) {
    dc::ChunkArgs ca{a, 0, c->kmap, c->vmap};
    const int per = dc::CH_M / a.group;
    ca.tiles = (b->max_tokens + per - 1) / per;
    const long long tiles = (long long)ca.tiles * c->d.n_kv_heads * b->n_seqs, steps = (seen + per) / dc::CH_N + 1;
    // Splits of a tile's rows over a cluster: while all CTAs are resident (two per SM) and each has two steps or more (chunks of 50 tokens, 8 sessions, 13 steps
    // of 64 rows: 21, 19, 18 and 25 us in 1, 2, 4 and 8).
    while (ca.a.splits < 16 && tiles * ca.a.splits * 2 <= 2ll * c->n_sm && ca.a.splits * 4 <= steps) ca.a.splits *= 2;
    if ((long long)ca.tiles * ca.a.splits > INT_MAX) DC_REFUSE(DC_ERR_ARG, "%s: too many tokens", who);
    return launched(dc::launch(chunk_fn(c->dtype, D, ca.a.splits > 1), dim3(ca.tiles * ca.a.splits, c->d.n_kv_heads, b->n_seqs), dc::CH_THREADS, chunk_smem_bytes(D), ca.a.splits,
                               (cudaStream_t)cuda_stream, &ca), who);
  }
  const bool two = a.group > 8;
  const int per = two ? 16 : 8, groups = (a.group + per - 1) / per;
  const long long units = seen * D * 2 / dc::STEP_HALF + 1, pairs = (long long)b->n_seqs * c->d.n_kv_heads * groups;
  // Splits: while every warp has a unit of its own, and either the CTAs are resident (two per SM) or, of many long rows, up to four
  // for the balance of the last wave (48 sessions x 8 heads of up to 4,100 rows: 112 us unsplit, 104 us in two, 98 us in four, 133 us in eight).
  while (a.splits < 16 && a.splits * 2 * 4 <= units && (pairs * a.splits * 2 <= 2ll * c->n_sm || (a.splits < 4 && units >= 64 * a.splits))) a.splits *= 2;
  // CTAs of 8 warps, one per SM, where there are fewer CTAs than SMs and rows enough: the copies in flight on an SM are what bounds it then (one session
  // of 32,768 rows: 20 us against 25 us in CTAs of 4).
  const bool wide = pairs * a.splits <= c->n_sm && (long long)a.splits * 8 * 2 <= units;
  return launched(dc::launch(step_fn(c->dtype, D, two, wide), dim3(a.splits, c->d.n_kv_heads * groups, b->n_seqs), wide ? 256 : 128, dc::step_smem(wide ? 8 : 4), a.splits,
                             (cudaStream_t)cuda_stream, &a), who);
}
