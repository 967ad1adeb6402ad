// Attention of chunks and prompts over a token cache (dc_cache_attend with several tokens of a sequence): included by
// dc_token_cache.cu, inside its namespace.
//
// Work: 4 D operations per (query head, attended row) against reads of K and V that all queries of a tile share, so a tile of
// 128 query rows is bound by the tensor cores and by the exponentials, 128 x 64 of each per step.  A tile holds
// 128 / G tokens with the G query heads that share a key/value head, so short chunks fill it and K/V is read once for the group.
// Two CTAs per SM, each with 256 columns of tensor memory: scores of two steps (64 columns each; the numerators, rounded to the
// cache's type, take the place of the scores that they come from and feed the second product from there) and the output.  One warp
// issues the copies, one the products, four hold a query row per thread: the product of step j + 1 runs under the exponentials of step
// j.  Keys are taken in the order of the cache's rows, 64 at a time: softmax does not mind their order, so a ring that has wrapped needs no
// gather, only masks, and steps whose rows no query of the tile sees are left out.
//
// The running maximum moves only when a row's new maximum exceeds it by 8 (in powers of two): the numerators then stay below 2^8,
// within fp16 too, and the output in tensor memory is rescaled in few of the steps.
//
// Measured: 8,192 tokens, 16 query heads over 4 of 128 values, window 2,048: 145 us in short bursts (831 TFLOP/s of what the masks leave), 163 us under
// lasting load, where the clock falls with the power.  A step of 64 rows takes a CTA 1,650 cycles with another on its SM; both CTAs' products hold the tensor pipe for 58 % of
// the cycles (40 % by the counter of its arithmetic: a product of 64 columns takes more than its share), the exponentials their unit for 44 %.

constexpr int CH_M = 128, CH_N = STEP_N, CH_STAGES = 2, CH_THREADS = 192;
constexpr uint32_t CH_TMEM = 256, CH_O = 128;   // columns: scores at 0 and 64, output at 128

// Never less than a third of an SM's: a third CTA on an SM would wait for tensor memory, and its cluster for it.
template <int D>
constexpr size_t chunk_smem() {
  const size_t need = 1024 + (size_t)CH_M * D * 2 + (size_t)CH_STAGES * 2 * CH_N * D * 2;
  return need < 80 * 1024 ? 80 * 1024 : need;
}

struct ChunkArgs {
  AttendArgs  a;
  int         tiles;       // of max_tokens
  CUtensorMap kmap, vmap;  // [sessions * kv_heads * rows][D], boxes of 64 rows x 64 values
};

template <typename T, int N>
__device__ __forceinline__ constexpr uint32_t chunk_idesc(int b_mn_major) {
  // fp32 accumulation, operand types (0: fp16, 1: bf16), N / 8, M / 16
  return (1u << 4) | (sizeof(T) && Num<T>::is_bf16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(CH_M >> 4) << 24);
}
// D[tmem] (+)= A[tmem] * B[smem]: a 32-bit column of A holds two neighbouring values of the reduction
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc)
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n"
      "tcgen05.wait::st.sync.aligned;" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st_cluster4(uint32_t addr, const float* v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }

// The bounded wait (about a second) of a warp: all lanes agree on its outcome, so that what the warp does together stays together.
constexpr uint32_t CH_POLLS = 1u << 18;
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait_limit(bar, parity, CH_POLLS)); }

// x * scale - m takes one rounding, and so leaves what the rounding of m, itself such a product, has lost: half a step of it, a common factor of a row's numerators.
// Up to here (2^24) that is 2^0.5 at most; far beyond it the factor leaves the types' range.
constexpr float CH_FAR = 16777216.f;

struct ChunkBars {
  uint64_t k_full[CH_STAGES], k_empty[CH_STAGES], v_full[CH_STAGES], v_empty[CH_STAGES];
  uint64_t s_full[2], p_full[2], q_full;
  uint64_t pv_done[2];   // of even and odd steps: a row's thread may see step j - 1's product done before it has looked for step j - 2's
  uint32_t tmem;
  int      failed;    // a bounded wait gave up
  int      odd;       // a row of V that some of the tile's queries see and others do not holds an infinity or a NaN, or a maximum lies beyond CH_FAR
  float    m[CH_M], l[CH_M];
};

// One query row with plain arithmetic over the steps' rows: o[0..16) of its columns c0.. .  Only for odd tiles (see ChunkBars):
// masked rows, whose weight of zero may not meet a value, are not read at all, and a score is rounded before the maximum is taken off.
// The query lies where the products read it, in row `row` of the swizzled tile.  Slow: one such tile over 2,048 rows of 128 values takes 23 ms, a prompt of 8,192 tokens of
// nothing else 83 ms (86 and 540 ms with the queries from memory, a row a lane).
template <typename T, int D>
__device__ __noinline__ void plain_row(const AttendArgs& a, const uint8_t* sQ, int row, const T* K, const T* V, const RowSet& mine, const StepList& steps, int n, float m, int c0, float* o,
                                       float* m_out, float* l_out) {
  float l = 0.f, top = -INFINITY;
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
  float base = m == -INFINITY ? 0.f : m;
  for (int pass = m_out ? 0 : 1; pass < 2; ++pass) {
    for (int j = 0; j < n; ++j) {
      const int r0 = steps.tile(j) * CH_N;
      const uint64_t on = mask64(mine, a.d.n_sink, r0);
      for (int i = 0; i < CH_N; ++i) {
        if (!(on >> i & 1)) continue;
        float2 dot = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(sQ + (c / 8) * (CH_M * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4));
          const uint4 y = *reinterpret_cast<const uint4*>(K + (long long)(r0 + i) * D + c * 8);
          dot = fma2(Num<T>::unpack(x.x), Num<T>::unpack(y.x), dot);
          dot = fma2(Num<T>::unpack(x.y), Num<T>::unpack(y.y), dot);
          dot = fma2(Num<T>::unpack(x.z), Num<T>::unpack(y.z), dot);
          dot = fma2(Num<T>::unpack(x.w), Num<T>::unpack(y.w), dot);
        }
        const float s = __fmul_rn(dot.x + dot.y, a.scale_log2e);
        if (pass == 0) {
          top = fmaxf(top, s);
        } else {
          const float p = ex2(s - base);
          l += p;
          for (int c = 0; c < 16; c += 2) {
            const float2 v = Num<T>::unpack(*reinterpret_cast<const uint32_t*>(V + (long long)(r0 + i) * D + c0 + c));
            o[c] = fmaf(p, v.x, o[c]);
            o[c + 1] = fmaf(p, v.y, o[c + 1]);
          }
        }
      }
    }
    if (pass == 0) base = top == -INFINITY ? 0.f : top;
  }
  if (m_out) {
    *m_out = top;
    *l_out = l;
  }
}

// SPLIT: a tile is shared by a cluster of a.splits CTAs, a kernel of its own for the registers that its way out takes.  (The bound of 3 caps the other form's at
// 96: a prompt of 8,192 tokens takes 145 us in short bursts, 151 without it; two CTAs of either fit on an SM.)
template <typename T, int D, bool SPLIT>
__global__ void __launch_bounds__(CH_THREADS, SPLIT ? 2 : 3) attend_chunk_kernel(const __grid_constant__ ChunkArgs args) {
  constexpr int BOXES = D / 64, QBOX = CH_M * 128, KVBOX = CH_N * 128, KVTILE = BOXES * KVBOX;
  extern __shared__ uint8_t smem_raw[];
  __shared__ ChunkBars bars;
  const AttendArgs& a = args.a;
  uint8_t* smem = smem_raw + ((1024 - (ptx::smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t *sQ = smem, *sK = sQ + BOXES * QBOX, *sV = sK + CH_STAGES * KVTILE;
  ptx::pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int splits = SPLIT ? a.splits : 1, rank = blockIdx.x % splits, tile = args.tiles - 1 - blockIdx.x / splits;   // late tokens see most rows: first
  const int kvh = blockIdx.y, G = a.group, per = CH_M / G;
  const TokenSeq s = load_seq(a.b, a.d, blockIdx.z);
  const int tok0 = tile * per;
  if (tok0 >= s.count) return;      // (the whole cluster)
  const int nt = min(per, s.count - tok0), n_rows = nt * G, q_lo = s.start + tok0, q_hi = q_lo + nt - 1;
  const int rows = a.d.n_sink + a.d.ring, n_sink = a.d.n_sink;
  const int plane = (s.session * a.d.n_kv_heads + kvh) * rows;     // (the cache has fewer than 2^31 rows)
  const RowSet any = seen_by_any(a.d, q_lo, q_hi), all = seen_by_all(a.d, q_lo, q_hi);
  StepList steps;
  const int n = steps.build(any, n_sink, rank, splits);

  if (threadIdx.x == 0) {
    for (int i = 0; i < CH_STAGES; ++i) {
      ptx::mbar_init(&bars.k_full[i], 1);
      ptx::mbar_init(&bars.k_empty[i], 1);
      ptx::mbar_init(&bars.v_full[i], 1);
      ptx::mbar_init(&bars.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&bars.s_full[i], 1);
      ptx::mbar_init(&bars.p_full[i], CH_M);
      ptx::mbar_init(&bars.pv_done[i], 1);
    }
    ptx::mbar_init(&bars.q_full, CH_M);
    bars.failed = bars.odd = 0;
    ptx::fence_barrier_init();
  }
  if (warp == 5) ptx::tmem_alloc(&bars.tmem, CH_TMEM);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = bars.tmem;
  ptx::pdl_launch();      // behind the allocation: a dependent that takes tensor memory before its own wait must not hold what this grid waits for

  const T* Kg = static_cast<const T*>(a.k) + (long long)plane * D;
  const T* Vg = static_cast<const T*>(a.v) + (long long)plane * D;
  const T* Qg = static_cast<const T*>(a.q) + (long long)(s.first + tok0) * a.q_stride + (long long)kvh * G * D;
  bool ok = true;
  const int tl = threadIdx.x / G, hh = threadIdx.x % G;      // this row's token and head (warps 0 .. 3)
  const bool live = (int)threadIdx.x < n_rows;
  RowSet mine = any;
  float m = -INFINITY, l = 0.f, m_odd, l_odd;

  if (warp == 4) {                                           // ---- copies
    if (ptx::elect_one()) {
      for (int j = 0; j < n && ok; ++j) {
        const int st = j % CH_STAGES, y = plane + steps.tile(j) * CH_N;
        const uint32_t ph = (j / CH_STAGES - 1) & 1;
        if (j >= CH_STAGES) ok = ptx::mbar_wait_limit(&bars.k_empty[st], ph, CH_POLLS);
        if (!ok) break;
        ptx::mbar_expect_tx(&bars.k_full[st], KVTILE);
#pragma unroll
        for (int b = 0; b < BOXES; ++b) ptx::tma_load_2d(sK + st * KVTILE + b * KVBOX, &args.kmap, b * 64, y, &bars.k_full[st]);
        if (j >= CH_STAGES) ok = ptx::mbar_wait_limit(&bars.v_empty[st], ph, CH_POLLS);
        if (!ok) break;
        ptx::mbar_expect_tx(&bars.v_full[st], KVTILE);
#pragma unroll
        for (int b = 0; b < BOXES; ++b) ptx::tma_load_2d(sV + st * KVTILE + b * KVBOX, &args.vmap, b * 64, y, &bars.v_full[st]);
      }
    }
    __syncwarp();
  } else if (warp == 5) {                                    // ---- products
    const uint64_t dq = ptx::umma_desc_sw128(ptx::smem_u32(sQ)), dk = ptx::umma_desc_sw128(ptx::smem_u32(sK)), dv = ptx::umma_desc_sw128(ptx::smem_u32(sV)) + ((uint64_t)(KVBOX / 16 - 1) << 16);   // (columns behind the 64th: the next box)
    auto scores = [&](int j) {
      const int st = j % CH_STAGES;
      if (!warp_wait(&bars.k_full[st], (j / CH_STAGES) & 1)) return false;
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          ptx::umma_bf16(tmem + (j & 1) * CH_N, dq + ((k / 4) * QBOX + (k % 4) * 32) / 16, dk + (st * KVTILE + (k / 4) * KVBOX + (k % 4) * 32) / 16, chunk_idesc<T, CH_N>(0), k > 0);
        ptx::umma_commit(&bars.k_empty[st]);
        ptx::umma_commit(&bars.s_full[j & 1]);
      }
      __syncwarp();
      return true;
    };
    ok = warp_wait(&bars.q_full, 0);
    if (ok && n > 0) ok = scores(0);
    if (ok && n > 1) ok = scores(1);
    for (int j = 0; j < n && ok; ++j) {
      const int st = j % CH_STAGES;
      ok = warp_wait(&bars.v_full[st], (j / CH_STAGES) & 1) && warp_wait(&bars.p_full[j & 1], (j >> 1) & 1);
      if (!ok) break;
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
#pragma unroll
        for (int k = 0; k < CH_N / 16; ++k)
          umma_ts(tmem + CH_O, tmem + (j & 1) * CH_N + k * 8, dv + (st * KVTILE + k * 2048) / 16, chunk_idesc<T, D>(1), j > 0 || k > 0);
        ptx::umma_commit(&bars.v_empty[st]);
        ptx::umma_commit(&bars.pv_done[j & 1]);
      }
      __syncwarp();
      if (j + 2 < n) ok = scores(j + 2);      // (into the columns that the product above has just read: products run in order)
    }
  } else {                                                   // ---- a query row per thread
    // the queries to the swizzled rows that the products read, all copies in flight at once (a row at a time it took 9,000 cycles)
    constexpr int CPR = D / 8;
    const uint32_t sq = ptx::smem_u32(sQ), inv_g = (65536u + G - 1) / G;      // r / G = r * inv_g >> 16 for r < 128, G <= 64
#pragma unroll
    for (int i = 0; i < CPR; ++i) {
      const int ch = i * 32 + lane, r = warp * 32 + ch / CPR, c = ch % CPR, tr = (int)(r * inv_g >> 16);
      const bool on = r < n_rows;
      cp16(sq + (c / 8) * QBOX + r * 128 + (((c & 7) ^ (r & 7)) << 4), Qg + (on ? (long long)tr * a.q_stride + (r - tr * G) * D + c * 8 : 0), on);
    }
    asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive(&bars.q_full);
    const int qp = q_lo + (live ? tl : 0);
    mine = seen_by_any(a.d, qp, qp);
    const uint32_t lane_base = tmem + ((uint32_t)warp << 21);      // lanes 32 warp .. of tensor memory
    for (int j = 0; j < n; ++j) {
      const int r0 = steps.tile(j) * CH_N, st = j % CH_STAGES;
      ok = warp_wait(&bars.s_full[j & 1], (j >> 1) & 1) && (j < 2 || warp_wait(&bars.pv_done[j & 1], ((j - 2) >> 1) & 1));    // (the second: step j - 2's, long done: no phase goes by unseen)
      if (!ok) break;
      ptx::tc_fence_after();
      float x[CH_N];
      ptx::tmem_ld64(lane_base + (j & 1) * CH_N, x);
      const uint64_t in_all = mask64(all, n_sink, r0);
      if (in_all != ~0ull) {                                 // some query of the tile does not see some row
        const uint64_t on = mask64(mine, n_sink, r0), in_any = mask64(any, n_sink, r0);
#pragma unroll
        for (int i = 0; i < CH_N; ++i) x[i] = (i < 32 ? (uint32_t)on >> i : (uint32_t)(on >> 32) >> (i - 32)) & 1 ? x[i] : -INFINITY;
        // rows of V that nobody sees become zeros; of those that only some see, infinities and NaN are noted
        ok = warp_wait(&bars.v_full[st], (j / CH_STAGES) & 1);
        if (!ok) break;
        // (half a row a thread; neighbouring rows' pieces lie in different banks)
        const int r = threadIdx.x & (CH_N - 1), c0 = (int)(threadIdx.x / CH_N) * (CPR / 2);
        uint8_t* row = sV + st * KVTILE + (c0 / 8) * KVBOX + r * 128;
        bool odd = false;
        if (!(in_all >> r & 1)) {
#pragma unroll
          for (int i = 0; i < CPR / 2; ++i) {
            uint4* p = reinterpret_cast<uint4*>(row + (((((c0 & 7) + i) & 7) ^ (r & 7)) << 4));
            if (in_any >> r & 1) {
              const uint4 v = *p;
              odd |= Num<T>::odd(v.x) | Num<T>::odd(v.y) | Num<T>::odd(v.z) | Num<T>::odd(v.w);
            } else {
              *p = make_uint4(0, 0, 0, 0);
            }
          }
        }
        if (odd) bars.odd = 1;
        ptx::fence_proxy_async_smem();
      }
      float t0 = x[0], t1 = x[1], t2 = x[2], t3 = x[3];
#pragma unroll
      for (int i = 4; i < CH_N; i += 4) {
        t0 = fmaxf(t0, x[i]);
        t1 = fmaxf(t1, x[i + 1]);
        t2 = fmaxf(t2, x[i + 2]);
        t3 = fmaxf(t3, x[i + 3]);
      }
      const float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * a.scale_log2e;
      const bool move = top > m + 8.f;                       // (m = -inf: at the first row that is seen)
      if (__any_sync(0xffffffffu, move)) {
        const float f = move ? ex2(m - top) : 1.f;
        if (move) {
          m = top;
          if (fabsf(top) > CH_FAR && top < INFINITY) bars.odd = 1;
        }
        l *= f;
        if (j > 0) {
          ok = warp_wait(&bars.pv_done[(j - 1) & 1], ((j - 1) >> 1) & 1);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            float o[16];
            ptx::tmem_ld16(lane_base + CH_O + c, o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= f;
            ptx::tmem_st16(lane_base + CH_O + c, o);
          }
        }
      }
      const float base = m == -INFINITY ? 0.f : m;
      const float2 sc2 = make_float2(a.scale_log2e, a.scale_log2e), nb2 = make_float2(-base, -base);
      float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
      uint32_t p[CH_N / 2];
#pragma unroll
      for (int i = 0; i < CH_N; i += 4) {
        float2 u = fma2(make_float2(x[i], x[i + 1]), sc2, nb2), v = fma2(make_float2(x[i + 2], x[i + 3]), sc2, nb2);
        u = make_float2(ex2(u.x), ex2(u.y));
        v = make_float2(ex2(v.x), ex2(v.y));
        sum0 = add2(sum0, u);
        sum1 = add2(sum1, v);
        p[i / 2] = Num<T>::pack(u.x, u.y);
        p[i / 2 + 1] = Num<T>::pack(v.x, v.y);
      }
      sum0 = add2(sum0, sum1);
      l += sum0.x + sum0.y;
      tmem_st32(lane_base + (j & 1) * CH_N, p);
      ptx::tc_fence_before();
      ptx::mbar_arrive(&bars.p_full[j & 1]);
    }
    if (ok && n > 1) ok = warp_wait(&bars.pv_done[n & 1], ((n - 2) >> 1) & 1);
    if (ok && n > 0) ok = warp_wait(&bars.pv_done[(n - 1) & 1], ((n - 1) >> 1) & 1);
    ptx::tc_fence_after();
  }
  if (!ok) {
    bars.failed = 1;
    *a.err = a.err_id;
  }
  __syncthreads();                                           // every product of this CTA has completed, or a wait has given up
  const bool failed = bars.failed != 0;
  if (failed) ptx::pause_for_copies();
  // Split tiles: CTA k finishes `own` rows from k * own on, and the others write their parts of those straight into its memory, [CTA][own][D] with the
  // 16-byte pieces of a row in the order piece ^ (row & 15).  (Writes are posted; reading the parts from the other CTAs took 8,000 cycles of a full tile, a
  // thousand a round.)
  const int own = (n_rows + splits - 1) / splits;
  const uint32_t part_s = ptx::smem_u32(sK), lane_base = tmem + ((uint32_t)warp << 21);
  const bool whole = warp < 4 && !failed && n > 0 && !bars.odd;      // this warp's rows are in tensor memory
  // the rows of a tile whose output is not there: none of this CTA's share is seen, or the odd ones
  auto apart = [&](auto emit) {
    float o[16] = {};
    if (n == 0) {
      for (int c = 0; c < D; c += 16) emit(c, o);
      return;
    }
#pragma unroll 1
    for (int c = 0; c < D; c += 16) {
      plain_row<T, D>(a, sQ, threadIdx.x, Kg, Vg, mine, steps, n, m, c, o, c == 0 ? &m_odd : nullptr, &l_odd);
      if (c == 0) {
        m = m_odd;
        l = l_odd;
      }
      emit(c, o);
    }
  };
  if constexpr (!SPLIT) {
    if (warp < 4 && !failed) {
      T* out = static_cast<T*>(a.out) + (long long)(s.first + tok0 + (live ? tl : 0)) * a.out_stride + (long long)(kvh * G + (live ? hh : 0)) * D;
      auto emit = [&](int c, const float* o) {                           // 16 columns
        if (!live) return;
        const float inv = 1.0f / l;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = Num<T>::pack(Num<T>::mean(o[2 * i] * inv), Num<T>::mean(o[2 * i + 1] * inv));
        *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
      };
      if (whole) {
#pragma unroll
        for (int c = 0; c < D; c += 64) {
          float o[64];
          ptx::tmem_ld64(lane_base + CH_O + c, o);
#pragma unroll
          for (int i = 0; i < 64; i += 16) emit(c + i, o + i);
        }
      } else {
        apart(emit);
      }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 5) ptx::tmem_dealloc(tmem, CH_TMEM);
    return;
  }
  // The output leaves tensor memory, and tensor memory is given back, before this CTA waits for the others of its cluster: one of those may
  // be waiting for columns that another kernel's CTA holds, which in turn may wait for these.
  float o_all[D];
  if (whole) {
#pragma unroll
    for (int c = 0; c < D; c += 64) ptx::tmem_ld64(lane_base + CH_O + c, o_all + c);
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 5) ptx::tmem_dealloc(tmem, CH_TMEM);
  __syncwarp();               // (the cluster's barrier is met by whole warps)
  ptx::cluster_arrive();      // every CTA of the cluster is through with its K and V: the parts go there
  ptx::cluster_wait();
  if (warp < 4 && !failed) {
    const int to = live ? threadIdx.x / own : 0, slot = rank * own + (live ? threadIdx.x % own : 0);
    const uint32_t part = ptx::map_to_cta(part_s + slot * D * 4, to);
    auto emit = [&](int c, const float* o) {
      if (!live) return;
#pragma unroll
      for (int i = 0; i < 4; ++i) st_cluster4(part + (((c / 4 + i) ^ (slot & 15)) << 4), o + 4 * i);
    };
    if (whole) {
#pragma unroll
      for (int c = 0; c < D; c += 16) emit(c, o_all + c);
    } else {
      apart(emit);
    }
    if (live) {
      st_cluster(ptx::map_to_cta(ptx::smem_u32(&bars.m[slot]), to), m);
      st_cluster(ptx::map_to_cta(ptx::smem_u32(&bars.l[slot]), to), l);
    }
  }
  __syncwarp();
  ptx::cluster_arrive();
  ptx::cluster_wait();      // (nobody reads or writes another CTA's memory behind this)
  const int r0 = rank * own, mine_n = min(own, n_rows - r0);
  float* weight = reinterpret_cast<float*>(sQ);      // [CTA][own]
  if ((int)threadIdx.x < mine_n) {
    const int r = threadIdx.x;
    float M = -INFINITY, L = 0.f;
    for (int k = 0; k < splits; ++k) M = fmaxf(M, bars.m[k * own + r]);
    const float base = M == -INFINITY ? 0.f : M;
    for (int k = 0; k < splits; ++k) L = fmaf(ex2(bars.m[k * own + r] - base), bars.l[k * own + r], L);
    const float inv = 1.0f / L;
    for (int k = 0; k < splits; ++k) weight[k * own + r] = ex2(bars.m[k * own + r] - base) * inv;
  }
  __syncthreads();
  const float* parts = reinterpret_cast<const float*>(sK);
  T* out = static_cast<T*>(a.out) + (long long)(s.first + tok0) * a.out_stride + (long long)kvh * G * D;
  constexpr int QUADS = D / 4;
#pragma unroll 4
  for (int e = threadIdx.x; e < mine_n * QUADS; e += CH_THREADS) {
    const int r = e / QUADS, c = e % QUADS, row = r0 + r, tr = (int)(row * ((65536u + G - 1) / G) >> 16);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    int slot = r;
#pragma unroll 2
    for (int k = 0; k < splits; ++k, slot += own) {
      const float f = weight[slot];
      const float4 v = *reinterpret_cast<const float4*>(parts + slot * D + ((c ^ (slot & 15)) << 2));
      o = make_float4(fmaf(f, v.x, o.x), fmaf(f, v.y, o.y), fmaf(f, v.z, o.z), fmaf(f, v.w, o.w));
    }
    *reinterpret_cast<uint2*>(out + (long long)tr * a.out_stride + (row - tr * G) * D + c * 4) =
        make_uint2(Num<T>::pack(Num<T>::mean(o.x), Num<T>::mean(o.y)), Num<T>::pack(Num<T>::mean(o.z), Num<T>::mean(o.w)));
  }
}
