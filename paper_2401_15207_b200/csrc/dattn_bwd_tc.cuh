// Differential attention backward on tcgen05 (bf16, heads of 64 and 128).  Included into gemm_tc.cu after dattn_fwd_tc.cuh.
//
// Two launches of one template, so that every output row has one writer and a fixed order of summation (no atomics):
//   MODE 0 (dk, dv): a CTA owns 128 keys of a key head and streams the queries of all heads of its group, 64 at a time
//   MODE 1 (dq)    : a CTA owns 128 queries and streams the keys, 64 at a time
//              F0   F1    X0   X1     S_m = F0_m X0_m^T, m = 1, 2     dP = F1 X1^T     accumulators
//   MODE 0     K    V     Q    g      scores^T                        (g V^T)^T        dv += (P_1 - lambda P_2)^T g,  dk_m += dS_m^T Q_m
//   MODE 1     Q    g     K    V      scores                          g V^T            dq_m += dS_m K_m
// (F0_m: the map's half of the columns; g: gradient of o.)  P_m = exp(scale S_m - lse_m),  dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2);
// dk and dq are multiplied by `scale` as they are stored.  dP is shared by the maps, and dv takes one product for both: 8 units of 128 x 64 x 64 a
// step against the 10 of two plain attentions.  P, dS and, behind a norm, g are rounded to bf16, the operand type of the products they feed (dqkv 2.4e-3 off relative to its norm, 3.0e-3
// with the norm, where its own rounding alone is 1.7e-3; what a rounding of g leaves would take a second product of dP and of dv, 4 units more); the accumulators are fp32.
//   warp 0    : TMA producer         warp 1: issues every product (one elected thread); owns the tensor memory
//   warp 2    : MODE 1 with key lengths, K's rows of hidden keys -> zeros
//   warps 4.. : element-wise, two or four warps to a lane quarter, their share of the 64 streamed columns each: S_1, S_2 -> registers, exponentials; dP, dS;
//               P and dS go back to tensor memory as bf16, the A operands of the accumulating products; at an item's end the accumulators -> global
// Two steps in flight (MODE 1, and heads of 64): two sets of S_1, S_2, dP (columns 192 u ..), accumulators behind 384.  P and dS lie over the scores, each
// warp's part over columns that it alone has read; the order of issue is  accumulating products of t, then S(t+2) and dP(t+2) into the same set.
// One step in flight (MODE 0 at heads of 128, whose accumulators take 256 columns): S_1 0, S_2 64, dP 128, [P_1 - lambda P_2 | dS_1] 192 (32 each), dS_2 over
// dP in the same way, accumulators 256.  S(t+1) is issued as soon as S(t) has been read, so that it runs beside the exponentials of step t; then
// the accumulating products of t; then dP(t+1), which finds both its buffer and the P / dS buffers of step t free when it is done.
// What bounds it: products 1276 cycles a step at heads of 128 (1024 in MODE 1), exponentials 1024 of the special function unit, and the element-wise warps' chain
// of them: scores, exponentials, dP, dS.  1 x 4096 x 16 heads of 128, causal, 114 steps a CTA: dk/dv 179 us and dq 135 by the profiler, each alone with cold caches; the whole call, with the
// preparation, 333 us in a run of calls.  With shared key heads a dk/dv item walks its whole group in sequence, and few items are left: the same case
// on 4 key heads 475 us, on one 1405.
#pragma once

constexpr int kDbX = 64;
template <int DH, int MODE> struct DattnBwdCfg {
  static constexpr int kSpans = DH / 64;
  static constexpr int kFBytes = 128 * DH * 2, kXBytes = kDbX * DH * 2;
  // Element-wise warps to a lane quarter.  MODE 0: two, of 32 streamed columns each (four: 180 -> 207 us at 4096 x 16 heads of 128, for each column's lse
  // and D are read from shared memory by every thread and the instructions bound it); MODE 1: four, of 16 (two: 135 -> 140 us)
  static constexpr int kParts = MODE == 0 ? 2 : 4, kEw = 4 * kParts, kThreads = 128 + 32 * kEw;
  static constexpr bool kTwo = MODE == 1 || DH == 64;              // two steps in flight: the accumulators leave tensor memory for two sets of S and dP
  static constexpr int kStages = kTwo ? 4 : 3;
  static constexpr int kNF = DH == 64 ? 2 : 1;                     // sets of fixed tiles: the next item's are fetched beside this one's steps
  static constexpr int kStage = kEw * 32 * (DH / kParts) * 2;      // a piece of 32 rows x this warp's share of the columns per element-wise warp
  static constexpr int kCol = MODE == 0 ? kEw * 2 * 512 : 0;       // per warp, two steps: lse and D of its 32 queries
  static constexpr int kSmem = kNF * 2 * kFBytes + kStages * 2 * kXBytes + kStage + kCol + 256 + 1024;
};

__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// loads and stores of as many columns as the array has registers
__device__ __forceinline__ void tm_load(uint32_t addr, uint32_t (&v)[32]) { tmem_ld32_nowait(addr, v); }
__device__ __forceinline__ void tm_load(uint32_t addr, uint32_t (&v)[16]) { tmem_ld16_nowait(addr, v); }
__device__ __forceinline__ void tm_loaded(uint32_t (&v)[32]) { tmem_ld_wait32(v); }
__device__ __forceinline__ void tm_loaded(uint32_t (&v)[16]) { tmem_ld_wait16(v); }
__device__ __forceinline__ void tm_store(uint32_t addr, const uint32_t (&v)[16]) { tmem_st16(addr, v); }
__device__ __forceinline__ void tm_store(uint32_t addr, const uint32_t (&v)[8]) { tmem_st8(addr, v); }
struct DattnBwdItem { int b, hk, f0, x_lo, per, nsteps, len; };    // hk: key head (MODE 0) or query head (MODE 1); per: steps of one head

template <int DH, int MODE>
__global__ void __launch_bounds__(DattnBwdCfg<DH, MODE>::kThreads, 1)
dattn_bwd_tc_kernel(const __grid_constant__ CUtensorMap map_f0, const __grid_constant__ CUtensorMap map_f1, const __grid_constant__ CUtensorMap map_x0,
                    const __grid_constant__ CUtensorMap map_x1, const __grid_constant__ CUtensorMap map_out, const DattnArgs a) {
  typedef DattnBwdCfg<DH, MODE> Cfg;
  constexpr int SP = Cfg::kSpans, HD = DH / 2, NS = Cfg::kStages, FB = Cfg::kFBytes, XB = Cfg::kXBytes, FSPAN = 128 * 128, XSPAN = kDbX * 128;
  constexpr int NF = Cfg::kNF, NP = Cfg::kParts, EW = Cfg::kEw, XC = kDbX / NP;        // XC: streamed columns of a thread
  constexpr bool TWO = Cfg::kTwo;
  extern __shared__ uint8_t smem_raw[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sF = base, sX = sF + NF * 2 * FB, sStage = sX + NS * 2 * XB, sCol = sStage + Cfg::kStage, bar = sCol + Cfg::kCol;
  // two steps in flight: s_full(u) covers S and dP of set u; one step: u = 0, and dP has a barrier of its own
  auto s_full = [&](int u) { return bar + (TWO ? 8u * u : 0u); };
  auto p_ready = [&](int u) { return bar + 16u + (TWO ? 8u * u : 0u); };
  const uint32_t s_free = bar + 32u, dp_full = bar + 40u, acc_full = bar + 48u, acc_free = bar + 56u, tmem_slot = bar + 160u;
  auto f_full = [&](int n) { return bar + 128u + 8u * (n % NF); };           // the set of fixed tiles of item n; its phase is n / NF
  auto f_empty = [&](int n) { return bar + 144u + 8u * (n % NF); };
  auto x_full = [&](int i) { return bar + 64u + 8u * i; };
  auto x_empty = [&](int i) { return bar + 96u + 8u * i; };
  auto x_ok = [&](int i) { return bar + 176u + 8u * i; };
  volatile uint32_t* slot_gen = reinterpret_cast<volatile uint32_t*>(gen + (tmem_slot - base));
  volatile uint32_t* poison_gen = slot_gen + 2;

  const int nfb = (a.S + 127) / 128, heads = MODE == 0 ? a.K : a.H, nbh = a.B * heads, nitems = nfb * nbh, group = a.H / a.K;
  auto item_of = [&](int idx) {
    DattnBwdItem it;
    const int rank = idx / nbh, bh = idx - rank * nbh;
    it.b = bh / heads;
    it.hk = bh - it.b * heads;
    it.len = a.lens ? max(0, min(a.lens[it.b], a.S)) : a.S;
    it.x_lo = 0;
    if (MODE == 0) {
      it.f0 = rank * 128;
      it.x_lo = a.causal ? it.f0 / kDbX : 0;
      it.per = (a.S + kDbX - 1) / kDbX - it.x_lo;
      it.nsteps = it.per * group;
      if (it.f0 >= it.len) it.nsteps = 1;                          // padding alone: one step, all of it masked, writes the zeros
    } else {
      it.f0 = (a.causal ? nfb - 1 - rank : rank) * 128;
      const int end = min(a.causal ? min(a.S, it.f0 + 128) : a.S, it.len);
      it.per = it.nsteps = max(1, (end + kDbX - 1) / kDbX);
    }
    return it;
  };

  if (threadIdx.x == 0) {
    for (int i = 0; i < NF; ++i) { mbar_init(f_full(i), 1); mbar_init(f_empty(i), 1); }
    for (int u = 0; u < (TWO ? 2 : 1); ++u) { mbar_init(s_full(u), 1); mbar_init(p_ready(u), EW); }
    mbar_init(s_free, EW); mbar_init(dp_full, 1);
    mbar_init(acc_full, 1); mbar_init(acc_free, EW);
    for (int i = 0; i < NS; ++i) { mbar_init(x_full(i), 1); mbar_init(x_empty(i), 1); mbar_init(x_ok(i), 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_wait();                                                    // no global access before it, the flag included
    *poison_gen = g_tc_error != 0 ? 1u : 0u;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = __shfl_sync(0xffffffffu, *slot_gen, 0);
  const bool poisoned = __any_sync(0xffffffffu, *poison_gen != 0);
  pdl_trigger();
  pdl_wait();
  auto t_s = [&](int m, int u) { return tm + (TWO ? 192u * u : 0u) + 64u * m; };
  auto t_dp = [&](int u) { return tm + (TWO ? 192u * u : 0u) + 128u; };
  const uint32_t tAcc = tm + (TWO ? 384u : 256u), tDv = tm + (TWO ? 448u : 384u);
  // packed P_1 - lambda P_2 (w = 0, MODE 0), dS_1 (1), dS_2 (2) of streamed column c (a multiple of 16, or of XC)
  auto t_p = [&](int w, int c, int u) -> uint32_t {
    const uint32_t own = (uint32_t)(c / XC * XC + c % XC / 2);     // over columns that the same warp has read
    if (TWO) return w == 2 ? t_s(1, u) + own : t_s(0, u) + own + (MODE == 0 && w == 1 ? XC / 2 : 0);
    return w == 2 ? t_dp(u) + own : tm + 192u + 32u * w + (uint32_t)(c / 2);
  };

  if (warp == 0) {
    if (!poisoned && elect_one()) {
      // ---------------- TMA producer
      int st = 0, n = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
        const DattnBwdItem it = item_of(idx);
        const int colF0 = (MODE == 0 ? a.H + it.hk : it.hk) * DH, colF1 = (MODE == 0 ? a.H + a.K + it.hk : it.hk) * DH;
        if (!mbar_wait(f_empty(n), (uint32_t)(((n / NF) & 1) ^ 1))) { atomicCAS(&g_tc_error, 0, 7); break; }
        mbar_expect_tx(f_full(n), 2 * FB);
        const uint32_t sF0 = sF + (n % NF) * 2 * FB;
#pragma unroll
        for (int sp = 0; sp < SP; ++sp) {
          tma_load_3d(sF0 + sp * FSPAN, &map_f0, f_full(n), colF0 + sp * 64, it.f0, it.b);
          tma_load_3d(sF0 + FB + sp * FSPAN, &map_f1, f_full(n), colF1 + sp * 64, it.f0, it.b);
        }
        int x = it.x_lo, h = MODE == 0 ? it.hk * group : it.hk / group;
        for (int t = 0; t < it.nsteps; ++t) {
          if (!mbar_wait(x_empty(st), ph)) { atomicCAS(&g_tc_error, 0, 7); ok = false; break; }
          const int colX0 = (MODE == 0 ? h : a.H + h) * DH, colX1 = (MODE == 0 ? h : a.H + a.K + h) * DH;
          const uint32_t s0 = sX + st * 2 * XB;
          mbar_expect_tx(x_full(st), 2 * XB);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) {
            tma_load_3d(s0 + sp * XSPAN, &map_x0, x_full(st), colX0 + sp * 64, x * kDbX, it.b);
            tma_load_3d(s0 + XB + sp * XSPAN, &map_x1, x_full(st), colX1 + sp * 64, x * kDbX, it.b);
          }
          if (++st == NS) { st = 0; ph ^= 1; }
          if (++x == it.x_lo + it.per) { x = it.x_lo; ++h; }
        }
      }
    }
  } else if (warp == 1) {
    if (!poisoned) {
      if (elect_one()) {
        // ---------------- MMA issuer
        const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | (((uint32_t)kDbX >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t idesc_h = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)HD >> 3) << 17) | ((128u >> 4) << 24);       // N = d
        const uint32_t idesc_v = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)DH >> 3) << 17) | ((128u >> 4) << 24);       // N = 2 d
        const uint64_t dF = desc_kmajor(sF), dX0 = desc_kmajor(sX);
        auto k_off = [](int e, int span) { return (uint64_t)(((e / 4) * span + (e % 4) * 32) >> 4); };       // 16 columns, number e, of a K-major tile
        auto issue_s = [&](int item, int st, int u) {
          const uint64_t dF0 = dF + (uint64_t)((item % NF) * (2 * FB >> 4)), x0 = dX0 + (uint64_t)(st * (2 * XB >> 4));
#pragma unroll
          for (int e = 0; e < DH / 16; ++e)
            tc_mma(t_s(e < HD / 16 ? 0 : 1, u), dF0 + k_off(e, FSPAN), x0 + k_off(e, XSPAN), idesc_s, e % (HD / 16) > 0 ? 1u : 0u);
        };
        auto issue_dp = [&](int item, int st, int u) {
          const uint64_t dF1 = dF + (uint64_t)(((item % NF) * 2 * FB + FB) >> 4), x1 = dX0 + (uint64_t)((st * 2 * XB + XB) >> 4);
#pragma unroll
          for (int e = 0; e < DH / 16; ++e) tc_mma(t_dp(u), dF1 + k_off(e, FSPAN), x1 + k_off(e, XSPAN), idesc_s, e > 0 ? 1u : 0u);
        };
        auto issue_acc = [&](int st, int u, bool first) {
          const uint64_t nX0 = desc_nmajor(sX, XSPAN) + (uint64_t)(st * (2 * XB >> 4)), nX1 = nX0 + (uint64_t)(XB >> 4);
#pragma unroll
          for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              // the map's half of X0's columns: the second span (heads of 128), or the second half of the one span
              const uint64_t b = nX0 + (uint64_t)((kk * 16 * 128 + m * (DH == 128 ? XSPAN : 64)) >> 4);
              tc_mma_ta(tAcc + (uint32_t)(m * HD), t_p(1 + m, kk * 16, u), b, idesc_h, (!first || kk > 0) ? 1u : 0u);
            }
          }
          if (MODE == 0) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) tc_mma_ta(tDv, t_p(0, kk * 16, u), nX1 + (uint64_t)((kk * 16 * 128) >> 4), idesc_v, (!first || kk > 0) ? 1u : 0u);
          }
          tc_commit(x_empty(st));
        };
        bool ok = true;
        int n = 0, t = 0, g = 0, st = 0;                           // g: steps over all items; st: its ring slot
        uint32_t ph = 0;
        int idx = dattn_item_at(0), nsteps = idx < nitems ? item_of(idx).nsteps : 0;
        if (TWO) {
          // the step whose S and dP are issued next, two ahead of the one whose products accumulate
          int sn = 0, sj = 0, sg = 0, sst = 0, ssteps = nsteps;
          uint32_t sph = 0;
          bool live = nsteps > 0;
          auto ahead = [&]() -> bool {
            if ((sj == 0 && !mbar_wait(f_full(sn), (uint32_t)((sn / NF) & 1))) || !mbar_wait(MODE == 1 && a.lens ? x_ok(sst) : x_full(sst), sph)) return false;
            tc_fence_after();
            issue_s(sn, sst, sg & 1);
            issue_dp(sn, sst, sg & 1);
            tc_commit(s_full(sg & 1));
            ++sg;
            if (++sst == NS) { sst = 0; sph ^= 1u; }
            if (++sj == ssteps) {
              tc_commit(f_empty(sn));
              sj = 0;
              const int i = dattn_item_at(++sn);
              live = i < nitems;
              if (live) ssteps = item_of(i).nsteps;
            }
            return true;
          };
          for (int i = 0; i < 2 && live && ok; ++i) ok = ahead();
          while (ok && idx < nitems) {
            ok = (t > 0 || n == 0 || mbar_wait(acc_free, (uint32_t)((n - 1) & 1))) && mbar_wait(p_ready(g & 1), (uint32_t)((g >> 1) & 1));
            if (!ok) break;
            tc_fence_after();
            issue_acc(st, g & 1, t == 0);
            const bool last = t + 1 == nsteps;
            if (last) tc_commit(acc_full);
            if (live) ok = ahead();
            ++g;
            if (++st == NS) st = 0;
            if (last) {
              t = 0;
              idx = dattn_item_at(++n);
              if (idx < nitems) nsteps = item_of(idx).nsteps;
            } else {
              ++t;
            }
          }
        } else {
          if (nsteps) {
            ok = mbar_wait(f_full(0), 0) && mbar_wait(x_full(0), 0);
            if (ok) {
              tc_fence_after();
              issue_s(0, 0, 0);
              tc_commit(s_full(0));
              issue_dp(0, 0, 0);
              tc_commit(dp_full);
              if (nsteps == 1) tc_commit(f_empty(0));
            }
          }
          while (ok && idx < nitems) {
            const bool last = t + 1 == nsteps;
            const int next_idx = last ? dattn_item_at(n + 1) : idx, st1 = st + 1 == NS ? 0 : st + 1;
            const uint32_t ph1 = st + 1 == NS ? ph ^ 1u : ph;
            const bool more = next_idx < nitems;
            if (!last) {                                           // scores of the next step beside the exponentials of this one
              ok = mbar_wait(s_free, (uint32_t)(g & 1)) && mbar_wait(x_full(st1), ph1);
              if (!ok) break;
              tc_fence_after();
              issue_s(n, st1, 0);
              tc_commit(s_full(0));
            }
            ok = (t > 0 || n == 0 || mbar_wait(acc_free, (uint32_t)((n - 1) & 1))) && mbar_wait(p_ready(0), (uint32_t)(g & 1));
            if (!ok) break;
            tc_fence_after();
            issue_acc(st, 0, t == 0);
            if (last) tc_commit(acc_full);
            int next_steps = nsteps;
            if (more) {
              if (last) {                                          // another item: its fixed tiles take the place of this one's
                next_steps = item_of(next_idx).nsteps;
                ok = mbar_wait(s_free, (uint32_t)(g & 1)) && mbar_wait(f_full(n + 1), (uint32_t)(((n + 1) / NF) & 1)) && mbar_wait(x_full(st1), ph1);
                if (!ok) break;
                tc_fence_after();
                issue_s(n + 1, st1, 0);
                tc_commit(s_full(0));
              }
              issue_dp(last ? n + 1 : n, st1, 0);
              tc_commit(dp_full);
              if (last ? next_steps == 1 : t + 2 == nsteps) tc_commit(f_empty(last ? n + 1 : n));
            }
            ++g;
            st = st1;
            ph = ph1;
            if (last) { t = 0; ++n; idx = next_idx; nsteps = next_steps; } else ++t;
          }
        }
        if (!ok) atomicCAS(&g_tc_error, 0, 8);
      }
      __syncwarp();
    }
  } else if (MODE == 1 && warp == 2) {
    if (!poisoned && a.lens) {
      // ---------------- hidden keys: rows of a block of K behind the entry's length become zeros (dS is 0 there, but 0 times NaN is not)
      int st = 0, n = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
        const DattnBwdItem it = item_of(idx);
        for (int t = 0; t < it.nsteps; ++t) {
          const bool ready = mbar_wait(x_full(st), ph);
          if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 7);
          ok = __all_sync(0xffffffffu, ready);
          if (!ok) break;
          zero_rows<SP, kDbX>(gen + (sX + st * 2 * XB - base), it.len - t * kDbX, lane);
          if (lane == 0) mbar_arrive(x_ok(st));
          if (++st == NS) { st = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp >= 4) {
    // ---------------- element-wise: thread = row of the fixed tile x XC streamed columns
    const int q = warp & 3, hc = (warp - 4) >> 2, r = q * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f;
    const uint64_t sc2 = f2_pack(sl2, sl2);
    const int64_t nrow = (int64_t)a.B * a.H * a.S;
    const uint32_t sPiece = sStage + (warp - 4) * (32 * (DH / NP) * 2);
    uint8_t* piece = gen + (sPiece - base);
    float* col = reinterpret_cast<float*>(gen + (sCol - base)) + (warp - 4) * 256;      // MODE 0: two buffers of XC / 2 column pairs x (-lse_1, -lse_2, -D_1, -D_2)
    bool ok = !poisoned;
    int n = 0, g = 0;
    // -lse in log2 units; a query that sees no key, or is none: P = 0 through -infinity
    auto neg_log2 = [](float v) { return v == -INFINITY ? -INFINITY : -v * 1.4426950408889634f; };
    for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
      const DattnBwdItem it = item_of(idx);
      const int frow = it.f0 + r;
      int x = it.x_lo, h = MODE == 0 ? it.hk * group : it.hk;
      // lse and D as they lie in memory, of this lane's column of the next step (MODE 0; nothing touches them before that step, so that no step waits
      // for them) or of this thread's row (MODE 1)
      float rl[2], rd[2];
      auto fetch = [&](int xx, int hh) {
        const int c = MODE == 0 ? xx * kDbX + hc * XC + (lane & (XC - 1)) : frow;
        const bool in = c < a.S;
        const int64_t at = ((int64_t)it.b * a.H + hh) * a.S + (in ? c : 0);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          rl[m] = in ? a.lse[m * nrow + at] : -INFINITY;
          rd[m] = in ? a.dsum[m * nrow + at] : 0.f;
        }
      };
      fetch(x, h);
      float lam = a.lam[h], lam_next = lam;
      float nl[2], nd[2];                                          // MODE 1
      if (MODE == 1) {
#pragma unroll
        for (int m = 0; m < 2; ++m) { nl[m] = neg_log2(rl[m]); nd[m] = -rd[m]; }
      }
      for (int t = 0; t < it.nsteps; ++t, ++g) {
        const int x0 = x * kDbX;
        const uint64_t nlam2 = f2_pack(-lam, -lam);
        float* cv = col + (g & 1) * 128;
        if (MODE == 0) {
          float* w = cv + ((lane & (XC - 1)) >> 1) * 8 + (lane & 1);
          if (lane < XC) { w[0] = neg_log2(rl[0]); w[2] = neg_log2(rl[1]); w[4] = -rd[0]; w[6] = -rd[1]; }
          __syncwarp();
        }
        int nx = x + 1, nh = h;
        if (MODE == 0 && nx == it.x_lo + it.per) { nx = it.x_lo; ++nh; }
        if (MODE == 0 && t + 1 < it.nsteps) {
          fetch(nx, nh);
          if (nh != h) lam_next = a.lam[nh];
        }
        const int u = TWO ? g & 1 : 0;
        const uint32_t par = (uint32_t)((TWO ? g >> 1 : g) & 1);
        bool ready = mbar_wait(s_full(u), par);
        if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 9);
        ok = __all_sync(0xffffffffu, ready);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[2][XC];
        tm_load(t_s(0, u) + lane_off + (uint32_t)(hc * XC), v[0]);
        tm_load(t_s(1, u) + lane_off + (uint32_t)(hc * XC), v[1]);
        tm_loaded(v[0]);
        tm_loaded(v[1]);
        if (!TWO) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_free);                      // the tensor core may overwrite the scores
        }
        // masks only where the tile meets the diagonal or the end of the keys (uniform): MODE 0 hides columns below `lo`, MODE 1 from `lo` on
        int lo;
        bool masked;
        if (MODE == 0) {
          masked = it.f0 + 128 > it.len || (a.causal && it.f0 + 127 > x0);
          lo = frow >= it.len ? kDbX : a.causal ? frow - x0 : 0;
        } else {
          masked = x0 + kDbX > min(it.len, a.causal ? it.f0 + 1 : a.S);
          lo = min(it.len, a.causal ? frow + 1 : a.S) - x0;
        }
        lo -= hc * XC;
        if (masked) {
#pragma unroll
          for (int i = 0; i < XC; ++i)
            if (MODE == 0 ? i < lo : i >= lo) v[0][i] = v[1][i] = 0xff800000u;
        }
#pragma unroll
        for (int i = 0; i < XC / 2; ++i) {
          uint64_t l1, l2;
          if (MODE == 0) {
            const float4 c = *reinterpret_cast<const float4*>(cv + i * 8);
            l1 = f2_pack(c.x, c.y);
            l2 = f2_pack(c.z, c.w);
          } else {
            l1 = f2_pack(nl[0], nl[0]);
            l2 = f2_pack(nl[1], nl[1]);
          }
          float p, s;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(v[0][2 * i]), __uint_as_float(v[0][2 * i + 1])), sc2, l1), p, s);
          v[0][2 * i] = __float_as_uint(ex2_approx(p));
          v[0][2 * i + 1] = __float_as_uint(ex2_approx(s));
          f2_unpack(f2_fma(f2_pack(__uint_as_float(v[1][2 * i]), __uint_as_float(v[1][2 * i + 1])), sc2, l2), p, s);
          v[1][2 * i] = __float_as_uint(ex2_approx(p));
          v[1][2 * i + 1] = __float_as_uint(ex2_approx(s));
        }
        if (!TWO) {
          ready = mbar_wait(dp_full, par);
          if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 9);
          ok = __all_sync(0xffffffffu, ready);
          if (!ok) break;
          tc_fence_after();
        }
        uint32_t d[XC], w1[XC / 2], w2[XC / 2], wv[XC / 2];
        tm_load(t_dp(u) + lane_off + (uint32_t)(hc * XC), d);
        tm_loaded(d);
        if (masked) {
#pragma unroll
          for (int i = 0; i < XC; ++i)
            if (MODE == 0 ? i < lo : i >= lo) d[i] = 0u;           // (what a hidden key's value holds does not matter)
        }
#pragma unroll
        for (int i = 0; i < XC / 2; ++i) {
          uint64_t d1, d2;
          if (MODE == 0) {
            const float4 c = *reinterpret_cast<const float4*>(cv + i * 8 + 4);
            d1 = f2_pack(c.x, c.y);
            d2 = f2_pack(c.z, c.w);
          } else {
            d1 = f2_pack(nd[0], nd[0]);
            d2 = f2_pack(nd[1], nd[1]);
          }
          const uint64_t dp = f2_pack(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1]));
          const uint64_t p1 = f2_pack(__uint_as_float(v[0][2 * i]), __uint_as_float(v[0][2 * i + 1]));
          const uint64_t p2 = f2_mul(f2_pack(__uint_as_float(v[1][2 * i]), __uint_as_float(v[1][2 * i + 1])), nlam2);
          float e0, e1;
          f2_unpack(f2_mul(p1, f2_add(dp, d1)), e0, e1);
          w1[i] = bf16_pair(e0, e1);
          f2_unpack(f2_mul(p2, f2_add(dp, d2)), e0, e1);
          w2[i] = bf16_pair(e0, e1);
          if (MODE == 0) {
            f2_unpack(f2_add(p1, p2), e0, e1);
            wv[i] = bf16_pair(e0, e1);
          }
        }
        // (one step in flight: dP of this step is behind the accumulating products of the last one, so what they read may be overwritten)
        if (MODE == 0) tm_store(t_p(0, hc * XC, u) + lane_off, wv);
        tm_store(t_p(1, hc * XC, u) + lane_off, w1);
        tm_store(t_p(2, hc * XC, u) + lane_off, w2);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(u));
        x = nx;
        h = nh;
        lam = lam_next;
      }
      if (!ok) break;
      // ---------------- accumulators -> global: this warp's 32 rows x its share of the columns (half of them, in MODE 1 a quarter), of dk (or dq) and of dv, through its piece
      const bool ready = mbar_wait(acc_full, (uint32_t)(n & 1));
      if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 9);
      ok = __all_sync(0xffffffffu, ready);
      if (!ok) break;
      tc_fence_after();
      constexpr int CW = DH / NP, CL = CW < 32 ? CW : 32;          // columns of this warp, and of one load
      uint32_t o1[CW / CL][CL], o0[MODE == 0 ? CW / CL : 1][CL];
#pragma unroll
      for (int c = 0; c < CW / CL; ++c) {
        tm_load(tAcc + lane_off + (uint32_t)(hc * CW + c * CL), o1[c]);
        if constexpr (MODE == 0) tm_load(tDv + lane_off + (uint32_t)(hc * CW + c * CL), o0[c]);
      }
#pragma unroll
      for (int c = 0; c < CW / CL; ++c) {
        tm_loaded(o1[c]);
        if constexpr (MODE == 0) tm_loaded(o0[c]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_free);
      const int row = it.f0 + q * 32;
      auto store = [&](const uint32_t (&o)[CW / CL][CL], float mul, int column) {
        if (lane == 0) bulk_wait_read();                           // what left through the piece before
        __syncwarp();
#pragma unroll
        for (int sg = 0; sg < CW / 8; ++sg) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = 8 * sg + 2 * i;
            w[i] = bf16_pair(__uint_as_float(o[e / CL][e % CL]) * mul, __uint_as_float(o[e / CL][e % CL + 1]) * mul);
          }
          // rows of 128, 64 or 32 bytes, swizzled over as many
          const int sw = CW == 64 ? lane & 7 : CW == 32 ? (lane >> 1) & 3 : (lane >> 2) & 1;
          const int at = lane * (CW * 2) + ((sg ^ sw) << 4);
          *reinterpret_cast<uint4*>(piece + at) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row < a.S) tma_store_3d(&map_out, sPiece, column + hc * CW, row, it.b);
          bulk_commit();
        }
      };
      store(o1, a.scale, (MODE == 0 ? a.H + it.hk : it.hk) * DH);
      if constexpr (MODE == 0) store(o0, 1.0f, (a.H + a.K + it.hk) * DH);
    }
    if (lane == 0) bulk_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "r"(512) : "memory");
  }
}
