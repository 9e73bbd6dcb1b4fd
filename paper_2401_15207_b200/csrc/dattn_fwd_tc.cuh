// Differential attention forward on tcgen05 (bf16, heads of 64 and 128): scores, probabilities and output accumulators in tensor memory.
// Included into gemm_tc.cu after attention_tc.cuh (shares its PTX wrappers, descriptors and bounded waits).
//
// Work item = one (batch, head) and 128 query rows; key blocks of 64.  Both maps read the same K and V tiles: the first map's half of a head's
// columns is the first half of the tile's row, the second map's the second.
//   warp 0     : TMA producer (Q per item, K and V blocks through 3-deep rings); the map has a batch dimension, so that rows beyond a
//                sequence are zeros and never the next entry's
//   warp 1     : issues everything (one elected thread), in the order  P_m V of block j, S_m of block j + 2  for m = 1, 2; owns the tensor
//                memory.  (An issuer for each map: 138 -> 153 us)
//   warp 2     : with key lengths, V's rows of hidden keys -> zeros
//   warps 4-11 : softmax, four warps to a map, one thread to a query row: S_m -> registers, mask, maximum, exponentials, P_m as bf16 over
//                S_m's columns in tensor memory (the A operand of P_m V: no shared-memory traffic for it).  The rounding of P to bf16 is the
//                operand type's; the row's sum takes the values before it
//   warps 12-15: epilogue: o = O_1 / l_1 - lambda O_2 / l_2, the head's norm; o, o_2, y leave by TMA.  The accumulators are free before the first store,
//                for the next item's products wait for them
// Each map has two buffers of scores, so that its warps find the next block's ready while the tensor core works on this one's P V and the one
// after next: with one buffer of 128 keys a map waited for its products and their latency in every block (2 x 2048 x 32 heads of 128, causal: 151 -> 134 us).
// What bounds it, both maps' 64 keys: products 890 cycles (at full rate), exponentials 1024 of the special function unit; measured 1450, and 1070 with
// the softmax left out; and about 3500 at the end of an item of heads of 128, whose accumulators the next item's products wait for.  142 us for that
// case in a run of calls (726 TFLOP/s), 124 in a short one.  Heads of 128 spill 44 bytes a thread at 128 registers, heads of 64 8 bytes.
// Tensor-memory columns: buffer u of S_m at 128 m + 64 u, O_m behind 256: one set of 2 x 128 (heads of 128), two sets of 2 x 64 by item parity
// (heads of 64).
#pragma once

constexpr int kDfThreads = 512, kDfKeys = 64, kDfStages = 3;
template <int DH> struct DattnFwdCfg {
  static constexpr int kSpans = DH / 64;
  static constexpr int kTileBytes = 128 * DH * 2;                  // Q
  static constexpr int kBlockBytes = kDfKeys * DH * 2;             // a block of K or V
  static constexpr int kNO = DH == 64 ? 2 : 1;                     // sets of output accumulators
  static constexpr int kStage = 4 * 2 * kSpans * 4096;             // pieces of 32 x 64 bf16 per epilogue warp: o (then o_2) and y
  // tiles, staging, barriers, row sums [kNO][2][128], gain
  static constexpr int kSmem = 2 * kTileBytes + 2 * kDfStages * kBlockBytes + kStage + 320 + kNO * 1024 + DH * 4 + 1024;
};
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// a [rows][64] bf16 piece, 128-byte swizzled, to global memory; rows beyond the tensor's are dropped
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"((uint64_t)map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }      // sources may be written again
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// A from tensor memory (lane = row, two bf16 to a column), B from shared memory
__device__ __forceinline__ void tc_mma_ta(uint32_t tmem_c, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_c), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accum) : "memory");
}
// One thread of a converged warp.  Products issued inside a branch on it take their operands from uniform registers and leave one behind the
// other at the tensor core's rate: 63 cycles for 128 x 128 x 16, against 120 to 170 in a branch on the lane's number or with a predicate per lane.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void tmem_ld8_nowait(uint32_t addr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_ld_wait8(uint32_t (&v)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]) :: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
                 "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
               : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Zeros in rows `from` .. ROWS - 1 of a tile of SP spans of ROWS rows x 128 bytes (a whole warp), before the tensor core reads them.
template <int SP, int ROWS> __device__ __forceinline__ void zero_rows(uint8_t* tile, int from, int lane) {
  if (from >= ROWS) return;
  for (int r = max(from, 0) + (lane >> 3); r < ROWS; r += 4) {
#pragma unroll
    for (int sp = 0; sp < SP; ++sp) *reinterpret_cast<uint4*>(tile + sp * (ROWS * 128) + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_async_smem();
  __syncwarp();
}
// Items: (batch, head, 128 query rows), the longest first, dealt forwards on even rounds and backwards on odd ones (as in attention_tc.cuh).
struct DattnItem { int b, h, q0, nblk, len; };
__device__ __forceinline__ DattnItem dattn_item(int idx, int nqb, int nbh, int H, int S, int causal, const int* __restrict__ lens) {
  DattnItem it;
  const int rank = idx / nbh, bh = idx - rank * nbh;
  it.b = bh / H;
  it.h = bh - it.b * H;
  it.q0 = (causal ? nqb - 1 - rank : rank) * 128;
  it.len = lens ? max(0, min(lens[it.b], S)) : S;
  const int end = min(causal ? min(S, it.q0 + 128) : S, it.len);
  it.nblk = max(1, (end + kDfKeys - 1) / kDfKeys);                             // no key at all: one block, all of it masked
  return it;
}
__device__ __forceinline__ int dattn_item_at(int n) {
  const int first = n * (int)gridDim.x;
  return (n & 1) ? first + (int)gridDim.x - 1 - (int)blockIdx.x : first + (int)blockIdx.x;
}

template <int DH>
__global__ void __launch_bounds__(kDfThreads, 1)
dattn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_kv, const __grid_constant__ CUtensorMap tmap_o,
                    const __grid_constant__ CUtensorMap tmap_o2, const __grid_constant__ CUtensorMap tmap_y, const DattnArgs a) {
  typedef DattnFwdCfg<DH> Cfg;
  constexpr int SP = Cfg::kSpans, NO = Cfg::kNO, HD = DH / 2, SPAN = 128 * 128, TB = Cfg::kTileBytes, BB = Cfg::kBlockBytes, KSPAN = kDfKeys * 128, NS = kDfStages;
  extern __shared__ uint8_t smem_raw[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (the role as a uniform value)
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base, sK = sQ + 2 * TB, sV = sK + NS * BB, sStage = sV + NS * BB, bar = sStage + Cfg::kStage;
  auto k_full = [&](int i) { return bar + 8u * i; };
  auto k_empty = [&](int i) { return bar + 32u + 8u * i; };
  auto v_full = [&](int i) { return bar + 64u + 8u * i; };
  auto v_empty = [&](int i) { return bar + 96u + 8u * i; };
  auto v_ok = [&](int i) { return bar + 24u + 32u * i; };          // (each fourth word of the rows above: three stages)
  auto q_full = [&](int i) { return bar + 128u + 8u * i; };
  auto q_empty = [&](int i) { return bar + 144u + 8u * i; };
  auto s_full = [&](int m, int u) { return bar + 160u + 16u * m + 8u * u; };
  auto p_ready = [&](int m, int u) { return bar + 192u + 16u * m + 8u * u; };
  auto pv_done = [&](int m) { return bar + 224u + 8u * m; };
  auto o_full = [&](int i) { return bar + 240u + 8u * i; };
  auto o_free = [&](int i) { return bar + 256u + 8u * i; };
  auto l_full = [&](int i) { return bar + 272u + 8u * i; };
  const uint32_t tmem_slot = bar + 288u;
  volatile uint32_t* slot_gen = reinterpret_cast<volatile uint32_t*>(gen + (tmem_slot - base));
  volatile uint32_t* poison_gen = slot_gen + 2;
  float* sums = reinterpret_cast<float*>(gen + (bar + 320u - base));                // [NO][2 maps][128 rows]
  float* sgain = sums + NO * 256;

  const int nqb = (a.S + 127) / 128, nbh = a.B * a.H, nitems = nqb * nbh;
  auto item_of = [&](int idx) { return dattn_item(idx, nqb, nbh, a.H, a.S, a.causal, a.lens); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); mbar_init(v_full(i), 1); mbar_init(v_empty(i), 1); mbar_init(v_ok(i), 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1); mbar_init(q_empty(i), 1); mbar_init(pv_done(i), 1);
      for (int u = 0; u < 2; ++u) { mbar_init(s_full(i, u), 1); mbar_init(p_ready(i, u), 4); }
      mbar_init(o_full(i), 1); mbar_init(o_free(i), 4); mbar_init(l_full(i), 8);
    }
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
  auto t_s = [&](int m, int u) { return tm + (uint32_t)(m * 128 + u * 64); };
  auto t_o = [&](int n, int m) { return tm + 256u + (uint32_t)((NO == 2 ? (n & 1) * 128 : 0) + m * DH); };

  if (warp < 4) {
    if (warp == 0 && !poisoned && elect_one()) {
      // ---------------- TMA producer
      int g = 0, n = 0;
      bool ok = true;
      for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
        const DattnItem it = item_of(idx);
        const int kh = it.h / (a.H / a.K), colQ = it.h * DH, colK = (a.H + kh) * DH, colV = (a.H + a.K + kh) * DH, qi = n & 1;
        if (!mbar_wait(q_empty(qi), (uint32_t)(((n >> 1) & 1) ^ 1))) { atomicCAS(&g_tc_error, 0, 4); break; }
        mbar_expect_tx(q_full(qi), TB);
#pragma unroll
        for (int sp = 0; sp < SP; ++sp) tma_load_3d(sQ + qi * TB + sp * SPAN, &tmap_q, q_full(qi), colQ + sp * 64, it.q0, it.b);
        for (int j = 0; j < it.nblk; ++j, ++g) {
          const int st = g % NS;
          const uint32_t ph = (uint32_t)((g / NS) & 1) ^ 1u;
          if (!mbar_wait(k_empty(st), ph)) { atomicCAS(&g_tc_error, 0, 4); ok = false; break; }
          mbar_expect_tx(k_full(st), BB);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) tma_load_3d(sK + st * BB + sp * KSPAN, &tmap_kv, k_full(st), colK + sp * 64, j * kDfKeys, it.b);
          if (!mbar_wait(v_empty(st), ph)) { atomicCAS(&g_tc_error, 0, 4); ok = false; break; }
          mbar_expect_tx(v_full(st), BB);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) tma_load_3d(sV + st * BB + sp * KSPAN, &tmap_kv, v_full(st), colV + sp * 64, j * kDfKeys, it.b);
        }
      }
    } else if (warp == 2 && !poisoned && a.lens) {
      // ---------------- values of hidden keys: rows of a block of V behind the entry's length become zeros (P is 0 there, but 0 times NaN is not)
      int st = 0, n = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
        const DattnItem it = item_of(idx);
        for (int j = 0; j < it.nblk; ++j) {
          const bool ready = mbar_wait(v_full(st), ph);
          if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 4);
          ok = __all_sync(0xffffffffu, ready);
          if (!ok) break;
          zero_rows<SP, kDfKeys>(gen + (sV + st * BB - base), it.len - j * kDfKeys, lane);
          if (lane == 0) mbar_arrive(v_ok(st));
          if (++st == NS) { st = 0; ph ^= 1; }
        }
      }
    } else if (warp == 1 && !poisoned) {
      if (elect_one()) {
        // ---------------- MMA issuer
        const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | (((uint32_t)kDfKeys >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((128u >> 4) << 24);
        // the block whose scores are issued next, number sg over all items: two ahead of the block whose P V is
        int sn = 0, sj = 0, sg = 0, sst = 0, sblk = 0;
        uint32_t sph = 0;
        bool live = dattn_item_at(0) < nitems, ok = true;
        if (live) sblk = item_of(dattn_item_at(0)).nblk;
        const uint64_t dQ0 = desc_kmajor(sQ), dK0 = desc_kmajor(sK), dV0 = desc_nmajor(sV, KSPAN);
        auto issue_s = [&](auto map) -> bool {                     // S_m = Q_m K_m^T: the map's half of the tiles' rows
          constexpr int m = decltype(map)::value;
          const int qi = sn & 1, u = sg & 1;
          if (m == 0) {
            if (!mbar_wait(k_full(sst), sph) || (sj == 0 && !mbar_wait(q_full(qi), (uint32_t)((sn >> 1) & 1)))) return false;
            tc_fence_after();
          }
          const uint64_t dQ = dQ0 + (uint64_t)(qi * (TB >> 4)), dK = dK0 + (uint64_t)(sst * (BB >> 4));
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const int e = m * (HD / 16) + kk;
            tc_mma(t_s(m, u), dQ + (uint64_t)(((e / 4) * SPAN + (e % 4) * 32) >> 4), dK + (uint64_t)(((e / 4) * KSPAN + (e % 4) * 32) >> 4), idesc_s, kk > 0 ? 1u : 0u);
          }
          tc_commit(s_full(m, u));
          if (m == 1) {
            tc_commit(k_empty(sst));
            ++sg;
            if (++sst == NS) { sst = 0; sph ^= 1; }
            if (++sj == sblk) {
              tc_commit(q_empty(qi));
              sj = 0;
              const int idx = dattn_item_at(++sn);
              live = idx < nitems;
              if (live) sblk = item_of(idx).nblk;
            }
          }
          return true;
        };
        int g = 0, n = 0, nblk = sblk, j = 0, st = 0;
        uint32_t ph = 0;
        auto half = [&](auto map) -> bool {                        // P_m V of block g, S_m of block g + 2
          constexpr int m = decltype(map)::value;
          const int u = g & 1;
          if (m == 0) {
            if (!mbar_wait(a.lens ? v_ok(st) : v_full(st), ph)) return false;
            // an item's first products overwrite an accumulator that its previous item's epilogue has read
            if (j == 0 && !mbar_wait(o_free(n % NO), (uint32_t)(((n / NO) & 1) ^ 1))) return false;
          }
          if (!mbar_wait(p_ready(m, u), (uint32_t)((g >> 1) & 1))) return false;
          tc_fence_after();
          const uint64_t dV = dV0 + (uint64_t)(st * (BB >> 4));
#pragma unroll
          for (int kk = 0; kk < kDfKeys / 16; ++kk)
            tc_mma_ta(t_o(n, m), t_s(m, u) + (uint32_t)(kk * 8), dV + (uint64_t)((kk * 16 * 128) >> 4), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
          tc_commit(pv_done(m));
          if (m == 1) {
            tc_commit(v_empty(st));
            if (j + 1 == nblk) tc_commit(o_full(n % NO));
          }
          // in the one issue order S_m of the block after next comes behind the products that read P_m out of its buffer
          return !live || issue_s(map);
        };
        typedef std::integral_constant<int, 0> M0;
        typedef std::integral_constant<int, 1> M1;
        for (int i = 0; i < 2 && live && ok; ++i) ok = issue_s(M0()) && issue_s(M1());
        for (int idx = dattn_item_at(n); idx < nitems && ok;) {
          ok = half(M0()) && half(M1());
          ++g;
          if (++st == NS) { st = 0; ph ^= 1; }
          if (++j == nblk) {
            j = 0;
            idx = dattn_item_at(++n);
            if (idx < nitems) nblk = item_of(idx).nblk;
          }
        }
        if (!ok) atomicCAS(&g_tc_error, 0, 5);
      }
      __syncwarp();
    }
  } else if (warp < 12) {
    // ---------------- softmax: one thread per query row
    const int m = (warp - 4) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f;
    bool ok = !poisoned;
    int g = 0, n = 0;
    for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
      const DattnItem it = item_of(idx);
      const int qrow = it.q0 + r;
      const int vis = min(it.len, a.causal ? qrow + 1 : a.S);      // keys this row may see
      const int all = min(it.len, a.causal ? it.q0 + 1 : a.S);     // keys that every row of the tile sees
      const uint32_t tO = t_o(n, m) + lane_off;
      float mx = -INFINITY, l = 0.f;                               // reference maximum (log2 units), sum
      for (int j = 0; j < it.nblk; ++j, ++g) {
        const uint32_t tS = t_s(m, g & 1) + lane_off;
        bool ready = mbar_wait(s_full(m, g & 1), (uint32_t)((g >> 1) & 1));
        if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 6);
        ok = __all_sync(0xffffffffu, ready);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[2][32];
        tmem_ld32_nowait(tS, v[0]);
        tmem_ld32_nowait(tS + 32u, v[1]);
        tmem_ld_wait32(v[0]);
        tmem_ld_wait32(v[1]);
        if ((j + 1) * kDfKeys > all) {                             // (uniform) some row of the tile sees less than the block
          const int lim = vis - j * kDfKeys;
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c * 32 + i >= lim) v[c][i] = 0xff800000u;        // -inf
        }
        float t4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) t4[e] = fmaxf(__uint_as_float(v[0][e]), __uint_as_float(v[1][e]));
#pragma unroll
        for (int i = 4; i < 32; i += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) t4[e] = fmaxf(t4[e], fmaxf(__uint_as_float(v[0][i + e]), __uint_as_float(v[1][i + e])));
        const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * sl2;
        // Lazy reference maximum: it moves, and O is rescaled, only when some row of the warp has grown by more than 2^8 over it
        const bool grow = __any_sync(0xffffffffu, top > mx + 8.0f);
        if (grow) {
          const float mnew = fmaxf(mx, top), corr = mnew == -INFINITY ? 1.0f : ex2_approx(mx - mnew);
          mx = mnew;
          l *= corr;
          if (j > 0) {
            // O_m is at rest once the last block's products are done (those of the block before are: this block's scores were issued behind them)
            ready = mbar_wait(pv_done(m), (uint32_t)((g - 1) & 1));
            if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 6);
            ok = __all_sync(0xffffffffu, ready);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = 0; c0 < DH; c0 += 16) {                  // (16 at a time: the scores stay in registers)
              uint32_t w[16];
              tmem_ld16_nowait(tO + (uint32_t)c0, w);
              tmem_ld_wait16(w);
#pragma unroll
              for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * corr);
              tmem_st16(tO + (uint32_t)c0, w);
            }
          }
        }
        const float neg = mx == -INFINITY ? 0.f : -mx;
        const uint64_t sc2 = f2_pack(sl2, sl2), ng2 = f2_pack(neg, neg);
        uint64_t acc[2] = {f2_pack(l, 0.f), f2_pack(0.f, 0.f)};
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float x, y;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(v[i / 16][2 * (i % 16)]), __uint_as_float(v[i / 16][2 * (i % 16) + 1])), sc2, ng2), x, y);
          x = ex2_approx(x);
          y = ex2_approx(y);
          acc[i & 1] = f2_add(acc[i & 1], f2_pack(x, y));
          w[i] = bf16_pair(x, y);
        }
        tmem_st32(tS, w);
        float s0, s1, s2, s3;
        f2_unpack(acc[0], s0, s1);
        f2_unpack(acc[1], s2, s3);
        l = (s0 + s1) + (s2 + s3);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(m, g & 1));
      }
      if (!ok) break;
      // the row's sum to the epilogue, once the buffer's last item has been read
      const bool ready = mbar_wait(o_free(n % NO), (uint32_t)(((n / NO) & 1) ^ 1));
      if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 6);
      ok = __all_sync(0xffffffffu, ready);
      if (!ok) break;
      sums[(n % NO) * 256 + m * 128 + r] = l;
      if (qrow < a.S) a.lse[(((int64_t)m * a.B + it.b) * a.H + it.h) * a.S + qrow] = (mx + log2f(l)) * 0.6931471805599453f;
      __syncwarp();
      if (lane == 0) mbar_arrive(l_full(n % NO));
    }
  } else {
    // ---------------- epilogue
    const int q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16;
    const uint32_t sPiece = sStage + q * (2 * SP * 4096);
    uint8_t* stage = gen + (sPiece - base);
    for (int i = threadIdx.x - 384; i < DH; i += 128) sgain[i] = a.gain ? __bfloat162float(((const __nv_bfloat16*)a.gain)[i]) * a.c : 0.f;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    bool ok = !poisoned;
    int n = 0;
    for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
      const DattnItem it = item_of(idx);
      const float lam = a.lam[it.h];
      const int ob = n % NO;
      const uint32_t ph = (uint32_t)((n / NO) & 1);
      const bool ready = mbar_wait(l_full(ob), ph) && mbar_wait(o_full(ob), ph);
      if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 6);
      ok = __all_sync(0xffffffffu, ready);
      if (!ok) break;
      tc_fence_after();
      const float l1 = sums[ob * 256 + r], l2 = sums[ob * 256 + 128 + r];
      const float r1 = l1 == 0.f ? 0.f : 1.0f / l1, r2 = l2 == 0.f ? 0.f : 1.0f / l2;        // a row that sees no key: zeros
      const uint64_t r1p = f2_pack(r1, r1), r2p = f2_pack(r2, r2), lamp = f2_pack(-lam, -lam);
      const uint32_t t1 = t_o(n, 0) + lane_off, t2 = t_o(n, 1) + lane_off;
      uint64_t rnp = 0;
      if (a.y) {
        uint64_t ss[2] = {0, 0};
        uint32_t u[2][16], w[2][16];
        tmem_ld16_nowait(t1, u[0]);
        tmem_ld16_nowait(t2, w[0]);
#pragma unroll
        for (int c = 0; c < DH / 16; ++c) {
          const int k = c & 1;
          tmem_ld_wait16(u[k]);
          tmem_ld_wait16(w[k]);
          if (c + 1 < DH / 16) {                                   // the next 16 columns arrive during this arithmetic
            tmem_ld16_nowait(t1 + (uint32_t)(16 * c + 16), u[k ^ 1]);
            tmem_ld16_nowait(t2 + (uint32_t)(16 * c + 16), w[k ^ 1]);
          }
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const uint64_t o2 = f2_mul(f2_pack(__uint_as_float(w[k][i]), __uint_as_float(w[k][i + 1])), r2p);
            const uint64_t o = f2_fma(f2_pack(__uint_as_float(u[k][i]), __uint_as_float(u[k][i + 1])), r1p, f2_mul(o2, lamp));
            ss[(i >> 1) & 1] = f2_fma(o, o, ss[(i >> 1) & 1]);
          }
        }
        float s0, s1;
        f2_unpack(f2_add(ss[0], ss[1]), s0, s1);
        const float rn = rsqrtf((s0 + s1) * (1.0f / DH) + a.eps);
        rnp = f2_pack(rn, rn);
      }
      if (lane == 0) bulk_wait_read();                             // the last item's stores have read the pieces
      __syncwarp();
      uint8_t* mine = stage + lane * 128;                          // pieces of 64 columns, 4 KB each: o, y
      uint32_t k2[SP][32];                                         // o_2 until o has left
      {
        uint32_t u[2][8], w[2][8];
        tmem_ld8_nowait(t1, u[0]);
        tmem_ld8_nowait(t2, w[0]);
#pragma unroll
        for (int c = 0; c < DH / 8; ++c) {
          const int k = c & 1;
          tmem_ld_wait8(u[k]);
          tmem_ld_wait8(w[k]);
          if (c + 1 < DH / 8) {
            tmem_ld8_nowait(t1 + (uint32_t)(8 * c + 8), u[k ^ 1]);
            tmem_ld8_nowait(t2 + (uint32_t)(8 * c + 8), w[k ^ 1]);
          }
          uint32_t po[4], py[4];
          const float4* gp = reinterpret_cast<const float4*>(sgain + 8 * c);
          const float4 g0 = gp[0], g1 = gp[1];
          const uint64_t gg[4] = {f2_pack(g0.x, g0.y), f2_pack(g0.z, g0.w), f2_pack(g1.x, g1.y), f2_pack(g1.z, g1.w)};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint64_t o2 = f2_mul(f2_pack(__uint_as_float(w[k][2 * i]), __uint_as_float(w[k][2 * i + 1])), r2p);
            const uint64_t o = f2_fma(f2_pack(__uint_as_float(u[k][2 * i]), __uint_as_float(u[k][2 * i + 1])), r1p, f2_mul(o2, lamp));
            const uint64_t y = f2_mul(f2_mul(o, rnp), gg[i]);
            float x0, x1;
            f2_unpack(o2, x0, x1);
            k2[c / 8][4 * (c % 8) + i] = bf16_pair(x0, x1);
            f2_unpack(o, x0, x1);
            po[i] = bf16_pair(x0, x1);
            f2_unpack(y, x0, x1);
            py[i] = bf16_pair(x0, x1);
          }
          const int at = ((c % 8) ^ (lane & 7)) << 4;
          *reinterpret_cast<uint4*>(mine + (c / 8) * 4096 + at) = make_uint4(po[0], po[1], po[2], po[3]);
          if (a.y) *reinterpret_cast<uint4*>(mine + (SP + c / 8) * 4096 + at) = make_uint4(py[0], py[1], py[2], py[3]);
        }
      }
      // everything read: the accumulators and sums may be reused, before anything is stored
      tc_fence_before();
      fence_async_smem();                                          // the pieces are read by the TMA (async proxy)
      __syncwarp();
      const int row = it.q0 + q * 32, col = it.h * DH;
      if (lane == 0) {
        mbar_arrive(o_free(ob));
        if (row < a.S) {
#pragma unroll
          for (int c = 0; c < SP; ++c) {
            tma_store_3d(&tmap_o, sPiece + c * 4096, col + 64 * c, row, it.b);
            if (a.y) tma_store_3d(&tmap_y, sPiece + (SP + c) * 4096, col + 64 * c, row, it.b);
          }
        }
        bulk_commit();
        if (a.o2) bulk_wait_read();
      }
      __syncwarp();
      if (a.o2) {
#pragma unroll
        for (int c = 0; c < SP; ++c)
#pragma unroll
          for (int sg = 0; sg < 8; ++sg)
            *reinterpret_cast<uint4*>(mine + c * 4096 + ((sg ^ (lane & 7)) << 4)) = make_uint4(k2[c][4 * sg], k2[c][4 * sg + 1], k2[c][4 * sg + 2], k2[c][4 * sg + 3]);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row < a.S) {
#pragma unroll
            for (int c = 0; c < SP; ++c) tma_store_3d(&tmap_o2, sPiece + c * 4096, col + 64 * c, row, it.b);
          }
          bulk_commit();
        }
      }
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
