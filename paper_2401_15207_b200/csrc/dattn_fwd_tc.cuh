// Differential attention forward on tcgen05 (bf16, heads of 64 and 128): scores, probabilities and output accumulators in tensor memory.
// Included into gemm_tc.cu after attention_tc.cuh (shares its PTX wrappers, descriptors and bounded waits).
//
// Work item = one (batch, head) and 128 query rows; key blocks of 128.  The two maps are the two streams that keep the tensor core fed: while
// one map's warps take exponentials, the tensor core works on the other map.  Both read the same K and V tiles: the first map's half of a
// head's columns is the first half of the tile's row, the second map's the second.
//   warp 0     : TMA producer (Q per item, K and V blocks through 2-deep rings); the map has a batch dimension, so that rows beyond a
//                sequence are zeros and never the next entry's
//   warp 1     : issues everything (one thread), in the order  P_m V of block j, S_m of block j + 1  for m = 1, 2; owns the tensor memory
//   warps 4-11 : softmax, four warps to a map, one thread to a query row: S_m -> registers, mask, maximum, exponentials, P_m as bf16 over
//                S_m's columns in tensor memory (the A operand of P_m V: no shared-memory traffic for it).  The rounding of P to bf16 is the
//                operand type's; the row's sum takes the values before it.  O_m is rescaled by the same thread when the reference maximum
//                grows by more than 2^8: S_m of block j is behind P_m V of block j - 1 in the one issue order, so O_m is at rest then
//   warps 12-15: epilogue: o = O_1 / l_1 - lambda O_2 / l_2, the head's norm, whole-line stores of o, o_2, y
// Tensor-memory columns: S_m at 128 m, O_m behind 256: one set of 2 x 128 (heads of 128), two sets of 2 x 64 by item parity (heads of 64).
#pragma once

constexpr int kDfThreads = 512;
template <int DH> struct DattnFwdCfg {
  static constexpr int kSpans = DH / 64;
  static constexpr int kTileBytes = 128 * DH * 2;
  static constexpr int kNO = DH == 64 ? 2 : 1;                     // sets of output accumulators
  static constexpr int kStage = 4 * 4096;                          // one 32 x 64 bf16 piece per epilogue warp
  // tiles, staging, barriers, row sums [kNO][2][128], gain
  static constexpr int kSmem = 6 * kTileBytes + kStage + 256 + kNO * 1024 + DH * 4 + 1024;
};
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// A from tensor memory (lane = row, two bf16 to a column), B from shared memory
__device__ __forceinline__ void tc_mma_ta(uint32_t tmem_c, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_c), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accum) : "memory");
}
template <int N> __device__ __forceinline__ void reg_alloc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void reg_dealloc() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
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
  it.nblk = max(1, (end + 127) / 128);                             // no key at all: one block, all of it masked
  return it;
}
__device__ __forceinline__ int dattn_item_at(int n) {
  const int first = n * (int)gridDim.x;
  return (n & 1) ? first + (int)gridDim.x - 1 - (int)blockIdx.x : first + (int)blockIdx.x;
}

template <int DH>
__global__ void __launch_bounds__(kDfThreads, 1)
dattn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmap, const DattnArgs a) {
  typedef DattnFwdCfg<DH> Cfg;
  constexpr int SP = Cfg::kSpans, NO = Cfg::kNO, HD = DH / 2, SPAN = 128 * 128, TB = Cfg::kTileBytes;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base, sK = sQ + 2 * TB, sV = sK + 2 * TB, sStage = sV + 2 * TB, bar = sStage + Cfg::kStage;
  auto q_full = [&](int i) { return bar + 8u * i; };
  auto q_empty = [&](int i) { return bar + 16u + 8u * i; };
  auto k_full = [&](int i) { return bar + 32u + 8u * i; };
  auto k_empty = [&](int i) { return bar + 48u + 8u * i; };
  auto v_full = [&](int i) { return bar + 64u + 8u * i; };
  auto v_empty = [&](int i) { return bar + 80u + 8u * i; };
  auto s_full = [&](int m) { return bar + 96u + 8u * m; };
  auto p_ready = [&](int m) { return bar + 112u + 8u * m; };
  auto o_full = [&](int i) { return bar + 128u + 8u * i; };
  auto o_free = [&](int i) { return bar + 144u + 8u * i; };
  auto l_full = [&](int i) { return bar + 160u + 8u * i; };
  const uint32_t tmem_slot = bar + 176u;
  volatile uint32_t* slot_gen = reinterpret_cast<volatile uint32_t*>(gen + (tmem_slot - base));
  volatile uint32_t* poison_gen = slot_gen + 2;
  float* sums = reinterpret_cast<float*>(gen + (bar + 256u - base));                // [NO][2 maps][128 rows]
  float* sgain = sums + NO * 256;

  const int nqb = (a.S + 127) / 128, nbh = a.B * a.H, nitems = nqb * nbh;
  auto item_of = [&](int idx) { return dattn_item(idx, nqb, nbh, a.H, a.S, a.causal, a.lens); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1); mbar_init(q_empty(i), 1);
      mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1);
      mbar_init(v_full(i), 1); mbar_init(v_empty(i), 1);
      mbar_init(s_full(i), 1); mbar_init(p_ready(i), 4);
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
  const uint32_t tm = *slot_gen;
  const bool poisoned = *poison_gen != 0;
  pdl_trigger();
  pdl_wait();
  auto t_o = [&](int n, int m) { return tm + 256u + (uint32_t)((NO == 2 ? (n & 1) * 128 : 0) + m * DH); };

  if (warp < 4) {
    // (48 + 96 + 2 * 184) * 128 threads = the 512 * 128 registers of the launch
    reg_dealloc<48>();
    if (warp == 0 && lane == 0 && !poisoned) {
      // ---------------- TMA producer
      int g = 0, n = 0;
      bool ok = true;
      for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
        const DattnItem it = item_of(idx);
        const int kh = it.h / (a.H / a.K), colQ = it.h * DH, colK = (a.H + kh) * DH, colV = (a.H + a.K + kh) * DH, qi = n & 1;
        if (!mbar_wait(q_empty(qi), (uint32_t)(((n >> 1) & 1) ^ 1))) { atomicCAS(&g_tc_error, 0, 4); break; }
        mbar_expect_tx(q_full(qi), TB);
#pragma unroll
        for (int sp = 0; sp < SP; ++sp) tma_load_3d(sQ + qi * TB + sp * SPAN, &tmap, q_full(qi), colQ + sp * 64, it.q0, it.b);
        for (int j = 0; j < it.nblk; ++j, ++g) {
          const int st = g & 1;
          const uint32_t ph = (uint32_t)((g >> 1) & 1) ^ 1u;
          if (!mbar_wait(k_empty(st), ph)) { atomicCAS(&g_tc_error, 0, 4); ok = false; break; }
          mbar_expect_tx(k_full(st), TB);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) tma_load_3d(sK + st * TB + sp * SPAN, &tmap, k_full(st), colK + sp * 64, j * 128, it.b);
          if (!mbar_wait(v_empty(st), ph)) { atomicCAS(&g_tc_error, 0, 4); ok = false; break; }
          mbar_expect_tx(v_full(st), TB);
#pragma unroll
          for (int sp = 0; sp < SP; ++sp) tma_load_3d(sV + st * TB + sp * SPAN, &tmap, v_full(st), colV + sp * 64, j * 128, it.b);
        }
      }
    } else if (warp == 1 && lane == 0 && !poisoned) {
      // ---------------- MMA issuer
      const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((128u >> 4) << 24);
      auto issue_s = [&](int m, int qi, int st) {                  // S_m = Q_m K_m^T: the map's half of the tiles' rows
        const uint64_t dQ = desc_kmajor(sQ + qi * TB), dK = desc_kmajor(sK + st * TB);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const int e = m * (HD / 16) + kk;
          const uint64_t off = (uint64_t)(((e / 4) * SPAN + (e % 4) * 32) >> 4);
          tc_mma(tm + (uint32_t)(m * 128), dQ + off, dK + off, idesc_s, kk > 0 ? 1u : 0u);
        }
        tc_commit(s_full(m));
      };
      int g = 0, n = 0, idx = dattn_item_at(0);
      bool ok = idx < nitems;
      DattnItem it = ok ? item_of(idx) : DattnItem{};
      if (ok) {
        ok = mbar_wait(q_full(0), 0) && mbar_wait(k_full(0), 0);
        if (!ok) atomicCAS(&g_tc_error, 0, 5);
        else {
          tc_fence_after();
          issue_s(0, 0, 0);
          issue_s(1, 0, 0);
          tc_commit(k_empty(0));
          if (it.nblk == 1) tc_commit(q_empty(0));
        }
      }
      while (ok && idx < nitems) {
        const int next_idx = dattn_item_at(n + 1);
        const bool more = next_idx < nitems;
        DattnItem next = it;
        if (more) next = item_of(next_idx);
        for (int j = 0; j < it.nblk && ok; ++j, ++g) {
          const int st = g & 1, ns = (g + 1) & 1;
          const bool last = j + 1 == it.nblk, follow = !last || more;          // a next block, of this item or the next
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            ok = mbar_wait(p_ready(m), (uint32_t)(g & 1));
            if (ok && m == 0) ok = mbar_wait(v_full(st), (uint32_t)((g >> 1) & 1));
            // an item's first products overwrite an accumulator that its previous item's epilogue has read
            if (ok && m == 0 && j == 0) ok = mbar_wait(o_free(n % NO), (uint32_t)(((n / NO) & 1) ^ 1));
            if (!ok) break;
            tc_fence_after();
            const uint64_t dV = desc_nmajor(sV + st * TB, SPAN);
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              tc_mma_ta(t_o(n, m), tm + (uint32_t)(m * 128 + kk * 8), dV + (uint64_t)((kk * 16 * 128) >> 4), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
            if (m == 1) {
              tc_commit(v_empty(st));
              if (last) tc_commit(o_full(n % NO));
            }
            if (follow) {
              const int nq = last ? (n + 1) & 1 : n & 1;
              if (m == 0) {
                ok = mbar_wait(k_full(ns), (uint32_t)(((g + 1) >> 1) & 1)) && (!last || mbar_wait(q_full(nq), (uint32_t)(((n + 1) >> 1) & 1)));
                if (!ok) break;
                tc_fence_after();
              }
              issue_s(m, nq, ns);
              if (m == 1) {
                tc_commit(k_empty(ns));
                if (last ? next.nblk == 1 : j + 2 == it.nblk) tc_commit(q_empty(nq));
              }
            }
          }
          if (!ok) atomicCAS(&g_tc_error, 0, 5);
        }
        it = next;
        idx = next_idx;
        ++n;
      }
    }
  } else if (warp < 12) {
    // ---------------- softmax: one thread per query row
    reg_alloc<184>();
    const int m = (warp - 4) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16, tS = tm + lane_off + (uint32_t)(m * 128);
    const float sl2 = a.scale * 1.4426950408889634f;
    bool ok = !poisoned;
    int g = 0, n = 0;
    for (int idx = dattn_item_at(n); idx < nitems && ok; idx = dattn_item_at(++n)) {
      const DattnItem it = item_of(idx);
      const int qrow = it.q0 + r;
      const int vis = min(it.len, a.causal ? qrow + 1 : a.S);      // keys this row may see
      const uint32_t tO = t_o(n, m) + lane_off;
      float mx = -INFINITY, l = 0.f;                               // reference maximum (log2 units), sum
      for (int j = 0; j < it.nblk; ++j, ++g) {
        const bool ready = mbar_wait(s_full(m), (uint32_t)(g & 1));
        if (!ready && lane == 0) atomicCAS(&g_tc_error, 0, 6);
        ok = __all_sync(0xffffffffu, ready);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_nowait(tS + 32u * c, v[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_wait32(v[c]);
        if ((j + 1) * 128 > min(it.len, a.causal ? it.q0 + 1 : a.S)) {         // (uniform) some row of the tile sees less than the block
          const int lim = vis - j * 128;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c * 32 + i >= lim) v[c][i] = 0xff800000u;        // -inf
        }
        float t4[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          t4[c] = __uint_as_float(v[c][0]);
#pragma unroll
          for (int i = 1; i < 32; ++i) t4[c] = fmaxf(t4[c], __uint_as_float(v[c][i]));
        }
        const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * sl2;
        // Lazy reference maximum: it moves, and O is rescaled, only when some row of the warp has grown by more than 2^8 over it
        const bool grow = __any_sync(0xffffffffu, top > mx + 8.0f);
        if (grow) {
          const float mnew = fmaxf(mx, top), corr = mnew == -INFINITY ? 1.0f : ex2_approx(mx - mnew);
          mx = mnew;
          l *= corr;
          if (j > 0) {
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
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const int c = 2 * hf + i / 16, e = 2 * (i % 16);
            float x, y;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])), sc2, ng2), x, y);
            x = ex2_approx(x);
            y = ex2_approx(y);
            acc[i & 1] = f2_add(acc[i & 1], f2_pack(x, y));
            w[i] = bf16_pair(x, y);
          }
          tmem_st32(tS + 32u * hf, w);
        }
        float s0, s1, s2, s3;
        f2_unpack(acc[0], s0, s1);
        f2_unpack(acc[1], s2, s3);
        l = (s0 + s1) + (s2 + s3);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(m));
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
    reg_dealloc<96>();
    const int q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16;
    uint8_t* stage = gen + (sStage - base) + q * 4096;
    if (a.gain)
      for (int i = threadIdx.x - 384; i < DH; i += 128) sgain[i] = __bfloat162float(((const __nv_bfloat16*)a.gain)[i]) * a.c;
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
      const bool none = l1 == 0.f;                                 // a row that sees no key: zeros
      const float r1 = 1.0f / l1, r2 = 1.0f / l2, c2 = lam * r2;
      const uint32_t t1 = t_o(n, 0) + lane_off, t2 = t_o(n, 1) + lane_off;
      const int row = it.b * a.S + it.q0 + r, row_end = it.b * a.S + a.S;
      const int64_t ld = (int64_t)a.H * DH;
      float rn = 0.f;
      if (a.y) {
        float ss[2] = {0.f, 0.f};
#pragma unroll 1
        for (int c0 = 0; c0 < DH; c0 += 16) {
          uint32_t u[16], w[16];
          tmem_ld16_nowait(t1 + (uint32_t)c0, u);
          tmem_ld16_nowait(t2 + (uint32_t)c0, w);
          tmem_ld_wait16(u);
          tmem_ld_wait16(w);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float o = fmaf(__uint_as_float(u[i]), r1, -c2 * __uint_as_float(w[i]));
            ss[i & 1] = fmaf(o, o, ss[i & 1]);
          }
        }
        rn = 1.0f / sqrtf((ss[0] + ss[1]) * (1.0f / DH) + a.eps);
      }
#pragma unroll 1
      for (int c0 = 0; c0 < DH; c0 += 64) {
        // o, o_2, y: 64 columns of each through the warp's 4 KB
#pragma unroll 1
        for (int out = 0; out < 3; ++out) {
          __nv_bfloat16* dst = (__nv_bfloat16*)(out == 0 ? a.o : out == 1 ? a.o2 : a.y);
          if (!dst) continue;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t u[32], w[32];
            tmem_ld32_nowait(t1 + (uint32_t)(c0 + 32 * hf), u);
            tmem_ld32_nowait(t2 + (uint32_t)(c0 + 32 * hf), w);
            tmem_ld_wait32(u);
            tmem_ld_wait32(w);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float o = out == 1 ? __uint_as_float(w[i]) * r2 : fmaf(__uint_as_float(u[i]), r1, -c2 * __uint_as_float(w[i]));
              if (out == 2) o *= rn * sgain[c0 + 32 * hf + i];
              u[i] = __float_as_uint(none ? 0.f : o);
            }
            att_stage32(u, 1.0f, stage, lane, 4 * hf);
          }
          const bool done = c0 + 64 == DH && (out == 2 || (!a.y && (out == 1 || !a.o2)));
          if (done) {                                              // everything read: the accumulators and sums may be reused
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free(ob));
          }
          att_flush64(stage, dst, ld, row, lane, row_end, it.h * DH + c0);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "r"(512) : "memory");
  }
}
