// The whole orthogonalisation of a matrix with a short side of 17 to 128 and a long one of at most 4096 in one launch; included by
// gemm_tc.cu.
//
// Through separate products such a matrix is 18 launches of a few microseconds each, whatever its size (64 x 300: 80 us, most of it
// launch latency, and 65 us of host time).  Here the matrix, turned so that the short side are the rows, stays on chip: a cluster of up to 16
// CTAs holds 128 NH columns each, the fp32 iterate in tensor memory (read and written by chunks of 32 columns in rolled loops: in registers
// the unrolled code was so long that the kernel waited for instructions, 67 us at 128 x 128), its fp16 image in shared memory, where the same 128-byte-swizzled tiles serve the Gram matrix as K-major and the step as N-major operand.
// Per step (arithmetic as in ns_epilogue.cuh):
//   A = X X^T: every CTA's part by tcgen05.mma over its own columns; the 32 x 32 units of the lower triangle are summed by one CTA
//   each (fixed order) and handed to all as fp16 E and fp32 diagonal, through distributed shared memory;
//   P(A): every CTA for itself, one 128 x 128 x 128 product;  the new X: its own columns.
constexpr int kSmThreads = 512;                        // 16 warps: lane quarter q = warp mod 4, of every 128 columns the 32-column chunk warp / 4
constexpr int kSmTile = 128 * 128;                     // bytes of a [128][64] fp16 tile
struct NsSmallArgs {
  const void* g; float* mom;                           // the matrix (fp32 or bf16), and the momentum to update or nullptr
  __nv_bfloat16* o; float* master; __nv_bfloat16* param;   // where the result goes: o, or master (and param)
  int rows, cols, steps, nesterov;
  float mu, decay, size;
};
template <int NH> constexpr int ns_small_smem = 1024 + (2 * NH + 4) * kSmTile + 64 * 1024 + 3 * 512 + 16 * 8 + 64;

// shared-memory descriptor, 128-byte swizzle, 8-row groups 1024 bytes apart; `lead`: bytes to the next 64-wide box of an MN-major tile
__device__ __forceinline__ uint64_t ns_desc(uint32_t saddr, uint32_t lead) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint32_t ns_peer(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void ns_peer_st16(uint32_t addr, const uint4& v) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
// byte offset of 16-byte segment `seg` (8 columns) of a row in a swizzled [128][64] tile
__device__ __forceinline__ uint32_t ns_seg(int row, int seg) { return (uint32_t)(row * 128 + ((seg ^ (row & 7)) << 4)); }
__device__ __forceinline__ uint4 ns_half8(const float* f) {
  uint4 o;
  __half2* h = reinterpret_cast<__half2*>(&o);
#pragma unroll
  for (int t = 0; t < 4; ++t) h[t] = __floats2half2_rn(f[2 * t], f[2 * t + 1]);
  return o;
}

// 32 columns of this thread's lane into tensor memory; complete (for this thread's later loads) on return
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float (&f)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(addr), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "f"(f[8]), "f"(f[9]), "f"(f[10]),
        "f"(f[11]), "f"(f[12]), "f"(f[13]), "f"(f[14]), "f"(f[15]), "f"(f[16]), "f"(f[17]), "f"(f[18]), "f"(f[19]), "f"(f[20]), "f"(f[21]),
        "f"(f[22]), "f"(f[23]), "f"(f[24]), "f"(f[25]), "f"(f[26]), "f"(f[27]), "f"(f[28]), "f"(f[29]), "f"(f[30]), "f"(f[31]) : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

template <typename T, int NH>
__global__ void __launch_bounds__(kSmThreads, 1) ns_small_kernel(NsSmallArgs a) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t xt = base, et = xt + 2 * NH * kSmTile, ft = et + 2 * kSmTile, recv = ft + 2 * kSmTile;
  const uint32_t stg = ft;                              // 2 KB per warp to turn a unit over: F is written later
  const uint32_t da_s = recv + 64 * 1024, df_s = da_s + 512, red_s = df_s + 512, nrm_s = red_s + 512, bar = nrm_s + 128, slot_s = bar + 8;
  auto gen = [&](uint32_t s) { return sm + (s - base); };
  float *dA = (float*)gen(da_s), *dF = (float*)gen(df_s);
  double *red = (double*)gen(red_s), *nrm = (double*)gen(nrm_s);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, q = warp & 3, sub = warp >> 2;
  uint32_t C, me;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
  me = cluster_ctarank();

  if (tid == 0) {
    mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  constexpr int kCols = 512;                           // X [128 NH] | Gram matrix and polynomial [128] | step [128]
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_s), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)gen(slot_s);
  pdl_trigger();
  pdl_wait();                                          // nothing global before this
  const uint32_t lanes = (uint32_t)(q * 32) << 16, xtm = tmem, acc1 = tmem + 128 * NH;
  // the step's accumulator of column block h; the second block's takes the place of the polynomial's, which is done by then
  auto acc2 = [&](int h) { return h == 0 ? acc1 + 128 : acc1; };

  // ---- the matrix: this thread's row m of the turned matrix and, of every 128 columns, one chunk of 32
  const bool wide = a.rows <= a.cols;
  const int S0 = wide ? a.rows : a.cols, L0 = wide ? a.cols : a.rows;
  const int m = q * 32 + lane;
  auto col = [&](int k) { return k * 128 + sub * 32; };                                           // of this CTA's columns
  // A chunk is 32 x 32: lines of 32 consecutive elements in memory, ni of them with nl elements that exist.  If the rows are as
  // in memory a line is a row and goes to its lane through shared memory (the receive buffer, free at both ends); else it is a column.
  struct Chunk { size_t at; int ni, nl; };
  auto chunk = [&](int k) {
    const int j = (int)me * (128 * NH) + col(k), rows_left = max(0, min(32, S0 - q * 32)), cols_left = max(0, min(32, L0 - j));
    return wide ? Chunk{(size_t)(q * 32) * a.cols + j, rows_left, cols_left} : Chunk{(size_t)j * a.cols + q * 32, cols_left, rows_left};
  };
  float* turn = reinterpret_cast<float*>(gen(recv)) + warp * 1024;
  auto turned = [&](float (&f)[32]) {                  // f[i] of lane l <-> f[l] of lane i
    if (!wide) return;
#pragma unroll
    for (int i = 0; i < 32; ++i) turn[i * 32 + (lane ^ i)] = f[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = turn[lane * 32 + (lane ^ i)];
    __syncwarp();
  };
  const int raised = tid == 0 ? *(volatile int*)&g_tc_error : 0;      // of an earlier launch
  double s = 0.0;
#pragma unroll 1
  for (int k = 0; k < NH; ++k) {
    const Chunk ch = chunk(k);
    const bool in = lane < ch.nl;
    const T* gp = reinterpret_cast<const T*>(a.g) + ch.at + lane;
    float u[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      u[i] = 0.f;
      if (in && i < ch.ni) {
        const T v = gp[(size_t)i * a.cols];
        u[i] = sizeof(T) == 4 ? *reinterpret_cast<const float*>(&v) : __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(&v));
      }
    }
    if (a.mom) {
      float* mp = a.mom + ch.at + lane;
      float b[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) b[i] = in && i < ch.ni ? mp[(size_t)i * a.cols] : 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        b[i] = fmaf(a.mu, b[i], u[i]);
        u[i] = a.nesterov ? fmaf(a.mu, b[i], u[i]) : b[i];
        if (in && i < ch.ni) mp[(size_t)i * a.cols] = b[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) s = fma((double)u[i], (double)u[i], s);
    turned(u);
    tmem_st32(xtm + lanes + col(k), u);
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) red[warp] = s;
  int* const raised_s = reinterpret_cast<int*>(red + 16);
  if (tid == 0) *raised_s = raised;
  cluster_sync_all();                                  // and every CTA of the cluster has started
  if (tid < (int)C) {                                  // this CTA's sum to all
    double t = 0.0;
    for (int w = 0; w < kSmThreads / 32; ++w) t += red[w];
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ns_peer(nrm_s + 8 * me, tid)), "d"(t) : "memory");
  }
  cluster_sync_all();
  float inv;
  {
    double t = 0.0;
    for (int w = 0; w < (int)C; ++w) t += nrm[w];
    const double n = sqrt(t);
    inv = (float)(1.0 / (n < 1e-30 ? 1e-30 : n));      // a NaN stays one
  }
  // chunk k of the iterate: kept in tensor memory, and its fp16 image in the operand tiles
  auto put_x = [&](int k, float (&f)[32]) {
    tmem_st32(xtm + lanes + col(k), f);
    uint8_t* tile = gen(xt) + (2 * k + (sub >> 1)) * kSmTile;
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] *= kNsScale;
#pragma unroll
    for (int sg = 0; sg < 4; ++sg) *reinterpret_cast<uint4*>(tile + ns_seg(m, (sub & 1) * 4 + sg)) = ns_half8(f + 8 * sg);
  };
#pragma unroll 1
  for (int k = 0; k < NH; ++k) {
    uint32_t v[32];
    float f[32];
    tmem_ld32(xtm + lanes + col(k), v);
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]) * inv;
    put_x(k, f);
  }
  fence_proxy_async_all();

  uint32_t phase = 0;
  bool ok = true;
  auto run = [&](auto&& issue) {                       // all threads: operands are ready; one issues, all wait for the products
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) {
      if (lane == 0) { issue(); tc_commit(bar); }
      __syncwarp();
    }
    if (!mbar_wait(bar, phase)) { ok = false; atomicCAS(&g_tc_error, 0, 3); }       // the result is then not written
    phase ^= 1;
    tc_fence_after();
  };
  // instruction descriptors: fp32 accumulator, fp16 operands, 128 x 128; the step's B operand is N-major
  constexpr uint32_t kIdesc = (1u << 4) | (16u << 17) | (8u << 24), kIdescN = kIdesc | (1u << 16);
  const int units_per = (10 + (int)C - 1) / (int)C;    // lower-triangle units that a CTA sums

#pragma unroll 1
  for (int step = 0; step < a.steps; ++step) {
    run([&] {
#pragma unroll 1
      for (int t = 0; t < 2 * NH; ++t) {
        const uint64_t d = ns_desc(xt + t * kSmTile, 16);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tc_mma(acc1, d + kk * 2, d + kk * 2, kIdesc, (t | kk) != 0);
      }
    });
    // ---- sum of the parts: unit (q, c), c <= q, number l = q (q + 1) / 2 + c, belongs to CTA l mod C, to the warp (q, c) of it
    const int c = sub, l = q * (q + 1) / 2 + c, o = l % (int)C;
    if (c <= q && o != (int)me) {                      // uniform across the warp
      uint32_t v[32];
      tmem_ld32(acc1 + lanes + 32 * c, v);
      const int from = (int)me < o ? (int)me : (int)me - 1;
      const uint32_t dst = ns_peer(recv + (uint32_t)((from * units_per + l / (int)C) * 4096 + lane * 16), o);
#pragma unroll
      for (int g = 0; g < 8; ++g) ns_peer_st16(dst + g * 512, make_uint4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]));
    }
    __syncwarp();
    cluster_sync_all();
    if (c <= q && o == (int)me) {
      uint32_t v[32];
      tmem_ld32(acc1 + lanes + 32 * c, v);
      float f[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
#pragma unroll 1
      for (int from = 0; from < (int)C - 1; ++from) {
        const uint8_t* src = gen(recv) + (from * units_per + l / (int)C) * 4096 + lane * 16;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float4 y = *reinterpret_cast<const float4*>(src + g * 512);
          f[4 * g] += y.x; f[4 * g + 1] += y.y; f[4 * g + 2] += y.z; f[4 * g + 3] += y.w;
        }
      }
      float d = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        f[j] *= 1.0f / (kNsScale * kNsScale);
        if (c == q && j == lane) { d = f[j]; f[j] = 0.f; }
      }
      // the unit, and below the diagonal its transpose, to every CTA's E
      uint4 row[4], col[4];
#pragma unroll
      for (int sg = 0; sg < 4; ++sg) row[sg] = ns_half8(f + 8 * sg);
      __half* st = reinterpret_cast<__half*>(gen(stg) + warp * 2048);
#pragma unroll
      for (int j = 0; j < 32; ++j) st[j * 32 + lane] = __float2half_rn(f[j]);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) col[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<uint8_t*>(st) + (8 * i + (lane >> 2)) * 64 + (lane & 3) * 16);
      __syncwarp();
#pragma unroll 1
      for (uint32_t p = 0; p < C; ++p) {
        const uint32_t e = ns_peer(et, p);
#pragma unroll
        for (int sg = 0; sg < 4; ++sg) ns_peer_st16(e + (c >> 1) * kSmTile + ns_seg(m, (c & 1) * 4 + sg), row[sg]);
        if (c < q) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            ns_peer_st16(e + (q >> 1) * kSmTile + ns_seg(32 * c + 8 * i + (lane >> 2), (q & 1) * 4 + (lane & 3)), col[i]);
        } else {
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ns_peer(da_s + 4 * m, p)), "f"(d) : "memory");
        }
      }
    }
    fence_proxy_async_all();
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();
    fence_proxy_async_all();
    run([&] {
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        const uint64_t d = ns_desc(et + t * kSmTile, 16);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tc_mma(acc1, d + kk * 2, d + kk * 2, kIdesc, (t | kk) != 0);
      }
    });
    // ---- F = b E + c (E E + (d_i + d_j) E), the diagonal apart
    const float dm = dA[m];
    {
      uint32_t v[32];
      tmem_ld32(acc1 + lanes + 32 * c, v);
      const uint8_t* er = gen(et) + (c >> 1) * kSmTile;
      uint8_t* fr = gen(ft) + (c >> 1) * kSmTile;
#pragma unroll
      for (int sg = 0; sg < 4; ++sg) {
        const uint4 e8 = *reinterpret_cast<const uint4*>(er + ns_seg(m, (c & 1) * 4 + sg));
        const __half2* he = reinterpret_cast<const __half2*>(&e8);
        float f[8];
        const float4 d4[2] = {*reinterpret_cast<const float4*>(dA + 32 * c + 8 * sg), *reinterpret_cast<const float4*>(dA + 32 * c + 8 * sg + 4)};
        const float* dn = reinterpret_cast<const float*>(d4);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float2 e2 = __half22float2(he[t]);
          const int i = 8 * sg + 2 * t;
          f[2 * t] = fmaf(kNsB, e2.x, kNsC * fmaf(dm + dn[2 * t], e2.x, __uint_as_float(v[i])));
          f[2 * t + 1] = fmaf(kNsB, e2.y, kNsC * fmaf(dm + dn[2 * t + 1], e2.y, __uint_as_float(v[i + 1])));
        }
        if (c == q) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (8 * sg + i == lane) { dF[m] = fmaf(kNsB, dm, kNsC * fmaf(dm, dm, __uint_as_float(v[8 * sg + i]))); f[i] = 0.f; }
        }
        *reinterpret_cast<uint4*>(fr + ns_seg(m, (c & 1) * 4 + sg)) = ns_half8(f);
      }
    }
    fence_proxy_async_all();
    run([&] {
#pragma unroll 1
      for (int t = 0; t < 2 * NH; ++t) {
        const uint64_t da = ns_desc(ft + (t & 1) * kSmTile, 16), db = ns_desc(xt + (t & ~1) * kSmTile, kSmTile) + (t & 1) * (64 * 128 >> 4);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tc_mma(acc2(t >> 1), da + kk * 2, db + kk * (16 * 128 >> 4), kIdescN, ((t & 1) | kk) != 0);
      }
    });
    const float df = dF[m];
    const int late = step + 2 >= a.steps;
#pragma unroll 1
    for (int k = 0; k < NH; ++k) {
      uint32_t v[32], xo[32];
      float f[32];
      tmem_ld32_nowait(acc2(k) + lanes + 32 * sub, v);
      tmem_ld32(xtm + lanes + col(k), xo);
      tmem_ld_wait32(v);
#pragma unroll
      for (int i = 0; i < 32; ++i) f[i] = ns_new_x(__uint_as_float(xo[i]), df, __uint_as_float(v[i]), late);
      put_x(k, f);
    }
    fence_proxy_async_all();
  }
  // ---- the result, unless a product gave up on a wait: here, in another CTA of the cluster, or before this launch.  Every CTA sends what it
  // knows round, so that all decide alike and no matrix is half updated.
  const int gave_up = __syncthreads_or(!ok);
  if (tid < (int)C)                                    // (the norm's slots have been read)
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ns_peer(nrm_s + 4 * me, tid)), "r"(*raised_s | gave_up) : "memory");
  __syncwarp();
  cluster_sync_all();
  int hold = 0;
  for (int w = 0; w < (int)C; ++w) hold |= reinterpret_cast<const int*>(nrm)[w];
  const bool write = hold == 0;
#pragma unroll 1
  for (int k = 0; k < NH; ++k) {
    uint32_t v[32];
    float f[32];
    tmem_ld32(xtm + lanes + col(k), v);
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
    turned(f);
    const Chunk ch = chunk(k);
    const bool in = write && lane < ch.nl;
    const size_t at = ch.at + lane;
    if (a.o) {
#pragma unroll
      for (int i = 0; i < 32; ++i) if (in && i < ch.ni) a.o[at + (size_t)i * a.cols] = __float2bfloat16_rn(f[i]);
    }
    if (a.master) {
      float b[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) b[i] = in && i < ch.ni ? a.master[at + (size_t)i * a.cols] : 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        b[i] = b[i] * a.decay - a.size * f[i];
        if (in && i < ch.ni) {
          a.master[at + (size_t)i * a.cols] = b[i];
          if (a.param) a.param[at + (size_t)i * a.cols] = __float2bfloat16_rn(b[i]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
  }
}
