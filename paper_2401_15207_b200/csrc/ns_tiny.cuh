// The whole orthogonalisation of a matrix with a short side of at most 16 in one launch, in fp32 on the CUDA cores; included by
// gemm_tc.cu.  Products this thin would fill a sixteenth of a tensor-core tile, and with few terms in a sum their 16-bit roundings do
// not average out (update off by 1e-3 to 2.5e-3 at short sides below 8).  A thread keeps CP columns of the turned matrix (short side = rows)
// in registers; a cluster of up to 16 CTAs of 512 threads holds the matrix.  Per step: the Gram matrix from a copy of the columns in
// shared memory, one thread per 2 x 2 entries and slice of columns, summed over the slices and, through distributed shared memory, over
// the CTAs in a fixed order; P = a I + b A + c A A by one thread per entry; X <- P X by every thread for its columns.
// Bound by latency: 2 to 4 us a step.  Against the tensor-core kernels: 16 x 16 43 -> 21 us, 8 x 700 64 -> 17, updates of 4695 x 2
// 107 -> 17 and of 4096 x 16 86 -> 52 us.
constexpr int kTinyRows = 16, kTinyThreads = 512;
template <int CP> constexpr int kTinyPitch = kTinyThreads * CP + 4;      // floats between rows of the copy: float4 reads of 16 rows, two per bank
template <int CP> constexpr int ns_tiny_smem = (kTinyRows * kTinyPitch<CP> + 2048 + 2 * 16 * 256 + 2 * 256) * 4 + 2 * 16 * 8 + 17 * 4;

template <typename T, int CP>
__global__ void __launch_bounds__(kTinyThreads, 1) ns_tiny_kernel(NsSmallArgs a) {
  extern __shared__ __align__(16) float ts[];
  float* xs = ts;                                      // [16][pitch]
  float* red = xs + kTinyRows * kTinyPitch<CP>;        // partial sums of the slices
  float* gather = red + 2048;                          // [step parity][CTA][entry]
  float* A = gather + 2 * 16 * 256;
  float* P = A + 256;
  double* dred = reinterpret_cast<double*>(P + 256);   // [16] of this CTA, [16] of the cluster's CTAs
  int* held = reinterpret_cast<int*>(dred + 32);       // results held back after a time-out: [16] as the cluster's CTAs read the flag, then this CTA's reading
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t C;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
  const uint32_t me = cluster_ctarank();
  pdl_trigger();
  pdl_wait();
  const bool wide = a.rows <= a.cols;
  const int S0 = wide ? a.rows : a.cols, L0 = wide ? a.cols : a.rows;
  auto column = [&](int p) { return ((int)me * CP + p) * kTinyThreads + tid; };
  auto at = [&](int m, int j) { return wide ? (size_t)m * a.cols + j : (size_t)j * a.cols + m; };

  // No product of this kernel can time out, but the matrix may come out of one that did.  Other streams may raise the flag meanwhile, so
  // each CTA takes one reading and sends it round with its sum: all decide alike.
  const int raised = tid == 0 ? *(volatile int*)&g_tc_error : 0;
  float x[CP][kTinyRows];
  double s = 0.0;
#pragma unroll
  for (int p = 0; p < CP; ++p) {
    const int j = column(p);
#pragma unroll
    for (int m = 0; m < kTinyRows; ++m) {
      float u = 0.f;
      if (m < S0 && j < L0) {
        const T v = reinterpret_cast<const T*>(a.g)[at(m, j)];
        u = sizeof(T) == 4 ? *reinterpret_cast<const float*>(&v) : __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(&v));
      }
      x[p][m] = u;
    }
    if (a.mom) {
      float b[kTinyRows];
#pragma unroll
      for (int m = 0; m < kTinyRows; ++m) b[m] = m < S0 && j < L0 ? a.mom[at(m, j)] : 0.f;
#pragma unroll
      for (int m = 0; m < kTinyRows; ++m) {
        b[m] = fmaf(a.mu, b[m], x[p][m]);
        x[p][m] = a.nesterov ? fmaf(a.mu, b[m], x[p][m]) : b[m];
        if (m < S0 && j < L0) a.mom[at(m, j)] = b[m];
      }
    }
#pragma unroll
    for (int m = 0; m < kTinyRows; ++m) s = fma((double)x[p][m], (double)x[p][m], s);
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) dred[warp] = s;
  if (tid == 0) held[16] = raised != 0;
  cluster_sync_all();                                  // and every CTA of the cluster has started
  if (tid < (int)C) {
    double t = 0.0;
    for (int w = 0; w < kTinyThreads / 32; ++w) t += dred[w];
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ns_peer(smem_u32(dred + 16 + me), tid)), "d"(t) : "memory");
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ns_peer(smem_u32(held + me), tid)), "r"(held[16]) : "memory");
  }
  cluster_sync_all();
  {
    double t = 0.0;
    for (int w = 0; w < (int)C; ++w) t += dred[16 + w];
    const double n = sqrt(t);
    const float inv = (float)(1.0 / (n < 1e-30 ? 1e-30 : n));        // a NaN stays one
#pragma unroll
    for (int p = 0; p < CP; ++p)
#pragma unroll
      for (int m = 0; m < kTinyRows; ++m) x[p][m] *= inv;
  }
  int S2 = 2;                                          // rows as a power of two
  while (S2 < S0) S2 *= 2;
  // the Gram matrix in 2 x 2 tiles, one thread per tile and slice of the columns (in fours, those that exist)
  const int entries = S2 * S2, er = tid / S2, ec = tid % S2;                           // entry of threads below `entries`
  const int tiles = entries / 4, tile = tid % tiles, slice = tid / tiles, slices = kTinyThreads / tiles;
  const int tr = tile / (S2 / 2) * 2, tc = tile % (S2 / 2) * 2;
  const int units = (max(0, min(kTinyThreads * CP, L0 - (int)me * (kTinyThreads * CP))) + 3) / 4;
  const int rows = tiles < 32 ? kTinyThreads / 32 : slices;                            // of red

#pragma unroll 1
  for (int step = 0; step < a.steps; ++step) {
#pragma unroll
    for (int p = 0; p < CP; ++p)
#pragma unroll
      for (int m = 0; m < kTinyRows; ++m)
        if (m < S2) xs[m * kTinyPitch<CP> + p * kTinyThreads + tid] = x[p][m];
    __syncthreads();
    float g[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = slice; k < units; k += slices) {
      float4 u[2], v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u[i] = *reinterpret_cast<const float4*>(xs + (tr + i) * kTinyPitch<CP> + 4 * k);
        v[i] = *reinterpret_cast<const float4*>(xs + (tc + i) * kTinyPitch<CP> + 4 * k);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 &p = u[i >> 1], &q = v[i & 1];
        g[i] = fmaf(p.x, q.x, g[i]); g[i] = fmaf(p.y, q.y, g[i]); g[i] = fmaf(p.z, q.z, g[i]); g[i] = fmaf(p.w, q.w, g[i]);
      }
    }
    for (int o = tiles; o < 32; o <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] += __shfl_xor_sync(0xffffffffu, g[i], o);
    if (tiles >= 32 || lane < tiles) {
      float* r = red + (tiles >= 32 ? slice : warp) * entries;
#pragma unroll
      for (int i = 0; i < 4; ++i) r[(tr + (i >> 1)) * S2 + tc + (i & 1)] = g[i];
    }
    __syncthreads();
    float* mine = gather + (step & 1) * (16 * 256);
    if (tid < entries) {
      float t = 0.f;
      for (int r = 0; r < rows; ++r) t += red[r * entries + tid];
      for (uint32_t p = 0; p < C; ++p)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ns_peer(smem_u32(mine + me * 256 + tid), p)), "f"(t) : "memory");
    }
    cluster_sync_all();                                // (the other parity's slots are read until every CTA has come here)
    if (tid < entries) {
      float t = 0.f;
      for (uint32_t p = 0; p < C; ++p) t += mine[p * 256 + tid];
      A[tid] = t;
    }
    __syncthreads();
    if (tid < entries) {
      float t = 0.f;
      for (int k = 0; k < S2; ++k) t = fmaf(A[er * S2 + k], A[k * S2 + ec], t);
      P[er * kTinyRows + ec] = fmaf(kNsC, t, kNsB * A[tid]) + (er == ec ? kNsA : 0.f);
    }
    __syncthreads();
    float y[CP][kTinyRows];
#pragma unroll
    for (int m = 0; m < kTinyRows; ++m) {
#pragma unroll
      for (int p = 0; p < CP; ++p) y[p][m] = 0.f;
      if (m >= S2) continue;
#pragma unroll
      for (int k = 0; k < kTinyRows; k += 4) {
        if (k >= S2) continue;
        const float4 w = *reinterpret_cast<const float4*>(P + m * kTinyRows + k);
        const float ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (k + i >= S2) continue;                   // (P holds nothing there)
#pragma unroll
          for (int p = 0; p < CP; ++p) y[p][m] = fmaf(ws[i], x[p][k + i], y[p][m]);
        }
      }
    }
#pragma unroll
    for (int p = 0; p < CP; ++p)
#pragma unroll
      for (int m = 0; m < kTinyRows; ++m) x[p][m] = y[p][m];
  }
  int hold = 0;
  for (int w = 0; w < (int)C; ++w) hold |= held[w];
  if (hold) return;                                    // (no peer reads this CTA's shared memory any more)
#pragma unroll
  for (int p = 0; p < CP; ++p) {
    const int j = column(p);
    if (j >= L0) continue;
#pragma unroll
    for (int m = 0; m < kTinyRows; ++m) {
      if (m >= S0) continue;
      const size_t k = at(m, j);
      if (a.o) a.o[k] = __float2bfloat16_rn(x[p][m]);
      if (a.master) {
        const float t = a.master[k] * a.decay - a.size * x[p][m];
        a.master[k] = t;
        if (a.param) a.param[k] = __float2bfloat16_rn(t);
      }
    }
  }
}
