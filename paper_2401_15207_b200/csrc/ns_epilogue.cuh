// Epilogues of the Newton-Schulz products (kernels_muon.cuh) in the tensor-core GEMM kernels; included by gemm_tc.cu.
//
// One step X <- a X + P(A) X, A = X X^T, P(A) = b A + c A A, is three products of fp16 operands with fp32 accumulators.  What
// 16 bits would lose is kept out of them:
//   - the iterate itself stays fp32 (x32); its fp16 image, scaled by 2^10 so that entries of 1 / sqrt(m n) are normal numbers,
//     is only an operand.  a X, which carries the small singular values up, is never rounded to 16 bits.
//   - the diagonals of A and P(A), which near the end are 1 and -2.7 against off-diagonal entries of about 1 / sqrt(n), stay
//     fp32 vectors; the fp16 matrices E and F hold zeros there.  With A = D + E:
//         P(A)_ij = b E_ij + c ((E E)_ij + (d_i + d_j) E_ij),   P(A)_ii = b d_i + c ((E E)_ii + d_i^2),
//         X_new = a X + P(A)_ii Y + F X16 / 2^10.
//     Y is the iterate as the products see it (rounded) in all but the last two steps, so that P(A) as a whole acts on one and the same
//     matrix: if P(A) has a low rank so has the rounding noise that it passes on, which the later steps would amplify like a signal
//     (with the fp32 iterate there, a rank-1 16 x 300 matrix comes out 2e-2 off).  In the last two steps nothing amplifies any more,
//     and Y is the fp32 iterate, which spares the large diagonals that rounding.
// Relative error of the result of five steps before its own rounding, from a CPU model of these roundings and as measured.  Where the
// roundings average out (Gaussian, low-rank, decaying, sparse, one-row and outlier matrices of 4 x 40 to 4096 x 11008): at most 2.4e-3,
// typically 3e-4 to 1e-3 (all-bf16 products: 7e-3 on full-rank matrices, 5e-2 to 1 on low-rank ones).  Where they line up, because there
// are few distinct values: constant 64 x 67 6e-3, blocks of 4 x 4 ones at 32 x 32 9e-3, the model's worst single singular value 3.6e-2 (it
// starts at 0.63, so that four steps amplify).  High and low halves of X and F (three products each) would give 2e-3, of E too 2e-5, at
// up to three times the tensor work.  Further steps: up to 1.6 times each on what is there, 3.44 on the null space's noise, which is the product
// of two roundings (2^-24): rank 3 at 4096 x 4096 1.7e-3 after five steps, 4.6e-2 after eight (fp32 products: 2.4e-4, 6.3e-3); no digit after 15.
// A and P(A) are symmetric: only tiles that touch the lower triangle are computed, and a 32 x 32 chunk below the diagonal is
// stored a second time transposed.  All dimensions are multiples of 64 (zero-padded scratch), so a chunk exists or not as a whole.
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kNsScale = 1024.0f;

// one element of the new iterate: x the old one, d the diagonal of P(A), acc = (F X16)
__device__ __forceinline__ float ns_new_x(float x, float d, float acc, int late) {
  const float y = late ? x * kNsScale : __half2float(__float2half_rn(x * kNsScale));
  return fmaf(kNsA, x, fmaf(d, y, acc) * (1.0f / kNsScale));
}

struct NsArgs {
  int mode;                // 0: A from X, 1: P(A) from E, 2: the new X
  int by_column;           // mode 2: the diagonal belongs to the columns (right-hand product)
  int late;                // mode 2: one of the last two steps: the diagonal acts on the fp32 iterate
  __half* out16;           // E, F or the fp16 image of the new X (nullptr: not wanted)
  const __half* e;         // mode 1: E
  const float* din;        // mode 1: diagonal of A, mode 2: of P(A)
  float* dout;             // modes 0, 1: the diagonal of the result
  float* x32;              // mode 2: the iterate, replaced in place
  int64_t ld;              // of out16, e and x32
  int split;               // modes 0, 1: CTAs (or CTA pairs) of a cluster that share a tile, each with its part of k; 1 otherwise
};
// Which 32-column chunks of a tile's lane quarter q are finished by member z of a split (`split` members, 2, 4 or 8 of them; 8 for
// tiles of 128 columns only, where a member takes one chunk of two quarters): chunk `first`, every `step`-th after it.
struct NsShare {
  int split, z;
  __device__ __forceinline__ int ways() const { return split < 4 ? split : 4; }
  __device__ __forceinline__ int owner(int chunk, int q) const { return split == 8 ? chunk * 2 + (q >> 1) : chunk % split; }
  __device__ __forceinline__ int first(int q) const { return split == 8 ? ((q >> 1) == (z & 1) ? z >> 1 : 1 << 20) : z; }
  // place of a unit (chunk, q) among those that its owner receives from one peer
  __device__ __forceinline__ int unit(int chunk, int q) const { return split == 8 ? (q & 1) : (chunk / split) * 4 + q; }
  __device__ __forceinline__ int units(int chunks) const { return split == 8 ? 2 : chunks / split * 4; }
};
// A split tile: each member's accumulator holds its part of k.  Every warp sends the 32 x 32 units that it does not finish to their
// owners' shared memory (the operand ring, which nobody reads any more), as [peer][unit][8 column groups][32 lanes] of 16 bytes.
// `stride`, `base`: cluster rank of member i = i * stride + base.
__device__ __forceinline__ void ns_send_units(uint32_t taddr, int chunks, int half, int q, const NsShare& s, uint32_t ring, int stride, int base, int lane) {
  const int units = s.units(chunks);
#pragma unroll 1
  for (int c = half; c < chunks; c += 2) {
    const int o = s.owner(c, q);
    if (o == s.z) continue;                            // uniform across the warp
    uint32_t v[32], dst;
    tmem_ld32(taddr + 32 * c, v);
    const int slot = s.z < o ? s.z : s.z - 1;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(ring + (uint32_t)((slot * units + s.unit(c, q)) * 4096 + lane * 16)), "r"(o * stride + base));
#pragma unroll
    for (int g = 0; g < 8; ++g)
      asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + g * 512), "r"(v[4 * g]), "r"(v[4 * g + 1]), "r"(v[4 * g + 2]), "r"(v[4 * g + 3]) : "memory");
  }
}
// adds what the peers sent for this unit, in the order of their places
__device__ __forceinline__ void ns_add_units(uint32_t (&v)[32], int chunk, int chunks, int q, const NsShare& s, const uint8_t* ring, int lane) {
  const int units = s.units(chunks);
#pragma unroll 1
  for (int slot = 0; slot < s.split - 1; ++slot) {
    const uint8_t* src = ring + (size_t)(slot * units + s.unit(chunk, q)) * 4096 + lane * 16;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      const float4 x = *reinterpret_cast<const float4*>(src + g * 512);
      v[4 * g] = __float_as_uint(__uint_as_float(v[4 * g]) + x.x);
      v[4 * g + 1] = __float_as_uint(__uint_as_float(v[4 * g + 1]) + x.y);
      v[4 * g + 2] = __float_as_uint(__uint_as_float(v[4 * g + 2]) + x.z);
      v[4 * g + 3] = __float_as_uint(__uint_as_float(v[4 * g + 3]) + x.w);
    }
  }
}

// tile index -> tile of the lower triangle; per_row = column tiles per row tile's width (1: square tiles, 2: half as wide)
__device__ __forceinline__ void ns_tri_tile(int t, int per_row, int& tm, int& tn) {
  const float k = per_row == 1 ? 8.0f : 4.0f;
  int r = (int)((sqrtf(k * (float)t + 1.0f) - 1.0f) * 0.5f);
  auto before = [&](int i) { return per_row == 1 ? i * (i + 1) / 2 : i * (i + 1); };
  while (before(r + 1) <= t) ++r;
  while (before(r) > t) --r;
  tm = r;
  tn = t - before(r);
}

// lane = row; 32 halves of a row as whole lines (see epi_store32_lines), every row and column of the chunk exists
__device__ __forceinline__ void ns_store_half(const float (&f)[32], uint8_t* __restrict__ stage, __half* __restrict__ out, int64_t ld,
                                              int row_base, int n, int lane) {
  uint8_t* mine = stage + lane * 64;
#pragma unroll
  for (int sg = 0; sg < 4; ++sg) {
    uint4 o;
    __half2* ho = reinterpret_cast<__half2*>(&o);
#pragma unroll
    for (int t = 0; t < 4; ++t) ho[t] = __floats2half2_rn(f[8 * sg + 2 * t], f[8 * sg + 2 * t + 1]);
    *reinterpret_cast<uint4*>(mine + ((sg ^ ((lane >> 1) & 3)) << 4)) = o;
  }
  __syncwarp();
  const int sg = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 2);
    *reinterpret_cast<uint4*>(out + (int64_t)(row_base + r) * ld + n + 8 * sg) =
        *reinterpret_cast<const uint4*>(stage + r * 64 + ((sg ^ ((r >> 1) & 3)) << 4));
  }
  __syncwarp();
}
// the same chunk transposed: element (lane, j) goes to row n + j, column row_base + lane
__device__ __forceinline__ void ns_store_half_transposed(const float (&f)[32], uint8_t* __restrict__ stage, __half* __restrict__ out,
                                                         int64_t ld, int row_base, int n, int lane) {
  __half* s = reinterpret_cast<__half*>(stage);
#pragma unroll
  for (int j = 0; j < 32; ++j) s[j * 32 + lane] = __float2half_rn(f[j]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = 8 * i + (lane >> 2);
    *reinterpret_cast<uint4*>(out + (int64_t)(n + j) * ld + row_base + 8 * (lane & 3)) = *reinterpret_cast<const uint4*>(stage + j * 64 + (lane & 3) * 16);
  }
  __syncwarp();
}

// One warp's rows of an output tile: the 32-column chunks first, first + step, ... below `end` of the tile, from tensor memory at
// taddr.  `ready()` waits for the accumulator (false: the wait gave up); what the first chunk reads from memory is fetched
// before it.  `more(v, chunk)` adds what a split tile's other members hold.
// STEP: mode 2, otherwise modes 0 and 1.
template <bool STEP, typename Ready, typename More>
__device__ __forceinline__ bool epi_ns(uint32_t taddr, int first, int end, int step, int m, int M, int n0, int N, const NsArgs& a,
                                       uint8_t* __restrict__ stage, int lane, Ready&& ready, More&& more) {
  const int row_base = m - lane, lo = 32 * first;
  step *= 32;
  end = min(end, N - n0);
  if (row_base >= M || lo >= end) return ready();      // uniform across the warp
  if constexpr (STEP) {
    float4 xn[8];
    lines_fetch_f32(xn, a.x32, a.ld, row_base, lane, M, n0 + lo);
    const float drow = a.by_column ? 0.f : a.din[m];
    if (!ready()) return false;
#pragma unroll 1
    for (int c0 = lo; c0 < end; c0 += step) {
      uint32_t v[32];
      tmem_ld32_nowait(taddr + c0, v);
      float4 xc[8];
      lines_to_own_row_f32(xn, xc, stage, lane);
      if (c0 + step < end) lines_fetch_f32(xn, a.x32, a.ld, row_base, lane, M, n0 + c0 + step);
      tmem_ld_wait32(v);
      float f[32];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float4 d = make_float4(drow, drow, drow, drow);
        if (a.by_column) d = *reinterpret_cast<const float4*>(a.din + n0 + c0 + 4 * j);
        const float xs[4] = {xc[j].x, xc[j].y, xc[j].z, xc[j].w}, ds[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f[4 * j + i] = ns_new_x(xs[i], ds[i], __uint_as_float(v[4 * j + i]), a.late);
      }
      epi_store32_lines<true>(f, stage, a.x32, a.ld, m, lane, M, n0 + c0, nullptr);
      if (a.out16) {
#pragma unroll
        for (int j = 0; j < 32; ++j) f[j] *= kNsScale;
        ns_store_half(f, stage, a.out16, a.ld, row_base, n0 + c0, lane);
      }
    }
    return true;
  } else {
  const float drow = a.mode == 1 ? a.din[m] : 0.f;
  const int last = min(end, row_base - n0 + 32);       // chunks above the diagonal are stored from below it
  uint4 en[4];
  const __nv_bfloat16* e16 = reinterpret_cast<const __nv_bfloat16*>(a.e);             // 16-bit lines, whatever they hold
  if (a.mode == 1 && last > lo) lines_fetch_bf16(en, e16, a.ld, row_base, lane, M, n0 + lo);
  if (!ready()) return false;
#pragma unroll 1
  for (int c0 = lo; c0 < last; c0 += step) {
    const int n = n0 + c0;
    uint32_t v[32];
    tmem_ld32_nowait(taddr + c0, v);
    float f[32];
    if (a.mode == 0) {
      tmem_ld_wait32(v);
      more(v, c0 >> 5);
#pragma unroll
      for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]) * (1.0f / (kNsScale * kNsScale));
    } else {
      uint4 ec[4];
      lines_park_bf16(en, stage, lane);
      __syncwarp();
      lines_own_row_bf16(ec, stage, lane);
      __syncwarp();
      if (c0 + step < last) lines_fetch_bf16(en, e16, a.ld, row_base, lane, M, n + step);
      tmem_ld_wait32(v);
      more(v, c0 >> 5);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half2* he = reinterpret_cast<const __half2*>(&ec[j]);
        const float4 d4[2] = {*reinterpret_cast<const float4*>(a.din + n + 8 * j), *reinterpret_cast<const float4*>(a.din + n + 8 * j + 4)};
        const float* dc = reinterpret_cast<const float*>(d4);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int i = 8 * j + 2 * t;
          const float2 e2 = __half22float2(he[t]);
          f[i] = fmaf(kNsB, e2.x, kNsC * fmaf(drow + dc[2 * t], e2.x, __uint_as_float(v[i])));
          f[i + 1] = fmaf(kNsB, e2.y, kNsC * fmaf(drow + dc[2 * t + 1], e2.y, __uint_as_float(v[i + 1])));
        }
      }
    }
    if (n == row_base) {                               // the chunk on the diagonal: its diagonal leaves as fp32
      float d = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (j == lane) { d = a.mode == 0 ? f[j] : fmaf(kNsB, drow, kNsC * fmaf(drow, drow, __uint_as_float(v[j]))); f[j] = 0.f; }
      }
      a.dout[m] = d;
    }
    ns_store_half(f, stage, a.out16, a.ld, row_base, n, lane);
    if (n < row_base) ns_store_half_transposed(f, stage, a.out16, a.ld, row_base, n, lane);
  }
  return true;
  }
}
