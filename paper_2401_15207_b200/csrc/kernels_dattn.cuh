// Differential attention on CUDA cores, fp32 arithmetic, every type and head size; and the small kernels that the tensor-core path shares.
//
//   a_m = softmax(q_m k_m^T / sqrt(d) + mask), m = 1, 2;   o_m = a_m v;   o = o_1 - lambda_h o_2;   y = c gain o / rms(o)
// A head has D = 2 d columns: q and k are the two maps' halves behind one another, v is D wide.  qkv[T, (H + 2 K) D]: H query heads, K key
// heads, K value heads; query head h reads key head h / (H / K).  Nothing of size S x S is stored: one pass over the keys with each map's
// running maximum and sum (its log-sum-exp saved), one tile of probabilities at a time in shared memory.
//
// Backward: with g the gradient of o, dP = g v^T is shared by the maps, and with D_1 = g.o_1 = g.(o + lambda o_2), D_2 = g.o_2
//   dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2),  dv = (P_1 - lambda P_2)^T g,  dq_m = dS_m k_m,  dk_m = dS_m^T q_m,
//   dlambda = -sum D_2.
// One kernel owns query rows (dq), one owns key rows (dk, dv; it walks the query heads of its key head in order): every output element has
// one writer and a fixed order of summation.
//
// Tile 64 x 64 with 256 threads: a thread owns 4 x 4 scores (rows 4 ty .., columns tx + 16 j, so that with rows padded by 4 words the reads of
// 16 bytes along a row are free of bank conflicts) and 4 rows x 4 or 8 columns of each output.  Where that leaves most of 148 SMs without a block, tiles
// of 16 rows (RI = 1: one row a thread), whose blocks take a quarter of the time.
#pragma once
#include "common.cuh"
#include "dattn_args.h"

namespace hift {

__device__ __forceinline__ int dattn_len(const int32_t* __restrict__ lens, int b, int S) { return lens ? max(0, min(lens[b], S)) : S; }

constexpr int kDaT = 64;                                   // streamed columns of a tile
template <int D> constexpr int kDaLd = D + 4;              // words between rows of a staged tile
constexpr int kDaPLd = kDaT + 4;
// RI: rows of a thread, so 16 RI owned rows of a tile
template <int D, int RI> constexpr int kDaFwdSmem = ((16 * RI + 2 * kDaT) * kDaLd<D> + 16 * RI * kDaPLd) * 4;
template <int D, int RI> constexpr int kDaDqSmem = (2 * (16 * RI + kDaT) * kDaLd<D> + 16 * RI * kDaPLd) * 4;
template <int D, int RI> constexpr int kDaDkvSmem = (2 * (16 * RI + kDaT) * kDaLd<D> + 3 * 16 * RI * kDaPLd + 4 * kDaT) * 4;

// ROWS rows of D elements, rows at or beyond `rows` as zeros; `vec`: rows start at 16-byte boundaries
template <typename T, int D, int ROWS>
__device__ __forceinline__ void da_stage(float* dst, const T* __restrict__ src, int64_t ld, int rows, bool vec) {
  if (vec) {
    constexpr int N = ROWS * D / 8;                        // groups of 8 elements
#pragma unroll
    for (int k = 0; k < (N + 255) / 256; ++k) {
      const int i = threadIdx.x + 256 * k, r = i / (D / 8), c = i % (D / 8) * 8;
      if (N % 256 && i >= N) break;
      float v[8] = {};
      if (r < rows) load8(src + r * ld + c, v);
      store8(dst + r * kDaLd<D> + c, v);
    }
    return;
  }
  for (int i = threadIdx.x; i < ROWS * D; i += 256) {
    const int r = i / D, c = i % D;
    dst[r * kDaLd<D> + c] = r < rows ? to_f(src[r * ld + c]) : 0.f;
  }
}
// s[i][j] = a[row RI ty + i] . b[row tx + 16 j] over W words
template <int D, int W, int RI>
__device__ __forceinline__ void da_dots(float (&s)[RI][4], const float* a, const float* b, int ty, int tx) {
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int e = 0; e < W; e += 4) {
    float4 x[RI], y[4];
#pragma unroll
    for (int i = 0; i < RI; ++i) x[i] = *reinterpret_cast<const float4*>(a + (RI * ty + i) * kDaLd<D> + e);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * kDaLd<D> + e);
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j]))));
  }
}
// An output tile of 16 RI rows x N columns: a thread owns rows RI ty .. and CW columns.  Narrow tiles (N < 64) leave lanes over, which take a share of
// the 64 k each (KS shares), so that four columns to a thread keep 16 products to each pair of 16-byte reads; the shares are added at the end.
template <int N, int RI> struct DaOut {
  static constexpr int G = N < 64 ? N / 4 : 16, KS = 16 / G, CW = N <= 64 ? 4 : N / 16;
  static __device__ __forceinline__ int col(int n, int tx) { return n / 4 * 64 + tx % G * 4 + n % 4; }
  // acc[i][n] += sum over this thread's k of p[row RI ty + i][k] x[k][its column n]
  static __device__ __forceinline__ void accumulate(float (&acc)[RI][CW], const float* p, const float* x, int ld, int ty, int tx) {
    const int k0 = tx / G * (kDaT / KS);
#pragma unroll 2
    for (int kk = 0; kk < kDaT / KS; kk += 4) {
      const int k = k0 + kk;
      float4 w[RI];
#pragma unroll
      for (int i = 0; i < RI; ++i) w[i] = *reinterpret_cast<const float4*>(p + (RI * ty + i) * kDaPLd + k);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[CW];
#pragma unroll
        for (int n = 0; n < CW; n += 4) {
          const float4 f = *reinterpret_cast<const float4*>(x + (k + j) * ld + col(n, tx));
          v[n] = f.x; v[n + 1] = f.y; v[n + 2] = f.z; v[n + 3] = f.w;
        }
#pragma unroll
        for (int i = 0; i < RI; ++i) {
          const float f = j == 0 ? w[i].x : j == 1 ? w[i].y : j == 2 ? w[i].z : w[i].w;
#pragma unroll
          for (int n = 0; n < CW; ++n) acc[i][n] = fmaf(f, v[n], acc[i][n]);
        }
      }
    }
  }
  static __device__ __forceinline__ void join(float (&acc)[RI][CW]) {         // every lane ends with the whole sums
#pragma unroll
    for (int o = G; o < 16; o *= 2)
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int n = 0; n < CW; ++n) acc[i][n] += __shfl_xor_sync(0xffffffffu, acc[i][n], o);
  }
  static __device__ __forceinline__ bool writes(int tx) { return tx < G; }
};
__device__ __forceinline__ float half_warp_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float half_warp_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Blocks of one launch are numbered along x alone (no limit of 65535 on heads or batch): the tiles with the most work first.
template <typename T, int D, int RI>
__global__ void __launch_bounds__(256) dattn_fwd_kernel(DattnArgs a) {
  typedef DaOut<D, RI> Out;
  constexpr int CW = Out::CW, HD = D / 2;
  constexpr int TR = 16 * RI;                              // rows this block owns
  extern __shared__ float da_smem[];
  float *sq = da_smem, *sk = sq + TR * kDaLd<D>, *sv = sk + kDaT * kDaLd<D>, *sp = sv + kDaT * kDaLd<D>;
  pdl_launch_next();
  pdl_wait_prior();
  const int ntile = (a.S + TR - 1) / TR, tile = ntile - 1 - (int)(blockIdx.x / (unsigned)(a.B * a.H));
  const int bh = (int)(blockIdx.x % (unsigned)(a.B * a.H)), b = bh / a.H, h = bh % a.H, kh = h / (a.H / a.K);
  const int q0 = tile * TR, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int len = dattn_len(a.lens, b, a.S), kend = a.causal ? min(len, min(q0 + TR, a.S)) : len;
  const int64_t ld = (int64_t)(a.H + 2 * a.K) * D;
  const T* base = (const T*)a.qkv + (int64_t)b * a.S * ld;
  da_stage<T, D, TR>(sq, base + q0 * ld + h * D, ld, a.S - q0, a.vec);
  float acc[2][RI][CW], m[2][RI], l[2][RI];
#pragma unroll
  for (int z = 0; z < 2; ++z)
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      m[z][i] = -INFINITY; l[z][i] = 0.f;
#pragma unroll
      for (int n = 0; n < CW; ++n) acc[z][i][n] = 0.f;
    }
  for (int k0 = 0; k0 < kend; k0 += kDaT) {
    __syncthreads();
    da_stage<T, D, kDaT>(sk, base + k0 * ld + (a.H + kh) * D, ld, a.S - k0, a.vec);
    da_stage<T, D, kDaT>(sv, base + k0 * ld + (a.H + a.K + kh) * D, ld, len - k0, a.vec);          // (rows of padding may hold anything: 0 * NaN)
    __syncthreads();
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      float s[RI][4];
      da_dots<D, HD, RI>(s, sq + z * HD, sk + z * HD, ty, tx);
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = k0 + tx + 16 * j;
          s[i][j] = key >= len || (a.causal && key > q0 + RI * ty + i) ? -INFINITY : s[i][j] * a.scale;
          top = fmaxf(top, s[i][j]);
        }
        const float mn = fmaxf(m[z][i], half_warp_max(top)), ref = mn == -INFINITY ? 0.f : mn, corr = expf(m[z][i] - ref);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = expf(s[i][j] - ref);
          sum += p;
          sp[(RI * ty + i) * kDaPLd + tx + 16 * j] = p;
        }
        l[z][i] = l[z][i] * corr + half_warp_sum(sum);
        m[z][i] = mn;
#pragma unroll
        for (int n = 0; n < CW; ++n) acc[z][i][n] *= corr;
      }
      __syncwarp();                                        // a warp's 8 rows of P are its own
      Out::accumulate(acc[z], sp, sv, kDaLd<D>, ty, tx);
      __syncwarp();
    }
  }
  const float lam = a.lam[h];
  Out::join(acc[0]);
  Out::join(acc[1]);
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int q = q0 + RI * ty + i;
    const float r1 = l[0][i] > 0.f ? 1.f / l[0][i] : l[0][i] == 0.f ? 0.f : l[0][i];          // no key: zeros; NaN stays
    const float r2 = l[1][i] > 0.f ? 1.f / l[1][i] : l[1][i] == 0.f ? 0.f : l[1][i];
    float o[CW], o2[CW], sq2 = 0.f;
#pragma unroll
    for (int n = 0; n < CW; ++n) {
      o2[n] = acc[1][i][n] * r2;
      o[n] = fmaf(-lam, o2[n], acc[0][i][n] * r1);
      sq2 = fmaf(o[n], o[n], sq2);
    }
    float r = 0.f;
    if (a.y) r = a.c / sqrtf(half_warp_sum(sq2) * (1.0f / (D * Out::KS)) + a.eps);      // (each column KS times)
    if (q >= a.S) continue;
    const int64_t at = ((int64_t)b * a.S + q) * a.H * D + h * D;
#pragma unroll
    for (int n = 0; n < CW && Out::writes(tx); ++n) {
      const int c = Out::col(n, tx);
      ((T*)a.o)[at + c] = from_f<T>(o[n]);
      if (a.o2) ((T*)a.o2)[at + c] = from_f<T>(o2[n]);
      if (a.y) ((T*)a.y)[at + c] = from_f<T>(o[n] * r * to_f(((const T*)a.gain)[c]));
    }
    if (tx < 2) {
      const int64_t row = ((int64_t)b * a.H + h) * a.S + q;
      a.lse[(int64_t)tx * a.B * a.H * a.S + row] = tx == 0 ? m[0][i] + logf(l[0][i]) : m[1][i] + logf(l[1][i]);
    }
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------------------------
// Groups of D / 8 lanes (heads of 16 to 128: 2 to 16 lanes) take (token, head) rows of one head: the gradient g of o (through the norm), D_1, D_2, and per block
// the sums for dlambda and dgain.  D_1 and D_2 are taken with g as the products will read it (rounded to T, their operand type): what is common to all of a row's dP
// then cancels in dP - D.  dlambda is taken with g in fp32.  Memory bounds it: dy, o and o_2 are read once.  VEC: 16-byte accesses.
struct DattnPrep { DattnArgs a; void* g_out; float* dsum_out; float* dlam_part; float* dgain_part; int chunks, rows_per_chunk; };
template <bool VEC, typename T> __device__ __forceinline__ void da_load8(const T* p, float (&v)[8]) {
  if (VEC) { load8(p, v); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_f(p[i]);
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(256) dattn_prep_kernel(DattnPrep p) {
  constexpr int L = D / 8, R = 256 / L;                    // lanes of a row, rows of a block at a time
  __shared__ float red[R][D + 1];
  pdl_launch_next();
  pdl_wait_prior();
  const DattnArgs& a = p.a;
  // the heads of a chunk of rows behind one another: what runs at once reads whole rows
  const int ch = blockIdx.x / a.H, h = blockIdx.x % a.H, slot = h * p.chunks + ch, part = threadIdx.x % L, r = threadIdx.x / L;
  const int64_t rows = (int64_t)a.B * a.S, first = (int64_t)ch * p.rows_per_chunk, last = min(rows, first + p.rows_per_chunk);
  const float lam = a.lam[h];
  float gain[8], dgain[8], dlam = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) { gain[e] = a.gain ? to_f(((const T*)a.gain)[part * 8 + e]) * a.c : 0.f; dgain[e] = 0.f; }
#pragma unroll 2
  for (int64_t t0 = first; t0 < last; t0 += R) {           // (whole warps: the sums below are over lanes)
    const int64_t t = t0 + r;
    const bool in = t < last;
    const int64_t at = (t * a.H + h) * D + part * 8;
    float g[8], o[8], o2[8];
    if (in) {
      da_load8<VEC>((const T*)a.dy + at, g);
      da_load8<VEC>((const T*)a.o + at, o);
      da_load8<VEC>((const T*)a.o2 + at, o2);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = o[e] = o2[e] = 0.f;
    }
    if (a.gain) {
      float ss = 0.f, wo = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) { ss = fmaf(o[e], o[e], ss); wo = fmaf(g[e] * gain[e], o[e], wo); }
      ss = lanes_sum<L>(ss);
      wo = lanes_sum<L>(wo);
      // rn may be up to eps^-1/2: its square fits fp32 (eps is a normal number), its cube need not, so the third factor goes to o first
      const float rn = rsqrtf(ss * (1.0f / D) + a.eps), k = rn * rn * wo * (1.0f / D);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float gr = g[e] * rn;
        dgain[e] = fmaf(gr, o[e], dgain[e]);               // (times c at the end)
        g[e] = fmaf(gr, gain[e], -k * (rn * o[e]));
      }
    }
    float d1 = 0.f, d2 = 0.f;
    if (p.g_out && sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dlam = fmaf(-g[e], o2[e], dlam);
        g[e] = to_f(from_f<T>(g[e]));
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      d2 = fmaf(g[e], o2[e], d2);
      d1 = fmaf(g[e], o[e], d1);
    }
    if (!p.g_out || sizeof(T) == 4) dlam -= d2;            // g was not rounded
    d2 = lanes_sum<L>(d2);
    d1 = fmaf(lam, d2, lanes_sum<L>(d1));                  // g . (o + lambda o_2)
    if (in) {
      if (p.g_out) store8((T*)p.g_out + at, g);            // (the scratch is aligned)
      if (part == 0) {
        const uint32_t b = (uint32_t)t / (uint32_t)a.S;
        const int64_t row = ((int64_t)b * a.H + h) * a.S + (t - (int64_t)b * a.S);
        p.dsum_out[row] = d1;
        p.dsum_out[(int64_t)a.B * a.H * a.S + row] = d2;
      }
    }
  }
  dlam = lanes_sum<L>(dlam);
  if (part == 0) red[r][D] = dlam;
#pragma unroll
  for (int e = 0; e < 8; ++e) red[r][part * 8 + e] = dgain[e] * a.c;
  __syncthreads();
  if (threadIdx.x <= D && (threadIdx.x == D || a.gain)) {
    float s = 0.f;
#pragma unroll 8
    for (int i = 0; i < R; ++i) s += red[i][threadIdx.x];
    if (threadIdx.x == D) p.dlam_part[slot] = s;
    else p.dgain_part[(int64_t)slot * D + threadIdx.x] = s;
  }
}
// The partial sums' sums, in a fixed order: blocks 0 .. H - 1 one head's dlambda each, the others 8 columns of dgain each.
__global__ void __launch_bounds__(1024) dattn_sums_kernel(const float* __restrict__ dlam_part, const float* __restrict__ dgain_part,
                                                          float* __restrict__ dlam, float* __restrict__ dgain, int H, int chunks, int D) {
  __shared__ float red[33];
  __shared__ float col[128][9];
  pdl_launch_next();
  pdl_wait_prior();
  if ((int)blockIdx.x < H) {
    if (!dlam) return;
    float s = 0.f;
    for (int i = threadIdx.x; i < chunks; i += 1024) s += dlam_part[(int64_t)blockIdx.x * chunks + i];
    s = block_sum(s, red);
    if (threadIdx.x == 0) dlam[blockIdx.x] = s;
    return;
  }
  const int c8 = threadIdx.x & 7, c = ((int)blockIdx.x - H) * 8 + c8, w = threadIdx.x >> 3;       // D is a multiple of 8
  float s = 0.f;
#pragma unroll 4
  for (int i = w; i < H * chunks; i += 128) s += dgain_part[(int64_t)i * D + c];
  col[w][c8] = s;
  __syncthreads();
  if (threadIdx.x < 8) {
    s = 0.f;
#pragma unroll 16
    for (int i = 0; i < 128; ++i) s += col[i][threadIdx.x];
    dgain[((int)blockIdx.x - H) * 8 + threadIdx.x] = s;
  }
}

template <typename T, int D, int RI>
__global__ void __launch_bounds__(256) dattn_dq_kernel(DattnArgs a) {
  constexpr int HD = D / 2, CW = DaOut<HD, RI>::CW;
  typedef DaOut<HD, RI> Out;
  constexpr int TR = 16 * RI;                              // rows this block owns
  extern __shared__ float da_smem[];
  float *sq = da_smem, *sg = sq + TR * kDaLd<D>, *sk = sg + TR * kDaLd<D>, *sv = sk + kDaT * kDaLd<D>, *sp = sv + kDaT * kDaLd<D>;
  pdl_launch_next();
  pdl_wait_prior();
  const int ntile = (a.S + TR - 1) / TR, tile = ntile - 1 - (int)(blockIdx.x / (unsigned)(a.B * a.H));
  const int bh = (int)(blockIdx.x % (unsigned)(a.B * a.H)), b = bh / a.H, h = bh % a.H, kh = h / (a.H / a.K);
  const int q0 = tile * TR, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int len = dattn_len(a.lens, b, a.S), kend = a.causal ? min(len, min(q0 + TR, a.S)) : len;
  const int64_t ld = (int64_t)(a.H + 2 * a.K) * D, nrow = (int64_t)a.B * a.H * a.S;
  const T* base = (const T*)a.qkv + (int64_t)b * a.S * ld;
  da_stage<T, D, TR>(sq, base + q0 * ld + h * D, ld, a.S - q0, a.vec);
  da_stage<T, D, TR>(sg, (const T*)a.g + ((int64_t)b * a.S + q0) * a.H * D + h * D, (int64_t)a.H * D, a.S - q0, a.vec);
  const float lam = a.lam[h];
  float acc[2][RI][CW], lse[2][RI], ds[2][RI];
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int64_t row = ((int64_t)b * a.H + h) * a.S + min(q0 + RI * ty + i, a.S - 1);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      lse[z][i] = a.lse[z * nrow + row];
      ds[z][i] = a.dsum[z * nrow + row];
#pragma unroll
      for (int n = 0; n < CW; ++n) acc[z][i][n] = 0.f;
    }
  }
  for (int k0 = 0; k0 < kend; k0 += kDaT) {
    __syncthreads();
    da_stage<T, D, kDaT>(sk, base + k0 * ld + (a.H + kh) * D, ld, len - k0, a.vec);
    da_stage<T, D, kDaT>(sv, base + k0 * ld + (a.H + a.K + kh) * D, ld, len - k0, a.vec);
    __syncthreads();
    float dp[RI][4];
    da_dots<D, D, RI>(dp, sg, sv, ty, tx);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      float s[RI][4];
      da_dots<D, HD, RI>(s, sq + z * HD, sk + z * HD, ty, tx);
      const float w = z == 0 ? a.scale : -lam * a.scale;
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = k0 + tx + 16 * j, q = q0 + RI * ty + i;
          const bool seen = key < len && q < a.S && (!a.causal || key <= q);
          sp[(RI * ty + i) * kDaPLd + tx + 16 * j] = seen ? w * expf(fmaf(s[i][j], a.scale, -lse[z][i])) * (dp[i][j] - ds[z][i]) : 0.f;
        }
      __syncwarp();
      Out::accumulate(acc[z], sp, sk + z * HD, kDaLd<D>, ty, tx);
      __syncwarp();
    }
  }
  Out::join(acc[0]);
  Out::join(acc[1]);
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int q = q0 + RI * ty + i;
    if (q >= a.S || !Out::writes(tx)) continue;
    T* row = (T*)a.dqkv + ((int64_t)b * a.S + q) * ld + h * D;
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int n = 0; n < CW; ++n) row[z * HD + Out::col(n, tx)] = from_f<T>(acc[z][i][n]);
  }
}

template <typename T, int D, int RI>
__global__ void __launch_bounds__(256) dattn_dkv_kernel(DattnArgs a) {
  typedef DaOut<D / 2, RI> Half;
  typedef DaOut<D, RI> Whole;
  constexpr int HD = D / 2, CW = Half::CW, VW = Whole::CW;
  constexpr int TR = 16 * RI;                              // rows this block owns
  extern __shared__ float da_smem[];
  float *sk = da_smem, *sv = sk + TR * kDaLd<D>, *sq = sv + TR * kDaLd<D>, *sg = sq + kDaT * kDaLd<D>;
  float* st[3];
  st[0] = sg + kDaT * kDaLd<D>; st[1] = st[0] + TR * kDaPLd; st[2] = st[1] + TR * kDaPLd;
  float* rowv = st[2] + TR * kDaPLd;                     // [lse 1 | lse 2 | D 1 | D 2][64 queries]
  pdl_launch_next();
  pdl_wait_prior();
  const int tile = (int)(blockIdx.x / (unsigned)(a.B * a.K));                          // the first keys meet the most queries
  const int bh = (int)(blockIdx.x % (unsigned)(a.B * a.K)), b = bh / a.K, kh = bh % a.K, group = a.H / a.K;
  const int k0 = tile * TR, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int len = dattn_len(a.lens, b, a.S);
  const int64_t ld = (int64_t)(a.H + 2 * a.K) * D, nrow = (int64_t)a.B * a.H * a.S;
  const T* base = (const T*)a.qkv + (int64_t)b * a.S * ld;
  da_stage<T, D, TR>(sk, base + k0 * ld + (a.H + kh) * D, ld, len - k0, a.vec);
  da_stage<T, D, TR>(sv, base + k0 * ld + (a.H + a.K + kh) * D, ld, len - k0, a.vec);
  float dk[2][RI][CW], dv[RI][VW];
#pragma unroll
  for (int i = 0; i < RI; ++i) {
#pragma unroll
    for (int n = 0; n < VW; ++n) dv[i][n] = 0.f;
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int n = 0; n < CW; ++n) dk[z][i][n] = 0.f;
  }
  if (k0 < len) {                                          // the whole block
    for (int h = kh * group; h < (kh + 1) * group; ++h) {
      const float lam = a.lam[h];
      for (int q0 = a.causal ? k0 / kDaT * kDaT : 0; q0 < a.S; q0 += kDaT) {
        __syncthreads();
        da_stage<T, D, kDaT>(sq, base + q0 * ld + h * D, ld, a.S - q0, a.vec);
        da_stage<T, D, kDaT>(sg, (const T*)a.g + ((int64_t)b * a.S + q0) * a.H * D + h * D, (int64_t)a.H * D, a.S - q0, a.vec);
        {
          const int z = threadIdx.x >> 6;
          const int64_t row = ((int64_t)b * a.H + h) * a.S + min(q0 + (int)(threadIdx.x & 63), a.S - 1);
          rowv[threadIdx.x] = z < 2 ? a.lse[z * nrow + row] : a.dsum[(z - 2) * nrow + row];
        }
        __syncthreads();
        float dp[RI][4], mix[RI][4];
        da_dots<D, D, RI>(dp, sv, sg, ty, tx);                 // [key][query]
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          float s[RI][4];
          da_dots<D, HD, RI>(s, sk + z * HD, sq + z * HD, ty, tx);
          const float w = z == 0 ? a.scale : -lam * a.scale;
#pragma unroll
          for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int c = tx + 16 * j, key = k0 + RI * ty + i, q = q0 + c;
              const bool seen = key < len && q < a.S && (!a.causal || key <= q);
              const float p = seen ? expf(fmaf(s[i][j], a.scale, -rowv[z * kDaT + c])) : 0.f;
              mix[i][j] = z == 0 ? p : fmaf(-lam, p, mix[i][j]);
              st[z][(RI * ty + i) * kDaPLd + c] = seen ? w * p * (dp[i][j] - rowv[(2 + z) * kDaT + c]) : 0.f;
              if (z == 1) st[2][(RI * ty + i) * kDaPLd + c] = mix[i][j];
            }
        }
        __syncwarp();
        Whole::accumulate(dv, st[2], sg, kDaLd<D>, ty, tx);
        Half::accumulate(dk[0], st[0], sq, kDaLd<D>, ty, tx);
        Half::accumulate(dk[1], st[1], sq + HD, kDaLd<D>, ty, tx);
      }
    }
  }
  Whole::join(dv);
  Half::join(dk[0]);
  Half::join(dk[1]);
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int key = k0 + RI * ty + i;
    if (key >= a.S) continue;                              // rows of padding get zeros
    T* row = (T*)a.dqkv + ((int64_t)b * a.S + key) * ld;
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int n = 0; n < CW && Half::writes(tx); ++n) row[(a.H + kh) * D + z * HD + Half::col(n, tx)] = from_f<T>(dk[z][i][n]);
#pragma unroll
    for (int n = 0; n < VW && Whole::writes(tx); ++n) row[(a.H + a.K + kh) * D + Whole::col(n, tx)] = from_f<T>(dv[i][n]);
  }
}

// ---- lambda -----------------------------------------------------------------------------------------------------------------------
// lambda_h = exp(q1_h . k1_h) - exp(q2_h . k2_h) + init.  w: fp32 q1 | k1 | q2 | k2, each [sets, d]; one set for all heads, or one each.
__global__ void __launch_bounds__(32) diff_lambda_kernel(const float* __restrict__ w, int sets, int d, float init, float* __restrict__ lam, int H) {
  pdl_launch_next();
  pdl_wait_prior();
  const int64_t n = (int64_t)sets * d;
  const float* p = w + (int64_t)(sets == 1 ? 0 : blockIdx.x) * d;
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x; i < d; i += 32) { a = fmaf(p[i], p[n + i], a); b = fmaf(p[2 * n + i], p[3 * n + i], b); }
  a = warp_sum(a);
  b = warp_sum(b);
  if (threadIdx.x == 0) lam[blockIdx.x] = expf(a) - expf(b) + init;
}
__global__ void __launch_bounds__(32) diff_lambda_bwd_kernel(const float* __restrict__ w, int sets, int d, const float* __restrict__ dlam,
                                                             float* __restrict__ dw, int H) {
  pdl_launch_next();
  pdl_wait_prior();
  const int64_t n = (int64_t)sets * d, at = (int64_t)blockIdx.x * d;
  const float* p = w + at;
  float a = 0.f, b = 0.f, g = 0.f;
  for (int i = threadIdx.x; i < d; i += 32) { a = fmaf(p[i], p[n + i], a); b = fmaf(p[2 * n + i], p[3 * n + i], b); }
  a = expf(warp_sum(a));
  b = expf(warp_sum(b));
  if (sets == 1) {                                         // one set serves every head
    for (int i = threadIdx.x; i < H; i += 32) g += dlam[i];
    g = warp_sum(g);
  } else {
    g = dlam[blockIdx.x];
  }
  for (int i = threadIdx.x; i < d; i += 32) {
    dw[at + i] = g * a * p[n + i];
    dw[n + at + i] = g * a * p[i];
    dw[2 * n + at + i] = -g * b * p[3 * n + i];
    dw[3 * n + at + i] = -g * b * p[2 * n + i];
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------
inline bool dattn_head_ok(int D) { return D == 16 || D == 32 || D == 64 || D == 128; }
#define HIFT_DATTN_SWITCH(D, CALL) switch (D) { case 16: return CALL(16); case 32: return CALL(32); case 64: return CALL(64); default: return CALL(128); }

// (the attribute belongs to a device and is idempotent; 1 us beside a launch)
template <typename A>
cudaError_t dattn_launch(void (*kernel)(A), int64_t blocks, int smem, cudaStream_t st, const A& a) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e != cudaSuccess ? e : launch_pdl(kernel, dim3((unsigned)blocks), dim3(256), smem, st, a);
}
// Small tiles where four times the blocks still find an SM each, or two (2 x 131 x 4 heads of 32: gradient 67 -> 48 us, forward 15.1 -> 14.8).
inline bool dattn_small(int S, int64_t heads) { return (int64_t)((S + 15) / 16) * heads <= 2 * 148; }
template <typename T, int D> cudaError_t launch_dattn_fwd_d(cudaStream_t st, const DattnArgs& a) {
  const int64_t bh = (int64_t)a.B * a.H;
  if (dattn_small(a.S, bh)) return dattn_launch(dattn_fwd_kernel<T, D, 1>, (a.S + 15) / 16 * bh, kDaFwdSmem<D, 1>, st, a);
  return dattn_launch(dattn_fwd_kernel<T, D, 4>, (a.S + 63) / 64 * bh, kDaFwdSmem<D, 4>, st, a);
}
template <typename T> cudaError_t launch_dattn_fwd(cudaStream_t st, int D, const DattnArgs& a) {
#define CALL(N) launch_dattn_fwd_d<T, N>(st, a)
  HIFT_DATTN_SWITCH(D, CALL)
#undef CALL
}
template <typename T, int D> cudaError_t launch_dattn_bwd_d(cudaStream_t st, const DattnArgs& a) {
  const int64_t bh = (int64_t)a.B * a.H, bk = (int64_t)a.B * a.K, small = (a.S + 15) / 16, tiles = (a.S + 63) / 64;
  const cudaError_t e = dattn_small(a.S, bh) ? dattn_launch(dattn_dq_kernel<T, D, 1>, small * bh, kDaDqSmem<D, 1>, st, a)
                                             : dattn_launch(dattn_dq_kernel<T, D, 4>, tiles * bh, kDaDqSmem<D, 4>, st, a);
  if (e != cudaSuccess) return e;
  return dattn_small(a.S, bk) ? dattn_launch(dattn_dkv_kernel<T, D, 1>, small * bk, kDaDkvSmem<D, 1>, st, a)
                              : dattn_launch(dattn_dkv_kernel<T, D, 4>, tiles * bk, kDaDkvSmem<D, 4>, st, a);
}
template <typename T> cudaError_t launch_dattn_bwd(cudaStream_t st, int D, const DattnArgs& a) {
#define CALL(N) launch_dattn_bwd_d<T, N>(st, a)
  HIFT_DATTN_SWITCH(D, CALL)
#undef CALL
}
template <typename T> cudaError_t launch_dattn_prep(cudaStream_t st, int D, const DattnPrep& p) {
  const bool vec = (((uintptr_t)p.a.dy | (uintptr_t)p.a.o | (uintptr_t)p.a.o2) & 15) == 0;
#define CALL(N) launch_pdl(vec ? dattn_prep_kernel<T, N, true> : dattn_prep_kernel<T, N, false>, dim3((unsigned)(p.a.H * p.chunks)), dim3(256), 0, st, p)
  HIFT_DATTN_SWITCH(D, CALL)
#undef CALL
}

// The backward call's scratch: D_1 | D_2, the gradient of o where there is a norm, the partial sums.  Chunks of rows: blocks over the heads for eight
// on each of 148 SMs, 32 rows at least.
struct DattnPlan { int chunks, rows_per_chunk; size_t dsum, g, part, bytes; };
inline DattnPlan dattn_plan(int es, int64_t B, int64_t S, int64_t H, int D, bool norm) {
  DattnPlan p;
  const int64_t rows = B * S;
  int64_t want = (148 * 8 + H - 1) / H, most = (rows + 31) / 32;
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.rows_per_chunk = (int)((rows + want - 1) / want);
  p.chunks = (int)((rows + p.rows_per_chunk - 1) / p.rows_per_chunk);
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  p.dsum = 0;
  p.g = up((size_t)(2 * B * H * S) * 4);
  p.part = p.g + (norm ? up((size_t)(rows * H * D) * es) : 0);
  p.bytes = p.part + up((size_t)H * p.chunks * (norm ? D + 1 : 1) * 4);
  return p;
}

}  // namespace hift
