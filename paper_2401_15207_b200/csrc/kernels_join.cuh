// The junction of a block's output h with the residual stream x, and its gradient:
//
//   u = N1(h),  x' = a x + q o u,  y = N2(x')          N: LayerNorm (kind 0) or RMSNorm (kind 1); q: the gate
//   d = dx' + N2'(dy; x'),  dx = a d,  dq = sum d o u,  du = d o q,  dh = N1'(du; h)
//   N'(v): with hat = (t - mean) rstd and w = v o gain:  rstd (w - mean(w) - hat mean(w o hat)); no mean(w) for RMSNorm
//   dgain = sum v o hat, dbias = sum v over the rows (dq: over the rows of one gate).
// Either norm, and the gate, can be missing.  x, x' and their gradients are fp32 (the residual stream); h, y and the
// parameters have the operand type.  Every statistic and sum is fp32, the sums over row chunks double.
#pragma once
#include "common.cuh"

namespace hift {

constexpr int kJoinMaxCols = 16384;
constexpr int kJoinPlanes = 5;         // column sums of the backward pass: gain and bias of both norms, gate

// Sums of two values over the block (at most 16 warps).  The warps' two sums go through one run of shuffles: the lower half
// of the lanes carries a, the upper half b.  `red` is one of several buffers of 32 floats used in turn, so that one barrier does.
__device__ __forceinline__ float2 block_sum2(float a, float b, float* red) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool up = lane & 16;
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (nw > 1) {
    if ((lane & 15) == 0) red[(up ? 16 : 0) + w] = v;
    __syncthreads();
    v = (lane & 15) < nw ? red[lane] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
}
// four values: two runs of the above behind one barrier; `red` holds 64 floats
__device__ __forceinline__ float4 block_sum4(float a, float b, float c, float d, float* red) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool up = lane & 16;
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 16);
  float u = (up ? d : c) + __shfl_xor_sync(0xffffffffu, up ? c : d, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) { v += __shfl_xor_sync(0xffffffffu, v, o); u += __shfl_xor_sync(0xffffffffu, u, o); }
  if (nw > 1) {
    if ((lane & 15) == 0) { red[(up ? 16 : 0) + w] = v; red[32 + (up ? 16 : 0) + w] = u; }
    __syncthreads();
    v = (lane & 15) < nw ? red[lane] : 0.f;
    u = (lane & 15) < nw ? red[32 + lane] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) { v += __shfl_xor_sync(0xffffffffu, v, o); u += __shfl_xor_sync(0xffffffffu, u, o); }
  }
  return make_float4(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16), __shfl_sync(0xffffffffu, u, 0), __shfl_sync(0xffffffffu, u, 16));
}
__device__ __forceinline__ float block_sum1(float a, float* red) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
  a = warp_sum(a);
  if (nw > 1) {
    if (lane == 0) red[w] = a;
    __syncthreads();
    a = (lane & 15) < nw ? red[lane & 15] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  }
  return a;
}

// A thread's columns: NC chunks of 8, each two groups of 4 that lie 128 columns apart, so that a warp's access to a group is one
// contiguous run of 512 bytes (fp32) or 256 (bf16).  (8 columns in a row per thread put half of every 32-byte sector into
// each of two instructions: 289 instead of 216 us for the backward kernel at 16384 x 4096.)  cols is a multiple of 8, so a
// group exists or not as a whole; where only the first one does, the second is held at zero.
__device__ __forceinline__ int join_col(int k, int half) {
  return ((k * (int)(blockDim.x >> 5) + (int)(threadIdx.x >> 5)) << 8) + (half << 7) + ((int)(threadIdx.x & 31) << 2);
}
__device__ __forceinline__ void ld4(const float* p, float* v) { const float4 a = *reinterpret_cast<const float4*>(p); v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
__device__ __forceinline__ void ld4(const bf16* p, float* v) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u); v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
}
__device__ __forceinline__ void st4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void st4(bf16* p, const float* v) {
  uint2 a;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&a);
  h[0] = __floats2bfloat162_rn(v[0], v[1]);
  h[1] = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = a;
}
template <typename T>
__device__ __forceinline__ void join_ld(const T* row, int k, int cols, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (join_col(k, h) < cols) ld4(row + join_col(k, h), v + 4 * h);
    else v[4 * h] = v[4 * h + 1] = v[4 * h + 2] = v[4 * h + 3] = 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void join_st(T* row, int k, int cols, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (join_col(k, h) < cols) st4(row + join_col(k, h), v + 4 * h);
}

struct JoinFwd {
  const float* x; const void* h;
  const void *gain1, *bias1, *gate, *gain2, *bias2;
  float* xo; void* y; float* stats;
  int64_t rows, rows_per_gate;
  int cols;
  float eps, scale;
};

// One block per row, the row in registers: NC chunks of 8 columns per thread.
template <typename P, int KIND, int NC>
__global__ void __launch_bounds__(512) join_fwd_kernel(JoinFwd p) {
  __shared__ float red[4][32];
  const int64_t row = blockIdx.x;
  const int64_t off = row * p.cols;
  const float inv = 1.0f / (float)p.cols;
  pdl_launch_next();
  pdl_wait_prior();
  float v[NC][8], xv[NC][8];                           // both streams are under way before the first sum
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    join_ld((const P*)p.h + off, k, p.cols, v[k]);
    join_ld(p.x + off, k, p.cols, xv[k]);
  }
  // mean and reciprocal deviation of the row held in v (two passes over registers)
  auto moments = [&](float* r0, float* r1, float& mean, float& rstd) {
    mean = 0.f;
    if (KIND == 0) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[k][i];
      mean = block_sum1(s, r0) * inv;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (join_col(k, h) >= p.cols) continue;
#pragma unroll
        for (int i = 4 * h; i < 4 * h + 4; ++i) q += (v[k][i] - mean) * (v[k][i] - mean);
      }
    rstd = 1.0f / sqrtf(block_sum1(q, r1) * inv + p.eps);
  };
  float mean = 0.f, rstd = 0.f;
  if (p.gain1) moments(red[0], red[1], mean, rstd);
  if (threadIdx.x == 0) { p.stats[row] = mean; p.stats[p.rows + row] = rstd; }
  const P* gate = p.gate ? (const P*)p.gate + (row / p.rows_per_gate) * p.cols : nullptr;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    float g[8], b[8];
    if (p.gain1) {
      join_ld((const P*)p.gain1, k, p.cols, g);
      if (KIND == 0) join_ld((const P*)p.bias1, k, p.cols, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = (v[k][i] - mean) * rstd * g[i] + (KIND == 0 ? b[i] : 0.f);
    }
    if (gate) {
      join_ld(gate, k, p.cols, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] *= g[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[k][i] = fmaf(p.scale, xv[k][i], v[k][i]);       // columns that do not exist stay 0
    join_st(p.xo + off, k, p.cols, v[k]);
  }
  mean = rstd = 0.f;
  if (p.gain2) moments(red[2], red[3], mean, rstd);
  if (threadIdx.x == 0) { p.stats[2 * p.rows + row] = mean; p.stats[3 * p.rows + row] = rstd; }
  if (!p.gain2) return;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    float g[8], b[8], o[8];
    join_ld((const P*)p.gain2, k, p.cols, g);
    if (KIND == 0) join_ld((const P*)p.bias2, k, p.cols, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (v[k][i] - mean) * rstd * g[i] + (KIND == 0 ? b[i] : 0.f);
    join_st((P*)p.y + off, k, p.cols, o);
  }
}

struct JoinBwd {
  const void* dy; const float* dxo; const float* xo; const void* h; const float* stats;
  const void *gain1, *bias1, *gate, *gain2;
  float* dx; void* dh; float* dgate;
  float* partial;          // [kJoinPlanes][ctas][cols]
  int64_t rows, rows_per_gate;
  int cols, ctas, stages;
  int split;               // > 0: every gate's rows are split over `split` blocks; 0: a block takes whole gates
  int64_t gates_per_cta;   // split == 0
  float scale;
};

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4cols(float* dst, const float* src) { cp_async16(dst, src); }
__device__ __forceinline__ void cp_async4cols(bf16* dst, const bf16* src) { cp_async8(dst, src); }
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// at most n (0 or 1: no more than two stages) of this thread's newest groups still under way
__device__ __forceinline__ void cp_async_wait_upto(int n) {
  if (n > 0) cp_async_wait<1>();
  else cp_async_wait<0>();
}
// rows a block works on at a time
template <int NC, bool ONE> constexpr int join_rows = NC == 1 && ONE ? 2 : 1;
// bytes a thread stages per chunk of 8 columns: x', dx' in fp32, dy, h in the operand type
template <typename P> constexpr int join_bytes = 2 * 32 + 2 * 8 * (int)sizeof(P);

// Two columns.  Packed: one instruction for both, in the LayerNorm variants, which are short of issue slots (main kernel at 16384 x 2048:
// 155 -> 122 us, at 16384 x 4096 310 -> 293; whole gradient at 8192 x 8192 with a gate per row 655 -> 569); the RMSNorm ones, nearer to the
// memory's rate, run faster on single registers (204 against 218 us).  So do bf16 LayerNorm rows beyond 8192 columns (NC = 4), where pairs
// spill more than they save (4096 x 16384: 542 -> 535 us, with a gate per row 1079 -> 959); in fp32 pairs stay ahead there (706 -> 696, 1174 -> 1161).
template <typename P, int KIND, int NC> constexpr bool kJoinPacked = KIND == 0 && (NC <= 2 || sizeof(P) == 4);
template <bool PACKED> struct JoinPair;
template <> struct JoinPair<true> {
  using T = uint64_t;
  __device__ static T make(float a, float b) { return f2_pack(a, b); }
  __device__ static void split(T v, float& a, float& b) { f2_unpack(v, a, b); }
  __device__ static T add(T a, T b) { return f2_add(a, b); }
  __device__ static T mul(T a, T b) { return f2_mul(a, b); }
  __device__ static T fma(T a, T b, T c) { return f2_fma(a, b, c); }
};
template <> struct JoinPair<false> {
  using T = float2;
  __device__ static T make(float a, float b) { return make_float2(a, b); }
  __device__ static void split(T v, float& a, float& b) { a = v.x; b = v.y; }
  __device__ static T add(T a, T b) { return make_float2(a.x + b.x, a.y + b.y); }
  __device__ static T mul(T a, T b) { return make_float2(a.x * b.x, a.y * b.y); }
  __device__ static T fma(T a, T b, T c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
};

// A block walks its rows; the column sums of its rows stay in registers (each thread owns its columns) and leave as one
// row of `partial` per plane: gain1, bias1, gain2, bias2, gate (the last only where a gate's rows are split).  Within one gate
// q everything after the block follows from two sums per column, S1 = sum d hat1 and S0 = sum d (S0 for LayerNorm only):
//     dq = gain1 S1 + bias1 S0,  dgain1 = q S1,  dbias1 = q S0
// (without a norm after the block dq = S1 = sum d h).  ONE: a block's rows share one gate, or there is none; otherwise the
// sums are turned over to dgate, dgain1 and dbias1 at each gate's end.
// A row is two block-wide sums in sequence, so what bounds a plain loop over rows is latency (one row's loads, two sums, its
// stores: 502 us at 16384 x 4096 bf16).  Three things against it, with the time that each left:
//   - the next rows are on their way into shared memory meanwhile: every thread copies its own columns
//     and reads them back itself, so the copies need no barrier (382 us of 502).  STAGED = false (rows too wide for shared memory): direct loads.
//   - gains and gate stay in registers where they fit (NC = 1): beside the staging buffers little L1 is left to re-read them
//     from (286 us).
//   - two rows at a time (R = 2, for NC = 1 and one gate), so that their sums share barriers and their work interleaves.
// The RMSNorm variants with one gate are given all 128 registers: left to itself the compiler may settle for 100 and order loads behind
// sums (254 instead of 205 us at 16384 x 4096).  The LayerNorm ones lose by it (16384 x 2048: 135 -> 157 us).
template <typename P, int KIND, int NC, bool STAGED, bool ONE>
__global__ void __launch_bounds__(512, KIND == 1 && ONE ? 1 : 0) join_bwd_kernel(JoinBwd p) {
  using Q = JoinPair<kJoinPacked<P, KIND, NC>>;
  using V = typename Q::T;
  constexpr int BYTES = join_bytes<P>;
  constexpr bool LN = KIND == 0, HOLD = NC == 1;
  constexpr int R = join_rows<NC, ONE>;
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ float red[4][64];
  const float inv = 1.0f / (float)p.cols;
  const int64_t rg = p.rows_per_gate;
  const int tid = threadIdx.x, nt = blockDim.x;
  const bool ragged = p.cols != NC * nt * 8;               // some threads hold columns that do not exist
  int64_t r0, r1, step = 1;                                // rows r0, r0 + step, ... below r1
  if (p.split > 0) {
    const int64_t gate = blockIdx.x / p.split, sub = blockIdx.x % p.split;
    r0 = gate * rg + sub;
    r1 = min(p.rows, (gate + 1) * rg);
    step = p.split;
  } else {
    r0 = min(p.rows, (int64_t)blockIdx.x * p.gates_per_cta * rg);
    r1 = min(p.rows, r0 + p.gates_per_cta * rg);
  }
  // staged groups of 4 columns: first x' and dx' (stream 0, 1), then dy and h (2, 3), each [half][thread]
  auto slot32 = [&](int place, int k, int stream, int half) {
    return reinterpret_cast<float*>(ring + (size_t)(place * NC + k) * BYTES * nt + (size_t)((stream * 2 + half) * nt + tid) * 16);
  };
  auto slotp = [&](int place, int k, int stream, int half) {
    return reinterpret_cast<P*>(ring + (size_t)(place * NC + k) * BYTES * nt + (size_t)64 * nt + (size_t)(((stream - 2) * 2 + half) * nt + tid) * 4 * sizeof(P));
  };
  auto fetch_row = [&](int64_t row, int place) {
    const int64_t off = row * p.cols;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = join_col(k, h);
        if (c >= p.cols) continue;
        if (p.gain2) {
          cp_async4cols(slotp(place, k, 2, h), (const P*)p.dy + off + c);
          cp_async4cols(slot32(place, k, 0, h), p.xo + off + c);
        }
        if (p.dxo) cp_async4cols(slot32(place, k, 1, h), p.dxo + off + c);
        cp_async4cols(slotp(place, k, 3, h), (const P*)p.h + off + c);
      }
  };
  auto fetch = [&](int64_t row, int stage) {               // the R rows from `row` on
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (row + j * step < r1) fetch_row(row + j * step, stage * R + j);
  };
  // 8 columns of a stream: from the staged row, or from memory
  auto get32 = [&](const float* base, int64_t off, int place, int k, int stream, float (&v)[8]) {
    if (!STAGED) { join_ld(base + off, k, p.cols, v); return; }
#pragma unroll
    for (int h = 0; h < 2; ++h) ld4(slot32(place, k, stream, h), v + 4 * h);
  };
  auto getp = [&](const void* base, int64_t off, int place, int k, int stream, float (&v)[8]) {
    if (!STAGED) { join_ld((const P*)base + off, k, p.cols, v); return; }
#pragma unroll
    for (int h = 0; h < 2; ++h) ld4(slotp(place, k, stream, h), v + 4 * h);
  };
  // (slots of columns that do not exist are never copied into: they are zeroed once, and stay so)
  if (STAGED && ragged) {
    for (int s = 0; s < p.stages * R; ++s)
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (join_col(k, h) < p.cols) continue;
          const float zero[4] = {0.f, 0.f, 0.f, 0.f};
          st4(slot32(s, k, 0, h), zero); st4(slot32(s, k, 1, h), zero); st4(slotp(s, k, 2, h), zero); st4(slotp(s, k, 3, h), zero);
        }
  }
  pdl_launch_next();
  pdl_wait_prior();
  if (STAGED)
    for (int s = 0; s < p.stages; ++s) {
      fetch(r0 + s * R * step, s);
      cp_async_commit();
    }
  constexpr int NB = LN ? NC : 1, NM = ONE ? 1 : NC, NMB = ONE || !LN ? 1 : NC;   // sums that this variant does not take shrink to one
  V S1[NC][4], S0[NB][4], a2[NC][4], b2[NB][4], a1[NM][4], b1[NMB][4];     // pairs of columns
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int k = 0; k < NC; ++k) S1[k][i] = a2[k][i] = Q::make(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < NB; ++k) S0[k][i] = b2[k][i] = Q::make(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < NM; ++k) a1[k][i] = Q::make(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < NMB; ++k) b1[k][i] = Q::make(0.f, 0.f);
  }
  float st[R][4], sn[R][4];                                              // statistics, an iteration ahead
  auto next_stats = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sn[j][i] = row + j * step < r1 ? p.stats[i * p.rows + row + j * step] : 0.f;
  };
  next_stats(r0);
  int64_t gate_row = r0 / rg, gate_end = (gate_row + 1) * rg;
  auto pairs = [](const float (&v)[8], V (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = Q::make(v[2 * i], v[2 * i + 1]);
  };
  auto singles = [](const V (&v)[4], float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) Q::split(v[i], o[2 * i], o[2 * i + 1]);
  };
  auto load = [&](const void* base, int k, float other, V (&o)[4]) {        // a parameter's columns, or `other`
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = other;
    if (base) join_ld((const P*)base, k, p.cols, v);
    pairs(v, o);
  };
  // the sums of one gate, at its end: q S1 and q S0 into v1 and v0, the gate's own gradient into dq
  auto turn_over = [&](int k, V (&v1)[4], V (&v0)[4], V (&dq)[4]) {
    V q[4], g[4], b[4];
    load(p.gate ? (const P*)p.gate + gate_row * p.cols : nullptr, k, 1.f, q);
    load(p.gain1, k, 1.f, g);
    if (LN) load(p.gain1 ? p.bias1 : nullptr, k, 0.f, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v1[i] = Q::mul(q[i], S1[k][i]);
      v0[i] = LN ? Q::mul(q[i], S0[LN ? k : 0][i]) : Q::make(0.f, 0.f);
      dq[i] = LN ? Q::fma(g[i], S1[k][i], Q::mul(b[i], S0[LN ? k : 0][i])) : Q::mul(g[i], S1[k][i]);
    }
  };
  // gains and gate as the operand type, in registers (kept as fp32, gate times gain1 at once: 210 instead of 204 us at 16384 x 4096, RMSNorm)
  P hg2[HOLD ? 8 : 1], hg1[HOLD ? 8 : 1], hq[HOLD && ONE ? 8 : 1];
  if (HOLD) {
    auto hold = [&](const void* base, P* v) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * h + i] = join_col(0, h) < p.cols ? ((const P*)base)[join_col(0, h) + i] : from_f<P>(0.f);
    };
    if (p.gain2) hold(p.gain2, hg2);
    if (p.gain1) hold(p.gain1, hg1);
    if (ONE && p.gate) hold((const P*)p.gate + gate_row * p.cols, hq);
  }
  auto param = [&](const void* base, const P* held, bool is_held, int k, V (&v)[4]) {
    if (!is_held) { load(base, k, 1.f, v); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = Q::make(to_f(held[2 * i]), to_f(held[2 * i + 1]));
  };
  auto gain2_of = [&](int k, V (&g)[4]) { param(p.gain2, hg2, HOLD, k, g); };
  auto gated_gain1_of = [&](int k, V (&g)[4]) {              // gate times gain1, of what there is
    if (p.gain1) param(p.gain1, hg1, HOLD, k, g);
    if (p.gate) {
      V q[4];
      param((const P*)p.gate + gate_row * p.cols, hq, HOLD && ONE, k, q);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = p.gain1 ? Q::mul(q[i], g[i]) : q[i];
    }
  };
  // the sums of R rows behind one barrier: c1 = scale mean(w), c2 = scale mean(w hat)
  auto means = [&](const float (&s1)[R], const float (&s2)[R], int which, float (&c1)[R], float (&c2)[R], float* buf) {
    if constexpr (R == 2) {
      if (LN) {
        const float4 s = block_sum4(s1[0], s2[0], s1[1], s2[1], buf);
        c1[0] = s.x; c2[0] = s.y; c1[1] = s.z; c2[1] = s.w;
      } else {
        const float2 s = block_sum2(s2[0], s2[1], buf);
        c1[0] = c1[1] = 0.f; c2[0] = s.x; c2[1] = s.y;
      }
    } else {
      const float2 s = block_sum2(s1[0], s2[0], buf);
      c1[0] = s.x; c2[0] = s.y;
    }
#pragma unroll
    for (int j = 0; j < R; ++j) { c1[j] *= st[j][which] * inv; c2[j] *= st[j][which] * inv; }
  };
  int stage = 0, turn = 0;
  for (int64_t row = r0; row < r1; row += R * step) {
    V d[R][NC][4], t[R][NC][4], p1[R], p2[R];
    float s1[R], s2[R], c1[R], c2[R];
    auto sums = [&] {
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float a, b;
        Q::split(p1[j], a, b);
        s1[j] = a + b;
        Q::split(p2[j], a, b);
        s2[j] = a + b;
      }
    };
    // t <- (t - mean) rstd
    auto normalise = [&](V v, int j, int which) {
      if (LN) v = Q::add(v, Q::make(-st[j][which], -st[j][which]));
      return Q::mul(v, Q::make(st[j][which + 1], st[j][which + 1]));
    };
    // rstd w - c1 - c2 hat
    auto norm_grad = [&](V w, V hat, int j, int which) {
      const V r = Q::make(st[j][which + 1], st[j][which + 1]);
      return Q::fma(Q::make(-c2[j], -c2[j]), hat, LN ? Q::fma(r, w, Q::make(-c1[j], -c1[j])) : Q::mul(r, w));
    };
#pragma unroll
    for (int j = 0; j < R; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) st[j][i] = sn[j][i];
      p1[j] = p2[j] = Q::make(0.f, 0.f);
      c1[j] = c2[j] = 0.f;
    }
    next_stats(row + R * step);
    if (STAGED) cp_async_wait_upto(p.stages - 1);
    if (p.gain2) {                                                       // d = rstd2 w - c1 - c2 hat2 (+ dx')
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (R > 1 && row + j * step >= r1) continue;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          float v[8];
          V g[4];
          getp(p.dy, (row + j * step) * p.cols, stage * R + j, k, 2, v);
          pairs(v, d[j][k]);
          get32(p.xo, (row + j * step) * p.cols, stage * R + j, k, 0, v);
          pairs(v, t[j][k]);
          gain2_of(k, g);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            t[j][k][i] = normalise(t[j][k][i], j, 2);
            a2[k][i] = Q::fma(d[j][k][i], t[j][k][i], a2[k][i]);
            if (LN) b2[LN ? k : 0][i] = Q::add(b2[LN ? k : 0][i], d[j][k][i]);
            d[j][k][i] = Q::mul(d[j][k][i], g[i]);
            if (LN) p1[j] = Q::add(p1[j], d[j][k][i]);
            p2[j] = Q::fma(d[j][k][i], t[j][k][i], p2[j]);
          }
        }
      }
      sums();
      means(s1, s2, 3, c1, c2, red[turn]);
    }
    const V scale = Q::make(p.scale, p.scale);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      p1[j] = p2[j] = Q::make(0.f, 0.f);
      if (R > 1 && row + j * step >= r1) continue;
      const int64_t off = (row + j * step) * p.cols;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        float v[8];
        V w[4];
        if (p.gain2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][k][i] = norm_grad(d[j][k][i], t[j][k][i], j, 2);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][k][i] = Q::make(0.f, 0.f);
        }
        if (p.dxo) {
          get32(p.dxo, off, stage * R + j, k, 1, v);
          pairs(v, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][k][i] = Q::add(d[j][k][i], w[i]);
        }
        if (ragged) {                                              // columns that do not exist take no part in the sums below
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][k][i] = join_col(k, i >> 1) < p.cols ? d[j][k][i] : Q::make(0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Q::mul(scale, d[j][k][i]);
        singles(w, v);
        join_st(p.dx + off, k, p.cols, v);
        getp(p.h, off, stage * R + j, k, 3, v);
        pairs(v, t[j][k]);
        if (p.gain1) {
          gated_gain1_of(k, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            t[j][k][i] = normalise(t[j][k][i], j, 0);
            S1[k][i] = Q::fma(d[j][k][i], t[j][k][i], S1[k][i]);
            if (LN) S0[LN ? k : 0][i] = Q::add(S0[LN ? k : 0][i], d[j][k][i]);
            d[j][k][i] = Q::mul(d[j][k][i], w[i]);
            if (LN) p1[j] = Q::add(p1[j], d[j][k][i]);
            p2[j] = Q::fma(d[j][k][i], t[j][k][i], p2[j]);
          }
        } else {
          if (p.gate) gated_gain1_of(k, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            S1[k][i] = Q::fma(d[j][k][i], t[j][k][i], S1[k][i]);
            if (p.gate) d[j][k][i] = Q::mul(d[j][k][i], w[i]);
          }
        }
      }
    }
    sums();
    if (STAGED) {                                                        // these rows' slots have been read: the rows after the staged ones
      fetch(row + (int64_t)p.stages * R * step, stage);
      cp_async_commit();
      if (++stage == p.stages) stage = 0;
    }
    if (p.gain1) means(s1, s2, 1, c1, c2, red[turn + 1]);
    turn ^= 2;
    const bool gate_done = !ONE && (row + 1 == r1 || row + 1 == gate_end);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (R > 1 && row + j * step >= r1) continue;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        if (p.gain1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) d[j][k][i] = norm_grad(d[j][k][i], t[j][k][i], j, 0);
        }
        float v[8];
        singles(d[j][k], v);
        join_st((P*)p.dh + (row + j * step) * p.cols, k, p.cols, v);
        if (!ONE && gate_done) {
          V v1[4], v0[4], dq[4];
          turn_over(k, v1, v0, dq);
          singles(dq, v);
          if (p.dgate) join_st(p.dgate + gate_row * p.cols, k, p.cols, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a1[ONE ? 0 : k][i] = Q::add(a1[ONE ? 0 : k][i], v1[i]);
            S1[k][i] = Q::make(0.f, 0.f);
            if (LN) { b1[ONE || !LN ? 0 : k][i] = Q::add(b1[ONE || !LN ? 0 : k][i], v0[i]); S0[LN ? k : 0][i] = Q::make(0.f, 0.f); }
          }
        }
      }
    }
    if (!ONE && gate_done) { ++gate_row; gate_end += rg; }
  }
  const size_t plane = (size_t)p.ctas * p.cols;
  float* out = p.partial + (size_t)blockIdx.x * p.cols;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    V v1[4], v0[4], dq[4];
    float v[8];
    auto put = [&](int plane_no, const V (&s)[4]) { singles(s, v); join_st(out + plane_no * plane, k, p.cols, v); };
    if (ONE) {
      turn_over(k, v1, v0, dq);
      if (p.gate) put(4, dq);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) { v1[i] = a1[ONE ? 0 : k][i]; v0[i] = b1[ONE || !LN ? 0 : k][i]; }
    }
    if (p.gain1) put(0, v1);
    if (LN && p.gain1) put(1, v0);
    if (p.gain2) put(2, a2[k]);
    if (LN && p.gain2) put(3, b2[LN ? k : 0]);
  }
}

struct JoinSums { float* out[kJoinPlanes]; };     // nullptr: not wanted
// Sums the planes of `partial` over the blocks, in a fixed order: blockIdx.y = plane; the gate's plane holds one sum per
// gate, over the `split` blocks of that gate.  A CUDA block takes 32 columns,
// four a thread, in blockDim / 8 runs of blocks: as many as leave a thread four loads, which are in flight together.  (32 runs of single
// columns: 10 us for 148 blocks of 4096 columns, 5 like this; with 32 runs always, 592 blocks of 1024 columns took 20 us, 6 like this.)
__global__ void __launch_bounds__(1024) join_sums_kernel(const float* partial, JoinSums o, int ctas, int cols, int split) {
  __shared__ double sh[32][32];
  pdl_launch_next();
  const int plane = min((int)blockIdx.y, kJoinPlanes - 1);
  const int gate = (int)blockIdx.y - (kJoinPlanes - 1);
  float* out = o.out[plane];
  if (out == nullptr) return;
  const int c0 = plane == kJoinPlanes - 1 ? gate * split : 0, cn = plane == kJoinPlanes - 1 ? split : ctas;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, col = blockIdx.x * 32 + (tid & 7) * 4;
  pdl_wait_prior();
  double a[4] = {0.0, 0.0, 0.0, 0.0};
  if (col < cols) {                                        // cols is a multiple of 8
    const float* src = partial + ((size_t)plane * ctas + c0) * cols + col;
#pragma unroll 4
    for (int i = tid >> 3; i < cn; i += blockDim.x >> 3) {
      float v[4];
      ld4(src + (size_t)i * cols, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] += v[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {                            // the warp's four runs
    a[k] += __shfl_xor_sync(0xffffffffu, a[k], 8);
    a[k] += __shfl_xor_sync(0xffffffffu, a[k], 16);
    if (lane < 8) sh[warp][lane * 4 + k] = a[k];
  }
  __syncthreads();
  const int mine = blockIdx.x * 32 + lane;
  if (warp != 0 || mine >= cols) return;
  double b = 0.0;
  for (int w = 0; w < (int)blockDim.x >> 5; ++w) b += sh[w][lane];
  out[(plane == kJoinPlanes - 1 ? (size_t)gate * cols : 0) + mine] = (float)b;
}

}  // namespace hift
