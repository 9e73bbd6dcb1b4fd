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

// sums of two values over the block; `red` is one of two buffers of 64 floats used in turn, so that one barrier does
__device__ __forceinline__ float2 block_sum2(float a, float b, float* red) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
  a = warp_sum(a);
  b = warp_sum(b);
  if (nw == 1) return make_float2(a, b);
  if (lane == 0) { red[w] = a; red[32 + w] = b; }
  __syncthreads();
  a = 0.f; b = 0.f;
  for (int i = 0; i < nw; ++i) { a += red[i]; b += red[32 + i]; }
  return make_float2(a, b);
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
  __shared__ float red[4][64];
  const int64_t row = blockIdx.x;
  const int64_t off = row * p.cols;
  const float inv = 1.0f / (float)p.cols;
  float v[NC][8], xv[NC][8];                           // both streams are under way before the first sum
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    if (c < p.cols) {
      load8((const P*)p.h + off + c, v[k]);
      load8(p.x + off + c, xv[k]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = xv[k][i] = 0.f;
    }
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
      mean = block_sum2(s, 0.f, r0).x * inv;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      if ((int)(threadIdx.x + k * blockDim.x) * 8 >= p.cols) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) q += (v[k][i] - mean) * (v[k][i] - mean);
    }
    rstd = 1.0f / sqrtf(block_sum2(q, 0.f, r1).x * inv + p.eps);
  };
  auto normed = [&](int k, int i, float mean, float rstd, const float (&g)[8], const float (&b)[8]) {
    return (v[k][i] - mean) * rstd * g[i] + (KIND == 0 ? b[i] : 0.f);
  };
  float mean = 0.f, rstd = 0.f;
  if (p.gain1) moments(red[0], red[1], mean, rstd);
  if (threadIdx.x == 0) { p.stats[row] = mean; p.stats[p.rows + row] = rstd; }
  const P* gate = p.gate ? (const P*)p.gate + (row / p.rows_per_gate) * p.cols : nullptr;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    if (c >= p.cols) continue;
    float g[8], b[8];
    if (p.gain1) {
      load8((const P*)p.gain1 + c, g);
      if (KIND == 0) load8((const P*)p.bias1 + c, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = normed(k, i, mean, rstd, g, b);
    }
    if (gate) {
      load8(gate + c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] *= g[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[k][i] = fmaf(p.scale, xv[k][i], v[k][i]);
    store8(p.xo + off + c, v[k]);
  }
  mean = rstd = 0.f;
  if (p.gain2) moments(red[2], red[3], mean, rstd);
  if (threadIdx.x == 0) { p.stats[2 * p.rows + row] = mean; p.stats[3 * p.rows + row] = rstd; }
  if (!p.gain2) return;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    if (c >= p.cols) continue;
    float g[8], b[8], o[8];
    load8((const P*)p.gain2 + c, g);
    if (KIND == 0) load8((const P*)p.bias2 + c, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = normed(k, i, mean, rstd, g, b);
    store8((P*)p.y + off + c, o);
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
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// at most n of this thread's newest groups still under way
__device__ __forceinline__ void cp_async_wait_upto(int n) {
  if (n >= 3) cp_async_wait<3>();
  else if (n == 2) cp_async_wait<2>();
  else if (n == 1) cp_async_wait<1>();
  else cp_async_wait<0>();
}
// 16-byte units a thread stages per chunk of 8 columns: dy, x', dx', h
template <typename P> constexpr int join_units = 4 + 2 * ((int)sizeof(P) / 2);

// A block walks its rows; the column sums of its rows stay in registers (each thread owns its columns) and leave as one
// row of `partial` per plane: gain1, bias1, gain2, bias2, gate (the last only where a gate's rows are split).
// A row is two block-wide sums in sequence, so what bounds a plain loop over rows is latency (one row's loads, two sums, its
// stores: 502 us at 16384 x 4096 bf16).  Here the next `stages` rows are on their way into shared memory meanwhile: every thread
// copies the 16-byte units of its own columns and reads them back itself, so the copies need no barrier, and one block per SM
// keeps 100 to 200 KB of loads in flight.  STAGED = false (rows too wide for shared memory) loads directly.
template <typename P, int KIND, int NC, bool STAGED>
__global__ void __launch_bounds__(512) join_bwd_kernel(JoinBwd p) {
  constexpr int UP = (int)sizeof(P) / 2, UNITS = join_units<P>;     // units of an operand chunk; of a whole chunk
  extern __shared__ uint4 ring[];
  __shared__ float red[4][64];
  const float inv = 1.0f / (float)p.cols;
  const int64_t rg = p.rows_per_gate;
  const int tid = threadIdx.x, nt = blockDim.x;
  int64_t r0, r1;
  if (p.split > 0) {
    const int64_t gate = blockIdx.x / p.split, sub = blockIdx.x % p.split;
    const int64_t g0 = gate * rg, gn = min(rg, p.rows - g0), per = (gn + p.split - 1) / p.split;
    r0 = g0 + min(gn, sub * per);
    r1 = g0 + min(gn, (sub + 1) * per);
  } else {
    r0 = min(p.rows, (int64_t)blockIdx.x * p.gates_per_cta * rg);
    r1 = min(p.rows, r0 + p.gates_per_cta * rg);
  }
  auto slot = [&](int stage, int k, int unit) { return ring + ((stage * NC + k) * UNITS + unit) * nt + tid; };
  auto fetch = [&](int64_t row, int stage) {
    const int64_t off = row * p.cols;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + k * nt) * 8;
      if (c >= p.cols) continue;
      if (p.gain2) {
#pragma unroll
        for (int q = 0; q < UP; ++q) cp_async16(slot(stage, k, q), (const P*)p.dy + off + c + q * 4);
#pragma unroll
        for (int q = 0; q < 2; ++q) cp_async16(slot(stage, k, UP + q), p.xo + off + c + q * 4);
      }
      if (p.dxo) {
#pragma unroll
        for (int q = 0; q < 2; ++q) cp_async16(slot(stage, k, UP + 2 + q), p.dxo + off + c + q * 4);
      }
#pragma unroll
      for (int q = 0; q < UP; ++q) cp_async16(slot(stage, k, UP + 4 + q), (const P*)p.h + off + c + q * 4);
    }
  };
  auto words = [&](const uint4& a, const uint4& b, float (&v)[8]) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
  };
  // 8 columns of a stream: unit `u` of the staged row, or from memory
  auto get32 = [&](const float* base, int64_t off, int c, int stage, int k, int u, float (&v)[8]) {
    if (STAGED) words(*slot(stage, k, u), *slot(stage, k, u + 1), v);
    else load8(base + off + c, v);
  };
  auto getp = [&](const void* base, int64_t off, int c, int stage, int k, int u, float (&v)[8]) {
    if (!STAGED) { load8((const P*)base + off + c, v); return; }
    if (UP == 2) { words(*slot(stage, k, u), *slot(stage, k, u + UP - 1), v); return; }
    load8((const P*)slot(stage, k, u), v);
  };
  if (STAGED)
    for (int s = 0; s < p.stages; ++s) {
      if (r0 + s < r1) fetch(r0 + s, s);
      cp_async_commit();
    }
  float aq[NC][8], a1[NC][8], b1[NC][8], a2[NC][8], b2[NC][8];
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) aq[k][i] = a1[k][i] = b1[k][i] = a2[k][i] = b2[k][i] = 0.f;
  float st[4], sn[4] = {0.f, 0.f, 0.f, 0.f};                             // statistics, a row ahead
  if (r0 < r1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sn[i] = p.stats[i * p.rows + r0];
  }
  int64_t gate_row = r0 / rg, gate_end = (gate_row + 1) * rg;
  int stage = 0;
  for (int64_t row = r0; row < r1; ++row) {
    const int64_t off = row * p.cols;
    float d[NC][8], t[NC][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { st[i] = sn[i]; if (row + 1 < r1) sn[i] = p.stats[i * p.rows + row + 1]; }
    if (row == gate_end) { ++gate_row; gate_end += rg; }
    if (STAGED) cp_async_wait_upto(p.stages - 1);
    // d = dx' + N2'(dy; x')
    if (p.gain2) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = (tid + k * nt) * 8;
        if (c >= p.cols) continue;
        float g[8];
        getp(p.dy, off, c, stage, k, 0, d[k]);
        get32(p.xo, off, c, stage, k, UP, t[k]);
        load8((const P*)p.gain2 + c, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[k][i] = (t[k][i] - st[2]) * st[3];
          a2[k][i] += d[k][i] * t[k][i];
          if (KIND == 0) b2[k][i] += d[k][i];
          d[k][i] *= g[i];
          s1 += d[k][i];
          s2 += d[k][i] * t[k][i];
        }
      }
      const float2 s = block_sum2(KIND == 0 ? s1 : 0.f, s2, red[(row & 1) * 2]);
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = st[3] * (d[k][i] - (KIND == 0 ? s.x * inv : 0.f) - t[k][i] * (s.y * inv));
    } else {
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = 0.f;
    }
    const P* gate = p.gate ? (const P*)p.gate + gate_row * p.cols : nullptr;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + k * nt) * 8;
      if (c >= p.cols) continue;
      float w[8], q[8];
      if (p.dxo) {
        get32(p.dxo, off, c, stage, k, UP + 2, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] += w[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = p.scale * d[k][i];
      store8(p.dx + off + c, w);
      getp(p.h, off, c, stage, k, UP + 4, t[k]);
      if (gate) load8(gate + c, q);
      if (p.gain1) {
        float g[8], b[8];
        load8((const P*)p.gain1 + c, g);
        if (KIND == 0 && p.bias1) load8((const P*)p.bias1 + c, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[k][i] = (t[k][i] - st[0]) * st[1];
          if (gate) {
            aq[k][i] += d[k][i] * (t[k][i] * g[i] + (KIND == 0 && p.bias1 ? b[i] : 0.f));
            d[k][i] *= q[i];
          }
          a1[k][i] += d[k][i] * t[k][i];
          if (KIND == 0) b1[k][i] += d[k][i];
          d[k][i] *= g[i];
          s1 += d[k][i];
          s2 += d[k][i] * t[k][i];
        }
      } else if (gate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { aq[k][i] += d[k][i] * t[k][i]; d[k][i] *= q[i]; }
      }
    }
    if (STAGED) {                                                        // this row's slot has been read: the row after the staged ones
      if (row + p.stages < r1) fetch(row + p.stages, stage);
      cp_async_commit();
      if (++stage == p.stages) stage = 0;
    }
    float2 s = make_float2(0.f, 0.f);
    if (p.gain1) s = block_sum2(KIND == 0 ? s1 : 0.f, s2, red[(row & 1) * 2 + 1]);
    const bool gate_done = p.split == 0 && gate && (row + 1 == r1 || row + 1 == gate_end);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (tid + k * nt) * 8;
      if (c >= p.cols) continue;
      if (p.gain1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = st[1] * (d[k][i] - (KIND == 0 ? s.x * inv : 0.f) - t[k][i] * (s.y * inv));
      }
      store8((P*)p.dh + off + c, d[k]);
      if (gate_done) {
        if (p.dgate) store8(p.dgate + gate_row * p.cols + c, aq[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) aq[k][i] = 0.f;
      }
    }
  }
  const size_t plane = (size_t)p.ctas * p.cols;
  float* out = p.partial + (size_t)blockIdx.x * p.cols;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (tid + k * nt) * 8;
    if (c >= p.cols) continue;
    if (p.gain1) store8(out + c, a1[k]);
    if (KIND == 0 && p.gain1) store8(out + plane + c, b1[k]);
    if (p.gain2) store8(out + 2 * plane + c, a2[k]);
    if (KIND == 0 && p.gain2) store8(out + 3 * plane + c, b2[k]);
    if (p.split > 0 && p.gate) store8(out + 4 * plane + c, aq[k]);
  }
  pdl_launch_next();
}

struct JoinSums { float* out[kJoinPlanes]; };     // nullptr: not wanted
// Sums the planes of `partial` over the blocks, in a fixed order: blockIdx.y = plane; the gate's plane holds one sum per
// gate, over the `split` blocks of that gate.  32 columns x 32 runs of blocks per CUDA block.
__global__ void __launch_bounds__(1024) join_sums_kernel(const float* __restrict__ partial, JoinSums o, int ctas, int cols, int split) {
  __shared__ double sh[32][33];
  const int plane = min((int)blockIdx.y, kJoinPlanes - 1);
  const int gate = (int)blockIdx.y - (kJoinPlanes - 1);
  float* out = o.out[plane];
  if (out == nullptr) return;
  const int c0 = plane == kJoinPlanes - 1 ? gate * split : 0, cn = plane == kJoinPlanes - 1 ? split : ctas;
  const int col = blockIdx.x * 32 + threadIdx.x;
  pdl_wait_prior();
  double a = 0.0;
  if (col < cols) {
    const float* src = partial + ((size_t)plane * ctas + c0) * cols + col;
#pragma unroll 4
    for (int i = threadIdx.y; i < cn; i += 32) a += src[(size_t)i * cols];
  }
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  // warp y joins column y: lane = run
  double b = sh[threadIdx.x][threadIdx.y];
  for (int k = 16; k > 0; k >>= 1) b += __shfl_xor_sync(0xffffffffu, b, k);
  const int mine = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && mine < cols) out[(plane == kJoinPlanes - 1 ? (size_t)gate * cols : 0) + mine] = (float)b;
}

}  // namespace hift
