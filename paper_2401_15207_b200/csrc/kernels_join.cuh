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
constexpr int kJoinCtas = 592;         // most row chunks of a backward call: 4 per SM
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
  float v[NC][8];
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    if (c < p.cols) load8((const P*)p.h + off + c, v[k]);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
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
    float xv[8], g[8], b[8];
    load8(p.x + off + c, xv);
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
    for (int i = 0; i < 8; ++i) v[k][i] = fmaf(p.scale, xv[i], v[k][i]);
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
  int cols, ctas;
  int split;               // > 0: every gate's rows are split over `split` blocks; 0: a block takes whole gates
  int64_t gates_per_cta;   // split == 0
  float scale;
};

// A block walks its rows; the column sums of its rows stay in registers (each thread owns its columns) and leave as one
// row of `partial` per plane: gain1, bias1, gain2, bias2, gate (the last only where a gate's rows are split).
template <typename P, int KIND, int NC>
__global__ void __launch_bounds__(512) join_bwd_kernel(JoinBwd p) {
  __shared__ float red[4][64];
  const float inv = 1.0f / (float)p.cols;
  const int64_t rg = p.rows_per_gate;
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
  float aq[NC][8], a1[NC][8], b1[NC][8], a2[NC][8], b2[NC][8];
#pragma unroll
  for (int k = 0; k < NC; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) aq[k][i] = a1[k][i] = b1[k][i] = a2[k][i] = b2[k][i] = 0.f;
  for (int64_t row = r0; row < r1; ++row) {
    const int64_t off = row * p.cols;
    float d[NC][8], t[NC][8];
    const float mean1 = p.stats[row], rstd1 = p.stats[p.rows + row];
    // d = dx' + N2'(dy; x')
    if (p.gain2) {
      const float mean2 = p.stats[2 * p.rows + row], rstd2 = p.stats[3 * p.rows + row];
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int c = (threadIdx.x + k * blockDim.x) * 8;
        if (c >= p.cols) continue;
        float g[8];
        load8((const P*)p.dy + off + c, d[k]);
        load8(p.xo + off + c, t[k]);
        load8((const P*)p.gain2 + c, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[k][i] = (t[k][i] - mean2) * rstd2;
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
        for (int i = 0; i < 8; ++i) d[k][i] = rstd2 * (d[k][i] - (KIND == 0 ? s.x * inv : 0.f) - t[k][i] * (s.y * inv));
    } else {
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = 0.f;
    }
    const P* gate = p.gate ? (const P*)p.gate + (row / rg) * p.cols : nullptr;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (threadIdx.x + k * blockDim.x) * 8;
      if (c >= p.cols) continue;
      float w[8], q[8];
      if (p.dxo) {
        load8(p.dxo + off + c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] += w[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = p.scale * d[k][i];
      store8(p.dx + off + c, w);
      load8((const P*)p.h + off + c, t[k]);
      if (gate) load8(gate + c, q);
      if (p.gain1) {
        float g[8], b[8];
        load8((const P*)p.gain1 + c, g);
        if (KIND == 0 && p.bias1) load8((const P*)p.bias1 + c, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[k][i] = (t[k][i] - mean1) * rstd1;
          if (gate) {
            aq[k][i] += d[k][i] * (t[k][i] * g[i] + (KIND == 0 ? b[i] : 0.f));
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
    float2 s = make_float2(0.f, 0.f);
    if (p.gain1) s = block_sum2(KIND == 0 ? s1 : 0.f, s2, red[(row & 1) * 2 + 1]);
    const bool gate_done = gate && (row + 1 == r1 || (row + 1) % rg == 0);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int c = (threadIdx.x + k * blockDim.x) * 8;
      if (c >= p.cols) continue;
      if (p.gain1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = rstd1 * (d[k][i] - (KIND == 0 ? s.x * inv : 0.f) - t[k][i] * (s.y * inv));
      }
      store8((P*)p.dh + off + c, d[k]);
      if (gate_done && p.split == 0) {
        if (p.dgate) store8(p.dgate + (row / rg) * p.cols + c, aq[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) aq[k][i] = 0.f;
      }
    }
  }
  const size_t plane = (size_t)p.ctas * p.cols;
  float* out = p.partial + (size_t)blockIdx.x * p.cols;
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    if (c >= p.cols) continue;
    store8(out + c, a1[k]);
    if (KIND == 0) store8(out + plane + c, b1[k]);
    store8(out + 2 * plane + c, a2[k]);
    if (KIND == 0) store8(out + 3 * plane + c, b2[k]);
    if (p.split > 0) store8(out + 4 * plane + c, aq[k]);
  }
}

struct JoinSums { float* out[kJoinPlanes]; };     // nullptr: not wanted
// Sums the planes of `partial` over the blocks, in a fixed order: blockIdx.y = plane; the gate's plane holds one sum per
// gate, over the `split` blocks of that gate.
__global__ void join_sums_kernel(const float* __restrict__ partial, JoinSums o, int ctas, int cols, int split) {
  __shared__ double sh[8][33];
  const int plane = min((int)blockIdx.y, kJoinPlanes - 1);
  const int gate = (int)blockIdx.y - (kJoinPlanes - 1);
  float* out = o.out[plane];
  if (out == nullptr) return;
  const int c0 = plane == kJoinPlanes - 1 ? gate * split : 0, cn = plane == kJoinPlanes - 1 ? split : ctas;
  const int col = blockIdx.x * 32 + threadIdx.x;
  double a = 0.0;
  if (col < cols)
    for (int i = threadIdx.y; i < cn; i += 8) a += partial[((size_t)plane * ctas + c0 + i) * cols + col];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y == 0 && col < cols) {
    for (int i = 1; i < 8; ++i) a += sh[i][threadIdx.x];
    out[(plane == kJoinPlanes - 1 ? (size_t)gate * cols : 0) + col] = (float)a;
  }
}

}  // namespace hift
