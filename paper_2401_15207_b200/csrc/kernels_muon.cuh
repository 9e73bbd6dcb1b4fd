// Orthogonalised update of a weight matrix by Newton-Schulz products.
//
//   X_0 = G / |G|_F;  X <- a X + (b A + c A A) X,  A = X X^T taken on the short side  (right-hand products if rows > cols)
// maps every singular value s of X to a s + b s^3 + c s^5, which pushes all of them towards 1 in a few steps; X_steps is
// close to the orthogonal factor of G.  The update:  U = momentum' (or g + mu momentum'),  momentum' = mu momentum + g,
//   theta <- theta (1 - lr wd) - lr 0.2 sqrt(max(rows, cols)) X(U).
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "gemm_tc.h"

namespace hift {

constexpr float kNsOperandScale = 1024.0f;    // of the iterate's fp16 image (kNsScale in ns_epilogue.cuh)
constexpr int kNsParts = 592;

// momentum update (mom != nullptr) and the sum of squares of what will be orthogonalised, one double per block
template <typename T>
__global__ void ns_sumsq_kernel(const T* __restrict__ g, float* __restrict__ mom, size_t n, float mu, int nesterov,
                                double* __restrict__ part) {
  __shared__ double sh[32];
  double s = 0.0;
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
    float u = to_f(g[i]);
    if (mom) {
      const float m = fmaf(mu, mom[i], u);
      mom[i] = m;
      u = nesterov ? fmaf(mu, m, u) : m;
    }
    s += (double)u * u;
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < (int)blockDim.x / 32; ++i) s += sh[i];
    part[blockIdx.x] = s;
  }
}
// X_0 = U / |U| into the zero-padded scratch, fp32 and as the first products' fp16 operand.  One thread per 4 columns of a row.
template <typename T>
__global__ void ns_start_kernel(const T* __restrict__ g, const float* __restrict__ mom, int rows, int cols, float mu, int nesterov,
                                const double* __restrict__ part, int nparts, int prows, int pcols, float* __restrict__ x32, __half* __restrict__ x16) {
  __shared__ double sh[32];
  __shared__ float s_inv;
  double s = 0.0;
  for (int i = threadIdx.x; i < nparts; i += blockDim.x) s += part[i];
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < (int)blockDim.x / 32; ++i) s += sh[i];
    const double n = sqrt(s);
    s_inv = (float)(1.0 / (n < 1e-30 ? 1e-30 : n));     // a NaN stays one
  }
  __syncthreads();
  const float inv = s_inv;
  const int q = pcols / 4;
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < (size_t)prows * q; i += (size_t)gridDim.x * blockDim.x) {
    const int r = (int)(i / q), c = (int)(i % q) * 4;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = 0.f;
      if (r < rows && c + k < cols) {
        const size_t at = (size_t)r * cols + c + k;
        float u = to_f(g[at]);
        if (mom) u = nesterov ? fmaf(mu, mom[at], u) : mom[at];
        v[k] = u * inv;
      }
    }
    *reinterpret_cast<float4*>(x32 + (size_t)r * pcols + c) = make_float4(v[0], v[1], v[2], v[3]);
    __half2 h[2] = {__floats2half2_rn(v[0] * kNsOperandScale, v[1] * kNsOperandScale), __floats2half2_rn(v[2] * kNsOperandScale, v[3] * kNsOperandScale)};
    *reinterpret_cast<uint2*>(x16 + (size_t)r * pcols + c) = *reinterpret_cast<uint2*>(h);
  }
}
// The result out of the padded scratch: o in bf16, or the update of the master.  Writes nothing after a product gave up on a wait.
__global__ void ns_finish_kernel(const float* __restrict__ x, int rows, int cols, int pcols, bf16* __restrict__ o, float* __restrict__ master,
                                 bf16* __restrict__ param, float decay, float size, const int* __restrict__ tc_error) {
  if (tc_error != nullptr && *tc_error != 0) return;
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < (size_t)rows * cols; i += (size_t)gridDim.x * blockDim.x) {
    const float v = x[(i / cols) * pcols + i % cols];
    if (o) o[i] = __float2bfloat16_rn(v);
    if (master) {
      const float t = master[i] * decay - size * v;
      master[i] = t;
      if (param) param[i] = __float2bfloat16_rn(t);
    }
  }
}

inline int ns_pad(int64_t n) { return n < 128 ? 128 : (int)((n + 63) / 64 * 64); }
// scratch: partial sums | x32 | x16 twice | e | f | da | df, each a multiple of 256 bytes
inline size_t ns_scratch_bytes(int64_t rows, int64_t cols) {
  const size_t r = ns_pad(rows), c = ns_pad(cols), s = r < c ? r : c;
  return ((size_t)kNsParts * 8 + 255) / 256 * 256 + r * c * 8 + s * s * 4 + 2 * ((s * 4 + 255) / 256 * 256);
}
struct NsUpdate { bf16* o; float* master; bf16* param; float decay, size; };   // where the result goes: o, or master (and param)

template <typename T>
inline cudaError_t launch_orthogonalize(cudaStream_t st, int64_t rows, int64_t cols, const T* g, float* mom, float mu, int nesterov,
                                        int steps, const NsUpdate& to, void* scratch) {
  const size_t n = (size_t)rows * cols;
  const int pr = ns_pad(rows), pc = ns_pad(cols), s = pr < pc ? pr : pc;
  char* w = (char*)scratch;
  auto take = [&](size_t bytes) { char* p = w; w += (bytes + 255) / 256 * 256; return p; };
  double* part = (double*)take(kNsParts * 8);
  NsBuffers b;
  b.rows = pr; b.cols = pc;
  b.x32 = (float*)take((size_t)pr * pc * 4);
  b.x16[0] = take((size_t)pr * pc * 2);
  b.x16[1] = take((size_t)pr * pc * 2);
  b.e = take((size_t)s * s * 2);
  b.f = take((size_t)s * s * 2);
  b.da = (float*)take((size_t)s * 4);
  b.df = (float*)take((size_t)s * 4);
  const int grid = (int)((n + 255) / 256 < kNsParts ? (n + 255) / 256 : kNsParts);
  const size_t np = (size_t)pr * pc / 4;
  const int pgrid = (int)((np + 255) / 256 < 2 * kNsParts ? (np + 255) / 256 : 2 * kNsParts);
  ns_sumsq_kernel<T><<<grid, 256, 0, st>>>(g, mom, n, mu, nesterov, part);
  ns_start_kernel<T><<<pgrid, 256, 0, st>>>(g, mom, (int)rows, (int)cols, mu, nesterov, part, grid, pr, pc, b.x32, (__half*)b.x16[0]);
  const cudaError_t e = ns_products_launch(st, b, steps);
  if (e != cudaSuccess) return e;
  ns_finish_kernel<<<grid, 256, 0, st>>>(b.x32, (int)rows, (int)cols, pc, to.o, to.master, to.param, to.decay, to.size, gemm_tc_error_device_ptr());
  return cudaGetLastError();
}

}  // namespace hift
