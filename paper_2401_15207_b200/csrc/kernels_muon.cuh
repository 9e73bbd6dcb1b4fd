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

// Blocks are 256 threads as 256 / tx rows of tx threads, 4 columns a thread: a matrix row is walked without an index division.
// VEC: rows of the caller's matrices start on 16-byte boundaries (8-byte for bf16), so the 4 columns move at once.
template <bool VEC, typename T>
__device__ __forceinline__ void ns_ld4(const T* p, int left, float (&v)[4]) {       // left: columns that exist from here on
  if (VEC) {
    if (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(p);
      v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u); v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = k < left ? to_f(p[k]) : 0.f;
}
template <bool VEC>
__device__ __forceinline__ void ns_st4(float* p, int left, const float (&v)[4]) {
  if (VEC) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
  for (int k = 0; k < 4; ++k) if (k < left) p[k] = v[k];
}
template <bool VEC>
__device__ __forceinline__ void ns_st4(bf16* p, int left, const float (&v)[4]) {
  if (VEC) {
    uint2 a;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&a);
    h[0] = __floats2bfloat162_rn(v[0], v[1]);
    h[1] = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = a;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) if (k < left) p[k] = __float2bfloat16_rn(v[k]);
}

// momentum update (mom != nullptr) and the sum of squares of what will be orthogonalised, one double per block
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) ns_sumsq_kernel(const T* g, float* mom, int rows, int cols, float mu, int nesterov,
                                                       double* part) {
  __shared__ double sh[8];
  const int tid = threadIdx.y * blockDim.x + threadIdx.x;
  double s = 0.0;
  pdl_wait_prior();
  for (int r = blockIdx.x * blockDim.y + threadIdx.y; r < rows; r += gridDim.x * blockDim.y) {
    const size_t off = (size_t)r * cols;
#pragma unroll 2
    for (int c = threadIdx.x * 4; c < cols; c += blockDim.x * 4) {
      float u[4];
      ns_ld4<VEC>(g + off + c, cols - c, u);
      if (mom) {
        float m[4];
        ns_ld4<VEC>(mom + off + c, cols - c, m);
#pragma unroll
        for (int k = 0; k < 4; ++k) { m[k] = fmaf(mu, m[k], u[k]); u[k] = nesterov ? fmaf(mu, m[k], u[k]) : m[k]; }
        ns_st4<VEC>(mom + off + c, cols - c, m);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) s = fma((double)u[k], (double)u[k], s);
    }
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) sh[tid >> 5] = s;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < 8; ++i) s += sh[i];
    part[blockIdx.x] = s;
  }
}
// X_0 = U / |U| into the zero-padded scratch, fp32 and as the first products' fp16 operand.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) ns_start_kernel(const T* g, const float* mom, int rows, int cols, float mu, int nesterov,
                                                       const double* part, int nparts, int prows, int pcols, float* x32,
                                                       __half* x16, int* verdict) {
  __shared__ double sh[8];
  __shared__ float s_inv;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x;
  double s = 0.0;
  pdl_wait_prior();
  if (blockIdx.x == 0 && tid == 0) *verdict = 0;        // for ns_finish_kernel
  for (int i = tid; i < nparts; i += 256) s += part[i];
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) sh[tid >> 5] = s;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < 8; ++i) s += sh[i];
    const double n = sqrt(s);
    s_inv = (float)(1.0 / (n < 1e-30 ? 1e-30 : n));     // a NaN stays one
  }
  __syncthreads();
  const float inv = s_inv;
  for (int r = blockIdx.x * blockDim.y + threadIdx.y; r < prows; r += gridDim.x * blockDim.y) {
    const size_t off = (size_t)r * cols;
#pragma unroll 2
    for (int c = threadIdx.x * 4; c < pcols; c += blockDim.x * 4) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (r < rows && c < cols) {
        ns_ld4<VEC>(g + off + c, cols - c, v);
        if (mom) {
          float m[4];
          ns_ld4<VEC>(mom + off + c, cols - c, m);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = nesterov ? fmaf(mu, m[k], v[k]) : m[k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] *= inv;
      }
      *reinterpret_cast<float4*>(x32 + (size_t)r * pcols + c) = make_float4(v[0], v[1], v[2], v[3]);
      __half2 h[2] = {__floats2half2_rn(v[0] * kNsOperandScale, v[1] * kNsOperandScale), __floats2half2_rn(v[2] * kNsOperandScale, v[3] * kNsOperandScale)};
      *reinterpret_cast<uint2*>(x16 + (size_t)r * pcols + c) = *reinterpret_cast<uint2*>(h);
    }
  }
  pdl_launch_next();
}
// The result out of the padded scratch: o in bf16, or the update of the master.  Writes nothing after a product gave up on a wait: the first
// block to come reads the flag for all, since another stream's products may raise it while this kernel runs, and no matrix is to be half updated.
template <bool VEC>
__global__ void __launch_bounds__(256) ns_finish_kernel(const float* x, int rows, int cols, int pcols, bf16* o,
                                                        float* master, bf16* param, float decay, float size,
                                                        const int* tc_error, int* verdict) {
  __shared__ int go;
  pdl_wait_prior();
  if (threadIdx.x == 0 && threadIdx.y == 0) {
    const int mine = *(const volatile int*)tc_error != 0 ? 2 : 1, first = atomicCAS(verdict, 0, mine);
    go = (first == 0 ? mine : first) == 1;
  }
  __syncthreads();
  if (!go) return;
  for (int r = blockIdx.x * blockDim.y + threadIdx.y; r < rows; r += gridDim.x * blockDim.y) {
    const size_t off = (size_t)r * cols;
#pragma unroll 2
    for (int c = threadIdx.x * 4; c < cols; c += blockDim.x * 4) {
      float v[4];
      ns_ld4<true>(x + (size_t)r * pcols + c, 4, v);
      if (o) ns_st4<VEC>(o + off + c, cols - c, v);
      if (master) {
        float t[4];
        ns_ld4<VEC>(master + off + c, cols - c, t);
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = t[k] * decay - size * v[k];
        ns_st4<VEC>(master + off + c, cols - c, t);
        if (param) ns_st4<VEC>(param + off + c, cols - c, t);
      }
    }
  }
}

inline int ns_pad(int64_t n) { return n < 128 ? 128 : (int)((n + 63) / 64 * 64); }
// scratch: partial sums, the verdict on the result behind them | x32 | x16 twice | e | f | da | df, each a multiple of 256 bytes
inline size_t ns_scratch_bytes(int64_t rows, int64_t cols) {
  const size_t r = ns_pad(rows), c = ns_pad(cols), s = r < c ? r : c;
  return ((size_t)kNsParts * 8 + 8 + 255) / 256 * 256 + r * c * 8 + s * s * 4 + 2 * ((s * 4 + 255) / 256 * 256);
}
struct NsUpdate { bf16* o; float* master; bf16* param; float decay, size; };   // where the result goes: o, or master (and param)

template <typename T>
inline cudaError_t launch_orthogonalize(cudaStream_t st, int64_t rows, int64_t cols, const T* g, float* mom, float mu, int nesterov,
                                        int steps, const NsUpdate& to, void* scratch) {
  const int* flag = ns_device_flag();                  // sets this device up
  if (!flag) return cudaErrorNotSupported;
  if (ns_small_eligible(rows, cols))
    return ns_small_launch(st, sizeof(T) == 2, rows, cols, g, mom, mu, nesterov, steps, to.o, to.master, to.param, to.decay, to.size);
  const int pr = ns_pad(rows), pc = ns_pad(cols), s = pr < pc ? pr : pc;
  char* w = (char*)scratch;
  auto take = [&](size_t bytes) { char* p = w; w += (bytes + 255) / 256 * 256; return p; };
  double* part = (double*)take(kNsParts * 8 + 8);
  int* verdict = (int*)(part + kNsParts);
  NsBuffers b;
  b.rows = pr; b.cols = pc;
  b.x32 = (float*)take((size_t)pr * pc * 4);
  b.x16[0] = take((size_t)pr * pc * 2);
  b.x16[1] = take((size_t)pr * pc * 2);
  b.e = take((size_t)s * s * 2);
  b.f = take((size_t)s * s * 2);
  b.da = (float*)take((size_t)s * 4);
  b.df = (float*)take((size_t)s * 4);
  // threads across a row, rows per block, blocks
  int tx = 32;
  while (tx < 256 && tx * 4 < pc) tx *= 2;
  const dim3 block(tx, 256 / tx);
  auto blocks = [&](int r) { const int b = (r + (int)block.y - 1) / (int)block.y; return dim3((unsigned)(b < kNsParts ? b : kNsParts)); };
  const dim3 grid = blocks((int)rows), pgrid = blocks(pr);
  auto at = [](const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; };
  const bool vec = cols % 4 == 0 && at(g, 4 * sizeof(T)) && at(mom, 16) && at(to.o, 8) && at(to.master, 16) && at(to.param, 8);
  const int R = (int)rows, C = (int)cols;
  cudaError_t e = launch_pdl(vec ? ns_sumsq_kernel<T, true> : ns_sumsq_kernel<T, false>, grid, block, 0, st, g, mom, R, C, mu, nesterov, part);
  if (e != cudaSuccess) return e;
  e = vec ? launch_pdl(ns_start_kernel<T, true>, pgrid, block, 0, st, g, (const float*)mom, R, C, mu, nesterov, (const double*)part, (int)grid.x, pr, pc, b.x32, (__half*)b.x16[0], verdict)
          : launch_pdl(ns_start_kernel<T, false>, pgrid, block, 0, st, g, (const float*)mom, R, C, mu, nesterov, (const double*)part, (int)grid.x, pr, pc, b.x32, (__half*)b.x16[0], verdict);
  if (e != cudaSuccess) return e;
  e = ns_products_launch(st, b, steps);
  if (e != cudaSuccess) return e;
  return vec ? launch_pdl(ns_finish_kernel<true>, grid, block, 0, st, (const float*)b.x32, R, C, pc, to.o, to.master, to.param, to.decay, to.size, flag, verdict)
             : launch_pdl(ns_finish_kernel<false>, grid, block, 0, st, (const float*)b.x32, R, C, pc, to.o, to.master, to.param, to.decay, to.size, flag, verdict);
}

}  // namespace hift
