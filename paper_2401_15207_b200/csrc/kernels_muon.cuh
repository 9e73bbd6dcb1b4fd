// Orthogonalised update of a weight matrix by Newton-Schulz products.
//
//   X_0 = G / |G|_F;  X <- a X + (b A + c A A) X,  A = X X^T taken on the short side  (right-hand products if rows > cols)
// maps every singular value s of X to a s + b s^3 + c s^5, which pushes all of them towards 1 in a few steps; X_steps is
// close to the orthogonal factor of G.  The update:  U = momentum' (or g + mu momentum'),  momentum' = mu momentum + g,
//   theta <- theta (1 - lr wd) - lr 0.2 sqrt(max(rows, cols)) X(U).
#pragma once
#include "common.cuh"

namespace hift {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
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
template <typename T>
__global__ void ns_start_kernel(const T* __restrict__ g, const float* __restrict__ mom, size_t n, float mu, int nesterov,
                                const double* __restrict__ part, int nparts, float* __restrict__ x) {
  double s = 0.0;
  for (int i = 0; i < nparts; ++i) s += part[i];
  const float norm = (float)sqrt(s), inv = norm > 1e-30f ? 1.0f / norm : 1e30f;
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
    float u = to_f(g[i]);
    if (mom) u = nesterov ? fmaf(mu, mom[i], u) : mom[i];
    x[i] = u * inv;
  }
}
// C[m, n] = alpha sum_k A(m, k) B(k, n) + beta D[m, n], fp32; C and D row-major with leading dimension N
__global__ void ns_product_kernel(int M, int N, int K, const float* __restrict__ a, int64_t sam, int64_t sak, const float* __restrict__ b,
                                  int64_t sbk, int64_t sbn, float alpha, float beta, const float* __restrict__ d, float* __restrict__ c) {
  __shared__ float sa[16][17], sb[16][17];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int tn = (N + 15) / 16;
  const int m = (int)(blockIdx.x / tn) * 16 + ty, n = (int)(blockIdx.x % tn) * 16 + tx;
  float acc = 0.f;
  for (int k0 = 0; k0 < K; k0 += 16) {
    sa[ty][tx] = m < M && k0 + tx < K ? a[m * sam + (k0 + tx) * sak] : 0.f;
    sb[ty][tx] = n < N && k0 + ty < K ? b[(k0 + ty) * sbk + n * sbn] : 0.f;
    __syncthreads();
    for (int k = 0; k < 16; ++k) acc = fmaf(sa[ty][k], sb[k][tx], acc);
    __syncthreads();
  }
  if (m < M && n < N) c[(int64_t)m * N + n] = alpha * acc + (d ? beta * d[(int64_t)m * N + n] : 0.f);
}
__global__ void ns_finish_kernel(const float* __restrict__ x, size_t n, bf16* __restrict__ o, float* __restrict__ master,
                                 bf16* __restrict__ param, float decay, float size) {
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
    if (o) o[i] = __float2bfloat16_rn(x[i]);
    if (master) {
      const float t = master[i] * decay - size * x[i];
      master[i] = t;
      if (param) param[i] = __float2bfloat16_rn(t);
    }
  }
}

inline size_t ns_scratch_bytes(int64_t rows, int64_t cols) {
  const size_t k = (size_t)(rows < cols ? rows : cols);
  return kNsParts * sizeof(double) + sizeof(float) * (2 * (size_t)rows * cols + 2 * k * k);
}
struct NsUpdate { bf16* o; float* master; bf16* param; float decay, size; };   // where the result goes: o, or master (and param)

template <typename T>
inline cudaError_t launch_orthogonalize(cudaStream_t st, int64_t rows, int64_t cols, const T* g, float* mom, float mu, int nesterov,
                                        int steps, const NsUpdate& to, void* scratch) {
  const size_t n = (size_t)rows * cols, k = (size_t)(rows < cols ? rows : cols);
  double* part = (double*)scratch;
  float* x = (float*)(part + kNsParts);
  float *y = x + n, *A = y + n, *B = A + k * k;
  const int grid = (int)((n + 255) / 256 < kNsParts ? (n + 255) / 256 : kNsParts);
  ns_sumsq_kernel<T><<<grid, 256, 0, st>>>(g, mom, n, mu, nesterov, part);
  ns_start_kernel<T><<<grid, 256, 0, st>>>(g, mom, n, mu, nesterov, part, grid, x);
  const int R = (int)rows, C = (int)cols, S = (int)k;
  const unsigned gs = (unsigned)(((k + 15) / 16) * ((k + 15) / 16)), gx = (unsigned)(((rows + 15) / 16) * ((cols + 15) / 16));
  for (int i = 0; i < steps; ++i) {
    if (rows <= cols) ns_product_kernel<<<gs, 256, 0, st>>>(S, S, C, x, C, 1, x, 1, C, 1.f, 0.f, nullptr, A);
    else ns_product_kernel<<<gs, 256, 0, st>>>(S, S, R, x, 1, C, x, C, 1, 1.f, 0.f, nullptr, A);
    ns_product_kernel<<<gs, 256, 0, st>>>(S, S, S, A, S, 1, A, S, 1, kNsC, kNsB, A, B);
    if (rows <= cols) ns_product_kernel<<<gx, 256, 0, st>>>(R, C, S, B, S, 1, x, C, 1, 1.f, kNsA, x, y);
    else ns_product_kernel<<<gx, 256, 0, st>>>(R, C, S, x, C, 1, B, S, 1, 1.f, kNsA, x, y);
    float* t = x; x = y; y = t;
  }
  ns_finish_kernel<<<grid, 256, 0, st>>>(x, n, to.o, to.master, to.param, to.decay, to.size);
  return cudaGetLastError();
}

}  // namespace hift
