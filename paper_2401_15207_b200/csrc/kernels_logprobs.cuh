// Log-probabilities of given tokens, the entropy and the most likely alternatives of rows of logits, and the gradient of
// the first two into the logits.
//
//   z_i = x_i / T,  m = max_i x_i,  r = sum over i, without one occurrence of the maximum, of exp((x_i - m) / T)
//   L = log(1 + r),  log p_i = (x_i - m) / T - L
//   H = -sum_i p_i log p_i = L - sum_i exp((x_i - m) / T) (x_i - m) / T / (1 + r)
//   d x_i = (1 / T) ( g (delta_it - p_i) - h p_i (log p_i + H) )          g = d log p_t, h = d H
// The maximum's own 1 is kept out of r, so that log1p(r) is exact to fp32 for a row that is nearly sure of one token.
#pragma once
#include "common.cuh"

namespace hift {


constexpr float kLowest = -3.402823466e38f;

// One block per row, three passes over the row, then one pass per alternative.
template <typename T>
__global__ void token_logprobs_kernel(const T* __restrict__ logits, const int32_t* __restrict__ tokens, int vocab, int64_t ld,
                                      int64_t rows, float scale, int n_top, float* __restrict__ logp, float* __restrict__ entropy,
                                      float* __restrict__ stats, int32_t* __restrict__ top_ids, float* __restrict__ top_logp,
                                      int32_t* __restrict__ bad) {
  __shared__ float red[33];
  __shared__ int first_max;
  __shared__ unsigned long long best;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  const int tok = tokens[row];
  if (tok < 0 || tok >= vocab) {
    if (threadIdx.x == 0) {
      if (tok >= vocab && bad) *bad = 1;
      logp[row] = 0.f;
      if (entropy) entropy[row] = 0.f;
      if (stats) { stats[row] = 0.f; stats[rows + row] = 0.f; }
      for (int k = 0; k < n_top; ++k) { top_ids[row * n_top + k] = -1; top_logp[row * n_top + k] = -INFINITY; }
    }
    return;
  }
  float mx = -INFINITY;
  for (int c = threadIdx.x; c < vocab; c += blockDim.x) mx = fmaxf(mx, to_f(x[c]));
  mx = block_max(mx, red);
  const bool none = mx == -INFINITY;                              // nothing above -inf, but for NaN
  mx = fmaxf(mx, kLowest);
  if (threadIdx.x == 0) first_max = vocab;
  __syncthreads();
  for (int c = threadIdx.x; c < vocab; c += blockDim.x) if (to_f(x[c]) == mx) { atomicMin(&first_max, c); break; }
  __syncthreads();
  float r = 0.f, u = 0.f;
  for (int c = threadIdx.x; c < vocab; c += blockDim.x) {
    const float t = (to_f(x[c]) - mx) * scale, e = expf(t);     // a NaN, or +inf - +inf, makes r NaN
    if (c != first_max) r += e;
    u += e > 0.f ? e * t : 0.f;
  }
  r = block_sum(r, red);
  u = block_sum(u, red);
  const float nanv = __int_as_float(0x7fc00000);
  const bool poison = !(r < INFINITY) || mx == INFINITY, empty = none && !poison;
  const float L = log1pf(r);
  if (threadIdx.x == 0) {
    logp[row] = empty ? -INFINITY : poison ? nanv : (to_f(x[tok]) - mx) * scale - L;
    if (entropy) entropy[row] = empty ? 0.f : poison ? nanv : L - u / (1.0f + r);
    if (stats) { stats[row] = poison ? nanv : empty ? -INFINITY : mx; stats[rows + row] = empty ? 0.f : poison ? nanv : L; }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < n_top; ++k) {
    unsigned long long mine = 0ull;
    if (threadIdx.x == 0) best = 0ull;
    __syncthreads();
    if (!empty && !poison) {
      for (int c = threadIdx.x; c < vocab; c += blockDim.x) {
        const float v = to_f(x[c]);
        if (v == -INFINITY) continue;
        uint32_t o = __float_as_uint(v + 0.0f);
        o = (o & 0x80000000u) ? ~o : (o | 0x80000000u);
        const unsigned long long key = ((unsigned long long)o << 32) | (uint32_t)~c;
        if (key < last && key > mine) mine = key;
      }
      if (mine) atomicMax(&best, mine);
    }
    __syncthreads();
    last = best;
    if (threadIdx.x == 0) {
      const int c = last ? (int)~(uint32_t)last : -1;
      top_ids[row * n_top + k] = c;
      top_logp[row * n_top + k] = poison ? nanv : c < 0 ? -INFINITY : (to_f(x[c]) - mx) * scale - L;
    }
    __syncthreads();
    if (last == 0ull) last = 1ull;                               // nothing left: nothing is below this key
  }
}

// One block per row: the gradient from the saved maximum, L and H.
template <typename T>
__global__ void token_logprobs_bwd_kernel(const T* __restrict__ logits, const int32_t* __restrict__ tokens, int vocab, int64_t ld,
                                          int64_t rows, float scale, const float* __restrict__ stats, const float* __restrict__ entropy,
                                          const float* __restrict__ dlogp, const float* __restrict__ dentropy, T* __restrict__ dlogits) {
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  T* d = dlogits + row * ld;
  const int tok = tokens[row];
  const float m = stats[row], L = stats[rows + row];
  if (tok < 0 || tok >= vocab || m == -INFINITY) {
    for (int64_t c = threadIdx.x; c < ld; c += blockDim.x) d[c] = from_f<T>(0.f);
    return;
  }
  const float g = dlogp ? dlogp[row] : 0.f, h = dentropy ? dentropy[row] : 0.f, H = dentropy ? entropy[row] : 0.f;
  for (int64_t c = threadIdx.x; c < ld; c += blockDim.x) {
    float v = 0.f;
    if (c < vocab) {
      const float lp = (to_f(x[c]) - m) * scale - L, p = expf(lp);
      v = c == tok ? -expm1f(lp) * g : -p * g;
      if (p > 0.f) v -= h * p * (lp + H);
      v *= scale;
    }
    d[c] = from_f<T>(v);
  }
}

}  // namespace hift
