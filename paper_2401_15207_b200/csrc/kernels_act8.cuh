// Activations kept in 8 bits for the backward pass.  Blocks of 32 consecutive columns of a row share a scale 2^(byte - 127): the least power
// of two that brings the block's largest magnitude into the format's range (int8: 127, e4m3: 448), 2^-110 at least, so that every value
// that a block stands for is exact in bf16 and fp32.  A power of two costs up to one bit of int8's seven against a scale of top / 127, and
// makes quotient, rounding and product free of any other error: the same 8 bits on every path.  A block that holds a NaN or an infinity
// gets scale byte 255 (infinity as an fp32 exponent) and zeros: 0 * infinity is NaN, the whole block.
//
// Memory bounds packing, unpacking and SwiGLU (4.9 and 5.9 TB/s); GELU, with fewer bytes a value, is bound by the issue of instructions (83 to 86 % of the
// slots: forward 3.1 TB/s, gradient 4.6).  Rows whose columns are a multiple of 8 in aligned buffers
// go 8 columns to a thread (16 bytes of bf16, 8 bytes of q): four threads share a block, its maximum takes two shuffles.  Other rows go
// one column to a thread, one block to a warp.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace hift {

constexpr int kAct8Block = 32;

// scale byte of a block whose largest magnitude has these bits (of |x|; a NaN's bits are above infinity's)
template <int FMT> __device__ __forceinline__ int act8_byte(uint32_t top) {
  const int e = (int)(top >> 23);
  const uint32_t m = top & 0x7FFFFFu;
  if (e == 255) return 255;
  // int8: 127 = 1.984375 * 2^6, e4m3: 448 = 1.75 * 2^8
  const int b = FMT == 0 ? e - 6 + (m > 0x7E0000u) : e - 8 + (m > 0x600000u);
  return max(b, 17);
}
__device__ __forceinline__ float act8_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float act8_inverse(int byte) { return byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23); }

// At the topmost scale the codes from 64 (int8) or 256 (e4m3) on stand for 2^128: the largest one below it is kept instead.  (No other block pays for more
// than the comparison.)
template <int FMT> constexpr int kAct8TopByte = FMT == 0 ? 249 : 247;
template <int FMT> __device__ __forceinline__ float act8_below_top(float v) {
  constexpr float most = FMT == 0 ? 63.f : 240.f;
  return fminf(fmaxf(v, -most), most);
}
// four values, scaled into range, as four bytes; round to nearest even
template <int FMT> __device__ __forceinline__ uint32_t act8_quad(float a, float b, float c, float d) {
  if (FMT == 0) {
    // |v| <= 127: added to 1.5 * 2^23, whose step is 1, v is rounded to nearest even and its two's complement is the low byte (a conversion
    // instruction has an eighth of an addition's rate)
    const uint32_t lo = __byte_perm(__float_as_uint(a + 12582912.0f), __float_as_uint(b + 12582912.0f), 0x0040);
    return __byte_perm(lo, __byte_perm(__float_as_uint(c + 12582912.0f), __float_as_uint(d + 12582912.0f), 0x0040), 0x5410);
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  return lo | (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
template <int FMT> __device__ __forceinline__ void act8_unquad(uint32_t q, float (&v)[4]) {
  if (FMT == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i)                              // 2^23 + (value + 128) as fp32 from its bytes, less 2^23 + 128
      v[i] = __uint_as_float(__byte_perm(q ^ 0x80808080u, 0x4B000000u, 0x7540 + i)) - 8388736.0f;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> 16 * i), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
  }
}
template <int FMT> __device__ __forceinline__ float act8_one(uint8_t q) {
  float v[4];
  act8_unquad<FMT>(q, v);
  return v[0];
}

struct Act8 {
  const void* x;             // pre-activations [rows, ld] (KIND 2: gate | up, [rows, 2 f])
  const void* dy;            // gradient of the activation's output [rows, f]
  void* y;                   // activation's output [rows, f], or nullptr
  void* dx;                  // gradient of the pre-activations, or the unpacked values
  uint8_t* q; uint8_t* scales;
  int64_t rows, f, ld;       // ld: of x (packing alone) or of dx (unpacking alone)
  int rows_per_block;        // rows of a block column (blockIdx.x), dealt to its threads (blockIdx.y) behind one another
};
// This thread's row and unit of it; false beyond the last row.  `units` a row.
__device__ __forceinline__ bool act8_place(const Act8& p, int units, int64_t& row, int& unit) {
  const int i = blockIdx.y * 256 + threadIdx.x, rb = i / units;
  unit = i - rb * units;
  row = (int64_t)blockIdx.x * p.rows_per_block + rb;
  return rb < p.rows_per_block && row < p.rows;
}
// Rows to a block column: so many that the last of its blocks is at most a 32nd of them (a 64-bit division in every thread is dearer).
inline dim3 act8_grid(Act8& p, int64_t units) {
  p.rows_per_block = (int)((8191 + units) / units);
  if (p.rows_per_block > p.rows) p.rows_per_block = (int)p.rows;
  return dim3((unsigned)((p.rows + p.rows_per_block - 1) / p.rows_per_block), (unsigned)((units * p.rows_per_block + 255) / 256));
}

// KIND 0: none (packing alone), 1: GELU, 2: SwiGLU
// sigmoid(a), and 1 - sigmoid(a) = sigmoid(-a): with t = exp(-|a|) one is 1 / (1 + t) and the other t / (1 + t), so that neither loses digits to a
// difference, nor the small one its value where exp(|a|) is beyond what a quick division or fp32 itself holds.  (SwiGLU of 8192 x 11008
// bf16 forward 141 -> 144 us, the gradient as before; sums and products of pairs 151.)
__device__ __forceinline__ float act8_sigmoid(float a, float& rest) {
  const float t = __expf(-fabsf(a)), r = __fdividef(1.0f, 1.0f + t), s = t * r;
  rest = a < 0.f ? r : s;
  return a < 0.f ? s : r;
}
// Normal distribution cdf and e = exp(-a^2 / 2).  With z = |a| / sqrt(2) and t = 1 / (1 + 0.45 z), erfc(z) / 2 = exp(-z^2) t Q(t): Q, of nine degrees, fitted
// to the least largest relative error over all z >= 0 (3.2e-8; 5 half steps of fp32 as evaluated).  The lower tail is that product itself: in
// 1 + erf its digits cancel (4 % off at a = -5, nothing left at -5.5).  One exponential serves the density too.  (GELU of 16384 x 5120 bf16, int8:
// 135 us, gradient 128; with CUDA's erfcf 183 and 197.)
__device__ __forceinline__ float act8_normal(float a, float& e) {
  const float t = __fdividef(1.0f, fmaf(fabsf(a), 0.31819806f, 1.0f));
  const float c[9] = {0.0953436941f, -0.150290787f, 0.0712000579f, -0.0111787422f, 0.0599751472f, 0.0876260772f, 0.114135817f, 0.126941577f, 0.126942664f};
  float q = -0.0206954964f;
#pragma unroll
  for (int i = 0; i < 9; ++i) q = fmaf(q, t, c[i]);
  e = __expf(-0.5f * a * a);
  const float tail = e * (t * q);
  return a < 0.f ? tail : 1.0f - tail;
}
template <int KIND> __device__ __forceinline__ float act8_value(float a, float u) {
  float e;
  return KIND == 1 ? a * act8_normal(a, e) : a * act8_sigmoid(a, e) * u;
}
// dx (and the gradient of `up`), and the activation's value
template <int KIND> __device__ __forceinline__ void act8_grad(float g, float a, float u, float& da, float& du, float& y) {
  if (KIND == 1) {
    float e;
    const float cdf = act8_normal(a, e);
    da = g * fmaf(a, 0.39894228040143267794f * e, cdf);
    y = a * cdf;
  } else {
    float rest;
    const float sig = act8_sigmoid(a, rest), s = a * sig;
    da = g * u * sig * fmaf(a, rest, 1.0f);
    du = g * s;
    y = s * u;
  }
}

// 8 elements as they lie in memory; as floats; and the bits of the largest magnitude (those of a NaN are above infinity's)
template <typename T> struct Act8Raw { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ void act8_load(const T* p, Act8Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4*>(p)[i];
}
__device__ __forceinline__ uint32_t act8_floats(const Act8Raw<float>& r, float (&v)[8]) {
  const uint32_t w[8] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w, r.w[1].x, r.w[1].y, r.w[1].z, r.w[1].w};
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = __uint_as_float(w[j]);
    top = max(top, w[j] & 0x7FFFFFFFu);
  }
  return top;
}
__device__ __forceinline__ uint32_t act8_floats(const Act8Raw<bf16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
  __nv_bfloat162 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    const uint32_t b = w[i] & 0x7FFF7FFFu;
    h[i] = *reinterpret_cast<const __nv_bfloat162*>(&b);
  }
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  const uint32_t u = *reinterpret_cast<const uint32_t*>(&m);
  return max(u << 16, u & 0xFFFF0000u);
}

// ---- 8 columns a thread -------------------------------------------------------------------------------------------------------------
// Thread i of a row: half i / units, columns 8 (i mod units) ..; units = 4 * ceil(f / 32), those at or beyond f / 8 idle in the last block.
template <typename T, int FMT, int KIND>
__global__ void __launch_bounds__(256) act8_fwd_vec_kernel(Act8 p) {
  pdl_launch_next();
  pdl_wait_prior();
  constexpr int N = KIND == 2 ? 2 : 1;
  const int nb = (int)((p.f + kAct8Block - 1) / kAct8Block), units = 4 * nb;
  int64_t row;
  int c;
  const bool in = act8_place(p, units, row, c) && 8 * c < p.f;
  float v[N][8];
  Act8Raw<T> raw[N] = {};
  if (in) {
#pragma unroll
    for (int n = 0; n < N; ++n) act8_load((const T*)p.x + row * p.ld + n * p.f + 8 * c, raw[n]);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    uint32_t top = act8_floats(raw[n], v[n]);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int byte = act8_byte<FMT>(top);
    const float inv = act8_inverse(byte);
    if (in) {
      uint2 w = make_uint2(0u, 0u);
      if (byte != 255) {
        const uint64_t ip = f2_pack(inv, inv);
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) f2_unpack(f2_mul(f2_pack(v[n][j], v[n][j + 1]), ip), s[j], s[j + 1]);
        if (byte == kAct8TopByte<FMT>) {
#pragma unroll
          for (int j = 0; j < 8; ++j) s[j] = act8_below_top<FMT>(s[j]);
        }
        w.x = act8_quad<FMT>(s[0], s[1], s[2], s[3]);
        w.y = act8_quad<FMT>(s[4], s[5], s[6], s[7]);
      }
      *reinterpret_cast<uint2*>(p.q + (row * N + n) * p.f + 8 * c) = w;
      if ((c & 3) == 0) p.scales[(row * N + n) * nb + (c >> 2)] = (uint8_t)byte;
    }
  }
  if (KIND > 0 && in) {
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = act8_value<KIND>(v[0][j], v[N - 1][j]);
    store8((T*)p.y + row * p.f + 8 * c, y);
  }
}
template <typename T, int FMT, int KIND, bool AGAIN>
__global__ void __launch_bounds__(256) act8_bwd_vec_kernel(Act8 p) {
  pdl_launch_next();
  pdl_wait_prior();
  constexpr int N = KIND == 2 ? 2 : 1;
  const int nb = (int)((p.f + kAct8Block - 1) / kAct8Block), units = (int)(p.f / 8);
  int64_t row;
  int c;
  if (!act8_place(p, units, row, c)) return;
  uint2 w[N];
  int byte[N];
  float g[8], v[N][8];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    w[n] = *reinterpret_cast<const uint2*>(p.q + (row * N + n) * p.f + 8 * c);
    byte[n] = p.scales[(row * N + n) * nb + (c >> 2)];
  }
  if (KIND > 0) load8((const T*)p.dy + row * p.f + 8 * c, g);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float s = act8_scale(byte[n]);
    float a[4], b[4];
    act8_unquad<FMT>(w[n].x, a);
    act8_unquad<FMT>(w[n].y, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[n][j] = a[j] * s; v[n][4 + j] = b[j] * s; }
  }
  if constexpr (KIND == 0) {
    store8((T*)p.dx + row * p.ld + 8 * c, v[0]);
    return;
  }
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float da, du = 0.f;
    act8_grad<KIND>(g[j], v[0][j], v[N - 1][j], da, du, y[j]);
    v[0][j] = da;
    if (N == 2) v[1][j] = du;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) store8((T*)p.dx + (row * N + n) * p.f + 8 * c, v[n]);
  if (AGAIN) store8((T*)p.y + row * p.f + 8 * c, y);
}

// ---- any rows: one column a thread, one block of 32 a warp --------------------------------------------------------------------------
template <typename T, int FMT, int KIND>
__global__ void __launch_bounds__(256) act8_fwd_any_kernel(Act8 p) {
  pdl_launch_next();
  pdl_wait_prior();
  constexpr int N = KIND == 2 ? 2 : 1;
  const int nb = (int)((p.f + kAct8Block - 1) / kAct8Block), lane = threadIdx.x & 31;
  int64_t row;
  int c;
  if (!act8_place(p, nb * kAct8Block, row, c)) return;     // whole warps
  const int k = c / kAct8Block;
  const bool in = c < p.f;
  float v[N];
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = in ? to_f(((const T*)p.x)[row * p.ld + n * p.f + c]) : 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int byte = act8_byte<FMT>(__reduce_max_sync(0xffffffffu, __float_as_uint(v[n]) & 0x7FFFFFFFu));
    float s = v[n] * act8_inverse(byte);
    if (byte == kAct8TopByte<FMT>) s = act8_below_top<FMT>(s);
    const uint32_t w = byte == 255 ? 0u : act8_quad<FMT>(s, 0.f, 0.f, 0.f);
    if (in) p.q[(row * N + n) * p.f + c] = (uint8_t)w;
    if (lane == 0) p.scales[(row * N + n) * nb + k] = (uint8_t)byte;
  }
  if (KIND > 0 && in) ((T*)p.y)[row * p.f + c] = from_f<T>(act8_value<KIND>(v[0], v[N - 1]));
}
template <typename T, int FMT, int KIND, bool AGAIN>
__global__ void __launch_bounds__(256) act8_bwd_any_kernel(Act8 p) {
  pdl_launch_next();
  pdl_wait_prior();
  constexpr int N = KIND == 2 ? 2 : 1;
  const int nb = (int)((p.f + kAct8Block - 1) / kAct8Block);
  int64_t row;
  int c;
  if (!act8_place(p, (int)p.f, row, c)) return;
  float v[N];
#pragma unroll
  for (int n = 0; n < N; ++n)
    v[n] = act8_one<FMT>(p.q[(row * N + n) * p.f + c]) * act8_scale(p.scales[(row * N + n) * nb + c / kAct8Block]);
  if (KIND == 0) { ((T*)p.dx)[row * p.ld + c] = from_f<T>(v[0]); return; }
  float da, du = 0.f, y;
  act8_grad<KIND>(to_f(((const T*)p.dy)[row * p.f + c]), v[0], v[N - 1], da, du, y);
  ((T*)p.dx)[row * N * p.f + c] = from_f<T>(da);
  if (N == 2) ((T*)p.dx)[(row * N + 1) * p.f + c] = from_f<T>(du);
  if (AGAIN) ((T*)p.y)[row * p.f + c] = from_f<T>(y);
}

inline bool act8_aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
template <typename T, int FMT, int KIND>
cudaError_t launch_act8_fwd(cudaStream_t st, Act8 p) {
  const int64_t nb = (p.f + kAct8Block - 1) / kAct8Block;
  const bool vec = p.f % 8 == 0 && p.ld % 8 == 0 && act8_aligned(p.x, 16) && act8_aligned(p.y, 16) && act8_aligned(p.q, 8);
  const dim3 g = act8_grid(p, vec ? nb * 4 : nb * kAct8Block);
  return launch_pdl(vec ? act8_fwd_vec_kernel<T, FMT, KIND> : act8_fwd_any_kernel<T, FMT, KIND>, g, dim3(256), 0, st, p);
}
template <typename T, int FMT, int KIND, bool AGAIN>
cudaError_t launch_act8_bwd_y(cudaStream_t st, Act8 p) {
  const bool vec = p.f % 8 == 0 && p.ld % 8 == 0 && act8_aligned(p.dy, 16) && act8_aligned(p.dx, 16) && act8_aligned(p.y, 16) && act8_aligned(p.q, 8);
  const dim3 g = act8_grid(p, vec ? p.f / 8 : p.f);
  return launch_pdl(vec ? act8_bwd_vec_kernel<T, FMT, KIND, AGAIN> : act8_bwd_any_kernel<T, FMT, KIND, AGAIN>, g, dim3(256), 0, st, p);
}
template <typename T, int FMT, int KIND>
cudaError_t launch_act8_bwd(cudaStream_t st, const Act8& p) {
  if constexpr (KIND == 0) return launch_act8_bwd_y<T, FMT, 0, false>(st, p);
  else return p.y ? launch_act8_bwd_y<T, FMT, KIND, true>(st, p) : launch_act8_bwd_y<T, FMT, KIND, false>(st, p);
}

}  // namespace hift
