// Rotary positions on caller-owned buffers: the pairs of the first `rot` elements of every head turned by angle(pos, j),
//   y1 = x1 cos - x2 sin,   y2 = x2 cos + x1 sin     (the gradient: the same with -sin),
// pair j = (j, j + rot / 2) in the half layout, (2 j, 2 j + 1) in the interleaved one; the rest of a head is copied.
// Memory bounds it: every element is read and written once.  A thread takes 2 V elements (V pairs, two loads of 16 bytes) of one head; its V
// cosines and sines come from L1 and L2.  16384 rows x 40 heads x 128 bf16: half of each head turned 63 us (5.3 TB/s), whole heads in the half layout 54, in place
// 56 (6.0 TB/s).  (Four heads a thread, which load them once for the four, cost 90 registers: 69 -> 82 us for the first of these when it was tried.)
#pragma once
#include "common.cuh"

namespace hift {

struct RopeOp {
  const void* x; void* out;
  const float* cs;                    // [n_pos, rot / 2] cosines, then as many sines
  const int32_t* positions;           // one per row, or nullptr: row mod seq
  int32_t* bad;                       // set to 1 by a position outside the table, or nullptr
  int64_t rows, ld, ld_out;
  int heads, dh, rot, n_pos, seq, rows_per_block, copy_units;        // copy_units: per head, beyond the rotated ones (0 in place)
  float sign;
};

template <typename T, int V> struct alignas(sizeof(T) * V) RopeVec { T v[V]; };

template <typename T, int V, int LAYOUT>
__global__ void __launch_bounds__(256) rope_rows_kernel(RopeOp p) {
  pdl_launch_next();
  pdl_wait_prior();
  typedef RopeVec<T, V> Vec;
  const int half = p.rot / 2, turn_units = half / V, units = turn_units + p.copy_units;
  const int per_row = units * p.heads;
  const int i = blockIdx.y * 256 + threadIdx.x;
  const int rb = i / per_row, k = i - rb * per_row;
  const int64_t row = (int64_t)blockIdx.x * p.rows_per_block + rb;
  if (rb >= p.rows_per_block || row >= p.rows) return;
  const int h = k / units, u = k - h * units;
  const T* x = (const T*)p.x + row * p.ld + (int64_t)h * p.dh;
  T* y = (T*)p.out + row * p.ld_out + (int64_t)h * p.dh;
  if (u >= turn_units) {                                   // behind the rotated part: copied
    const int e = p.rot + (u - turn_units) * 2 * V;
    if (V > 1 || e + 1 < p.dh) {
      const Vec a = *reinterpret_cast<const Vec*>(x + e), b = *reinterpret_cast<const Vec*>(x + e + V);
      *reinterpret_cast<Vec*>(y + e) = a;
      *reinterpret_cast<Vec*>(y + e + V) = b;
    } else {
      y[e] = x[e];
    }
    return;
  }
  int pos = p.positions ? p.positions[row] : (int)((uint32_t)row % (uint32_t)p.seq);          // rows are below 2^31
  const bool in = pos >= 0 && pos < p.n_pos;
  if (!in) {                                               // the row stays as it is
    if (p.bad && k == 0) *p.bad = 1;
    pos = 0;
  }
  alignas(16) float c[V], s[V];
  const float* ct = p.cs + (int64_t)pos * half + u * V;
  const float* st = ct + (int64_t)p.n_pos * half;
  typedef RopeVec<float, (V < 4 ? V : 4)> Cs;
#pragma unroll
  for (int j = 0; j < V; j += (V < 4 ? V : 4)) {
    *reinterpret_cast<Cs*>(c + j) = *reinterpret_cast<const Cs*>(ct + j);
    *reinterpret_cast<Cs*>(s + j) = *reinterpret_cast<const Cs*>(st + j);
  }
  const int e0 = LAYOUT == 0 ? u * V : u * 2 * V, e1 = LAYOUT == 0 ? e0 + half : e0 + V;
  const Vec a = *reinterpret_cast<const Vec*>(x + e0), b = *reinterpret_cast<const Vec*>(x + e1);
  if (!in) {                                               // (cosine 1 and sine 0 would make a NaN of an infinity's partner; a branch in front of the loads: 59 -> 71 us for
    *reinterpret_cast<Vec*>(y + e0) = a;                   // 16384 rows x 40 heads x 128 bf16 in the half layout)
    *reinterpret_cast<Vec*>(y + e1) = b;
    return;
  }
  Vec o0, o1;
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] *= p.sign;
#pragma unroll
  for (int j = 0; j < V; ++j) {                            // fp32, rounded once
    if (LAYOUT == 0) {
      const float x1 = to_f(a.v[j]), x2 = to_f(b.v[j]);
      o0.v[j] = from_f<T>(x1 * c[j] - x2 * s[j]);
      o1.v[j] = from_f<T>(x2 * c[j] + x1 * s[j]);
    } else {                                               // pair j lies at elements 2 j, 2 j + 1 of the 2 V
      const float x1 = 2 * j < V ? to_f(a.v[(2 * j) % V]) : to_f(b.v[(2 * j) % V]);
      const float x2 = 2 * j + 1 < V ? to_f(a.v[(2 * j + 1) % V]) : to_f(b.v[(2 * j + 1) % V]);
      const T y1 = from_f<T>(x1 * c[j] - x2 * s[j]), y2 = from_f<T>(x2 * c[j] + x1 * s[j]);
      if (2 * j < V) o0.v[(2 * j) % V] = y1; else o1.v[(2 * j) % V] = y1;
      if (2 * j + 1 < V) o0.v[(2 * j + 1) % V] = y2; else o1.v[(2 * j + 1) % V] = y2;
    }
  }
  *reinterpret_cast<Vec*>(y + e0) = o0;
  *reinterpret_cast<Vec*>(y + e1) = o1;
}

// The table of cosines and sines: angle(pos, j) = pos * freq(j) in 64 bits, the cosine and sine rounded once, times `mag`.
//   kind 0 plain: base^(-2j/rot);  1 linear: that / factor;  2 NTK-aware: base grown so that the slowest pair turns `factor` times slower;
//   kind 3 (YaRN): per pair between plain (pairs that turn at least `fast` times over orig_len) and / factor (at most `slow` times), linear in j;
//   kind 4 (banded): plain above `fast` turns over orig_len, / factor below `slow`, in between linear in the number of turns.
struct RopeTable { int kind, n_pos, half; double base, factor, orig_len, fast, slow; float mag; float* cs; };
__host__ __device__ inline double rope_frequency(const RopeTable& t, int j) {
  const double rot = 2.0 * t.half, two_pi = 6.283185307179586476925286766559;
  double base = t.base;
  if (t.kind == 2 && t.half > 1) base *= pow(t.factor, rot / (rot - 2.0));
  const double f = pow(base, -2.0 * j / rot);
  if (t.kind == 0 || t.kind == 2) return f;
  if (t.kind == 1) return f / t.factor;
  if (t.kind == 3) {
    // the pair indices at which a pair turns `fast` and `slow` times over orig_len, outwards to whole ones
    const double lo = floor(rot * log(t.orig_len / (t.fast * two_pi)) / (2.0 * log(t.base)));
    const double hi = ceil(rot * log(t.orig_len / (t.slow * two_pi)) / (2.0 * log(t.base)));
    if (hi <= 0.0) return f / t.factor;                    // even the first pair turns `slow` times at most
    if (j <= lo) return f;
    const double from = lo < 0.0 ? 0.0 : lo, to = hi > rot - 1.0 ? rot - 1.0 : hi;
    if (j >= to) return f / t.factor;
    const double ramp = (j - from) / (to - from);          // from <= j < to
    return f * (1.0 - ramp) + f / t.factor * ramp;
  }
  const double turns = t.orig_len * f / two_pi;
  if (turns > t.fast) return f;
  if (turns < t.slow) return f / t.factor;
  const double w = (turns - t.slow) / (t.fast - t.slow);
  return (1.0 - w) * f / t.factor + w * f;
}
__global__ void __launch_bounds__(256) rope_table_kernel(RopeTable t) {
  pdl_launch_next();
  pdl_wait_prior();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)t.n_pos * t.half;
  if (i >= n) return;
  const int j = (int)(i % t.half);
  double s, c;
  sincos((double)(i / t.half) * rope_frequency(t, j), &s, &c);
  t.cs[i] = (float)(c * (double)t.mag);
  t.cs[n + i] = (float)(s * (double)t.mag);
}

template <typename T, int V>
cudaError_t launch_rope_v(cudaStream_t st, int layout, RopeOp p) {
  // the rest of a head is in place already where x is the output
  p.copy_units = p.x == p.out ? 0 : (p.dh - p.rot + 2 * V - 1) / (2 * V);
  const int64_t per_row = (int64_t)(p.rot / 2 / V + p.copy_units) * p.heads;
  // rows to a block column: so many that the last of its blocks is at most a 16th of them
  p.rows_per_block = (int)((4095 + per_row) / per_row);
  if (p.rows_per_block > p.rows) p.rows_per_block = (int)p.rows;
  const dim3 g((unsigned)((p.rows + p.rows_per_block - 1) / p.rows_per_block), (unsigned)((per_row * p.rows_per_block + 255) / 256));
  return launch_pdl(layout == 0 ? rope_rows_kernel<T, V, 0> : rope_rows_kernel<T, V, 1>, g, dim3(256), 0, st, p);
}
// The widest vector (16 bytes at most) that divides the halves of the rotated part, the rest of a head, heads and rows, and fits the addresses
// (the table's too: rot / 2 is a multiple of v).
template <typename T>
cudaError_t launch_rope(cudaStream_t st, int layout, const RopeOp& p) {
  auto fits = [&](int v) {
    const int64_t b = v * (int64_t)sizeof(T);
    return p.rot % (2 * v) == 0 && (p.dh - p.rot) % (2 * v) == 0 && p.ld % v == 0 && p.ld_out % v == 0 &&
           (((uintptr_t)p.x | (uintptr_t)p.out) & (uintptr_t)(b - 1)) == 0 && ((uintptr_t)p.cs & (uintptr_t)(v >= 4 ? 15 : 4 * v - 1)) == 0;
  };
  if (sizeof(T) == 2 && fits(8)) return launch_rope_v<T, sizeof(T) == 2 ? 8 : 4>(st, layout, p);
  if (fits(4)) return launch_rope_v<T, 4>(st, layout, p);
  if (fits(2)) return launch_rope_v<T, 2>(st, layout, p);
  return launch_rope_v<T, 1>(st, layout, p);
}

}  // namespace hift
