// Entry points of the block operators beside the training step: rotary positions, differential attention and activations kept in 8 bits
// (include/hift.h).  Argument checks and launches; the kernels are in the headers.
#include <math.h>

#include "hift.h"
#include "kernels_act8.cuh"
#include "kernels_dattn.cuh"
#include "kernels_rope.cuh"

using namespace hift;

static_assert(kAct8Block == HIFT_ACT8_BLOCK, "");

namespace {

hift_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return HIFT_OK;
  cudaGetLastError();                                      // an error does not stay behind for the next call's check
  return HIFT_ERR_CUDA;
}
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
template <typename... Ptr> bool words(const Ptr*... p) { return (aligned(p, 4) && ...); }       // buffers of fp32 or int32
bool elements(int32_t dtype, std::initializer_list<const void*> ps) {
  for (const void* p : ps) if (!aligned(p, dtype == 0 ? 4 : 2)) return false;
  return true;
}

hift_status dattn_cfg(int32_t dtype, int64_t B, int64_t S, int64_t H, int64_t K, int32_t D, const void* gain, double eps, double c) {
  if (dtype < 0 || dtype > 1 || B < 0 || S < 0 || H < 1 || K < 1 || H % K || !dattn_head_ok(D)) return HIFT_ERR_CFG;
  if (gain && (!(eps > 0.0) || !isnormal((float)eps) || !isfinite((float)c))) return HIFT_ERR_CFG;
  // rows of the buffers and the blocks of a launch are counted in 32 bits
  if (B * S > INT32_MAX / 2 || (H + 2 * K) * D > INT32_MAX / 4 || B * ((S + 63) / 64) > INT32_MAX / H) return HIFT_ERR_CAPACITY;
  return HIFT_OK;
}
DattnArgs dattn_args(int64_t B, int64_t S, int64_t H, int64_t K, int32_t D, int32_t causal, const void* qkv, const float* lam, const void* gain,
                     double eps, double c, const int32_t* lens) {
  DattnArgs a{};
  a.qkv = qkv; a.lam = lam; a.gain = gain; a.lens = lens;
  a.B = (int)B; a.S = (int)S; a.H = (int)H; a.K = (int)K; a.causal = causal != 0;
  a.scale = (float)(1.0 / sqrt(D / 2.0)); a.eps = (float)eps; a.c = (float)c;
  return a;
}

hift_status act8_cfg(int32_t dtype, int32_t format, int64_t rows, int64_t f) {
  if (dtype < 0 || dtype > 1 || format < 0 || format > 1 || rows < 0 || rows > INT32_MAX || f < 1) return HIFT_ERR_CFG;
  return f > HIFT_ACT8_MAX_COLS ? HIFT_ERR_CAPACITY : HIFT_OK;
}
template <int KIND> cudaError_t act8_fwd(cudaStream_t st, int32_t dtype, int32_t format, const Act8& p) {
  if (dtype == 0) return format == 0 ? launch_act8_fwd<float, 0, KIND>(st, p) : launch_act8_fwd<float, 1, KIND>(st, p);
  return format == 0 ? launch_act8_fwd<bf16, 0, KIND>(st, p) : launch_act8_fwd<bf16, 1, KIND>(st, p);
}
template <int KIND> cudaError_t act8_bwd(cudaStream_t st, int32_t dtype, int32_t format, const Act8& p) {
  if (dtype == 0) return format == 0 ? launch_act8_bwd<float, 0, KIND>(st, p) : launch_act8_bwd<float, 1, KIND>(st, p);
  return format == 0 ? launch_act8_bwd<bf16, 0, KIND>(st, p) : launch_act8_bwd<bf16, 1, KIND>(st, p);
}

}  // namespace

extern "C" {

hift_status hift_rope_table(int32_t scaling, int64_t n_pos, int32_t rot, double base, double factor, double orig_len, double fast, double slow,
                            float* cs, void* stream) {
  if (scaling < 0 || scaling > 4 || n_pos < 0 || n_pos > INT32_MAX || rot < 2 || rot % 2 || !(base > 1.0) || !isfinite(base)) return HIFT_ERR_CFG;
  if (scaling != 0 && (!(factor >= 1.0) || !isfinite(factor))) return HIFT_ERR_CFG;
  if (scaling >= 3 && (!(orig_len > 0.0) || !isfinite(orig_len) || !(slow > 0.0) || !(fast > slow) || !isfinite(fast))) return HIFT_ERR_CFG;
  const int64_t n = n_pos * (rot / 2);
  if (n > ((int64_t)INT32_MAX) * 256) return HIFT_ERR_CAPACITY;
  if (n_pos == 0) return HIFT_OK;
  if (!cs) return HIFT_ERR_INPUT;
  if (!words(cs)) return HIFT_ERR_CFG;
  const float mag = scaling == 3 ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  const RopeTable t{scaling, (int)n_pos, rot / 2, base, factor, orig_len, fast, slow, mag, cs};
  return status_of(launch_pdl(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, (cudaStream_t)stream, t));
}

hift_status hift_k_rope(int32_t dtype, int32_t layout, int64_t rows, int32_t n_heads, int32_t d_head, int32_t rot, const void* x, int64_t ld, void* out,
                        int64_t ld_out, const float* cs, int64_t n_pos, int64_t seq, const int32_t* positions, int32_t inverse, int32_t* bad,
                        void* stream) {
  const int64_t width = (int64_t)n_heads * d_head;
  if (dtype < 0 || dtype > 1 || layout < 0 || layout > 1 || rows < 0 || rows > INT32_MAX || n_heads < 1 || d_head < 2 || rot < 2 || rot % 2 || rot > d_head)
    return HIFT_ERR_CFG;
  if (n_pos < 1 || n_pos > INT32_MAX || (!positions && (seq < 1 || seq > n_pos)) || ld < width || ld_out < width) return HIFT_ERR_CFG;
  if (width > HIFT_ROPE_MAX_WIDTH) return HIFT_ERR_CAPACITY;
  if (rows == 0) return HIFT_OK;
  if (!x || !out || !cs) return HIFT_ERR_INPUT;
  if (!elements(dtype, {x, out}) || !words(cs, positions, bad) || (x == out && ld != ld_out)) return HIFT_ERR_CFG;
  const RopeOp p{x, out, cs, positions, bad, rows, ld, ld_out, n_heads, d_head, rot, (int)n_pos, positions ? 1 : (int)seq, 1, 0, inverse ? -1.f : 1.f};
  return status_of(dtype == 0 ? launch_rope<float>((cudaStream_t)stream, layout, p) : launch_rope<bf16>((cudaStream_t)stream, layout, p));
}

hift_status hift_k_diff_lambda(int32_t n_heads, int32_t sets, int32_t d, double init, const float* w, float* lam, void* stream) {
  if (n_heads < 1 || d < 1 || (sets != 1 && sets != n_heads) || !isfinite((float)init)) return HIFT_ERR_CFG;
  if (!w || !lam) return HIFT_ERR_INPUT;
  if (!words(w, lam)) return HIFT_ERR_CFG;
  return status_of(launch_pdl(diff_lambda_kernel, dim3((unsigned)n_heads), dim3(32), 0, (cudaStream_t)stream, w, sets, d, (float)init, lam, n_heads));
}
hift_status hift_k_diff_lambda_bwd(int32_t n_heads, int32_t sets, int32_t d, const float* w, const float* dlam, float* dw, void* stream) {
  if (n_heads < 1 || d < 1 || (sets != 1 && sets != n_heads)) return HIFT_ERR_CFG;
  if (!w || !dlam || !dw) return HIFT_ERR_INPUT;
  if (!words(w, dlam, dw)) return HIFT_ERR_CFG;
  return status_of(launch_pdl(diff_lambda_bwd_kernel, dim3((unsigned)sets), dim3(32), 0, (cudaStream_t)stream, w, sets, d, dlam, dw, n_heads));
}

hift_status hift_k_diff_attention_fwd(int32_t dtype, int32_t B, int32_t S, int32_t H, int32_t K, int32_t D, int32_t causal, const void* qkv,
                                      const float* lam, const void* gain, double eps, double out_scale, void* o, void* o2, void* y, float* lse,
                                      const int32_t* key_lens, void* stream) {
  const hift_status s = dattn_cfg(dtype, B, S, H, K, D, gain, eps, out_scale);
  if (s != HIFT_OK) return s;
  if (B == 0 || S == 0) return HIFT_OK;
  if (!qkv || !lam || !o || !lse || (gain && !y) || (y && !gain)) return HIFT_ERR_INPUT;
  if (!elements(dtype, {qkv, gain, o, o2, y}) || !words(lam, lse, key_lens)) return HIFT_ERR_CFG;
  DattnArgs a = dattn_args(B, S, H, K, D, causal, qkv, lam, gain, eps, out_scale, key_lens);
  a.o = o; a.o2 = o2; a.y = y; a.lse = lse;
  a.vec = aligned(qkv, 16);
  cudaStream_t st = (cudaStream_t)stream;
  if (dattn_tc_eligible(dtype, D, a)) return status_of(dattn_tc_fwd_launch(st, D, a));
  return status_of(dtype == 0 ? launch_dattn_fwd<float>(st, D, a) : launch_dattn_fwd<bf16>(st, D, a));
}

size_t hift_diff_attention_bwd_scratch_bytes(int32_t dtype, int32_t B, int32_t S, int32_t H, int32_t D, int32_t norm) {
  if (dattn_cfg(dtype, B, S, H, 1, D, nullptr, 0, 0) != HIFT_OK || B == 0 || S == 0) return 0;
  return dattn_plan(dtype == 0 ? 4 : 2, B, S, H, D, norm != 0).bytes;
}

hift_status hift_k_diff_attention_bwd(int32_t dtype, int32_t B, int32_t S, int32_t H, int32_t K, int32_t D, int32_t causal, const void* qkv,
                                      const float* lam, const void* gain, double eps, double out_scale, const void* o, const void* o2,
                                      const float* lse, const void* dy, void* dqkv, float* dlam, float* dgain, void* scratch, size_t scratch_bytes,
                                      const int32_t* key_lens, void* stream) {
  const hift_status s = dattn_cfg(dtype, B, S, H, K, D, gain, eps, out_scale);
  if (s != HIFT_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  if (dgain && !gain) return HIFT_ERR_INPUT;
  if (!words(dlam, dgain)) return HIFT_ERR_CFG;
  if (B == 0 || S == 0) {                                  // no rows: the sums over them are zero
    if (dlam && cudaMemsetAsync(dlam, 0, (size_t)H * 4, st) != cudaSuccess) return HIFT_ERR_CUDA;
    if (dgain && cudaMemsetAsync(dgain, 0, (size_t)D * 4, st) != cudaSuccess) return HIFT_ERR_CUDA;
    return HIFT_OK;
  }
  if (!qkv || !lam || !o || !o2 || !lse || !dy || !dqkv || !scratch) return HIFT_ERR_INPUT;
  if (!elements(dtype, {qkv, gain, o, o2, dy, dqkv}) || !words(lam, lse, key_lens) || !aligned(scratch, 256)) return HIFT_ERR_CFG;
  const DattnPlan pl = dattn_plan(dtype == 0 ? 4 : 2, B, S, H, D, gain != nullptr);
  if (scratch_bytes < pl.bytes) return HIFT_ERR_CAPACITY;
  char* w = (char*)scratch;
  DattnArgs a = dattn_args(B, S, H, K, D, causal, qkv, lam, gain, eps, out_scale, key_lens);
  a.o = (void*)o; a.o2 = (void*)o2; a.lse = (float*)lse; a.dy = dy; a.dqkv = dqkv;
  a.dsum = (float*)(w + pl.dsum);
  a.g = gain ? (void*)(w + pl.g) : dy;
  a.vec = aligned(qkv, 16) && aligned(a.g, 16);
  float* dlam_part = (float*)(w + pl.part);
  const DattnPrep p{a, gain ? (void*)(w + pl.g) : nullptr, (float*)(w + pl.dsum), dlam_part, dlam_part + (size_t)H * pl.chunks, pl.chunks, pl.rows_per_chunk};
  cudaError_t e = dtype == 0 ? launch_dattn_prep<float>(st, D, p) : launch_dattn_prep<bf16>(st, D, p);
  if (e == cudaSuccess && (dlam || dgain)) {
    const int blocks = H + (dgain ? D / 8 : 0);
    e = launch_pdl(dattn_sums_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, (const float*)p.dlam_part, (const float*)p.dgain_part, dlam, dgain, H, pl.chunks, D);
  }
  if (e != cudaSuccess) return status_of(e);
  if (dattn_tc_eligible(dtype, D, a)) return status_of(dattn_tc_bwd_launch(st, D, a));
  e = dtype == 0 ? launch_dattn_bwd<float>(st, D, a) : launch_dattn_bwd<bf16>(st, D, a);
  return status_of(e);
}

hift_status hift_k_act8_pack(int32_t dtype, int32_t format, int64_t rows, int64_t cols, const void* x, int64_t ld, void* q, uint8_t* scales, void* stream) {
  const hift_status s = act8_cfg(dtype, format, rows, cols);
  if (s != HIFT_OK) return s;
  if (ld < cols) return HIFT_ERR_CFG;
  if (rows == 0) return HIFT_OK;
  if (!x || !q || !scales) return HIFT_ERR_INPUT;
  if (!elements(dtype, {x})) return HIFT_ERR_CFG;
  return status_of(act8_fwd<0>((cudaStream_t)stream, dtype, format, Act8{x, nullptr, nullptr, nullptr, (uint8_t*)q, scales, rows, cols, ld, 0}));
}
hift_status hift_k_act8_unpack(int32_t dtype, int32_t format, int64_t rows, int64_t cols, const void* q, const uint8_t* scales, void* out, int64_t ld,
                               void* stream) {
  const hift_status s = act8_cfg(dtype, format, rows, cols);
  if (s != HIFT_OK) return s;
  if (ld < cols) return HIFT_ERR_CFG;
  if (rows == 0) return HIFT_OK;
  if (!out || !q || !scales) return HIFT_ERR_INPUT;
  if (!elements(dtype, {out})) return HIFT_ERR_CFG;
  return status_of(act8_bwd<0>((cudaStream_t)stream, dtype, format, Act8{nullptr, nullptr, nullptr, out, (uint8_t*)q, (uint8_t*)scales, rows, cols, ld, 0}));
}
hift_status hift_k_act8_fwd(int32_t dtype, int32_t format, int32_t kind, int64_t rows, int64_t f, const void* pre, void* act, void* q, uint8_t* scales,
                            void* stream) {
  const hift_status s = act8_cfg(dtype, format, rows, f);
  if (s != HIFT_OK) return s;
  if (kind < 1 || kind > 2) return HIFT_ERR_CFG;
  if (rows == 0) return HIFT_OK;
  if (!pre || !act || !q || !scales) return HIFT_ERR_INPUT;
  if (!elements(dtype, {pre, act})) return HIFT_ERR_CFG;
  const Act8 p{pre, nullptr, act, nullptr, (uint8_t*)q, scales, rows, f, kind == 2 ? 2 * f : f, 0};
  return status_of(kind == 1 ? act8_fwd<1>((cudaStream_t)stream, dtype, format, p) : act8_fwd<2>((cudaStream_t)stream, dtype, format, p));
}
hift_status hift_k_act8_bwd(int32_t dtype, int32_t format, int32_t kind, int64_t rows, int64_t f, const void* dact, const void* q, const uint8_t* scales,
                            void* dpre, void* act, void* stream) {
  const hift_status s = act8_cfg(dtype, format, rows, f);
  if (s != HIFT_OK) return s;
  if (kind < 1 || kind > 2) return HIFT_ERR_CFG;
  if (rows == 0) return HIFT_OK;
  if (!dact || !q || !scales || !dpre) return HIFT_ERR_INPUT;
  if (!elements(dtype, {dact, dpre, act})) return HIFT_ERR_CFG;
  const Act8 p{nullptr, dact, act, dpre, (uint8_t*)q, (uint8_t*)scales, rows, f, kind == 2 ? 2 * f : f, 0};
  return status_of(kind == 1 ? act8_bwd<1>((cudaStream_t)stream, dtype, format, p) : act8_bwd<2>((cudaStream_t)stream, dtype, format, p));
}

}  // extern "C"
