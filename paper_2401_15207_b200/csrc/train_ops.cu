// Entry points of the operators beside the training step: token log-probabilities, the residual junction and the
// orthogonalised update (include/hift.h).  Argument checks and launches; the kernels are in the headers.
#include <math.h>

#include "hift.h"
#include "kernels_join.cuh"
#include "kernels_logprobs.cuh"
#include "kernels_muon.cuh"

using namespace hift;

static_assert(kLpMaxTop == HIFT_MAX_TOP, "");

namespace {

// a launch's result; an error does not stay behind for the next call's check
hift_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return HIFT_OK;
  cudaGetLastError();
  return HIFT_ERR_CUDA;
}
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
template <typename... Ptr> bool words(const Ptr*... p) { return (aligned(p, 4) && ...); }       // buffers of fp32 or int32

hift_status logprobs_cfg(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, double temperature, float* scale, float* scale2) {
  if (dtype < 0 || dtype > 1 || rows < 0 || rows > INT32_MAX || vocab < 1 || ld < vocab || ld > INT32_MAX - 65536) return HIFT_ERR_CFG;
  *scale = (float)(1.0 / temperature);
  *scale2 = (float)(1.4426950408889634 / temperature);     // (from the rounded 1 / T: up to 1e-7 off, times |z - z_max| in every exponential)
  if (!(temperature > 0.0) || !isfinite(temperature) || !isnormal(*scale) || !isfinite(*scale2)) return HIFT_ERR_CFG;
  return HIFT_OK;
}

// threads of a junction kernel (a warp per 256 columns, `most` warps at most) and its chunks of 8 columns per thread
void join_shape(int64_t cols, int most, int* threads, int* chunks) {
  const int units = (int)((cols + 255) / 256), warps = units < most ? units : most;
  int nc = (units + warps - 1) / warps;
  if (nc == 3) nc = 4;
  *threads = 32 * warps;
  *chunks = nc;
}
hift_status join_cfg(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double res_scale, const void* gate, int64_t rows_per_gate) {
  if (dtype < 0 || dtype > 1 || kind < 0 || kind > 1 || rows < 0 || rows > INT32_MAX || cols < 8 || cols % 8) return HIFT_ERR_CFG;
  if (!isfinite((float)res_scale) || (gate && rows_per_gate < 1)) return HIFT_ERR_CFG;
  return cols > kJoinMaxCols ? HIFT_ERR_CAPACITY : HIFT_OK;
}

// Blocks of the backward kernel that an SM holds: its registers (128 a thread at most) and shared memory.
constexpr size_t kJoinSmem = 208 * 1024;
int join_ctas_per_sm(int th) { return th <= 64 ? 8 : 512 / th; }
// How a backward call deals its rows out: the number of blocks, and whether a gate's rows are split over several.  For 148 SMs whatever the
// device: the scratch size, which follows from it, is asked for without one, and only the speed depends on it.
struct JoinPlan { int ctas, split; int64_t gates_per_cta, rows_per_gate, n_gates; };
JoinPlan join_plan(int64_t rows, int64_t cols, int64_t rows_per_gate) {
  int th, nc;
  join_shape(cols, 16, &th, &nc);
  const int64_t most = 148 * join_ctas_per_sm(th);
  JoinPlan pl;
  pl.rows_per_gate = rows_per_gate < 1 || rows_per_gate > rows ? (rows > 0 ? rows : 1) : rows_per_gate;
  pl.n_gates = (rows + pl.rows_per_gate - 1) / pl.rows_per_gate;
  if (pl.n_gates > most) {
    pl.split = 0;
    pl.gates_per_cta = (pl.n_gates + most - 1) / most;
    pl.ctas = (int)((pl.n_gates + pl.gates_per_cta - 1) / pl.gates_per_cta);
    return pl;
  }
  int64_t split = pl.n_gates > 0 ? most / pl.n_gates : 1;
  const int64_t cap = (pl.rows_per_gate + 3) / 4;          // four rows at least for a block
  if (split > cap) split = cap;
  pl.split = (int)(split < 1 ? 1 : split);
  pl.gates_per_cta = 1;
  pl.ctas = (int)(pl.n_gates * pl.split);
  return pl;
}

template <typename P, int KIND>
cudaError_t launch_join_fwd(cudaStream_t st, int th, int nc, const JoinFwd& p) {
  auto kernel = nc == 1 ? join_fwd_kernel<P, KIND, 1> : nc == 2 ? join_fwd_kernel<P, KIND, 2> : join_fwd_kernel<P, KIND, 4>;
  return launch_pdl(kernel, dim3((unsigned)p.rows), dim3(th), 0, st, p);
}
template <typename P, int KIND, int NC, bool STAGED, bool ONE>
cudaError_t launch_join_bwd_nc(cudaStream_t st, int th, const JoinBwd& p) {
  const size_t smem = STAGED ? (size_t)p.stages * join_rows<NC, ONE> * NC * join_bytes<P> * th : 0;
  if (smem > 40 * 1024) {                                  // idempotent, and cheap beside the launch
    const cudaError_t e = cudaFuncSetAttribute(join_bwd_kernel<P, KIND, NC, STAGED, ONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(join_bwd_kernel<P, KIND, NC, STAGED, ONE>, dim3((unsigned)p.ctas), dim3(th), smem, st, p);
}
// Iterations (of one or two rows) staged ahead: two, or what fits.  None fits: fp32 operands beyond 8192 columns, the direct variant.
template <typename P, int KIND, bool ONE>
cudaError_t launch_join_bwd_one(cudaStream_t st, int th, int nc, JoinBwd p) {
  const size_t stage = (size_t)nc * join_bytes<P> * th * (nc == 1 ? join_rows<1, ONE> : 1), budget = kJoinSmem / (size_t)join_ctas_per_sm(th);
  p.stages = (int)(budget / stage < 2 ? budget / stage : 2);
  if (p.stages == 0) return launch_join_bwd_nc<P, KIND, 4, false, ONE>(st, th, p);
  if (nc == 1) return launch_join_bwd_nc<P, KIND, 1, true, ONE>(st, th, p);
  if (nc == 2) return launch_join_bwd_nc<P, KIND, 2, true, ONE>(st, th, p);
  return launch_join_bwd_nc<P, KIND, 4, true, ONE>(st, th, p);
}
template <typename P, int KIND>
cudaError_t launch_join_bwd(cudaStream_t st, int th, int nc, const JoinBwd& p) {
  return p.split > 0 ? launch_join_bwd_one<P, KIND, true>(st, th, nc, p) : launch_join_bwd_one<P, KIND, false>(st, th, nc, p);
}

hift_status ns_cfg(int64_t rows, int64_t cols, int32_t steps, const void* scratch, size_t scratch_bytes) {
  if (rows < 1 || cols < 1 || steps < 1 || steps > HIFT_ORTHOGONALIZE_MAX_STEPS) return HIFT_ERR_CFG;
  if (rows > HIFT_ORTHOGONALIZE_MAX_DIM || cols > HIFT_ORTHOGONALIZE_MAX_DIM) return HIFT_ERR_CAPACITY;
  if (!scratch) return HIFT_ERR_INPUT;
  if (!aligned(scratch, 256)) return HIFT_ERR_CFG;
  return scratch_bytes < ns_scratch_bytes(rows, cols) ? HIFT_ERR_CAPACITY : HIFT_OK;
}

}  // namespace

extern "C" {

hift_status hift_k_token_logprobs(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const void* logits, const int32_t* tokens,
                                  double temperature, int32_t n_top, float* logp, float* entropy, float* stats, int32_t* top_ids,
                                  float* top_logp, int32_t* bad, void* stream) {
  float scale, scale2;
  const hift_status s = logprobs_cfg(dtype, rows, vocab, ld, temperature, &scale, &scale2);
  if (s != HIFT_OK) return s;
  if (n_top < 0) return HIFT_ERR_CFG;
  if (n_top > HIFT_MAX_TOP) return HIFT_ERR_CAPACITY;
  if (rows == 0) return HIFT_OK;
  if (!logits || !tokens || !logp || (n_top > 0 && (!top_ids || !top_logp))) return HIFT_ERR_INPUT;
  if (!aligned(logits, dtype == 0 ? 4 : 2) || !words(tokens, logp, entropy, stats, top_ids, top_logp, bad)) return HIFT_ERR_CFG;
  const LpArgs a{tokens, (int)vocab, n_top, ld, rows, scale, scale2, logp, entropy, stats, top_logp, top_ids, bad};
  const cudaError_t e = dtype == 0 ? launch_token_logprobs((cudaStream_t)stream, (const float*)logits, a)
                                   : launch_token_logprobs((cudaStream_t)stream, (const bf16*)logits, a);
  return status_of(e);
}

hift_status hift_k_token_logprobs_bwd(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const void* logits, const int32_t* tokens,
                                      double temperature, const float* stats, const float* entropy, const float* dlogp,
                                      const float* dentropy, void* dlogits, void* stream) {
  float scale, scale2;
  const hift_status s = logprobs_cfg(dtype, rows, vocab, ld, temperature, &scale, &scale2);
  if (s != HIFT_OK) return s;
  if (rows == 0) return HIFT_OK;
  if (!logits || !tokens || !stats || !dlogits || (!dlogp && !dentropy) || (dentropy && !entropy)) return HIFT_ERR_INPUT;
  if (!aligned(logits, dtype == 0 ? 4 : 2) || !aligned(dlogits, dtype == 0 ? 4 : 2) || !words(tokens, stats, entropy, dlogp, dentropy)) return HIFT_ERR_CFG;
  const LpBwdArgs a{tokens, (int)vocab, 0, ld, rows, scale, stats, entropy, dlogp, dentropy};
  const cudaError_t e = dtype == 0 ? launch_token_logprobs_bwd((cudaStream_t)stream, (const float*)logits, (float*)dlogits, a)
                                   : launch_token_logprobs_bwd((cudaStream_t)stream, (const bf16*)logits, (bf16*)dlogits, a);
  return status_of(e);
}

hift_status hift_k_join_fwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double eps, double res_scale, const float* x,
                            const void* h, const void* gain1, const void* bias1, const void* gate, int64_t rows_per_gate,
                            const void* gain2, const void* bias2, float* x_out, void* y, float* stats, void* stream) {
  const hift_status s = join_cfg(dtype, kind, rows, cols, res_scale, gate, rows_per_gate);
  if (s != HIFT_OK) return s;
  if (!(eps >= 0.0) || !isfinite((float)eps)) return HIFT_ERR_CFG;
  if (rows == 0) return HIFT_OK;
  if (!x || !h || !x_out || !stats || (gain2 && !y) || (kind == 0 && ((gain1 && !bias1) || (gain2 && !bias2)))) return HIFT_ERR_INPUT;
  if (!aligned(x, 16) || !aligned(h, 16) || !aligned(x_out, 16) || !aligned(gain1, 16) || !aligned(bias1, 16) || !aligned(gate, 16) ||
      !aligned(gain2, 16) || !aligned(bias2, 16) || (gain2 && !aligned(y, 16)) || !words(stats)) return HIFT_ERR_CFG;
  JoinFwd p{x, h, gain1, bias1, gate, gain2, bias2, x_out, y, stats, rows, gate ? rows_per_gate : rows, (int)cols, (float)eps, (float)res_scale};
  int th, nc;
  // up to 4096 columns 8 warps of 16 columns a thread: 123 us at 16384 x 4096 bf16, the copy rate; 16 warps of 8 columns: 138
  join_shape(cols, cols <= 4096 ? 8 : 16, &th, &nc);
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = dtype == 0 ? (kind == 0 ? launch_join_fwd<float, 0>(st, th, nc, p) : launch_join_fwd<float, 1>(st, th, nc, p))
                                   : (kind == 0 ? launch_join_fwd<bf16, 0>(st, th, nc, p) : launch_join_fwd<bf16, 1>(st, th, nc, p));
  return status_of(e);
}

size_t hift_join_bwd_scratch_bytes(int64_t rows, int64_t cols, int64_t rows_per_gate) {
  if (rows < 1 || cols < 8 || cols % 8 || rows > INT32_MAX || cols > kJoinMaxCols) return 0;
  return (size_t)join_plan(rows, cols, rows_per_gate).ctas * cols * kJoinPlanes * sizeof(float);
}

hift_status hift_k_join_bwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double res_scale, const void* dy,
                            const float* dx_out, const float* x_out, const void* h, const float* stats, const void* gain1,
                            const void* bias1, const void* gate, int64_t rows_per_gate, const void* gain2, float* dx, void* dh,
                            float* dgain1, float* dbias1, float* dgate, float* dgain2, float* dbias2, void* scratch,
                            size_t scratch_bytes, void* stream) {
  const hift_status s = join_cfg(dtype, kind, rows, cols, res_scale, gate, rows_per_gate);
  if (s != HIFT_OK) return s;
  if (!words(stats, dgain1, dbias1, dgain2, dbias2)) return HIFT_ERR_CFG;
  cudaStream_t st = (cudaStream_t)stream;
  if (rows == 0) {                                         // no rows: the sums over them are zero
    for (float* q : {dgain1, dbias1, dgain2, dbias2})
      if (q && cudaMemsetAsync(q, 0, (size_t)cols * sizeof(float), st) != cudaSuccess) return HIFT_ERR_CUDA;
    return HIFT_OK;
  }
  if (!h || !stats || !dx || !dh || !scratch || (gain2 && (!dy || !x_out)) || (!gain2 && !dx_out)) return HIFT_ERR_INPUT;
  if ((dgate && !gate) || ((dgain1 || dbias1) && !gain1) || ((dgain2 || dbias2) && !gain2) || (kind == 1 && (dbias1 || dbias2))) return HIFT_ERR_INPUT;
  if (kind == 0 && gain1 && dgate && !bias1) return HIFT_ERR_INPUT;
  const void* ptrs[] = {dy, dx_out, x_out, h, gain1, bias1, gate, gain2, dx, dh, dgate, scratch};
  for (const void* q : ptrs) if (!aligned(q, 16)) return HIFT_ERR_CFG;
  const JoinPlan pl = join_plan(rows, cols, gate ? rows_per_gate : rows);
  if (scratch_bytes < (size_t)pl.ctas * cols * kJoinPlanes * sizeof(float)) return HIFT_ERR_CAPACITY;
  JoinBwd p{dy, dx_out, x_out, h, stats, gain1, bias1, gate, gain2, dx, dh, dgate, (float*)scratch, rows, pl.rows_per_gate, (int)cols,
            pl.ctas, 0, pl.split, pl.gates_per_cta, (float)res_scale};
  int th, nc;
  join_shape(cols, 16, &th, &nc);
  cudaError_t e = dtype == 0 ? (kind == 0 ? launch_join_bwd<float, 0>(st, th, nc, p) : launch_join_bwd<float, 1>(st, th, nc, p))
                             : (kind == 0 ? launch_join_bwd<bf16, 0>(st, th, nc, p) : launch_join_bwd<bf16, 1>(st, th, nc, p));
  if (e == cudaSuccess && (dgain1 || dbias1 || dgain2 || dbias2 || (dgate && pl.split > 0))) {
    const JoinSums o{{dgain1, dbias1, dgain2, dbias2, pl.split > 0 ? dgate : nullptr}};
    const dim3 g((unsigned)((cols + 31) / 32), (unsigned)(kJoinPlanes - 1 + (dgate && pl.split > 0 ? pl.n_gates : 0)));
    int th = 256;
    while (th < 1024 && pl.ctas > th / 8 * 4) th *= 2;
    e = launch_pdl(join_sums_kernel, g, dim3(th), 0, st, (const float*)scratch, o, pl.ctas, (int)cols, pl.split);
  }
  return status_of(e);
}

size_t hift_orthogonalize_scratch_bytes(int64_t rows, int64_t cols) {
  return rows < 1 || cols < 1 || rows > HIFT_ORTHOGONALIZE_MAX_DIM || cols > HIFT_ORTHOGONALIZE_MAX_DIM ? 0 : ns_scratch_bytes(rows, cols);
}

hift_status hift_k_orthogonalize(int32_t dtype, int64_t rows, int64_t cols, const void* g, void* o, int32_t steps, void* scratch,
                                 size_t scratch_bytes, void* stream) {
  if (dtype < 0 || dtype > 1) return HIFT_ERR_CFG;
  const hift_status s = ns_cfg(rows, cols, steps, scratch, scratch_bytes);
  if (s != HIFT_OK) return s;
  if (!g || !o) return HIFT_ERR_INPUT;
  if (!aligned(g, dtype == 0 ? 4 : 2) || !aligned(o, 2)) return HIFT_ERR_CFG;
  const NsUpdate to{(bf16*)o, nullptr, nullptr, 0.f, 0.f};
  const cudaError_t e = dtype == 0 ? launch_orthogonalize((cudaStream_t)stream, rows, cols, (const float*)g, nullptr, 0.f, 0, steps, to, scratch)
                                   : launch_orthogonalize((cudaStream_t)stream, rows, cols, (const bf16*)g, nullptr, 0.f, 0, steps, to, scratch);
  return status_of(e);
}

hift_status hift_muon_step(int64_t rows, int64_t cols, void* param_bf16, float* master, const float* grad, float* momentum_buf,
                           void* scratch, size_t scratch_bytes, double lr, double momentum, int32_t nesterov, double weight_decay,
                           int32_t steps, void* stream) {
  const hift_status s = ns_cfg(rows, cols, steps, scratch, scratch_bytes);
  if (s != HIFT_OK) return s;
  const float decay = (float)(1.0 - lr * weight_decay), size = (float)(lr * 0.2 * sqrt((double)(rows > cols ? rows : cols)));
  if (!isfinite(lr) || !isfinite(weight_decay) || !isfinite(decay) || !isfinite(size) || !(momentum >= 0.0 && momentum < 1.0)) return HIFT_ERR_CFG;
  if (!master || !grad || !momentum_buf) return HIFT_ERR_INPUT;
  if (!aligned(master, 4) || !aligned(grad, 4) || !aligned(momentum_buf, 4) || !aligned(param_bf16, 2)) return HIFT_ERR_CFG;
  const NsUpdate to{nullptr, master, (bf16*)param_bf16, decay, size};
  const cudaError_t e = launch_orthogonalize((cudaStream_t)stream, rows, cols, grad, momentum_buf, (float)momentum, nesterov != 0, steps, to, scratch);
  return status_of(e);
}

}  // extern "C"
