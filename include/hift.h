/*
 * hift.h -- C ABI of the B200 hierarchical fine-tuning (HiFT) training step.
 *
 * One context = one model on one GPU.  A call to hift_step() performs one
 * iteration of the paper's Algorithm 1: select the active group (steps c-g),
 * full forward pass (h), move that group's optimizer state to the GPU (i),
 * back-propagate only as far down as the group and form weight gradients only
 * inside it (the "Backpropagation" step), update the group with the chosen
 * optimizer, clear gradients, move the state back to host memory (k), and
 * advance the learning-rate schedule once every full cycle of groups (final
 * branch of Algorithm 1).  Only the active group's parameters change
 * (Eq. 2-3: the binary mask beta_i).
 *
 * Conventions
 *   - "dev" pointers are CUDA device pointers on the context's GPU, "host"
 *     pointers are ordinary host memory.  The caller owns every buffer it
 *     passes in; the library never frees or keeps them past the call.
 *   - Everything the context allocates (device and pinned host memory) is
 *     released by hift_destroy().
 *   - Every function returns a hift_status (or a plain value for getters);
 *     nothing aborts, throws, or traps on the device.
 *   - A context is not thread-safe.  Work is issued on the CUDA stream given to
 *     hift_create() plus copy streams the context owns.
 *   - Row-major everywhere.  Linear weights are [out_features, in_features].
 */
#ifndef HIFT_H_
#define HIFT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hift_ctx hift_ctx;

typedef enum {
  HIFT_OK = 0,
  HIFT_ERR_CFG = 1,          /* invalid or unsupported configuration / argument      */
  HIFT_ERR_OOM_DEVICE = 2,   /* cudaMalloc failed                                    */
  HIFT_ERR_OOM_PINNED = 3,   /* pinned host allocation failed                        */
  HIFT_ERR_INPUT = 4,        /* token id or label out of range, NULL pointer         */
  HIFT_ERR_NONFINITE = 5,    /* the loss of the step was NaN/Inf (no update was made)*/
  HIFT_ERR_TIMEOUT = 6,      /* a bounded device-side wait gave up (no update made)  */
  HIFT_ERR_CUDA = 7,         /* any other CUDA runtime/driver error                  */
  HIFT_ERR_CAPACITY = 8      /* size exceeds the library's built-in scratch capacity */
} hift_status;

/* Model description.  Units (the paper's "layers", Section "Hierarchical
 * Training": the embedding is the bottom layer, the head the top layer):
 * unit 0 = all embeddings, units 1..n_blocks = transformer blocks,
 * unit n_blocks+1 = head (final norm + LM matrix, or classifier). */
typedef struct {
  int32_t arch;        /* 0 pre-LN causal decoder (GELU, learned positions)
                          1 post-LN bidirectional encoder + classifier on token 0
                          2 LLaMA-style (RMSNorm, RoPE, SwiGLU, no biases)          */
  int32_t n_blocks, d_model, n_heads, d_ffn, vocab;
  int32_t max_pos;     /* rows of the learned position table (arch 0,1)            */
  int32_t n_classes;   /* arch 1 only                                              */
  int32_t causal;      /* 1: attention masks keys after the query                  */
  int32_t tie_head;    /* 1: LM head shares tok_emb; the matrix belongs to unit 0  */
  int32_t dtype;       /* 0: fp32 params+activations; 1: bf16 with fp32 master     */
  int32_t batch, seq;  /* fixed per context                                        */
  double  norm_eps, rope_base;
  double  dropout;     /* probability p in [0, 1) of dropping an element at the outputs of each block's
                          attention projection and feed-forward network (before the residual addition)
                          and at the embedding output; kept values are scaled by 1/(1-p); 0 = none.
                          The paper fine-tunes with the models' usual dropout without describing it.   */
  uint64_t dropout_seed; /* the mask is Philox4x32-10(key = seed, counter = (element / 4, site, step)),
                          word element % 4, kept iff word >= floor(p 2^32); site 0 = embedding,
                          1 + 2 i = block i attention output, 2 + 2 i = its feed-forward output;
                          step = t.  Reproducible from (seed, t) alone, also across checkpoints.     */
  double  attn_dropout; /* probability in [0, 1) of dropping an attention probability, after the softmax and
                          before the product with V (kept ones scaled by 1/(1-p)); 0 = none.  Same seed;
                          site 1000 + i for block i; the probabilities are numbered ((b H + h) S + q) S' + k
                          with S' = seq rounded up to a multiple of 4.  The tensor-core (tcgen05) and the
                          CUDA-core attention kernels apply it; the warp-level fallback kernels do not, so a
                          bf16 launch they would have taken goes to the CUDA-core kernels.            */
} hift_model_cfg;

/* Grouping and order (paper: Notation paragraph; Algorithm 1 "UpdateStrategy"). */
typedef struct {
  int32_t layers_per_group;  /* m: consecutive units per group, last group short   */
  int32_t split_emb_head;    /* 1: embedding | blocks in chunks of m | head        */
  int32_t order;             /* 0 bottom2up, 1 top2down, 2 random (shuffled once)  */
  uint64_t order_seed;       /* seed of the one-time shuffle                       */
  const int32_t *group_sizes;/* host; NULL = the uniform rule above.  Otherwise n_group_sizes counts of
                                consecutive units per group, bottom first, each >= 1, summing to
                                n_blocks + 2 (groups of unequal size: the paper's grouping is uniform,
                                this is the same fixed partition with the chunk lengths chosen by the
                                caller); read during hift_create only, not kept            */
  int32_t n_group_sizes;
  int32_t literal_queue;     /* 1: Algorithm 1, steps c-d, taken literally: a queue of the n units in the strategy's
                                order (random: shuffled once); every step pops m units from its head and appends
                                them to its tail.  When m divides n this is the fixed partition above.  When it does
                                not, the sets drift: a set can wrap around (top and bottom units together) and a unit
                                is trained ceil- or floor-many times per pass; every unit then keeps its own master,
                                state and update count, a step trains a SET of units (hift_num_sets() distinct sets,
                                set id = step mod that; hift_active_group() returns the set id and hift_set_units()
                                its units), and the learning rate still moves every k = floor(n/m) + 1 steps
                                (hift_num_groups()).  State paging uses one slot in this mode (sets share units).
                                Not with group_sizes, split_emb_head or sharded state.                            */
} hift_group_cfg;

/* Optimizer P and schedule eta_t of Algorithm 1's "Require" list; state residency
 * per its steps i and k ("MoveOptimizerState2GPU/2CPU") and the adapted mixed
 * precision of Section "Mixing Precision" (only the active group's fp32 master
 * is on the GPU). */
typedef struct {
  int32_t kind;              /* 0 AdamW, 1 AdaGrad, 2 SGD with momentum, 3 plain SGD
                                (no optimizer state: only the fp32 master, if any, is paged),
                                4 Adafactor (factored second moment: rows + cols floats of state per
                                matrix; `lr` caps the relative step, `eps` is its epsilon_1;
                                epsilon_2 = 1e-3, clipping d = 1, decay exponent -0.8, no momentum) */
  int32_t sched;             /* 0 constant, 1 linear: warm-up, then decay to 0     */
  int32_t total_cycles;      /* horizon C of the linear schedule, in cycles        */
  int32_t offload_state;     /* 1: inactive groups' master+state in pinned host    */
  int32_t prefetch_groups;   /* state slots on the GPU beyond the first, 0..3 (each the size of the largest
                                group's paged state).  0: one slot, upload issued after the forward pass
                                (the paper's order).  1: two slots, upload at the start of the group's
                                own step, overlapped with the previous write-back.  p >= 2: p + 1 slots,
                                the uploads of the next p - 1 steps' groups are issued ahead (the order
                                is known), so transfers stream across steps and a step no longer lasts
                                at least one transfer.  Residency rule of Algorithm 1 steps i/k kept:
                                only the active group and groups whose transfer is in flight are on
                                the GPU.  Same bits in every mode.                                   */
  int32_t recompute;         /* 1: frozen blocks above the active group keep only their input during the
                                forward pass; what their backward (dX) needs is recomputed block by block in
                                the backward pass.  Same bits, less HBM (the paper's concern), one extra
                                forward of those blocks per step.  0: keep (default)                */
  int32_t warmup_cycles;     /* W (sched 1; the warm-up the paper's hyper-parameter tables list, counted in
                                cycles because the rate moves once per cycle): cycle c < W runs at
                                lr*c/W, cycle c >= W at lr*max(0, (C-c)/(C-W)); 0 = none             */
  int32_t shard_rank;        /* data-parallel ranks may split the optimizer state (ZeRO stage 1): with   */
  int32_t shard_world;       /* shard_world = W > 1 this context holds fp32 master and state (device     */
                             /* slots, pinned blobs, paging) only for piece shard_rank of every group's  */
                             /* span (W contiguous pieces of whole 128-element lines, hift_shard_range), */
                             /* and hift_step_end / hift_step_finish update only that piece; the caller  */
                             /* reduces each piece of the gradient to its owner before, and broadcasts   */
                             /* each piece of the updated parameters (hift_param_view) from its owner    */
                             /* after.  The update is element-wise, so the pieces together are exactly   */
                             /* the unsharded update.  0 or 1 = off.  Not with Adafactor (its statistics */
                             /* span rows and columns); checkpoints are refused while sharded; outside   */
                             /* its piece hift_get_param returns the model value, hift_get_state zeros.  */
  int32_t grad_bf16;         /* 1: the active group's gradient is kept in bf16: the weight-gradient GEMMs store  */
                             /* bf16 from their fp32 accumulators, the other gradient producers round once, the   */
                             /* optimizer reads bf16; half the gradient buffer, half the exchange volume of a     */
                             /* data-parallel step, 2 bytes per element less optimizer traffic.  One rounding of  */
                             /* 2^-9 relative per gradient element (within the 2e-2 gradient tolerance; the       */
                             /* update given that gradient is exact as before).  bf16 models with AdamW, AdaGrad, */
                             /* SGD-momentum or SGD only.  0: fp32 gradients.                                     */
  double lr, beta1, beta2, eps, weight_decay, momentum;
} hift_opt_cfg;

/* Build a context.  `cuda_stream` is a cudaStream_t (NULL = default stream).
 * Parameters start as zeros; fill them with hift_set_param() or
 * hift_init_synthetic().  Fails with HIFT_ERR_OOM_* and leaves *out NULL if the
 * device or pinned memory cannot be had (everything allocated so far is released).
 * One process drives one GPU: the tensor-core kernels' time-out flag, the SM count and the
 * driver entry point for tensor maps are looked up once per process, for the device that
 * was current at the first call; contexts on two different GPUs in one process are not
 * supported (several contexts on the same GPU are).
 * batch * seq <= 65536 tokens a step (HIFT_ERR_CFG beyond it). */
hift_status hift_create(const hift_model_cfg *model, const hift_group_cfg *groups,
                        const hift_opt_cfg *opt, void *cuda_stream, hift_ctx **out);
void hift_destroy(hift_ctx *ctx);

/* One iteration of Algorithm 1 on the group hift_active_group() names.
 * tokens_dev: int32 [batch, seq].  labels_dev: int32 [batch, seq] (arch 0, 2;
 * -1 = position ignored) or int32 [batch] (arch 1).  The mean cross-entropy of
 * the batch, computed before the update, is written to *loss_host.  Returns
 * after the loss is on the host; state write-back may still be in flight.
 * A step that fails changes nothing: when a bounded device-side wait gave up
 * (HIFT_ERR_TIMEOUT), a token id or label was out of range (HIFT_ERR_INPUT; the
 * id is clamped on the device so that the pass itself stays in bounds) or the
 * loss is not finite (HIFT_ERR_NONFINITE), the optimizer kernels see the
 * failure on the device and store nothing, so every parameter, master value and
 * optimizer-state value of every group keeps its bits, the group's update
 * count and t do not advance, and the next call trains the same group again.
 * (Gradients that overflow while the loss stays finite are not detected.) */
hift_status hift_step(hift_ctx *ctx, const int32_t *tokens_dev, const int32_t *labels_dev,
                      float *loss_host);
/* Same, with the batch in host memory (validated on the host, then copied to
 * the GPU inside the call; invalid input is rejected before anything runs). */
hift_status hift_step_host(hift_ctx *ctx, const int32_t *tokens_host, const int32_t *labels_host,
                           float *loss_host);

/* Batches of unequal length, padded on the right to `seq` (what fine-tuning on the paper's tasks feeds a
 * model; the paper does not discuss it): lens_host[b] in [1, seq] is the number of real tokens of batch
 * entry b.  From the next step on, attention lets every query of entry b see keys 0 .. lens_host[b]-1 only
 * (on top of the causal mask, if any); NULL switches the table off again.  Padded positions still run
 * through the model; the caller keeps them out of the loss with label -1 (arch 0, 2; arch 1 reads
 * token 0 only), and then no gradient flows through them.  The table is copied during the call.
 * HIFT_ERR_INPUT if a length is out of range. */
hift_status hift_set_key_lengths(hift_ctx *ctx, const int32_t *lens_host);

/* The same step in two halves, for data-parallel training (several contexts, one per GPU, each
 * on its shard of the batch; the paper's method itself is single-device).  hift_step_begin runs
 * the forward pass and the truncated backward pass and returns the loss; the active group's flat
 * fp32 gradient (its tensors in layout order, zero in the alignment gaps) is then exposed by
 * hift_grad_view as a device pointer the caller may reduce over ranks and scale (1/k of the
 * volume a full-parameter step would exchange); hift_step_end applies the optimizer to the group,
 * starts the state write-back and advances t.  Work the caller enqueued on the stream given to
 * hift_create is ordered before the update.  begin/end must alternate; hift_step in between is
 * refused with HIFT_ERR_CFG.  A hift_step_begin that fails leaves no update pending.
 * hift_step_abort drops a pending update instead of applying it (t does not advance): what
 * every rank calls when any rank's first half failed, so that replicas stay identical. */
hift_status hift_step_begin(hift_ctx *ctx, const int32_t *tokens_dev, const int32_t *labels_dev,
                            float *loss_host);
hift_status hift_grad_view(hift_ctx *ctx, void **grad_dev, size_t *n);   /* n elements of hift_grad_elem_bytes() each */
int32_t     hift_grad_elem_bytes(const hift_ctx *ctx);                    /* 4: fp32 gradients, 2: bf16 (grad_bf16) */
hift_status hift_step_end(hift_ctx *ctx);
hift_status hift_step_abort(hift_ctx *ctx);

/* The exchange overlapped with the backward pass.  The truncated backward pass finishes the group's
 * gradient from the top of its flat span downwards (the last block's down projection first, the lowest
 * unit's first norm last), so the tail of the buffer can be reduced over the ranks while the head is
 * still being computed: with one all-reduce per chunk this hides all but the last chunk's exchange
 * behind the remaining dX / dW GEMMs.
 *   hift_step_begin_async  enqueues forward + truncated backward and returns without waiting;
 *   hift_grad_num_chunks / hift_grad_chunk  list the chunks of hift_grad_view's buffer in the order
 *       they become final (offset and length in elements; together they tile the span exactly once;
 *       each at least the size set by hift_set_grad_chunk_bytes, default 32 MiB, except the last);
 *   hift_grad_chunk_wait   makes `cuda_stream` (the caller's communication stream) wait until chunk
 *       i is final; waiting for the last chunk also covers the step's gate word;
 *   hift_gate_view         device address of the step's gate word (int32): 0 = the update goes ahead,
 *       otherwise a positive code of what failed.  Ranks reduce it with MAX next to the last chunk,
 *       so that all of them call the update off when one of them failed;
 *   hift_step_finish       = hift_step_end that also returns the loss: orders itself after the work
 *       enqueued on the stream given to hift_create (make that stream wait for the communication
 *       stream first), applies the optimizer, starts the write-back, waits for the step and returns
 *       its status.  A rank whose own pass was fine but whose gate word a peer raised returns the
 *       peer's failure.
 * The chunk plan itself is host logic; hift_plan_grad_chunks runs it on a caller-given tensor list
 * (ascending offsets) and completion order without touching a GPU: chunk_off / chunk_n receive the
 * chunks, chunk_after[i] the index into completion_order after which chunk i is final.  Returns the
 * number of chunks, or -1 (bad arguments, max_chunks too small). */
hift_status hift_step_begin_async(hift_ctx *ctx, const int32_t *tokens_dev, const int32_t *labels_dev);
int32_t     hift_grad_num_chunks(const hift_ctx *ctx);
hift_status hift_grad_chunk(const hift_ctx *ctx, int32_t i, size_t *offset, size_t *n);
hift_status hift_grad_chunk_wait(hift_ctx *ctx, int32_t i, void *cuda_stream);
hift_status hift_gate_view(hift_ctx *ctx, int32_t **gate_dev);
hift_status hift_set_grad_chunk_bytes(hift_ctx *ctx, size_t bytes);
/* Sharded optimizer state (hift_opt_cfg.shard_world): the piece of group g's flat span that `rank` holds, as
 * offset and length in elements of hift_grad_view / hift_param_view; and the parameters of the group trained
 * by the step in flight (or the last one) as the forward pass reads them (bf16: elem_bytes 2, or fp32: 4),
 * a device pointer to the group's whole span, for the exchange of the updated pieces. */
hift_status hift_shard_range(const hift_ctx *ctx, int32_t g, int32_t rank, size_t *offset, size_t *n);
hift_status hift_param_view(hift_ctx *ctx, void **param_dev, size_t *n, int32_t *elem_bytes);
hift_status hift_step_finish(hift_ctx *ctx, float *loss_host);
int32_t     hift_plan_grad_chunks(const size_t *offsets, const size_t *sizes, int32_t n_tensors, size_t span_elems,
                                  const int32_t *completion_order, int32_t n_completed, size_t min_chunk_elems,
                                  size_t *chunk_off, size_t *chunk_n, int32_t *chunk_after, int32_t max_chunks);

int32_t hift_active_group(const hift_ctx *ctx);   /* group the NEXT hift_step trains */
int32_t hift_num_groups(const hift_ctx *ctx);     /* k: steps per learning-rate cycle */
int32_t hift_num_sets(const hift_ctx *ctx);       /* distinct sets of units the schedule trains (= k unless the queue drifts) */
/* Units of set `set_id` (ascending) into units_out[0 .. cap); *n_units receives their number. */
hift_status hift_set_units(const hift_ctx *ctx, int32_t set_id, int32_t *units_out, int32_t cap, int32_t *n_units);
int64_t hift_step_count(const hift_ctx *ctx);     /* t, steps taken so far           */
double  hift_current_lr(const hift_ctx *ctx);     /* lr the NEXT step will use       */
/* Units of group (set) g: writes the first and last unit id (inclusive); HIFT_ERR_CFG for a set of the drifting
 * queue that is not an interval of units (use hift_set_units). */
hift_status hift_group_units(const hift_ctx *ctx, int32_t g, int32_t *unit_lo, int32_t *unit_hi);
/* Force the group trained by the next steps (depth sweeps); -1 restores the schedule. */
hift_status hift_force_group(hift_ctx *ctx, int32_t g);
/* The same for a list: the next steps train groups[0], groups[1], ..., groups[n-1], groups[0], ...
 * (host array, copied; n = 0 restores the schedule; a forced single group takes precedence).  Unlike
 * a group forced step by step, the list is known ahead, so look-ahead paging works on it: what a
 * benchmark uses to time an even sample of the cycle.  t, the learning rate and the update counts
 * advance as always. */
hift_status hift_force_sequence(hift_ctx *ctx, const int32_t *groups, int32_t n);

/* High-water mark, in bytes, of all device memory the context holds. */
size_t hift_peak_hbm_bytes(const hift_ctx *ctx);
/* Bytes of pinned host memory the context holds. */
size_t hift_pinned_host_bytes(const hift_ctx *ctx);

/* ---- parameter / gradient access (tests and checkpoints) ---------------- */
int32_t hift_num_tensors(const hift_ctx *ctx);
/* name_out: at least 64 bytes.  A vector has rows = 1. */
hift_status hift_tensor_info(const hift_ctx *ctx, int32_t tensor, char *name_out,
                             int32_t *unit, int64_t *rows, int64_t *cols);
/* fp32 master values of one tensor, host memory, `n` = rows*cols elements.
 * set: also refreshes the bf16 model copy (round to nearest even). */
hift_status hift_set_param(hift_ctx *ctx, int32_t tensor, const float *src_host, size_t n);
hift_status hift_get_param(hift_ctx *ctx, int32_t tensor, float *dst_host, size_t n);
/* The value the forward pass reads (bf16 widened to fp32, or the fp32 itself). */
hift_status hift_get_model_param(hift_ctx *ctx, int32_t tensor, float *dst_host, size_t n);
/* Optimizer state `which` (0: first moment / accumulator / momentum, 1: second moment). */
hift_status hift_get_state(hift_ctx *ctx, int32_t tensor, int32_t which, float *dst_host, size_t n);
/* Adafactor only: which = 0 the row statistics R [rows] (for a vector, rows = 1: its second
 * moment V [cols]), which = 1 the column statistics C [cols]. */
hift_status hift_get_factored_state(hift_ctx *ctx, int32_t tensor, int32_t which, float *dst_host, size_t n);
/* fp32 gradient of a tensor of the group trained by the LAST step. */
hift_status hift_get_grad(hift_ctx *ctx, int32_t tensor, float *dst_host, size_t n);
/* Fill every parameter on the device: matrices N(0, std^2) from a counter-based
 * hash of (seed, element index), gains 1, biases 0; optimizer state zero. */
hift_status hift_init_synthetic(hift_ctx *ctx, uint64_t seed, double std);

/* Weights from a file in the library's container format ("HIFTWTS1": magic[8], uint32 n, then n records of
 * { char name[64]; uint32 dtype (0 fp32, 1 bf16); uint64 rows, cols; rows*cols elements }, names and shapes
 * as hift_tensor_info reports them).  Each record goes through hift_set_param (fp32 master and bf16 model
 * copy; optimizer state is left alone).  strict != 0: every tensor of the model must be in the file.
 * *n_loaded (may be NULL) receives the number of tensors set.  HIFT_ERR_INPUT for a missing / short /
 * foreign file, an unknown or repeated tensor, a wrong shape; tensors set before the error stay set.
 * The package's weights.py writes this format and converts safetensors checkpoints with the public
 * LLaMA / GPT-2 / RoBERTa tensor names into it. */
hift_status hift_load_weights(hift_ctx *ctx, const char *path, int32_t strict, int32_t *n_loaded);

/* Checkpoint: the whole training state is the fp32 master (or fp32 parameters), the optimizer
 * state and update count of every group (which Algorithm 1 keeps on the host between a group's
 * turns anyway), and the step counter t; the group order follows from the configuration.
 * hift_load needs a context created with the same configuration (HIFT_ERR_CFG otherwise) and
 * rebuilds the bf16 model copy.  A missing / short / foreign file gives HIFT_ERR_INPUT. */
hift_status hift_save(hift_ctx *ctx, const char *path);
hift_status hift_load(hift_ctx *ctx, const char *path);

/* ---- instrumentation ------------------------------------------------------ */
/* Kernel classes for hift_profile(). */
enum { HIFT_K_GEMM_FWD = 0, HIFT_K_GEMM_DX = 1, HIFT_K_GEMM_DW = 2, HIFT_K_ATTN_FWD = 3,
       HIFT_K_ATTN_BWD = 4, HIFT_K_NORM = 5, HIFT_K_ELEMWISE = 6, HIFT_K_CE = 7,
       HIFT_K_EMBED = 8, HIFT_K_OPT = 9, HIFT_K_REDUCE = 10, HIFT_K_NUM = 11 };
/* on=1: bracket every kernel launch of the following steps with CUDA events on
 * the launching stream and accumulate per class; on=0 stops.  Resets counters. */
hift_status hift_profile_enable(hift_ctx *ctx, int32_t on);
/* Accumulated since enable: launches, device milliseconds and algorithmic work
 * (flops for GEMM/attention classes, bytes for the others). */
hift_status hift_profile(hift_ctx *ctx, int32_t kernel_class, int64_t *launches,
                         double *millis, double *work);
/* Kernel launches issued by the last hift_step (all classes). */
int64_t hift_last_step_launches(const hift_ctx *ctx);
/* Bytes paged host->device and device->host by the last step. */
hift_status hift_last_step_paging(const hift_ctx *ctx, size_t *h2d_bytes, size_t *d2h_bytes);

/* Device timeline of the last step's state paging (Algorithm 1 steps i and k), in milliseconds
 * after the step's first kernel: [0] H2D begin, [1] H2D end (of the upload that made the group
 * resident: negative when an earlier step issued it ahead), [2] optimizer reaches its wait
 * for the state, [3] wait over, [4] D2H begin, [5] D2H end.  NaN where there is nothing to
 * report (offload off).  Waits for the copies to finish. */
hift_status hift_last_step_timeline(hift_ctx *ctx, double *ms6);

/* The tensor-core GEMM bounds every device-side wait; a wait that gives up records a code in a
 * device flag, after which every tensor-core GEMM launch returns at once and hift_step reports
 * HIFT_ERR_TIMEOUT.  This call reads the flag (set_value < 0) or overwrites it first
 * (set_value >= 0; 0 clears it, which is how a caller resumes after a time-out, and a non-zero
 * value lets a test walk the time-out path without stalling anything).  Returns the flag, or -1
 * if the tensor-core path is unavailable.  Synchronises the device. */
int32_t hift_tc_error_flag(int32_t set_value);

/* Code-path switches for tests and A/B timing; every one defaults to 1, the fast path.  which = 0: CTA-pair
 * tiles in the tensor-core GEMM (0 = one CTA per tile); 1: programmatic dependent launch (0 = plain stream
 * order); 2: tcgen05 attention forward, 3: tcgen05 attention backward (0 = the warp-level mma.sync kernels); 6: the
 * orthogonalised update of small matrices in one launch (0 = the products of the large ones, which also run where a
 * device cannot hold the cluster of up to 16 blocks that the one launch takes).
 * value >= 0 sets the switch, value < 0 only reads it; returns the previous value, or -1 for an unknown
 * switch.  Process-wide, consulted at every launch, not thread-safe.  Results do not depend on switches 0
 * and 1 (same bits); 2, 3 and 6 select kernels with a different summation order (6: and other roundings).
 * Two more, for fault-path tests that need no faulting GPU: which = 4: the value-th pinned host allocation
 * from now on (0 = the next one) fails as if the host were out of pinned memory, once (value -1 = off),
 * so that hift_create's HIFT_ERR_OOM_PINNED path and its clean-up run; which = 5: contexts created while it
 * is 1 run in checked mode: every slice of the activation arena is followed by a 256-byte guard region that
 * each step paints before its first kernel, and hift_check_arena() counts the regions a step wrote into. */
int32_t hift_test_switch(int32_t which, int32_t value);
/* Checked mode only (-1 otherwise): guard regions of the last step's arena plan that no longer hold their
 * pattern (0 = no kernel wrote past the end of its buffer), and how many regions there are. */
int64_t hift_check_arena(hift_ctx *ctx);
int64_t hift_arena_guard_count(const hift_ctx *ctx);

/* ---- the group-local fused optimizer on caller-owned flat buffers --------
 * One streaming pass over n elements (the update Algorithm 1 applies to the
 * active group once "UpdateOptimizerParameter" has pointed P at theta_s).  All
 * pointers are device pointers, 16-byte aligned.  master/grad/s0/s1 are fp32;
 * s1 is used by AdamW only (may be NULL otherwise), s0 by all but plain SGD
 * (kind 3; may be NULL there); param_bf16 may be NULL
 * (fp32 configs).  tau >= 1 is the number of updates this group has had,
 * including this one (bias correction).  Launches on `cuda_stream`, does not
 * synchronise. */
hift_status hift_opt_step(int32_t kind, size_t n, void *param_bf16_dev, float *master_dev,
                          const float *grad_dev, float *s0_dev, float *s1_dev,
                          double lr, double beta1, double beta2, double eps,
                          double weight_decay, double momentum, int64_t tau,
                          void *cuda_stream);

/* Adafactor (one of the optimizers the paper profiles, without formulas; built in the form
 * torch.optim.Adafactor uses for Shazeer & Stern 2018, Algorithms 4-5: epsilon_1 is a lower clamp on the
 * factored second-moment estimate and on the root of it, not a term added to the squared gradient)
 * on one caller-owned tensor [rows, cols] (rows = 1: a vector, unfactored).
 * master/grad: fp32 [rows*cols]; state: fp32, R[rows] | C[cols] for a matrix, V[cols] for a
 * vector; scratch: fp32, 2*rows + 64*cols + 8 floats; param_bf16 may be NULL.  tau >= 1 as in
 * hift_opt_step.  Launches several small kernels on `cuda_stream`; does not synchronise. */
hift_status hift_adafactor_step(int64_t rows, int64_t cols, void *param_bf16_dev, float *master_dev,
                                const float *grad_dev, float *state_dev, float *scratch_dev,
                                double lr, double eps1, double weight_decay, int64_t tau, void *cuda_stream);

/* ---- single kernels on caller-owned device buffers (per-kernel parity) ----
 * These are the pieces of Algorithm 1's "ForwardPropagation"/"Backpropagation"
 * steps.  dtype 0: fp32 operands, 1: bf16 operands.  All launch on `cuda_stream`
 * and do not synchronise. */
/* form 0: y[M,N]  = x[M,K] * w[N,K]^T (+ bias[N]);             out has operand type
 * form 1: dx[M,K] = dy[M,N] * w[N,K];                          out has operand type
 * form 2: dw[N,K] = dy[M,N]^T * x[M,K];                        out is fp32
 * residual_dev (forms 0,1; optional): fp32 [M, out cols]; when given the output
 * is fp32 too (the residual stream is kept in fp32).
 * `path`: 0 = pick automatically, 1 = force the CUDA-core kernel, 2 = force the
 * tcgen05 tensor-core kernel (bf16 only; HIFT_ERR_CFG if the shape is not eligible). */
hift_status hift_k_linear(int32_t form, int32_t dtype, int32_t path, int64_t M, int64_t N, int64_t K,
                          const void *a_dev, const void *b_dev, void *out_dev,
                          const void *bias_dev, const float *residual_dev, void *cuda_stream);
/* qkv[T,3d] (q|k|v column blocks, head h at columns h*d_h) -> o[T,d], lse[B,H,S] fp32.
 * key_lens_dev: int32 [batch] or NULL; entry b attends to keys 0 .. key_lens[b]-1 only (values are
 * clamped to [1, seq] on the device). */
hift_status hift_k_attention_fwd(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads,
                                 int32_t d_head, int32_t causal, const void *qkv_dev, void *o_dev,
                                 float *lse_dev, const int32_t *key_lens_dev, void *cuda_stream);
/* -> dqkv[T,3d]; dsum_dev is fp32 scratch of batch*seq*n_heads elements.  Rows of dk, dv at padded
 * keys are written as zeros. */
hift_status hift_k_attention_bwd(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads,
                                 int32_t d_head, int32_t causal, const void *qkv_dev,
                                 const void *o_dev, const float *lse_dev, const void *do_dev,
                                 void *dqkv_dev, float *dsum_dev, const int32_t *key_lens_dev,
                                 void *cuda_stream);
/* The same two with dropout on the probabilities (hift_model_cfg.attn_dropout): rate p in [0, 1), the generator's
 * seed, site and step as the step would pass them (site 1000 + block, step t).  p = 0 is the plain kernel. */
hift_status hift_k_attention_fwd_drop(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads,
                                      int32_t d_head, int32_t causal, const void *qkv_dev, void *o_dev,
                                      float *lse_dev, const int32_t *key_lens_dev, double p, uint64_t seed,
                                      int32_t site, int64_t step, void *cuda_stream);
hift_status hift_k_attention_bwd_drop(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads,
                                      int32_t d_head, int32_t causal, const void *qkv_dev,
                                      const void *o_dev, const float *lse_dev, const void *do_dev,
                                      void *dqkv_dev, float *dsum_dev, const int32_t *key_lens_dev, double p,
                                      uint64_t seed, int32_t site, int64_t step, void *cuda_stream);
/* Rotary models (RoPE on q and k, as in the LLaMA-shaped configuration the paper profiles) on the
 * tensor-core path: the rotation is fused into the epilogue of the qkv projection, and this hook
 * exposes exactly that kernel: out[M,N] = rope(x[M,K] w[N,K]^T + bias) on columns [0, rope_cols),
 * plain beyond.  cs_dev: fp32 [seq, d_head/2] cosines followed by [seq, d_head/2] sines of
 * angle(pos, j) = pos * base^(-2j/d_head); pair (j, j + d_head/2); row r has position r mod seq.
 * HIFT_ERR_CFG when the fused kernel does not apply (d_head != 128, operands not 16-byte aligned,
 * N or rope_cols not a multiple of 128). */
hift_status hift_k_linear_rope(int64_t M, int64_t N, int64_t K, const void *a_dev, const void *b_dev, void *out_dev,
                               const void *bias_dev, const float *cs_dev, int32_t seq, int32_t d_head,
                               int64_t rope_cols, void *cuda_stream);
/* SwiGLU blocks on the tensor-core path: the gate | up projection (w[2f, K]: f gate rows, then f up rows) and
 * the activation are one kernel.  s_dev[M, f] = silu(gate) * up (bf16); gu_dev[M, 2f] receives the two
 * pre-activations, or may be NULL when nothing will read them (blocks below the active group keep no
 * activations).  HIFT_ERR_CFG when the fused kernel does not apply (f not a multiple of 128, M < 128,
 * operands not 16-byte aligned). */
hift_status hift_k_linear_swiglu(int64_t M, int64_t f, int64_t K, const void *a_dev, const void *b_dev, void *gu_dev,
                                 void *s_dev, const void *bias_dev, void *cuda_stream);
/* ... and its backward: dgu_dev[M, 2f] = swiglu_bwd(dy[M,N] w[N,f]; gu_dev[M, 2f]), i.e. the dX product of the
 * down projection (w is the down matrix [N = d_model, f]) with the activation's backward applied in
 * its epilogue: d gate in columns [0, f), d up in [f, 2f).  HIFT_ERR_CFG when the fused kernel does not
 * apply (f not a multiple of 32, M < 128, operands not 16-byte aligned). */
hift_status hift_k_linear_dx_swiglu_bwd(int64_t M, int64_t N, int64_t f, const void *dy_dev, const void *w_dev,
                                        const void *gu_dev, void *dgu_dev, void *cuda_stream);
/* GELU blocks (the GPT-2- and RoBERTa-shaped configurations), same two fusions:
 *   hift_k_linear_gelu       : pre_dev[M,N] = x[M,K] w[N,K]^T + bias (may be NULL when not needed), act_dev[M,N] = gelu(pre)
 *   hift_k_linear_dx_gelu_bwd: da_dev[M,f] = (dy[M,N] w[N,f]) * gelu'(pre_dev[M,f])
 * exact (erf) GELU; HIFT_ERR_CFG when the fused kernel does not apply (output width not a multiple of 32, M < 128,
 * operands not 16-byte aligned). */
hift_status hift_k_linear_gelu(int64_t M, int64_t N, int64_t K, const void *a_dev, const void *b_dev, void *pre_dev,
                               void *act_dev, const void *bias_dev, void *cuda_stream);
hift_status hift_k_linear_dx_gelu_bwd(int64_t M, int64_t N, int64_t f, const void *dy_dev, const void *w_dev,
                                      const void *pre_dev, void *da_dev, void *cuda_stream);
/* kind 0 LayerNorm (gain, bias), 1 RMSNorm (gain).  x is the fp32 residual stream in every
 * dtype; gain/bias/y have the operand type.  stats: fp32 [2*rows] (mean|rstd). */
hift_status hift_k_norm_fwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double eps,
                            const float *x_dev, const void *gain_dev, const void *bias_dev,
                            void *y_dev, float *stats_dev, void *cuda_stream);
/* dx = norm_bwd(dy) (+ add).  dy and gain have the operand type; x, add and dx are fp32
 * (residual stream and its gradient).  dx may be NULL (skipped).  dgain/dbias fp32 [cols]
 * may be NULL (skipped); partial_dev: fp32 scratch of 2*64*cols elements, needed when
 * dgain != NULL. */
hift_status hift_k_norm_bwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols,
                            const void *dy_dev, const float *x_dev, const float *stats_dev,
                            const void *gain_dev, const float *add_dev, float *dx_dev,
                            float *dgain_dev, float *dbias_dev, float *partial_dev,
                            void *cuda_stream);
/* The paper has no counterpart for this entry point; it exists for callers that must not
 * allocate.  It computes exactly what hift_k_norm_bwd computes (same kernels, same summation
 * order, same results), but takes no `partial_dev` argument: the column-reduction scratch lives
 * in a fixed array that is part of the library image (4 MiB of device memory per GPU that loads
 * the library, held until the process exits).  Nothing is allocated or freed, on the host or on
 * the device, by this call: no cudaMalloc, no cudaFree, no allocating library routine.  That is
 * what code needs which runs where the allocator is off limits - inside a memory pool whose
 * budget is already committed, in a latency-critical loop that cannot afford an allocator's
 * implicit synchronisation, or in a host process that was handed its buffers by someone else
 * and has no allocator of its own for this device.
 *   - cols must be <= HIFT_STATIC_SCRATCH_MAX_COLS, else HIFT_ERR_CAPACITY (nothing is launched).
 *   - The first call on each device looks up the device address of the array (with that
 *     device current).  Make that first call before starting any stream capture.  The address is
 *     kept for the life of the process: it does not survive a cudaDeviceReset of that device.
 *   - dy, x, stats and gain must not be NULL when dx or dgain is requested (HIFT_ERR_INPUT;
 *     hift_k_norm_bwd checks the same).
 *   - All calls on one GPU share the one array, which keeps whatever the previous call left.
 *     Every word a call reads it has written earlier in the same call, so stale contents
 *     are harmless and nothing needs clearing; but two calls that overlap on the GPU (different
 *     streams, or different host threads) race on it.  Serialise them.
 * Inputs and outputs are the caller's, as for hift_k_norm_bwd. */
#define HIFT_STATIC_SCRATCH_MAX_COLS 8192
hift_status hift_k_norm_bwd_static(int32_t dtype, int32_t kind, int64_t rows, int64_t cols,
                                   const void *dy_dev, const float *x_dev, const float *stats_dev,
                                   const void *gain_dev, const float *add_dev, float *dx_dev,
                                   float *dgain_dev, float *dbias_dev, void *cuda_stream);

/* Softmax cross-entropy over rows of logits[rows, ld] (columns >= vocab are
 * padding).  Overwrites logits with d loss / d logits.  loss_dev: 4 fp32 words,
 * [0] = mean loss over rows with label >= 0, [1] = that row count (int32 bits),
 * [2] = 1 (int32) if a label was >= vocab.  rowloss_dev: fp32 scratch [rows]. */
hift_status hift_k_cross_entropy(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                                 void *logits_dev, const int32_t *labels_dev, float *rowloss_dev,
                                 float *loss_dev, void *cuda_stream);

/* ---- operators beside the step ---------------------------------------------
 * What fine-tuning with objectives and updates other than the step's own needs, on caller-owned device buffers.  All
 * launch on `cuda_stream` (on the device that is current, whose buffers they are given), do not synchronise and do
 * not allocate.  They can be captured into a CUDA graph; the first call of an operator on a device sets its kernels up
 * and is made before any capture.  Calls that overlap on the GPU need scratch buffers of their own.  Inputs and outputs
 * must not overlap except where it is said.  A call that is refused launches nothing: HIFT_ERR_CFG also for a buffer that
 * does not start where its elements may, and for factors that are beyond fp32. */

/* Log-probabilities of given tokens under rows of logits[rows, ld] (columns >= vocab are padding and not read):
 *     z = x / temperature,  log p = z - log sum exp z,  logp_dev[r] = log p[tokens_dev[r]],
 *     entropy_dev[r] = -sum_i p_i log p_i (0 log 0 = 0; may be NULL),
 *     top_ids_dev / top_logp_dev [rows, n_top]: the n_top most likely tokens in falling order of the logit, equal logits in
 *     rising order of the id; places without a token whose logit is above -inf hold id -1 and -inf.
 *     stats_dev fp32 [2*rows] (may be NULL): the row's largest logit x | log sum_i exp(z_i - z_max): what the gradient takes.
 * The logits are read once and left as they are; sums are fp32, a log p below the range of fp32 is -inf.  A logit of -inf is a
 * token that cannot occur.  tokens_dev[r] < 0: the row is ignored, whatever it holds (0, 0, stats 0 | 0, ids -1, -inf);
 * tokens_dev[r] >= vocab: likewise, and *bad_dev (int32, may be NULL) is set to 1 (and never cleared by the library).  A row
 * with nothing above -inf: logp -inf, entropy 0, stats -inf | 0, no alternatives.  A row that holds a NaN or +inf: NaN
 * everywhere, ids -1.
 * dtype 0: fp32 logits, 1: bf16; the rows may start anywhere an element may (any ld >= vocab).  rows = 0 is allowed.
 * HIFT_ERR_CAPACITY if n_top > HIFT_MAX_TOP. */
#define HIFT_MAX_TOP 32
hift_status hift_k_token_logprobs(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const void *logits_dev,
                                  const int32_t *tokens_dev, double temperature, int32_t n_top, float *logp_dev,
                                  float *entropy_dev, float *stats_dev, int32_t *top_ids_dev, float *top_logp_dev,
                                  int32_t *bad_dev, void *cuda_stream);
/* The gradient of sum_r dlogp[r] logp[r] + dentropy[r] entropy[r] into the logits, from what the call above saved:
 *     dlogits[r, i] = ( dlogp[r] (delta_it - p_i) - dentropy[r] p_i (log p_i + entropy[r]) ) / temperature,
 * rounded once to the logits' type.  dlogp_dev or dentropy_dev may be NULL (not both; entropy_dev is read with dentropy_dev
 * only).  dlogits_dev [rows, ld] may be logits_dev itself; padding columns, ignored rows and rows with nothing above -inf
 * get zeros. */
hift_status hift_k_token_logprobs_bwd(int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const void *logits_dev,
                                      const int32_t *tokens_dev, double temperature, const float *stats_dev,
                                      const float *entropy_dev, const float *dlogp_dev, const float *dentropy_dev,
                                      void *dlogits_dev, void *cuda_stream);

/* The junction of a block's output h with the residual stream x, norms after the block and before the next one included:
 *     x_out = res_scale * x + gate o N1(h),    y = N2(x_out)
 * N: LayerNorm (kind 0: gain, bias) or RMSNorm (kind 1: gain; biases are not read), both with `eps`.  gain1_dev NULL: no norm
 * after the block (N1(h) = h); gain2_dev NULL: none before the next (y_dev is not written); gate_dev NULL: no gate.  The
 * gate is [ceil(rows / rows_per_gate), cols]: row r takes row r / rows_per_gate of it (rows_per_gate >= rows: one learned
 * vector; the sequence length: one per batch entry; 1: one per token).
 * x and x_out (which may be x itself) are fp32, the residual stream; h, y, gains, biases and gate have the operand type
 * (dtype 0 fp32, 1 bf16).  stats_dev: fp32 [4*rows], mean1 | rstd1 | mean2 | rstd2 (means 0 for RMSNorm, zeros for a
 * norm that is missing).  cols a multiple of 8, at most 16384 (HIFT_ERR_CAPACITY); buffers 16-byte aligned.  rows = 0 is
 * allowed. */
hift_status hift_k_join_fwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double eps, double res_scale,
                            const float *x_dev, const void *h_dev, const void *gain1_dev, const void *bias1_dev,
                            const void *gate_dev, int64_t rows_per_gate, const void *gain2_dev, const void *bias2_dev,
                            float *x_out_dev, void *y_dev, float *stats_dev, void *cuda_stream);
/* Its gradient.  dy_dev [rows, cols] (operand type) is the gradient of y (read if gain2_dev is given), dx_out_dev (fp32; may be
 * NULL if gain2_dev is given) the gradient that reaches x_out past the norm; x_out_dev, h_dev and stats_dev are the forward
 * pass's.  With d = dx_out + N2'(dy):
 *     dx = res_scale * d (fp32; may be dx_out_dev itself),  dh = N1'(gate o d) (operand type),
 *     dgate = sum of d o N1(h) over a gate's rows (fp32, the gate's shape),  dgain1, dbias1, dgain2, dbias2 fp32 [cols].
 * Each of the last five may be NULL (not wanted); one that belongs to a missing norm, gate or bias is refused.  bias1_dev is
 * read for dgate only.  Sums over rows run in a fixed order.  scratch_dev: hift_join_bwd_scratch_bytes(rows, cols,
 * rows_per_gate) bytes (rows_per_gate = rows without a gate; 0 for rows and columns that the call does not take),
 * HIFT_ERR_CAPACITY if scratch_bytes is less. */
size_t      hift_join_bwd_scratch_bytes(int64_t rows, int64_t cols, int64_t rows_per_gate);
hift_status hift_k_join_bwd(int32_t dtype, int32_t kind, int64_t rows, int64_t cols, double res_scale, const void *dy_dev,
                            const float *dx_out_dev, const float *x_out_dev, const void *h_dev, const float *stats_dev,
                            const void *gain1_dev, const void *bias1_dev, const void *gate_dev, int64_t rows_per_gate,
                            const void *gain2_dev, float *dx_dev, void *dh_dev, float *dgain1_dev, float *dbias1_dev,
                            float *dgate_dev, float *dgain2_dev, float *dbias2_dev, void *scratch_dev, size_t scratch_bytes,
                            void *cuda_stream);

/* Orthogonalisation of a matrix by Newton-Schulz products:
 *     X_0 = G / max(|G|_F, 1e-30),   X <- a X + (b A + c A A) X,  A = X X^T  (right-hand products when rows > cols),
 * `steps` times, (a, b, c) = (3.4445, -4.7750, 2.0315): every singular value s of X goes to a s + b s^3 + c s^5, which brings
 * all of 0.01 and more to between 0.68 and 1.14 in five steps.  g_dev [rows, cols] fp32 (dtype 0) or bf16 (1), o_dev bf16
 * [rows, cols].
 * The products run in 16-bit floating point with fp32 sums, around an iterate kept in fp32 (all in fp32 for a short side of at most 16
 * beside a long one of at most 16384).  Before its rounding to bf16 and relative to its Frobenius norm, the result of up to five steps is
 * within 2^-8 of the definition where the products' roundings average out, as over random entries and gradients of any rank, up to a
 * short side of 4096 (found: 2e-4 to 2.4e-3), and within 2^-4 where they line up, in matrices of few distinct values (all entries
 * equal, equal blocks, diagonal ones; found: up to 9e-3, 3.6e-2 on a single singular value).  Every further step multiplies what is
 * there by up to 1.6, and noise in directions that the matrix lacks, which fp32 sums have too, by 3.44: 2^-4 and 2^-2 after eight.
 * More would keep no digit of a low-rank matrix.  A zero matrix stays zero; NaN or infinity anywhere makes the whole result NaN.
 * 1 <= rows, cols <= HIFT_ORTHOGONALIZE_MAX_DIM (HIFT_ERR_CAPACITY), 1 <= steps <= HIFT_ORTHOGONALIZE_MAX_STEPS.  scratch_dev: 256-byte
 * aligned, hift_orthogonalize_scratch_bytes(rows, cols) bytes.  A call after a time-out (hift_tc_error_flag) writes no result. */
#define HIFT_ORTHOGONALIZE_MAX_DIM 65536
#define HIFT_ORTHOGONALIZE_MAX_STEPS 8
size_t      hift_orthogonalize_scratch_bytes(int64_t rows, int64_t cols);
hift_status hift_k_orthogonalize(int32_t dtype, int64_t rows, int64_t cols, const void *g_dev, void *o_dev, int32_t steps,
                                 void *scratch_dev, size_t scratch_bytes, void *cuda_stream);
/* One update of a weight matrix with it, beside hift_opt_step and hift_adafactor_step (what the Muon optimiser does):
 *     momentum <- mu momentum + grad;   U = grad + mu momentum (nesterov != 0) or momentum;   X from U as above;
 *     master <- master (1 - lr weight_decay) - lr 0.2 sqrt(max(rows, cols)) X
 * (the factor gives the update the size of an AdamW update at the same lr); param_bf16_dev (may be NULL) receives the
 * bf16 image of the new master.  master, grad and momentum_dev are fp32 [rows, cols].  The update is as exact as
 * hift_k_orthogonalize's result before rounding.  After a time-out master and param keep their values, while momentum has
 * been updated. */
hift_status hift_muon_step(int64_t rows, int64_t cols, void *param_bf16_dev, float *master_dev, const float *grad_dev,
                           float *momentum_dev, void *scratch_dev, size_t scratch_bytes, double lr, double momentum,
                           int32_t nesterov, double weight_decay, int32_t steps, void *cuda_stream);

/* ---- operators of a transformer block beside the step ------------------------
 * For blocks that the step's own architectures do not have, with the conventions of the operators above: caller-owned buffers, the stream
 * and the current device given by the caller, no synchronisation, no allocation, capture into a CUDA graph after one first call on a
 * device, scratch buffers of their own for calls that overlap.  Inputs and outputs must not overlap except where it is said. */

/* Cosines and sines for rotary positions: cs_dev fp32 [n_pos, rot/2] cosines of pos * freq(j), then as many sines (what hift_k_linear_rope
 * and hift_k_rope take).  Angles are formed in 64 bits.  With plain frequencies base^(-2j/rot), `scaling` for contexts longer than trained:
 *   0 none;  1 linear: all frequencies / factor;  2 NTK-aware: base * factor^(rot/(rot-2)) for base (the fastest pair keeps its frequency,
 *   the slowest gets 1/factor of it);
 *   3 YaRN: plain for pairs that turn at least `fast` times over orig_len positions, / factor for at most `slow` times, in between linear in the pair's
 *   index, and cosines and sines times 0.1 ln(factor) + 1.  The ramp runs from the index at which a pair turns `fast` times, rounded down (0 at least), to that
 *   of `slow` times, rounded up (rot - 1 at most);
 *   4 banded: plain above `fast` turns over orig_len, / factor below `slow`, linear in the number of turns in between.
 * factor >= 1 (read for 1 to 4), orig_len > 0 and 0 < slow < fast (read for 3 and 4).  rot even. */
hift_status hift_rope_table(int32_t scaling, int64_t n_pos, int32_t rot, double base, double factor, double orig_len, double fast,
                            double slow, float *cs_dev, void *cuda_stream);
/* Rotary positions on the first n_heads * d_head columns of x_dev [rows, ld] into out_dev [rows, ld_out] (which may be x_dev itself, with
 * the same ld): the first `rot` elements of every head are turned, the rest of it is copied; columns beyond the heads are neither read nor
 * written.  For a qkv buffer: n_heads = the q and the k heads; for the two maps of differential attention: twice as many of half the size.
 * layout 0: pair (j, j + rot/2), 1: pair (2j, 2j+1).  positions_dev int32 [rows], or NULL: row r has position r mod seq.  A position
 * outside [0, n_pos) leaves its row unturned and sets *bad_dev (int32, may be NULL) to 1, which the library never clears.
 * inverse != 0 turns back: the gradient of the turned rows into the rows before.  dtype 0 fp32, 1 bf16; computed in fp32, rounded once; any
 * alignment of an element, any ld >= n_heads * d_head.  rows = 0 is allowed.  HIFT_ERR_CAPACITY if n_heads * d_head > HIFT_ROPE_MAX_WIDTH. */
#define HIFT_ROPE_MAX_WIDTH 8388608
hift_status hift_k_rope(int32_t dtype, int32_t layout, int64_t rows, int32_t n_heads, int32_t d_head, int32_t rot, const void *x_dev,
                        int64_t ld, void *out_dev, int64_t ld_out, const float *cs_dev, int64_t n_pos, int64_t seq,
                        const int32_t *positions_dev, int32_t inverse, int32_t *bad_dev, void *cuda_stream);

/* Differential attention: the difference of two softmax maps with a learned weight per head,
 *     a_m = softmax(q_m k_m^T / sqrt(d_head/2) + mask),   o_m = a_m v  (m = 1, 2),   o = o_1 - lambda_h o_2,
 *     y = out_scale * gain * o / sqrt(mean(o^2) + eps)    per head (gain_dev NULL: no norm, y_dev NULL).
 * qkv_dev [batch*seq, (n_heads + 2 n_kv_heads) * d_head]: the column blocks q | k | v of hift_k_attention_fwd; in a head of q or k the first
 * half of its columns belongs to the first map, the second half to the second, while v is d_head wide.  Query head h reads key and value
 * head h / (n_heads / n_kv_heads).  Masks as in hift_k_attention_fwd (causal; key_lens_dev int32 [batch] or NULL), but a length of
 * 0 leaves nothing: zeros, lse = -inf, no gradient.  What k and v hold at padded keys does not matter, NaN included; a NaN or an infinity elsewhere may
 * reach any row of its batch entry, rows that the causal mask hides it from among them (0 times NaN), but no other entry.
 * lambda_dev fp32 [n_heads], gain_dev [d_head] of the operand type.  Out, all [batch*seq, n_heads * d_head] of the operand type: o_dev, o2_dev (o_2, what
 * the gradient needs; may be NULL), y_dev; lse_dev fp32 [2, batch, n_heads, seq], the maps' log-sum-exps.
 * d_head 16, 32, 64 or 128; dtype 0 fp32, 1 bf16.  bf16 heads of 64 and 128 with qkv, o, o2 and y (in the gradient qkv, dqkv and, without a norm, dy)
 * 16-byte aligned run on the tensor cores, with probabilities, their gradients and, behind a norm, the gradient of o rounded to bf16 as operands and
 * sums in fp32; the rest runs on the CUDA cores in fp32.
 * batch = 0 or seq = 0 is allowed. */
hift_status hift_k_diff_attention_fwd(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                      int32_t causal, const void *qkv_dev, const float *lambda_dev, const void *gain_dev, double eps,
                                      double out_scale, void *o_dev, void *o2_dev, void *y_dev, float *lse_dev,
                                      const int32_t *key_lens_dev, void *cuda_stream);
/* Its gradient, from o_dev, o2_dev and lse_dev as the forward pass stored them.  dy_dev: the gradient of y (of o without a norm).  dqkv_dev has qkv's
 * shape and is written whole (zeros at padded keys; shared key heads get the sum over their query heads); dlambda_dev fp32 [n_heads] and
 * dgain_dev fp32 [d_head] may be NULL.  Sums run in a fixed order.  scratch_dev: 256-byte aligned,
 * hift_diff_attention_bwd_scratch_bytes(...) bytes (norm != 0 with a gain; 0 for what the call does not take), HIFT_ERR_CAPACITY if
 * scratch_bytes is less. */
size_t      hift_diff_attention_bwd_scratch_bytes(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads, int32_t d_head, int32_t norm);
hift_status hift_k_diff_attention_bwd(int32_t dtype, int32_t batch, int32_t seq, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                      int32_t causal, const void *qkv_dev, const float *lambda_dev, const void *gain_dev, double eps,
                                      double out_scale, const void *o_dev, const void *o2_dev, const float *lse_dev, const void *dy_dev,
                                      void *dqkv_dev, float *dlambda_dev, float *dgain_dev, void *scratch_dev, size_t scratch_bytes,
                                      const int32_t *key_lens_dev, void *cuda_stream);
/* The weights as they are learned: lambda_h = exp(q1 . k1) - exp(q2 . k2) + init, w_dev fp32 [4, sets, d]: q1 | k1 | q2 | k2; sets = 1 (the
 * same vectors for all heads, whose gradients are summed) or n_heads.  dw_dev has w's shape. */
hift_status hift_k_diff_lambda(int32_t n_heads, int32_t sets, int32_t d, double init, const float *w_dev, float *lambda_dev, void *cuda_stream);
hift_status hift_k_diff_lambda_bwd(int32_t n_heads, int32_t sets, int32_t d, const float *w_dev, const float *dlambda_dev, float *dw_dev,
                                   void *cuda_stream);

/* Activations kept in 8 bits for the backward pass, beside recomputing them.  Blocks of HIFT_ACT8_BLOCK consecutive columns of a row
 * (the last one of a row may be shorter) share a scale 2^(byte - 127), the least power of two, 2^-110 at least, that brings the block's
 * largest magnitude to at most 127 (format 0: int8) or 448 (format 1: e4m3); q = x / scale rounded to nearest even, and q * scale is exact in bf16 and
 * fp32; only where that would be 2^128 the largest code that is finite is kept (63 * 2^122, or 240 * 2^120: less than a step away).  A block that holds a
 * NaN or an infinity has byte 255 and comes back as NaNs.  q_dev: one byte a value; scales_dev:
 * ceil(cols / HIFT_ACT8_BLOCK) bytes a row.
 *   pack:   x_dev [rows, ld] -> q, scales          unpack: q, scales -> out_dev [rows, ld]    (columns beyond `cols` are left alone)
 *   fwd:    act_dev[rows, f] = activation of pre_dev, and pre packed.  kind 1: GELU (erf), pre [rows, f]; 2: SwiGLU, pre [rows, 2f] = gate | up,
 *           act = silu(gate) * up, q [rows, 2f] and the scale bytes of gate | up per row, each part with blocks of its own
 *   bwd:    dpre_dev (pre's shape) from dact_dev [rows, f] at the packed values; act_dev [rows, f] (may be NULL): the activation at them, what the next
 *           weight's gradient takes
 * dtype: of x, out, pre, act, dact and dpre.  rows = 0 is allowed.  HIFT_ERR_CAPACITY for more than HIFT_ACT8_MAX_COLS columns. */
#define HIFT_ACT8_BLOCK 32
#define HIFT_ACT8_MAX_COLS 8388608
hift_status hift_k_act8_pack(int32_t dtype, int32_t format, int64_t rows, int64_t cols, const void *x_dev, int64_t ld, void *q_dev,
                             uint8_t *scales_dev, void *cuda_stream);
hift_status hift_k_act8_unpack(int32_t dtype, int32_t format, int64_t rows, int64_t cols, const void *q_dev, const uint8_t *scales_dev,
                               void *out_dev, int64_t ld, void *cuda_stream);
hift_status hift_k_act8_fwd(int32_t dtype, int32_t format, int32_t kind, int64_t rows, int64_t f, const void *pre_dev, void *act_dev,
                            void *q_dev, uint8_t *scales_dev, void *cuda_stream);
hift_status hift_k_act8_bwd(int32_t dtype, int32_t format, int32_t kind, int64_t rows, int64_t f, const void *dact_dev, const void *q_dev,
                            const uint8_t *scales_dev, void *dpre_dev, void *act_dev, void *cuda_stream);

const char *hift_strerror(hift_status s);

#ifdef __cplusplus
}
#endif
#endif /* HIFT_H_ */
