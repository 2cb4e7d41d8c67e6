/*
 * vit.h — C boundary of the ViT pipeline-stage forward library for NVIDIA B200 (sm_100a).
 *
 * The library computes the forward pass of one pipeline stage: a contiguous range of layers
 * [layer_begin, layer_end) of a pre-LN Vision Transformer encoder applied to one microbatch of
 * activations, plus the two book-ends (patch embedding before the first stage, classification
 * head after the last) and a stage runner that issues microbatches on CUDA streams.
 *
 * Conventions for every entry point
 *   - All functions return an int status: VIT_OK (0) or a negative VIT_ERR_* code.  Arguments
 *     are validated on the host before anything is launched; a failed call launches nothing.
 *   - "dev" pointers are device memory owned by the caller (for example the data_ptr() of a
 *     PyTorch tensor) and must stay alive until the stream has drained.  They must be 16-byte
 *     aligned.  "host" pointers are ordinary (preferably pinned) host memory.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Calls are
 *     asynchronous on that stream, allocate no device memory and never synchronise the host,
 *     except where stated (while vit_profile_enable is on, every launch also creates a pair of
 *     CUDA events).
 *   - A handle belongs to the CUDA device that was current in vit_create; every call that takes
 *     the handle must be made with that device current (otherwise VIT_ERR_INVALID_ARG).
 *   - Activations are row-major [microbatch, T, H] (T = patches + 1 class token, H = hidden).
 *     Their element type is the model's activation type: bf16 when config.dtype == VIT_BF16
 *     (bf16 operands, fp32 accumulation), fp32 when config.dtype == VIT_FP32.
 *   - A workspace must not be shared by two calls that may overlap on the GPU.
 *   - A handle may be used from several host threads at once with distinct streams and
 *     workspaces; parameters are read-only after vit_create.
 */
#ifndef VIT_B200_H
#define VIT_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  VIT_OK = 0,
  VIT_ERR_INVALID_ARG = -1, /* null or misaligned pointer, microbatch < 1 or > max_microbatch */
  VIT_ERR_RANGE = -2,       /* not 0 <= layer_begin < layer_end <= layers (empty range is an error) */
  VIT_ERR_CONFIG = -3,      /* inconsistent or unsupported model shape */
  VIT_ERR_WORKSPACE = -4,   /* workspace smaller than the size query says */
  VIT_ERR_CUDA = -5,        /* a CUDA runtime/driver call or a launch failed */
  VIT_ERR_TIMEOUT = -6,     /* a bounded wait inside a kernel gave up (device status word) */
  VIT_ERR_NO_DEVICE = -7,   /* no sm_100 device / driver available */
  VIT_ERR_TOO_LARGE = -8,   /* problem exceeds the fixed scratch of an allocation-free entry point,
                               or the partitioner's tables do not fit in host memory */
  VIT_ERR_INFEASIBLE = -9,  /* the partitioner found no assignment that fits the devices' memory */
  VIT_ERR_OFFSETS = -10     /* device status word: a packed sequence's or group's offsets were out of order or range */
};

enum { VIT_BF16 = 0, VIT_FP32 = 1 };

typedef struct vit_config {
  int32_t image_size;     /* pixels per side, e.g. 224 */
  int32_t patch_size;     /* 16 or 14; must divide image_size */
  int32_t channels;       /* 3 */
  int32_t hidden;         /* H, multiple of 64 */
  int32_t layers;         /* L */
  int32_t heads;          /* H / heads must be a multiple of 16 and <= 128 */
  int32_t mlp_dim;        /* F, multiple of 64 */
  int32_t num_classes;
  float   ln_eps;         /* LayerNorm epsilon (inside the square root) */
  int32_t dtype;          /* VIT_BF16 or VIT_FP32 */
  int32_t max_microbatch; /* largest microbatch any call will use */
  int32_t extra_tokens;   /* 0, or 1 for a distillation token after the class token (see below) */
} vit_config;

typedef struct vit_handle vit_handle; /* opaque */

/* Number of fp32 values in the host parameter blob for this configuration (0 if the
 * configuration is invalid).  Blob layout, tensors back to back, matrices [out, in] row-major:
 *   patch.W [H, C*P*P] (column = c*P*P + i*P + j), patch.b [H], cls [H], (dist [H]), pos [T, H],
 *   per layer: ln1.g ln1.b Wqkv[3H,H] bqkv[3H] Wo[H,H] bo[H] ln2.g ln2.b W1[F,H] b1[F] W2[H,F] b2[H],
 *   lnf.g [H], lnf.b [H], head.W [classes, H], head.b [classes], (head_dist.W, head_dist.b).
 * The entries in parentheses exist when extra_tokens == 1: the compressed models of the paper's
 * Section 5.5 are distilled transformers with a distillation token; then T = patches + 2, token 1
 * is dist + pos[1], patch tokens start at 2, and the head averages two classifiers.
 * Wqkv rows [0,H) produce Q, [H,2H) K, [2H,3H) V; head h owns rows h*d..(h+1)*d of each. */
size_t vit_param_count(const vit_config* cfg);

/* Bytes of scratch one call of vit_patch_embed / vit_run_stage / vit_head needs for
 * `microbatch` images (the maximum over the three).  0 if arguments are invalid. */
size_t vit_workspace_bytes(const vit_config* cfg, int microbatch);

/* Bytes of scratch one stream of vit_run_pipeline[_host] needs for `microbatch` images:
 * the stage scratch above plus the token buffer and pixel/logit staging. */
size_t vit_pipeline_workspace_bytes(const vit_config* cfg, int microbatch);

/* Creates a model instance on the current CUDA device.
 * The transformer to partition is given to the system as a configuration plus its weights
 * (paper Section 3.1: the model configuration is the partitioner's input; Section 4: the
 * models are standard ViT definitions).
 *   host_params: host, fp32 blob in the layout above, n_params == vit_param_count(cfg).
 *     In bf16 mode matrices are rounded to bf16 (nearest even) on upload; vectors stay fp32.
 * Allocates device memory for the parameters (freed by vit_destroy), synchronises.
 * Errors: INVALID_ARG, CONFIG, NO_DEVICE, CUDA. */
int vit_create(const vit_config* cfg, const float* host_params, size_t n_params, vit_handle** out);

/* Frees the handle and the device memory it allocated.  Synchronises the device. */
int vit_destroy(vit_handle* h);

/* Embedding book-end (paper Section 4: inputs pass an embedding layer that gives them the
 * uniform dimension the transformer layers expect).
 *   pixels: dev, fp32 [microbatch, C, S, S] (NCHW).
 *   tokens_out: dev, activations [microbatch, T, H].  Token 1 + extra_tokens + py*(S/P) + px is
 *     patch.W . vec(patch(py,px)) + patch.b + pos[token]; token 0 is cls + pos[0] (and token 1
 *     dist + pos[1] when extra_tokens == 1).
 *   ws: dev scratch of at least vit_workspace_bytes(cfg, microbatch). */
int vit_patch_embed(vit_handle* h, int microbatch, const float* pixels, void* tokens_out,
                    void* ws, size_t ws_bytes, void* stream);

/* One pipeline stage T_i (paper Section 3.1: the model is split into parts T_1..T_k of
 * consecutive layers, the output of stage i is the input of stage i+1, and
 * Y = T_k(...T_1(X))).  Applies layers [layer_begin, layer_end) to `in`, writes `out`.
 * Each layer is x += Wo.attention(LN1(x).Wqkv^T + bqkv) + bo;  x += W2.gelu(W1.LN2(x) + b1) + b2
 * (Section 2.1: self-attention, MLP, two layer normalisations, residual connections).  In bf16
 * mode the two layer normalisations are applied inside the QKV and fc1 products (row statistics
 * from a small kernel, gain and shift folded into the weights at vit_create).
 *   in, out: dev, activations [microbatch, T, H]; in == out is allowed (in place), any other
 *     overlap is INVALID_ARG.
 * Running [a,b) then [b,c) gives bit-identical results to one call on [a,c). */
int vit_run_stage(vit_handle* h, int layer_begin, int layer_end, int microbatch,
                  const void* in, void* out, void* ws, size_t ws_bytes, void* stream);

/* Classification book-end (paper Section 3.1: the device of the final stage produces the
 * final result; Section 4: the task is image classification).  Final LayerNorm of each image's
 * class token, then logits = f . head.W^T + head.b.  With extra_tokens == 1 the distillation
 * token (row 1) goes through the same LayerNorm and the classifier head_dist, and the logits are
 * the mean of the two classifiers' outputs.
 *   tokens: dev, activations [microbatch, T, H];  logits: dev, fp32 [microbatch, classes]. */
int vit_head(vit_handle* h, int microbatch, const void* tokens, float* logits,
             void* ws, size_t ws_bytes, void* stream);

/* vit_head for callers that cannot allocate device memory.  (The paper has no counterpart; this
 * is a convenience of the library.)  Some code that wants the classification result runs where
 * cudaMalloc is off limits: a real-time loop that must never enter the allocator (it can block
 * and synchronise the device), a plugin whose host application owns all device memory and hands
 * out only the input and output buffers, or a process whose memory pool was given away whole to
 * another framework at start-up.  vit_head needs a scratch buffer for
 * the normalised class-token features; this variant keeps that scratch in an array that is part
 * of the library itself, so the caller passes only tokens and logits.
 *   - Same arithmetic and same results as vit_head.
 *   - Limit: microbatch * (1 + extra_tokens) * hidden <= VIT_HEAD_STATIC_MAX_FLOATS (2 MiB of floats); anything
 *     larger returns VIT_ERR_TOO_LARGE and launches nothing.  Every GPU on which the library
 *     is loaded carries the array (2 MiB) until the process exits.
 *   - The first call on each device looks up the array's device address (a runtime query, not
 *     an allocation); make that first call before starting any stream capture.  It must be
 *     made with the handle's device current, like every other call.
 *   - There is ONE array per device, shared by all handles and streams, and it keeps whatever
 *     the last call left in it.  Nothing in it has to be cleared: a call overwrites every value
 *     before reading it.  Two calls that may run on the GPU at the same time (different
 *     streams, no dependency between them) would overwrite each other's features: order them.
 *   - Calls no cudaMalloc / cudaFree and no allocating library routine. */
#define VIT_HEAD_STATIC_MAX_FLOATS (512 * 1024)
int vit_head_static(vit_handle* h, int microbatch, const void* tokens, float* logits, void* stream);

/* Stage runner (paper Section 2.1/3.1: the minibatch is split into equal microbatches that
 * flow through the stages in order).  Splits `batch` images into microbatches of `microbatch`
 * (the last may be smaller), and for microbatch m issues, on streams[m % n_streams]:
 * patch embed, every stage in order (stage s covers stage_layers[s] layers; the counts must
 * sum to L), head.  A microbatch never changes stream, so stream order carries the
 * stage-to-stage dependency; different microbatches overlap across streams.
 *   pixels: dev fp32 [batch, C, S, S];  logits: dev fp32 [batch, classes].
 *   ws_per_stream[i]: dev scratch of at least vit_pipeline_workspace_bytes(cfg, microbatch).
 * Does not synchronise; the caller waits on the streams. */
int vit_run_pipeline(vit_handle* h, const int32_t* stage_layers, int n_stages, int batch,
                     int microbatch, const float* pixels, float* logits,
                     void* const* ws_per_stream, size_t ws_bytes, void* const* streams,
                     int n_streams);

/* vit_run_pipeline with `group` consecutive microbatches carried through every kernel launch
 * together (paper Section 5.4 studies the microbatch size: small microbatches keep the memory
 * per stage low but leave a large GPU underused; images are independent, so several of them in
 * flight can share a launch without changing any result).  Microbatch m still consists of images
 * [m * microbatch, (m + 1) * microbatch); groups go round-robin over the streams.
 *   ws_per_stream[i]: at least vit_pipeline_workspace_bytes(cfg, group * microbatch);
 *   group * microbatch <= max_microbatch. */
int vit_run_pipeline_grouped(vit_handle* h, const int32_t* stage_layers, int n_stages, int batch,
                             int microbatch, int group, const float* pixels, float* logits,
                             void* const* ws_per_stream, size_t ws_bytes, void* const* streams,
                             int n_streams);

/* Same as vit_run_pipeline with HOST pixels and logits: each microbatch's pixels are copied to
 * the device, and its logits back, on that microbatch's stream (copies are asynchronous only
 * if the host memory is pinned).  Does not synchronise. */
int vit_run_pipeline_host(vit_handle* h, const int32_t* stage_layers, int n_stages, int batch,
                          int microbatch, const float* host_pixels, float* host_logits,
                          void* const* ws_per_stream, size_t ws_bytes, void* const* streams,
                          int n_streams);

/* Returns and clears the device status word after everything queued on `stream` has finished
 * (synchronises that stream): VIT_OK, or VIT_ERR_TIMEOUT if a bounded wait in a kernel gave up
 * since the last check, or VIT_ERR_CUDA if the stream reported an error.  There is one word per
 * handle, shared by all its streams; it is read and cleared in one atomic step on the device, so
 * a timeout raised on another stream while this call runs is reported by the next check.  To
 * know that a multi-stream run was clean, check after each of its streams. */
int vit_check_status(vit_handle* h, void* stream);

/* Failure-detection self-test.  Every wait inside the tensor-core kernels is bounded: when it
 * expires the kernel raises the device status word and returns.  This call launches a one-warp
 * kernel whose wait can never be satisfied, with a limit of `limit_cycles` SM cycles (at most
 * 2^31, about a second), so that the path can be exercised without a stuck kernel: afterwards
 * vit_check_status returns VIT_ERR_TIMEOUT once and the handle keeps working. */
int vit_debug_wait_probe(vit_handle* h, int64_t limit_cycles, void* stream);

/* Number of kernels this handle has launched so far (host counter). */
uint64_t vit_launch_count(const vit_handle* h);

const char* vit_status_string(int status);

/* Per-kernel timing.  While enabled, every kernel launch of this handle is bracketed by a pair
 * of CUDA events on the stream it is launched on.  vit_profile_collect synchronises the device,
 * adds the elapsed milliseconds and launch counts per class into the two arrays of
 * VIT_PROF_CLASSES entries, and clears the records.  Use from one host thread only. */
enum {
  VIT_PROF_LAYERNORM = 0, VIT_PROF_QKV = 1, VIT_PROF_ATTENTION = 2, VIT_PROF_OUTPROJ = 3,
  VIT_PROF_FC1 = 4, VIT_PROF_FC2 = 5, VIT_PROF_EMBED = 6, VIT_PROF_HEAD = 7, VIT_PROF_OP = 8,
  VIT_PROF_CLASSES = 9
};
int vit_profile_enable(vit_handle* h, int on);
int vit_profile_collect(vit_handle* h, double* ms_by_class, uint64_t* launches_by_class);

/* ---- pipeline partitioner (host only, no GPU work) -------------------------------------------
 * Chooses which consecutive layers run on which device so that the slowest pipeline stage is as
 * fast as possible (paper Section 3.3: Eq. 1 T_comm = P_j / b(u,v); Eq. 2 T_period = max(T_comp,
 * T_comm); Eq. 3 the transition of the three-dimensional dynamic programme over layers done,
 * devices used and next device; Algorithm 1 with its memory check and precursor table).
 * All pointers are host memory. */
typedef struct vit_partition_problem {
  int32_t layers;            /* L */
  int32_t devices;           /* D (at most 16), or the number of categories (at most 8) */
  const double* layer_time;  /* [D][L] seconds layer j takes on device u; T_comp of a layer range is the sum */
  const double* out_bytes;   /* [L] P_j: bytes a stage ending with layer j sends to the next stage */
  const double* layer_mem;   /* [L] M_j: memory layer j needs */
  const double* device_mem;  /* [D] m_u */
  const double* bandwidth;   /* [D][D] bytes per second from device u to device v */
} vit_partition_problem;

/* t_opt: the slowest stage's period; n_stages, stage_layers[s] (layer counts in pipeline order,
 * summing to L) and stage_device[s] (device of stage s) describe one optimal mapping.  The two
 * output arrays need min(L, D) entries.  Every device is used at most once; not all need be used.
 * Errors: INVALID_ARG (null pointer, D > 16, a bandwidth that is not positive, a time, size or
 * memory that is negative or not a number), INFEASIBLE, TOO_LARGE (the tables of the dynamic
 * programme, about 8 * L * 2^D * D bytes, could not be allocated). */
int vit_partition(const vit_partition_problem* problem, double* t_opt, int32_t* n_stages,
                  int32_t* stage_layers, int32_t* stage_device);

/* The same problem with identical devices grouped (paper Section 3.3, last paragraph): `devices`
 * is the number of categories, category_count[c] the number of devices in category c, and
 * layer_time / device_mem / bandwidth are indexed by category (bandwidth[c][c] = between two
 * devices of category c).  stage_device receives category indices.  The state space shrinks from
 * 2^D to prod(count + 1).  Output arrays need min(L, total devices) entries. */
int vit_partition_categories(const vit_partition_problem* problem, const int32_t* category_count,
                             double* t_opt, int32_t* n_stages, int32_t* stage_layers,
                             int32_t* stage_device);

/* ---- single operations, exposed so that each kernel can be checked on its own ------------
 * All pointers dev; `dtype` selects the bf16 or fp32 kernel family as in vit_config.
 * They need a handle only for the device status word and the launch counter. */

/* y[r,:] = (x[r,:] - mean) / sqrt(var + eps) * gain + shift, biased variance, rows x cols.
 * x, y: activations; gain, shift: fp32 [cols]. */
int vit_op_layernorm(vit_handle* h, int dtype, int rows, int cols, const void* x,
                     const float* gain, const float* shift, float eps, void* y, void* stream);

/* out = epilogue(a[M,K] . w[N,K]^T + bias[N]); a, w, out, residual in the activation type,
 * bias fp32.  epilogue: 0 = none, 1 = erf-GELU, 2 = add residual[M,N] (residual may equal out).
 * bf16 family: K % 8 == 0 and N % 8 == 0. */
int vit_op_linear(vit_handle* h, int dtype, int M, int N, int K, const void* a, const void* w,
                  const float* bias, int epilogue, const void* residual, void* out, void* stream);

/* vit_op_linear with the tiling of the bf16 tensor-core kernel chosen by the caller instead of
 * by the library's shape-only cost model, so that every tiling can be checked on any shape.
 * VIT_TILING_PAIR_256x256 runs CTA pairs on 256 x 256 tiles.  fp32 family: AUTO only. */
enum { VIT_TILING_AUTO = 0, VIT_TILING_128x128 = 1, VIT_TILING_128x256 = 2, VIT_TILING_PAIR_256x256 = 3 };
int vit_op_linear_tiled(vit_handle* h, int dtype, int M, int N, int K, const void* a, const void* w,
                        const float* bias, int epilogue, const void* residual, void* out, int tiling,
                        void* stream);

/* The two halves of the LayerNorm that vit_run_stage folds into its QKV and fc1 products in bf16
 * mode (the normalised activations are never written to memory):
 *   vit_op_rowstats: stats[2 r] = mean of row r of x (bf16 [rows, cols]), stats[2 r + 1] =
 *     1 / sqrt(biased variance + eps); stats is fp32 [rows, 2].
 *   vit_op_linear_ln: out[m,n] = f(stats[m].rstd * (a[m,:] . wg[n,:] - stats[m].mean * c1[n]) + c0[n]),
 *     f = identity or erf-GELU.  With wg[n,k] = gain[k] w[n,k], c1[n] = sum_k wg[n,k] and
 *     c0[n] = bias[n] + sum_k shift[k] w[n,k] this equals f(LayerNorm(a)[m,:] . w[n,:] + bias[n]).
 *     a, wg, out bf16; c1, c0 fp32 [N]; `tiling` as in vit_op_linear_tiled. */
int vit_op_rowstats(vit_handle* h, int rows, int cols, const void* x, float eps, float* stats, void* stream);
int vit_op_linear_ln(vit_handle* h, int M, int N, int K, const void* a, const float* stats, const void* wg,
                     const float* c1, const float* c0, int gelu, void* out, int tiling, void* stream);

/* Multi-head self-attention for `images` sequences of T tokens: qkv [images*T, 3*heads*d]
 * (column blocks Q, K, V; head-major inside each), out [images*T, heads*d];
 * out_h = softmax_rows(Q_h K_h^T / sqrt(d)) V_h. */
int vit_op_attention(vit_handle* h, int dtype, int images, int T, int heads, int d,
                     const void* qkv, void* out, void* stream);

/* ---- packed images: position rotation, query/key norm, attention and their gradients ---------
 * A batch of images of different sizes is one buffer of tokens, image after image.  These operations
 * serve such a layer between its QKV product and its output product, forwards and backwards.  The gradients of the
 * layer's other parts (linear products, LayerNorm, GELU) are further below, and the stage calls above do not use
 * these operations: a caller's own training or serving loop does.
 * Rows have strides of their own (`ld...`, in elements), so that queries, keys and values can be read
 * from, and their gradients written to, the column blocks of one [rows, (heads + 2 kv_heads) * d] buffer.
 * Common rules, checked before anything is launched: pointers 16-byte aligned (offsets: 4); d a multiple
 * of 16, at most 128; heads * d below 2^31; a stride at least as wide as its heads and a multiple of 8; no
 * output may overlap an input or another output unless stated (column blocks of one buffer with the same
 * stride do not overlap).
 * Sums, norms and softmax statistics are fp32; bf16 results are rounded once.  In bf16 attention of more than a few
 * queries, probabilities and the gradients of the scores are rounded to bf16 as operands of their products (half a
 * step, 2^-8), and probabilities below 2^-126 count as zero.
 * Scratch holds nothing between calls; calls that may run at the same time (on two streams, or in graphs that are
 * replayed together) need scratch of their own.
 * Results do not depend on the schedule: the same call gives the same bits. */

/* Rotary positions on one to four axes (row and column of a patch, frame of a video).  Pair i of a head
 * (0 <= i < n, n = sum of pairs[a]) belongs to the axis whose section it lies in: the first pairs[0]
 * pairs to axis 0, the next pairs[1] to axis 1, and so on.  It is turned by the angle
 * positions[axis * rows + row] * freqs[i] (radians; whole turns are taken off in 64 bits and more, so that
 * angles of up to 2^52 keep 32 bits).  Channels from 2 n on are passed on as they are. */
typedef struct vit_rope {
  int32_t axes;               /* 1 ... 4 */
  int32_t pairs[4];           /* pairs of channels of each axis, >= 0; 2 n <= d */
  int32_t interleaved;        /* pair i is the channels (2 i, 2 i + 1) if not 0, else (i, n + i) */
  const int32_t* positions;   /* dev [axes][rows]; may be NULL if rows or n is 0 */
  const float* freqs;         /* dev [n]; may be NULL if n is 0 */
} vit_rope;

/* y = x with every head's pairs turned; inverse != 0 turns them back, which is also the gradient.
 *   x, y: activations [rows, heads * d] with strides ldx, ldy; x == y with ldx == ldy is allowed. */
int vit_op_rope_axes(vit_handle* h, int dtype, int rows, int heads, int d, const vit_rope* rope, int inverse,
                     const void* x, int64_t ldx, void* y, int64_t ldy, void* stream);

/* Norm of queries and keys, then the rotation: every head becomes gain * x / sqrt(mean(x^2) + eps), turned.
 *   x, y: activations [rows, (q_heads + k_heads) * d]: query heads first, then key heads;
 *   x == y with ldx == ldy is allowed.  q_gain, k_gain: dev fp32 [d].  rope: NULL for no rotation. */
int vit_op_qk_norm_rope(vit_handle* h, int dtype, int rows, int q_heads, int k_heads, int d, const float* q_gain,
                        const float* k_gain, float eps, const vit_rope* rope, const void* x, int64_t ldx, void* y,
                        int64_t ldy, void* stream);

/* Bytes of scratch for vit_op_qk_norm_rope_backward; 0 if an argument is invalid. */
size_t vit_qk_norm_rope_backward_bytes(int rows, int q_heads, int k_heads, int d);

/* Gradients of vit_op_qk_norm_rope: dx from x (its input) and dy, and the sums over rows and heads
 * dq_gain, dk_gain (dev fp32 [d], overwritten; zero for no rows).  dx == x or dx == dy with the same
 * stride is allowed. */
int vit_op_qk_norm_rope_backward(vit_handle* h, int dtype, int rows, int q_heads, int k_heads, int d,
                                 const float* q_gain, const float* k_gain, float eps, const vit_rope* rope,
                                 const void* x, int64_t ldx, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                                 float* dq_gain, float* dk_gain, void* ws, size_t ws_bytes, void* stream);

/* Softmax attention of packed sequences: the queries of sequence i are rows q_offsets[i] ... q_offsets[i+1] - 1
 * of q, its keys and values rows k_offsets[i] ... k_offsets[i+1] - 1 of k and v (self-attention passes the same
 * offsets twice; attention pooling has one query per image).  heads is a multiple of kv_heads; query head j
 * reads key head j / (heads / kv_heads).
 * The offsets are read on the device.  A sequence whose offsets are out of order, reach outside the buffers or
 * make it longer than max_q / max_k is skipped, its rows are left as they were, and vit_check_status reports
 * VIT_ERR_OFFSETS.  The other sequences are computed; where a step backwards makes two of them overlap, a row that they
 * share gets the result of either.  Rows that no sequence covers are left as they were. */
typedef struct vit_attention_problem {
  int32_t sequences, heads, kv_heads, d;
  int32_t q_rows, max_q;      /* rows of q; bound on the length of a sequence's queries (any, INT32_MAX too) */
  int32_t k_rows, max_k;      /* rows of k and v; bound on the length of its keys; rows: at most INT32_MAX - 1024 */
  const int32_t* q_offsets;   /* dev [sequences + 1] */
  const int32_t* k_offsets;   /* dev [sequences + 1] */
  float scale;                /* of the scores, usually 1 / sqrt(d); finite and positive */
} vit_attention_problem;

/* Bytes of scratch for vit_op_attention_packed (backward == 0; it needs none at present) or its gradients; 0 if none
 * is needed, an argument is invalid or the problem is too large. */
size_t vit_attention_packed_bytes(int dtype, const vit_attention_problem* problem, int backward);

/* out[r, j] = softmax(scale q[r, j] . k^T) v over the row's sequence, and lse[j * q_rows + r] = log of the sum
 * of exp(scale q[r, j] . k), which the gradients need.  A query without keys gives out = 0, lse = -infinity.
 *   q, out: activations [q_rows, heads * d]; k, v: [k_rows, kv_heads * d]; lse: dev fp32 [heads][q_rows], always
 *   written. */
int vit_op_attention_packed(vit_handle* h, int dtype, const vit_attention_problem* problem, const void* q, int64_t ldq,
                            const void* k, int64_t ldk, const void* v, int64_t ldv, void* out, int64_t ldo, float* lse,
                            void* ws, size_t ws_bytes, void* stream);

/* Gradients of vit_op_attention_packed from its operands, its two results and dout.  The probabilities are
 * computed again from lse.  dk and dv of a key head are summed over the query heads that share it.  Long sums are
 * cut where the lengths of all sequences of the call say, so that beside other sequences the last bit may differ.
 *   dq: activations [q_rows, heads * d]; dk, dv: [k_rows, kv_heads * d]. */
int vit_op_attention_packed_backward(vit_handle* h, int dtype, const vit_attention_problem* problem, const void* q,
                                     int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                     const void* out, int64_t ldo, const float* lse, const void* dout, int64_t lddo,
                                     void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv, int64_t lddv, void* ws,
                                     size_t ws_bytes, void* stream);

/* ---- training a layer: layer norm, linear layers of one or several weight matrices, gradient clipping ------------
 * What a training or fine-tuning loop needs beside the operations above: the other half of a layer forwards and
 * backwards, and the step at its end.  The common rules above hold (pointers 16-byte aligned, strides in elements, at
 * least as wide as their rows and multiples of 8, checks before anything is launched, outputs that overlap nothing
 * unless stated, sums and statistics in 32 bits or more, results rounded once, the same call gives the same bits). */

/* y[r,:] = (x[r,:] - mean) * rstd * gain + shift with rstd = 1 / sqrt(biased variance + eps), and the statistics that
 * the gradients need: stats[2 r] = mean, stats[2 r + 1] = rstd.  (vit_op_layernorm: rows without strides, no statistics.)
 *   x, y: activations [rows, cols]; x == y with ldx == ldy is allowed.  gain, shift: dev fp32 [cols].
 *   stats: dev fp32 [rows][2], may be NULL.  cols: a multiple of 8, at most 8192. */
int vit_op_layernorm_forward(vit_handle* h, int dtype, int rows, int cols, const void* x, int64_t ldx, const float* gain,
                             const float* shift, float eps, void* y, int64_t ldy, float* stats, void* stream);

/* Bytes of scratch for vit_op_layernorm_backward; 0 if an argument is invalid. */
size_t vit_layernorm_backward_bytes(int rows, int cols);

/* Gradients of vit_op_layernorm_forward from its input, its statistics and dy:
 * dx (+ dres where dres is given: the gradient that arrives on the residual path), and the sums over rows dgain and
 * dshift (dev fp32 [cols], overwritten; zero for no rows).
 *   dx may be x, dy or dres with the same stride.  dres: NULL for none (lddres is not looked at then). */
int vit_op_layernorm_backward(vit_handle* h, int dtype, int rows, int cols, const void* x, int64_t ldx, const float* gain,
                              const float* stats, const void* dy, int64_t lddy, const void* dres, int64_t lddres, void* dx,
                              int64_t lddx, float* dgain, float* dshift, void* ws, size_t ws_bytes, void* stream);

/* Linear layers whose rows come in groups, each with weights of its own: tokens sorted by expert.  One group is an
 * ordinary linear layer (vit_op_linear's product with strides, and the gradients that it lacks).
 * The rows of group g are offsets[g] ... offsets[g+1] - 1.  The offsets are read on the device.  A group whose offsets are
 * out of order or reach outside the rows is skipped, its rows (or weights' gradients) are left as they were, and
 * vit_check_status reports VIT_ERR_OFFSETS; the other groups are computed; where a step backwards makes two of them
 * overlap, what is written to the rows that they share is undefined.  Rows that no group covers are left as they were.
 * A problem whose tiles could not be counted in 32 bits, if every group had all rows, is refused (VIT_ERR_TOO_LARGE). */
typedef struct vit_grouped_problem {
  int32_t groups;                     /* >= 1 */
  int32_t rows;                       /* of the activations; at most INT32_MAX - 1024 */
  int32_t in_features, out_features;  /* multiples of 8 */
  const int32_t* offsets;             /* dev [groups + 1], or NULL for one group of all rows */
} vit_grouped_problem;

/* out[r,:] = f(x[r,:] . w[g]^T + bias[g]) for the rows r of every group g.
 *   x: activations [rows, in_features]; out: [rows, out_features]; w: [groups][out_features][in_features] in the
 *   activation type; bias: dev fp32 [groups][out_features], or NULL for none.
 *   epilogue: 0 = none, 1 = erf-GELU, 2 = add residual [rows, out_features] (residual == out with the same stride is allowed;
 *   residual is not looked at otherwise).  pre: with epilogue 1, NULL or [rows, out_features]: receives the argument of the
 *   GELU, which its gradient needs; not looked at otherwise.
 * Sums are fp32.  The GELU is taken of the sums before they are rounded. */
int vit_op_linear_grouped(vit_handle* h, int dtype, const vit_grouped_problem* problem, const void* x, int64_t ldx,
                          const void* w, const float* bias, int epilogue, const void* residual, int64_t ldr, void* out,
                          int64_t ldo, void* pre, int64_t ldp, void* stream);

/* Gradient of its rows: dx[r,:] = (dout[r,:] . w[g]) * gelu'(pre[r,:]).  pre: [rows, in_features], the argument of a GELU
 * that made x (so that dx is the gradient of that argument), or NULL for no such factor; pre == dx with the same stride is
 * allowed.  dx: [rows, in_features]. */
int vit_op_linear_grouped_backward_input(vit_handle* h, int dtype, const vit_grouped_problem* problem, const void* dout,
                                         int64_t lddout, const void* w, const void* pre, int64_t ldp, void* dx,
                                         int64_t lddx, void* stream);

/* Bytes of scratch for vit_op_linear_grouped_backward_weights; 0 if an argument is invalid or the problem is too large. */
size_t vit_linear_grouped_backward_weights_bytes(int dtype, const vit_grouped_problem* problem);

/* Gradients of its weights: dw[g] = sum over the rows r of group g of dout[r,:]^T x[r,:] ([groups][out_features]
 * [in_features], activation type) and dbias[g] = sum of dout[r,:] (dev fp32 [groups][out_features], or NULL for none).  Both
 * are overwritten, with zeros for a group without rows.  Long sums are cut where the lengths of all groups of the call say,
 * so that beside other groups the last bit may differ. */
int vit_op_linear_grouped_backward_weights(vit_handle* h, int dtype, const vit_grouped_problem* problem, const void* x,
                                           int64_t ldx, const void* dout, int64_t lddout, void* dw, float* dbias, void* ws,
                                           size_t ws_bytes, void* stream);

/* The gradients of all weights, scaled down together: norm = sqrt of the sum of all squares of all src, and
 * dst = src * min(1, max_norm / norm) for every tensor with a dst.  Sums are taken so that neither large nor small values
 * leave the range of 32 bits before the norm itself does.
 * (A norm beyond fp32 is written as infinity, and the tensors are scaled by what it is.)  An infinite value makes all dst
 * zero, and NaN in the infinite places, also where max_norm is infinite; a value that is not a number makes all dst NaN.
 *   tensors: HOST array of `count` entries, read before the call returns (a captured graph keeps what it said).
 *     dst == src scales in place (and writes nothing where the norm is within the bound); dst == NULL: the tensor only
 *     counts.  No dst may otherwise overlap a src, another dst, norm or ws.
 *   max_norm: >= 0, may be infinity.  norm: dev fp32 [1], may be NULL. */
typedef struct vit_tensor {
  const void* src;        /* dev, 16-byte aligned; may be NULL if count is 0 */
  void* dst;              /* dev, 16-byte aligned, or NULL */
  int64_t count;          /* values, 0 ... 2^40 */
  int32_t dtype;          /* VIT_BF16 or VIT_FP32, of src and dst */
} vit_tensor;

/* Bytes of scratch for vit_op_grad_clip with `count` tensors; 0 if count is negative. */
size_t vit_grad_clip_bytes(int count);

int vit_op_grad_clip(vit_handle* h, const vit_tensor* tensors, int count, float max_norm, float* norm, void* ws,
                     size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VIT_B200_H */
