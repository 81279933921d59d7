/*
 * rrm.h - C ABI of the MI355X (gfx950) Recurrent Residual Module library.
 *
 * The library keeps, for one linear layer (convolution or fully connected) of a CNN that runs
 * on video, the previous frame's input I_{t-1} and projection P_{t-1} = W (*) I_{t-1} + b on
 * the device and advances them with the paper's delta update (Eq. 5; Algorithm 1, inner loop)
 *
 *      P_t = P_{t-1} + W (*) (I_t - I_{t-1}),
 *
 * doing work only where the input changed.  Everything is asynchronous on the HIP stream the
 * caller passes; no call in the per-frame path synchronises with the host or allocates.
 *
 * Layouts (all row-major, innermost index last)
 *   activations  x  [n][h][w][c_in]            (FC: [n][c_in])
 *   conv weights    [c_out][kh][kw][c_in/groups]   cross-correlation, no kernel flip
 *   FC weights      [c_out][c_in]
 *   outputs      y  [n][h_out][w_out][c_out]   (FC: [n][c_out])
 *   n is the number of independent video streams (chunks of a video processed in parallel,
 *   Sec. 3.2 last paragraph); each has its own snapshots, weights are shared.
 *
 * Element types (rrm_dtype)
 *   RRM_I8_I32    x, weights int8; bias, y int32.  Exact.  A convolution needs differences of two inputs that
 *                 fit int8 (true whenever inputs are post-ReLU values in [0,127]); a violation
 *                 raises the sticky RRM_ERR_RANGE reported by rrm_get_stats.  FC layers take any inputs.
 *   RRM_BF16_F32  x, weights bfloat16 (16-bit patterns); bias, y float32.  Inputs must be
 *                 finite.
 *   RRM_BIN_I32   x, weights are +1/-1 values bit-packed along the channel axis into 32-bit
 *                 words, LSB first, bit 1 = +1 (c_in must be a multiple of 32; x is
 *                 [n][h][w][c_in/32] words, weights [c_out][kh][kw][c_in/groups/32] words);
 *                 bias, y int32.  Exact.  Convolution only; taps outside the image contribute 0.
 *
 * Pointers: `weights` and `bias` given to rrm_layer_create may be host or device memory and are
 * copied (the caller may free them on return).  x / y arguments of rrm_step and rrm_dense are
 * DEVICE pointers, 16-byte aligned, borrowed until the work enqueued on `hip_stream` has run.
 * `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).
 *
 * Errors: every call returns an rrm_status (never throws, never aborts).  rrm_last_error()
 * gives a human-readable description of the last failure on the calling thread.
 *
 * Threading: one handle is used from one stream at a time; distinct handles are independent.
 */
#ifndef RRM_H
#define RRM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct rrm_layer rrm_layer; /* opaque: device copies of W, b, snapshots, scratch */

typedef enum {
    RRM_OK = 0,
    RRM_ERR_NULL = -1,   /* a required pointer is NULL */
    RRM_ERR_SHAPE = -2,  /* shape not representable / not supported */
    RRM_ERR_DTYPE = -3,  /* unknown dtype, or dtype not valid for this kind */
    RRM_ERR_ALLOC = -4,  /* device or host allocation failed */
    RRM_ERR_HIP = -5,    /* a HIP runtime call failed */
    RRM_ERR_STATE = -6,  /* call not valid in the handle's current state */
    RRM_ERR_RANGE = -7,  /* an int8 difference did not fit int8 (sticky, see rrm_get_stats) */
    RRM_ERR_OPTION = -8, /* unknown option key or value */
    RRM_ERR_ALIGN = -9,  /* a device pointer is not aligned (16 bytes, where a call does not say otherwise) */
    RRM_ERR_WORKSPACE = -10 /* the caller's workspace is smaller than the call needs */
} rrm_status;

typedef enum { RRM_CONV = 0, RRM_FC = 1 } rrm_kind;
typedef enum { RRM_I8_I32 = 0, RRM_BF16_F32 = 1, RRM_BIN_I32 = 2 } rrm_dtype;

/* Layer description.  FC layers use n, c_in, c_out (h = w = kh = kw = stride = groups = 1,
 * pad = 0).  h_out = (h + 2*pad - kh)/stride + 1, likewise w_out. */
typedef struct {
    int kind; /* rrm_kind */
    int n, h, w, c_in, c_out, kh, kw, stride, pad, groups;
} rrm_shape;

/* Counters of a handle.  All are totals since creation or the last rrm_reset.  `steps` is counted by the host
 * when a call is enqueued (a captured graph that is replayed does not advance it); every other counter is kept
 * on the device by the kernels themselves and also advances under graph replay. */
typedef struct {
    uint64_t steps;           /* rrm_step calls enqueued by the host */
    uint64_t delta_steps;     /* steps executed on the sparse delta path */
    uint64_t changed_elems;   /* input elements (binary: bits) that differed from the snapshot */
    uint64_t changed_units;   /* 16-byte input units with any difference (FC: = changed_elems) */
    uint64_t active_tiles;    /* int8 / bf16 conv: output blocks recomputed (4x4 positions for the window-tile
                                 kernel, single positions for the position-gather kernel), or input positions
                                 multiplied (single-launch scatter path); binary conv: output
                                 positions updated (8x8 tiles for layers without bands); FC: columns
                                 streamed */
    uint64_t total_tiles;     /* the same unit, counted as a dense step would, summed over delta steps
                                 (FC: c_in per step).  Steps on different paths add different units: rrm_reset
                                 between them keeps the counters apart */
    int32_t range_error;      /* non-zero once an int8 difference overflowed */
    int32_t tile_positions;   /* positions per tile of active_tiles / total_tiles, as the last enqueued step counts
                                 them: 16, 1, 64; FC: 0 */
    uint64_t truncated_elems; /* BF16 with a threshold: differences below it (neither applied nor committed) */
    double truncated_sumsq;   /* and the sum of their squares: sum over steps of l2(u)^2 of Eq. 7's truncated maps */
} rrm_stats;

/* Create a layer handle (Eq. 3 defines the layer; Sec. 3.2 the state it keeps).
 *   weights  layout and element type as above; host or device; copied and repacked.
 *   bias     c_out values (int32 or float32), host or device, may be NULL (= 0); copied.
 *   shape    validated; unsupported combinations give RRM_ERR_SHAPE.  A convolution keeps the input window of
 *            a 4 x 4 output sub-tile (3*stride + kh rows, 3*stride + kw columns, one 16-byte channel chunk or
 *            more) and that chunk's weights of every filter tap in on-chip memory.  Of the windows up to
 *            11 x 11 at strides up to 4, all fit except BF16 11 x 11 at stride 4 with 16 or more channels per
 *            group; a layer that does not fit is refused here, with a message.  BIN layers keep the window of
 *            an 8 x 8 output tile (7*stride + kh rows) twice: 152 KB bounds it.
 *   out      receives the handle.  The initial state is I_0 = 0 (Algorithm 1, first line) and
 *            P_0 = b, so the first rrm_step yields the dense result of its frame. */
rrm_status rrm_layer_create(const void* weights, const void* bias, const rrm_shape* shape, int dtype,
                            rrm_layer** out);

/* One (layer, frame) iteration of Algorithm 1: difference with the stored input, weights times
 * the non-zero part of the difference, sum into the stored projection, snapshot of the input.
 *   x_t    device, this frame's input for all n streams.
 *   y_out  device, may be NULL; when given it receives a full copy of P_t (n*h_out*w_out*c_out
 *          values).  Without it, read the projection through rrm_snapshot.
 * After the enqueued work has run: y_snap == b + W (*) x_t (exactly for I8/BIN; to fp32
 * accumulation accuracy for BF16) and x_snap == x_t bitwise. */
rrm_status rrm_step(rrm_layer* layer, const void* x_t, void* y_out, void* hip_stream);

/* The standard (dense) layer of Eq. 3: y = b + W (*) x.  Stateless: snapshots are untouched. */
rrm_status rrm_dense(rrm_layer* layer, const void* x, void* y, void* hip_stream);

/* rrm_dense for callers that cannot allocate device memory while they run (code under HIP-graph capture, tight
 * serving loops, harnesses that forbid it): FC layers only; the partial sums of the row splits, which rrm_dense
 * keeps in a buffer the handle allocated at create, live in a static device array of 4 MiB that exists once per
 * GPU.  The call allocates and frees nothing.  Same arguments and result as rrm_dense (of a BF16 layer that rrm_dense
 * runs as one product, see "fc_batched", up to the order of the fp32 sums).  A layer whose partial
 * sums (n x row splits x c_out x 4 bytes) exceed the array gives RRM_ERR_SHAPE.  Every call on a GPU shares that
 * GPU's array: calls that overlap in time on one GPU (different streams, different handles) race.
 * Errors: RRM_ERR_NULL, RRM_ERR_ALIGN, RRM_ERR_SHAPE (not an FC layer, or too large), RRM_ERR_HIP. */
rrm_status rrm_dense_noalloc(rrm_layer* layer, const void* x, void* y, void* hip_stream);

/* Forget the stream history: I <- 0, P <- b, counters cleared (the "new precise inference"
 * of Sec. 3.4 starts from here: the next rrm_step recomputes its frame in full). */
rrm_status rrm_reset(rrm_layer* layer, void* hip_stream);

/* Borrowed device pointers to the stored input and projection (valid until destroy). */
rrm_status rrm_snapshot(rrm_layer* layer, const void** x_snap, const void** y_snap);

/* Copy the stored input and/or projection into caller-owned device buffers (either may be NULL),
 * enqueued on hip_stream: x_dst receives the bytes of x_snap (same format as x_t), y_dst the
 * n*h_out*w_out*c_out values of y_snap. */
rrm_status rrm_read_snapshot(rrm_layer* layer, void* x_dst, void* y_dst, void* hip_stream);

/* Options: how a step is carried out, never what it computes (every setting yields the P_t of Eq. 5 / Algorithm 1,
 * within the layer's tolerance).  Value semantics per key:
 *   "path"        0 auto, 1 sparse delta path always (scan + tile kernel, no switch to recomputation), 2 recompute
 *                 densely every step, 3 INT8 / BF16 conv: the single-launch scatter path always (one kernel compares,
 *                 multiplies the changed input positions and adds the products into the stored projection with
 *                 atomic adds: work proportional to the changed input positions; fp32 results then depend on the
 *                 order of the adds within the layer's tolerance).  Automatic mode takes path 3 for layers of few
 *                 such adds, and there the products alone behind a scan that another layer's projection feeds: ahead
 *                 while up to about half of the positions change; a sequence in which most of them do, frame after
 *                 frame, is better served by "path" 2, or by "conv_kernel" 1, which keeps the switch to recomputation.
 *   "fc_splits"   FC, dense path: number of row splits of the weight matrix, in [1, the default chosen at
 *                 create] (the partial-sum scratch is sized for the default).  Without effect where the dense layer
 *                 runs as one product (see "fc_batched"); rrm_dense_noalloc always splits so
 *   "fc_batched"  FC with 4 to 4096 streams (c_out off 16 or rows off 64 bytes: where it pays): 1 (default) =
 *                 the dense layer runs as one product on the matrix cores with W read once for all streams, and
 *                 so does a step where that is cheaper than the streams' column walks (many streams or output
 *                 channels, long rows): it commits x_t and recomputes b + W x_t, one pass over W whatever the density;
 *                 0 = one column walk per stream as at batch 1.  Layers with a truncation threshold
 *                 or "fc_sparse_weights" take the walk.  Such a layer keeps W twice, as the walk and as the product read it
 *   "fc_sparse_weights"  FC, delta step: 1 = walk the non-zero weights of the changed columns only (pruned
 *                 models, Sec. 4.3; the (row, value) lists exist when at most half of W is non-zero at create,
 *                 else RRM_ERR_OPTION), 0 = walk whole columns (default).  fp32 sums of the sparse walk
 *                 depend on the order of its atomic adds, within the layer's tolerance; integers are exact.
 *   "bf16_terms"  BF16 conv: 2 = difference carried as hi+lo bf16 pair (default), 1 = hi only
 *   "dense_switch_pct"  INT8 / BF16 conv: a delta step whose changes touch more than this percentage of the
 *                 4x4 output blocks recomputes the whole projection (same result; cheaper than reading and
 *                 re-writing most of it); 1..100, 100 = never; defaults 75 (int8) / 40 (bf16) for the window-tile
 *                 kernel, which decides per launch, and 90 / 50 for the position-gather kernel, which decides per
 *                 work unit.  Without effect on steps that take path 3
 *   "conv_kernel" INT8 / BF16 conv: 0 = automatic (the window-tile kernel), 1 = window-tile kernel (4x4 output
 *                 blocks with their input windows gathered into LDS; any stride), 2 = position-gather kernel
 *                 (single active output positions as columns of the product; stride 1 and channel runs of
 *                 16-byte multiples; faster where every stream changes sparsely and alike).  Set it before the
 *                 first rrm_step, or follow it with rrm_reset: the two kernels keep their change flags differently.
 *   "bin_single_launch"  binary conv, delta step: 1 (default) = the whole step in one launch where the layer allows
 *                 it (compare, products of the changed positions and commit in the band kernel), 0 = a
 *                 difference kernel followed by the band kernel.  Change it only right after create or rrm_reset
 *                 (the two forms keep the flip buffer differently).
 *   "bin_cout_per_wave"  binary conv, tile kernel: output channels per wavefront, 8 / 16 (0 = heuristic)
 *   "profile"     1 = bracket every kernel of the following rrm_step calls with HIP events on the
 *                 caller's stream (see rrm_get_kernel_times; not for use under graph capture), 0 = off */
rrm_status rrm_set_option(rrm_layer* layer, const char* key, long value);

/* Read the counters: how many inputs changed and how much of the projection a step touched, the measured
 * counterpart of the density rho in the cost model of Sec. 3.3 (Table 1, Eq. 6), and the truncated differences
 * of Sec. 3.4 (Eq. 7).  Synchronises with the device (copies a small block back); call it after
 * the stream has been synchronised, outside timed regions.  Returns RRM_ERR_RANGE (with *out
 * filled) if the sticky range flag is set. */
rrm_status rrm_get_stats(rrm_layer* layer, rrm_stats* out);

/* rrm_step for a layer whose input is f(P) of the layer before it, without materialising that input
 * (Algorithm 1: the non-linear map f is applied to the projection and the result is the next layer's
 * input I).  f is the benchmark's int8 map of rrm_aux_relu_requant_pool_i8: ReLU, arithmetic right shift, clamp
 * to 127, optional 3x3 / stride-2 max pooling.  Equivalent to rrm_step(layer, f(producer's y_snap), ...), but
 * an input entry is computed and compared only under the 4x4 blocks of the projection that the producer's last
 * step wrote: elsewhere neither P nor f(P) changed.  Both layers INT8 convolutions with equal n, layer's c_in ==
 * producer's c_out (a multiple of 16), layer's (h, w) == the mapped size of the producer's (h_out, w_out).
 * Call it once after every step of the producer, on the same stream, and feed `layer` through this call
 * only (its stored input must be the mapped projection of the producer's previous step; a freshly created or
 * reset `layer` compares everything).  Not available with "path" = 2.
 * Errors: RRM_ERR_NULL, RRM_ERR_DTYPE, RRM_ERR_SHAPE, RRM_ERR_STATE, RRM_ERR_ALIGN, RRM_ERR_HIP. */
rrm_status rrm_step_from_projection(rrm_layer* layer, rrm_layer* producer, int shift, int pool, void* y_out,
                                    void* hip_stream);

/* One frame through a stack of INT8 convolution layers: Algorithm 1's inner loop over the layers, with the
 * non-linear map f between them (ReLU, right shift, clamp to 127, optional 3x3 / 2 max pooling; see
 * rrm_step_from_projection) fused into the next layer's difference kernel, so that no layer input but the frame is
 * ever written to memory:
 *     layer 0                      rrm_step(entries[0].layer, x_t)
 *     layer i > 0                  rrm_step_from_projection(entries[i].layer, entries[i-1].layer,
 *                                                           entries[i-1].shift, entries[i-1].pool)
 *     f_out (may be NULL)          f of the last layer's stored projection, recomputed only where its last step
 *                                  wrote (rrm_aux_relu_requant_pool_changed_i8 with entries[n-1].shift / .pool);
 *                                  device, int8, must hold the previous call's result
 * The shape conditions are those of the calls above.  Everything is enqueued on hip_stream; nothing synchronises.
 * Errors: RRM_ERR_NULL, or the first error of a constituent call. */
typedef struct {
    rrm_layer* layer;
    int shift; /* right shift of f applied to this layer's projection */
    int pool;  /* non-zero: 3x3 / stride-2 max pooling in f */
} rrm_stack_entry;
rrm_status rrm_stack_step(const rrm_stack_entry* entries, int n_layers, const void* x_t, void* f_out, void* hip_stream);

/* Truncation threshold of a BF16 layer (Sec. 3.4, "Improving sparsity": small values of the difference are
 * truncated to zero to gain sparsity; the experiments use 1e-2).  An entry with |x_t - x_snap| < epsilon
 * (difference formed in fp32) is not applied to the stored projection and not committed to the stored input,
 * so y_snap == b + W (*) x_snap stays true and the entry is still pending at the next frame; x_snap then
 * differs from x_t by less than epsilon per entry.  epsilon = 0 (the default) is the exact method.  Takes
 * effect at the next rrm_step; steps with "path" = 2 ignore it.
 * Errors: RRM_ERR_NULL, RRM_ERR_DTYPE (not BF16), RRM_ERR_OPTION (negative or not finite). */
rrm_status rrm_set_threshold(rrm_layer* layer, float epsilon);

/* Kernel times of the rrm_step calls made since "profile" was switched on (or since the last call
 * of this function): sums, in microseconds, of the event-bracketed durations of the scan kernel
 * (delta + change map) and of the compute kernel (tile conv / column scatter / binary conv), and
 * the number of steps summed.  Synchronises with the recorded events.  At most 1024 steps are kept. */
rrm_status rrm_get_kernel_times(rrm_layer* layer, double* scan_us, double* compute_us, int* steps);

void rrm_layer_destroy(rrm_layer* layer);

const char* rrm_status_string(int status);
const char* rrm_last_error(void);

/* Harness helper, NOT part of the paper's linear-layer path: the nonlinear map f that the int8
 * conv-stack benchmark places between layers.  out = maxpool3x3/2( min(127, max(0, y) >> shift) )
 * (pooling only if pool != 0), y NHWC int32 -> out NHWC int8, both device pointers. */
rrm_status rrm_aux_relu_requant_pool_i8(const void* y, void* out, int n, int h, int w, int c, int shift,
                                        int pool, void* hip_stream);

/* The same map applied to the stored projection of an int8 convolution layer (c_out a multiple of 4),
 * recomputing only the outputs whose window touches a 4x4 block of output positions that the layer's last
 * rrm_step wrote (Algorithm 1 applies f to all of P; where P did not change, f(P) did not either).  `out`
 * ([n][ho'][wo'][c_out] int8, 4-byte aligned, device, caller-owned) must hold the result of the previous call
 * for this layer: entries that are not recomputed keep it.  Call it once after every rrm_step, on the same
 * stream; after rrm_layer_create, rrm_reset or a dense step everything is recomputed.
 * Errors: RRM_ERR_NULL, RRM_ERR_SHAPE (not an int8 conv layer, c_out % 4 != 0, bad shift / pool),
 * RRM_ERR_ALIGN, RRM_ERR_HIP. */
rrm_status rrm_aux_relu_requant_pool_changed_i8(rrm_layer* layer, void* out, int shift, int pool, void* hip_stream);

/* Measurement probes for the benchmark, NOT part of the method: what the device sustains, to price the
 * library's kernels against measured as well as published peaks.
 * rrm_aux_probe_mfma: `workgroups` workgroups of four wavefronts, each wavefront issuing 4 * iters
 *   matrix-core products of register-resident operands (dtype RRM_I8_I32: 32x32x32 int8 tiles, 65536
 *   operations each; RRM_BF16_F32: 32x32x16 bf16 tiles, 32768 each).  `sink` is a device word that the
 *   kernel practically never writes.  1 <= iters <= 1 << 20, 1 <= workgroups <= 1 << 16.
 * rrm_aux_probe_copy: copies bytes / 16 sixteen-byte vectors from src to dst (device pointers, 16-byte
 *   aligned, not overlapping): `bytes` read and `bytes` written.
 * Errors: RRM_ERR_NULL, RRM_ERR_DTYPE, RRM_ERR_SHAPE (counts out of range), RRM_ERR_ALIGN, RRM_ERR_HIP. */
rrm_status rrm_aux_probe_mfma(int dtype, void* sink, int iters, int workgroups, void* hip_stream);
rrm_status rrm_aux_probe_copy(void* dst, const void* src, size_t bytes, void* hip_stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Operators between and behind the linear layers of a video network (not part of the paper's method): the map f of a
 * bf16 layer that ends in a group norm, a gated recurrence over the frames' features, and a gated feed-forward block on
 * them, each with its backward pass.  They keep no handle and no state of their own: every pointer is a DEVICE pointer
 * that the caller owns, borrowed until the work enqueued on hip_stream has run, and aligned to its element.  Scratch
 * is the caller's `workspace` (256-byte aligned, at least as large as the *_workspace function says, contents
 * irrelevant before and after; NULL where that is 0); calls that overlap in time need one each.  Nothing
 * synchronises, allocates or depends on the host, so all of it can be captured into a HIP graph.  Inputs and outputs of
 * one call must not overlap unless a call says otherwise.  A tensor without elements may be NULL.
 *
 * Strides count elements; the innermost axis (channels) is adjacent, the two outer ones lie as the strides say (no two
 * elements of an output at one place).  Strides of tensors that a call does not take are not looked at.
 *
 * Sums, statistics, states and gates are held in 32 bits whatever the element type; a result is rounded once, to
 * nearest even.  Every sum has one order, and nothing depends on which workgroup comes first: the same call gives the same bits.
 * (A scan of few long videos is cut into blocks whose workgroups hand their states on through the workspace, with atomic counters, loads
 * and stores.  A block waits only for such as run already; the wait is bounded all the same, at some seconds.  Were it to run out, frames of
 * that block and of those behind it would be not-a-numbers where no input is one, with RRM_OK.)
 *
 * Errors of all of them: RRM_ERR_NULL, RRM_ERR_SHAPE (sizes, strides), RRM_ERR_DTYPE (element types), RRM_ERR_OPTION
 * (activation, eps), RRM_ERR_STATE (h_last given as h0), RRM_ERR_ALIGN, RRM_ERR_WORKSPACE (too small), RRM_ERR_HIP. */
typedef enum { RRM_F32 = 0, RRM_BF16 = 1 } rrm_elem;

/* act(z): z; max(z, 0); z * sigmoid(z); z * Phi(z) with the normal distribution function Phi (erf form) */
typedef enum { RRM_ACT_NONE = 0, RRM_ACT_RELU = 1, RRM_ACT_SILU = 2, RRM_ACT_GELU = 3 } rrm_act;

/* Group norm with an activation, channels last: over a sample's positions and the c / groups channels of a group
 *      mean, var = the mean and the (biased) variance      r = 1 / sqrt(var + eps)
 *      y = act(gamma_c * (x - mean) * r + beta_c)
 * x may be a convolution's stored projection (rrm_snapshot), y the next layer's input. */
typedef struct {
    int n, positions, c, groups; /* groups divides c; n or positions may be 0; n * c and positions at most 2^31 - 4096 */
    int x_elem, y_elem, act;     /* rrm_elem of x and dx, of y and dy; rrm_act */
    float eps;                   /* > 0 */
    int64_t x_sample, x_position, y_sample, y_position, dx_sample, dx_position; /* strides; dy lies by those of y */
} rrm_norm_desc;

size_t rrm_group_norm_workspace(const rrm_norm_desc* desc, int backward);

/* gamma, beta  float32 [c]; NULL = 1, 0
 * stats        float32 [n][groups][2] or NULL: receives mean and r, which the backward pass reads */
rrm_status rrm_group_norm_act(const rrm_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y,
                              float* stats, void* workspace, size_t workspace_bytes, void* hip_stream);

/* With dz = dy * act'(z), xh = (x - mean) * r and the means over a group's values (ReLU: act'(0) = 0):
 *      dgamma_c = sum dz * xh       dbeta_c = sum dz       dx = r * (gamma dz - mean(gamma dz) - xh * mean(gamma dz xh))
 * dx, dgamma, dbeta (float32 [c]) may each be NULL. */
rrm_status rrm_group_norm_act_backward(const rrm_norm_desc* desc, const void* x, const float* stats, const float* gamma,
                                       const float* beta, const void* dy, void* dx, float* dgamma, float* dbeta,
                                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gated linear recurrence over the t frames of n videos, each of the c features by itself:
 *      a_t = sigmoid(f_t)        h_t = a_t * h_{t-1} + (1 - a_t) * x_t        y_t = h_t
 * A video of lengths[i] < t frames ends there: what x, f and dy hold behind is not looked at (not-a-numbers included),
 * y, dx and df are 0 there, and h_last is the state after its last frame (h0 for a video of no frames).
 * One frame of live videos is t = 1, with h0 the state before and h_last the state after it; there h_last may be h0. */
typedef struct {
    int n, t, c; /* each may be 0; t at most 2^31 - 256 */
    int elem;    /* rrm_elem of x, f, y and their gradients */
    int64_t x_video, x_frame, f_video, f_frame, y_video, y_frame; /* strides; dy lies by those of y */
    int64_t dx_video, dx_frame, df_video, df_frame;
} rrm_scan_desc;

/* frames between two states that a forward pass of training keeps in `marks`, float32 [n][rrm_scan_marks(t)][c] */
#define RRM_SCAN_MARK_FRAMES 64
int rrm_scan_marks(int t); /* ceil(t / RRM_SCAN_MARK_FRAMES) */
size_t rrm_gated_scan_workspace(const rrm_scan_desc* desc, int backward);

/* h0       float32 [n][c], NULL = 0           lengths  int32 [n], NULL = t each (held to [0, t])
 * h_last   float32 [n][c] or NULL             marks    see above, or NULL: the state before every 64th frame */
rrm_status rrm_gated_scan(const rrm_scan_desc* desc, const void* x, const void* f, const float* h0, const int32_t* lengths,
                          void* y, float* h_last, float* marks, void* workspace, size_t workspace_bytes, void* hip_stream);

/* With g_t = dy_t + a_{t+1} g_{t+1}, from g = dy + dh_last at a video's last frame:
 *      dx_t = (1 - a_t) g_t        df_t = g_t (h_{t-1} - x_t) a_t (1 - a_t)        dh0 = a_1 g_1 (no frames: dh_last)
 * marks    as the forward pass on the same x, f, h0 and lengths left it (h is recomputed from it, not read back)
 * dh_last  float32 [n][c] or NULL (= 0)        dh0  float32 [n][c] or NULL */
rrm_status rrm_gated_scan_backward(const rrm_scan_desc* desc, const void* x, const void* f, const float* marks,
                                   const int32_t* lengths, const void* dy, const float* dh_last, void* dx, void* df,
                                   float* dh0, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gated feed-forward block on m rows of k features, bfloat16 throughout:
 *      G = X Wg^T        U = X Wu^T        H = act(G) * U            X [m][k], Wg and Wu [f][k], H, G, U [m][f]
 * both projections, the activation and the product in one pass; the weights lie as an FC layer's do. */
typedef struct {
    int m, k, f; /* m may be 0 */
    int act;     /* rrm_act */
    int64_t x_row, wg_row, wu_row, h_row, gu_row, dx_row, dwg_row, dwu_row; /* strides; dh lies by h_row */
    int unaligned; /* 0: x, wg and wu begin at whole 16 bytes; 1: at whole elements (the workspace then holds copies of
                      them, as it does where k or a row is not a multiple of 8 elements) */
} rrm_ff_desc;

size_t rrm_gated_ff_workspace(const rrm_ff_desc* desc, int backward);

/* g, u: both or neither; for a backward pass they receive G and U, rounded to bfloat16 (half the memory and traffic of 32 bits) */
rrm_status rrm_gated_ff(const rrm_ff_desc* desc, const void* x, const void* wg, const void* wu, void* h, void* g, void* u,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/*      dG = dH * U * act'(G)     dU = dH * act(G)     dX = dG Wg + dU Wu     dWg = dG^T X     dWu = dU^T X
 * dG and dU enter the products in bfloat16, as the matrix cores take them.  A gradient is off by 0.0030 of its norm, of which rounding the result
 * alone would leave 0.0017, G and U in 32 bits 0.0023, dG and dU in 32 bits 0.0025.  dx, or dwg and dwu together, may be NULL. */
rrm_status rrm_gated_ff_backward(const rrm_ff_desc* desc, const void* x, const void* wg, const void* wu, const void* g,
                                 const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* workspace,
                                 size_t workspace_bytes, void* hip_stream);

/* Linear attention over the t frames of n videos, h heads with keys of dk and values of dv features, each head with a decay of its own:
 *      lambda = exp(log_decay_head)        S_t = lambda S_{t-1} + k_t^T v_t        o_t = scale * q_t S_t        S [dk][dv]
 * A video of lengths[i] < t frames ends there: what q, k, v and do hold behind is not looked at (not-a-numbers included), o, dq, dk and dv
 * are 0 there, and s_last is the state after its last frame (s0 for a video of no frames).  One frame of live videos is t = 1, with s0 the state
 * before and s_last the state after it; there s_last may be s0.  Inputs of several heads may be one (a head's stride of 0); their gradients come head
 * by head.  log_decay is at most 0 in a memory that fades (minus infinity: nothing of the frames before); its decays are not learned, there is no gradient.  Above 0
 * the memory grows: what the recurrence holds in 32 bits comes out so, but a head that doubles in a frame (of a few long videos,
 * whose frames many workgroups share: that grows by 2^64 in a workgroup's) goes frame by frame, some microseconds each.
 * Infinities and not-a-numbers reach what the formulas take them into, a frame's neighbours of other videos, heads and times never; an infinity may come out
 * as a not-a-number.
 *
 * A bfloat16 call multiplies on the matrix cores in bfloat16: the scores with their decays, and the state where a query reads it, are rounded to
 * it; the state itself, and what it takes up of each frame, are held in 32 bits. */
typedef struct {
    int n, t, h, dk, dv; /* n, t and h may be 0; t at most 2^31 - 256, n * h 2^28, dk and dv 1 to 256 */
    int elem;            /* rrm_elem of q, k, v, o and their gradients */
    float scale;
    int64_t q_video, q_frame, q_head, k_video, k_frame, k_head, v_video, v_frame, v_head; /* strides */
    int64_t o_video, o_frame, o_head;                                                     /* do lies by those of o */
    int64_t dq_video, dq_frame, dq_head, dk_video, dk_frame, dk_head, dv_video, dv_frame, dv_head;
} rrm_decay_desc;

size_t rrm_decay_attention_workspace(const rrm_decay_desc* desc, int backward);

/* log_decay  float32 [h]                        lengths  int32 [n], NULL = t each (held to [0, t])
 * s0         float32 [n][h][dk][dv], NULL = 0   s_last   the same or NULL */
rrm_status rrm_decay_attention(const rrm_decay_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                               const float* s0, const int32_t* lengths, void* o, float* s_last, void* workspace,
                               size_t workspace_bytes, void* hip_stream);

/* With D_t = lambda D_{t+1} + scale * q_t^T do_t, from D = ds_last + scale * q^T do at a video's last frame:
 *      dq_t = scale * S_t do_t        dk_t = D_t v_t        dv_t = k_t D_t        ds0 = lambda D_1 (no frames: ds_last)
 * S is made again from s0, k and v.  ds_last and s0 may be NULL (= 0); dq, dk, dv and ds0 may each be NULL. */
rrm_status rrm_decay_attention_backward(const rrm_decay_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                                        const float* s0, const int32_t* lengths, const void* d_o, const float* ds_last, void* dq,
                                        void* dk, void* dv, float* ds0, void* workspace, size_t workspace_bytes, void* hip_stream);

/* What stands between two blocks of a residual network, on m rows of c features: the norm behind the one, its gate, the residual scale and sum,
 * and the norm before the next,
 *      p = b * rb * post, rb = 1 / sqrt(mean(b^2) + eps)  (post_norm = 0: p = b)
 *      r = x + scale * sigmoid(gate) * p
 *      u = r * rr * pre, rr = 1 / sqrt(mean(r^2) + eps)
 * in one pass over x, b and the gate.  Without b (NULL; no gate, scale or post_norm) r is x and not written: the norm before the first block. */
typedef struct {
    int m, c;           /* m may be 0; c 1 to 16384 */
    int x_elem, b_elem; /* rrm_elem of x, r and their gradients; of b, gate, u and theirs */
    int post_norm;
    float eps;          /* > 0 */
    int64_t x_row, b_row, gate_row, r_row, u_row, dx_row, db_row, dgate_row; /* strides; dr lies by r_row, du by u_row */
} rrm_residual_desc;

/* gate, b-typed [m][c], NULL = no gate (factor 1)         scale, post, pre  float32 [c], NULL = 1
 * r, u     either may be NULL; r may be x                   stats  float32 [m][2] or NULL: receives rb and rr for the backward pass */
rrm_status rrm_residual_norm(const rrm_residual_desc* desc, const void* x, const void* b, const void* gate, const float* scale,
                             const float* post, const float* pre, void* r, void* u, float* stats, void* hip_stream);

size_t rrm_residual_norm_workspace(const rrm_residual_desc* desc); /* of the backward pass */

/* With rh = r * rr, bh = b * rb, sg = sigmoid(gate), w = du * pre and means over a row:
 *      dx = dr + rr * (w - rh * mean(w rh))     dpre = sum du rh        dgate = dx * scale * p * sg (1 - sg)     dscale = sum dx sg p
 *      dp = dx * scale * sg                     dpost = sum dp bh       db = rb * (dp post - bh * mean(dp post bh))   (post_norm = 0: dp)
 * x and b as the forward pass took them (r is made again, in 32 bits).  dr or du may be NULL (= 0); every result may be NULL. */
rrm_status rrm_residual_norm_backward(const rrm_residual_desc* desc, const void* dr, const void* du, const void* x, const void* b,
                                      const float* stats, const void* gate, const float* scale, const float* post, const float* pre,
                                      void* dx, void* db, void* dgate, float* dscale, float* dpost, float* dpre, void* workspace,
                                      size_t workspace_bytes, void* hip_stream);

/* A weight's update made orthogonal by Newton-Schulz products: n matrices G [rows][cols], each by itself,
 *      X = G / (|G| + eps)  (|G|: root of the sum of squares)        `steps` times:  A = X X^T,  X = a X + (b A + c A^2) X
 * (with A = X^T X, X = a X + X (b A + c A^2) where rows > cols, which is the same).  The result is bfloat16.  Between the products X, A and
 * b A + c A^2 are held in half precision, X at 256 times its size, so that singular values down to some 1e-6 of the norm count: polynomials
 * that leave singular values below 200 are meant.  Not-a-numbers and infinities of a matrix are its own. */
typedef struct {
    int n, rows, cols; /* n 0 to 65535; rows and cols 1 to 65536, tensors of up to 2^40 elements */
    int elem;          /* rrm_elem of G */
    int steps;         /* 1 to 100 */
    float a, b, c;     /* the polynomial */
    float eps;         /* >= 0 */
    int64_t g_matrix, g_row, x_matrix, x_row; /* strides */
} rrm_orth_desc;

size_t rrm_orthogonalize_workspace(const rrm_orth_desc* desc);
rrm_status rrm_orthogonalize(const rrm_orth_desc* desc, const void* g, void* x, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Which form of its kernels a call with this descriptor takes (host only; for tests and measurements).
 * norm: layout[0] the size of workgroup, 0 to 3, that holds a sample in registers, -1: slices; [1] channels of a workgroup (slices: their number)
 * scan: layout[0] 0: a thread a feature, 1: a workgroup a chain of blocks, 2: many; [1] frames of a block (0: none)
 * ff:   asked: 0 the forward pass, else 1 (dX) + 2 (dW); layout[0], [1] the tile shape (0 to 3; -1: few rows) and the parts of the summed axis of
 *       the forward pass or dX, [2], [3] of dW, [4] whether one launch makes both (what is not asked for: -2, 0)
 * Errors: the descriptor's, RRM_ERR_NULL. */
rrm_status rrm_aux_norm_layout(const rrm_norm_desc* desc, int backward, int layout[2]);
rrm_status rrm_aux_scan_layout(const rrm_scan_desc* desc, int backward, int layout[2]);
rrm_status rrm_aux_ff_layout(const rrm_ff_desc* desc, int asked, int layout[5]);

#ifdef __cplusplus
}
#endif
#endif /* RRM_H */
