/*
 * sb.h -- C ABI of libsb, the MI355X (gfx950) compute library for one
 * SplitBrain worker's share of a training step (arXiv 2112.15317).
 *
 * The paper splits a CNN into two halves (sec. 3.1, Model Parallelism): the
 * convolutional layers, compute-heavy with few parameters, run data-parallel
 * on each worker's local batch; the fully connected layers, which hold most
 * parameters, are split to 1/K of their outputs and run on the batch that
 * the modulo layer gathers from the K workers.  One worker's compute is
 * therefore: 3x3 convolution forward / data gradient / weight gradient, the
 * ReLU and 2x2 max pooling between them (sec. 2.2), and the forward and
 * backward of its FC column shard.  Those are the calls below, together
 * with the data movement of the modulo and shard layers around the FC
 * shards for the case where every worker's buffers sit on one device.
 * Exchanges between devices and model averaging are not part of this
 * library.
 *
 * Conventions for every call
 * --------------------------
 *  * Tensor pointers are DEVICE pointers, owned by the caller, that stay
 *    valid until the enqueued work has finished.  The library never
 *    allocates, frees or synchronises inside these calls; scratch memory is
 *    the caller's workspace (query its size first).
 *  * The workspace holds split-reduction partial sums; its contents need no
 *    initialisation and are dead after the call.  Calls that share one
 *    workspace must not run concurrently (use one workspace per stream).
 *  * `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *    All work is enqueued on it, asynchronously.
 *  * Arguments are validated before anything is enqueued; on any error
 *    nothing is launched and the status says why.  A launch failure
 *    returns SB_ERR_HIP.  Faults during execution surface, as in HIP, at
 *    the caller's next synchronisation.
 *  * Outputs must not overlap inputs (checked by address range).
 *  * Layouts: activations NCHW row-major, or channel-blocked NCHW8C
 *    (sb_layout) for the conv and pooling calls; conv weights KCRS
 *    ([out][in][3][3]); FC input X [M][Kin] and shard weights
 *    W_shard [Kin][Ns] row-major.  Element strides are in elements.
 *  * dtype SB_F32: every tensor fp32.  SB_BF16: activations, activation
 *    gradients and conv weights are bfloat16 (round-to-nearest-even on
 *    store); accumulation is fp32; bias, weight gradient and bias gradient
 *    are fp32.  SB_F32 products are formed from bf16 parts of the operands
 *    where those hold all bits, else on fp32 operands: infinities, NaNs and
 *    subnormals come out as from fp32 sums, and the part of a call that
 *    meets one, or an operand below 2^-110, takes 3 to 7 times as long.
 *  * Calls are thread-safe; the library keeps no state between calls.
 */
#ifndef SB_H
#define SB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SB_OK = 0,
    SB_ERR_INVALID_ARG = 1,   /* null pointer, bad size, overlap, bad flag */
    SB_ERR_UNSUPPORTED = 2,   /* valid request this build does not provide */
    SB_ERR_WORKSPACE = 3,     /* workspace missing or smaller than needed  */
    SB_ERR_HIP = 4            /* a HIP runtime call or launch failed       */
} sb_status;

typedef enum { SB_F32 = 0, SB_BF16 = 1 } sb_dtype;

/* Activation layouts.  SB_NCHW: [n][c][h][w].  SB_NCHW8C (channel-blocked):
 * [n][c/8][h][w][c%8], i.e. element (n, c, h, w) at
 * ((n * C/8 + c/8) * H + h) * W + w) * 8 + c % 8, for channel counts that
 * are multiples of 8; the 8 channels of a pixel are one 16-byte bf16 piece.
 * Filters are KCRS in both. */
typedef enum { SB_NCHW = 0, SB_NCHW8C = 1 } sb_layout;

/* flags */
#define SB_FUSE_RELU 1u       /* apply ReLU to the output (conv fwd, FC fwd) */
#define SB_PACKED_FILTERS 2u  /* conv fwd / data gradient: `w` holds filters
                                 packed by sb_conv3x3_pack_filters */
#define SB_UNALIGNED 4u       /* gated FC: x or weights off 16-byte boundaries */
#define SB_TOP_PROBS 8u       /* token log-probabilities: alternatives' probabilities */

/* Returns a static string naming the status. */
const char *sb_status_string(sb_status s);

/* Library version as major*10000 + minor*100 + patch. */
int sb_version(void);

/* ------------------------------------------------------------------------
 * 3x3 convolution, stride 1, zero padding 1 (sec. 2.2: each convolutional
 * stage multiplies successive input patches with square filters; the
 * operation is the cross-correlation used by deep-learning frameworks).
 *
 *   x  [n][c][h][w]    input activations (or channel-blocked, see layout)
 *   w  [k][c][3][3]    filters
 *   y  [n][k][h][w]    output (same layout as x)
 * The layout applies to every activation tensor of a call (x, y, dy, dx,
 * the ReLU mask).  SB_NCHW8C is provided for SB_BF16 with c and k multiples
 * of 8 and w >= 8 (the bf16 MFMA kernels); other combinations return
 * SB_ERR_UNSUPPORTED.
 * ---------------------------------------------------------------------- */
typedef struct {
    int n, c, h, w;       /* batch, input channels, height, width (all > 0) */
    int k;                /* output channels (> 0)                          */
    int dtype;            /* sb_dtype                                       */
    unsigned flags;       /* SB_FUSE_RELU (forward only), SB_PACKED_FILTERS
                             (forward and data gradient)                    */
    int layout;           /* sb_layout of the activations                   */
} sb_conv3x3_desc;

/* SB_PASS_FWD_POOL: the forward with ReLU + 2x2 max pooling fused
 * (sb_conv3x3_fwd_pool); it takes the forward's workspace and packing. */
enum { SB_PASS_FWD = 0, SB_PASS_BWD_DATA = 1, SB_PASS_BWD_WEIGHT = 2, SB_PASS_FWD_POOL = 3 };

/* Workspace bytes that `pass` needs for `desc` (0 is a valid answer, and a
 * NULL workspace is then accepted).  With SB_PACKED_FILTERS set the answer
 * leaves out the room the call would otherwise use to pack the filters.
 * Returns (size_t)-1 for an invalid or unsupported descriptor. */
size_t sb_conv3x3_workspace_bytes(const sb_conv3x3_desc *desc, int pass);

/* Packed filters.  The forward and data-gradient kernels read the filters
 * rearranged into the order they stage them (slices per output-channel tile
 * and input-channel chunk; for the data gradient the filters transposed and
 * rotated by 180 degrees).  Every such call packs them first, into its
 * workspace.  A caller that runs several calls with the same filters (a
 * training step: forward, then data gradient), or wants the packing off the
 * critical path (on another stream, ahead of the call), packs them once with
 * sb_conv3x3_pack_filters and sets SB_PACKED_FILTERS on the calls, which
 * then take the packed buffer as `w`.
 *
 * sb_conv3x3_packed_bytes: bytes of the packed filters of `pass`
 * (SB_PASS_FWD or SB_PASS_BWD_DATA) for `desc`; 0 for an invalid descriptor
 * or pass.  The flags of desc other than the dtype's are ignored.
 *
 * sb_conv3x3_pack_filters: packs w [k][c][3][3] (desc->dtype, device) into
 * `packed` (device, packed_bytes >= sb_conv3x3_packed_bytes, not
 * overlapping w), on `stream`.  The result serves every call of that pass
 * on a descriptor with the same n, c, h, w, k and dtype, until w changes;
 * the caller orders it before those calls (same stream, or an event).
 * SB_ERR_INVALID_ARG for a bad descriptor, pass, pointer or size. */
size_t sb_conv3x3_packed_bytes(const sb_conv3x3_desc *desc, int pass);
sb_status sb_conv3x3_pack_filters(const sb_conv3x3_desc *desc, int pass,
                                  const void *w, void *packed,
                                  size_t packed_bytes, void *stream);

/* The packing of `count` (1..64) filter tensors in one launch, each as
 * sb_conv3x3_pack_filters(&descs[i], passes[i], w[i], packed[i],
 * packed_bytes[i]) would do it; all descriptors of one dtype, the packed
 * buffers disjoint.  A packing moves little data, so packing every layer of
 * a network this way costs about one launch instead of one per layer and
 * pass.  The host arrays are read before the call returns. */
sb_status sb_conv3x3_pack_filters_many(int count, const sb_conv3x3_desc *descs,
                                       const int *passes, const void *const *w,
                                       void *const *packed,
                                       const size_t *packed_bytes, void *stream);

/* Forward:  y[n,k,h,w] = bias[k] + sum_{c,r,s} x[n,c,h+r-1,w+s-1] * w[k,c,r,s]
 * (x = 0 outside the image), then max(y, 0) when SB_FUSE_RELU is set.
 * bias may be NULL (zero).  With SB_PACKED_FILTERS, w is the forward
 * packing of the filters (sb_conv3x3_pack_filters, SB_PASS_FWD). */
sb_status sb_conv3x3_fwd(const sb_conv3x3_desc *desc, const void *x,
                         const void *w, const float *bias, void *y,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Forward followed by ReLU + 2x2 / stride 2 max pooling in one call
 * (sec. 2.2: a convolution, its ReLU and the pooling layer after it; the
 * pooled layer's pre-activation is read by nothing else in a step, so it is
 * never written): the forward's output z as sb_conv3x3_fwd would store it
 * without SB_FUSE_RELU (bias added, rounded to the storage type), then
 * y and idx exactly as sb_relu_maxpool_fwd computes them from z.  y is
 * [n][k][h/2][w/2] and idx one byte per element of y, both in desc->layout.
 * Supported with even h and w for SB_NCHW8C bf16 when the forward's channel
 * loop is not split, and for SB_NCHW fp32 (an unsplit plan pools in the
 * kernel, a split one in its split reduction; not the few-output-channel
 * kernel): sb_conv3x3_workspace_bytes(desc, SB_PASS_FWD_POOL) is then not
 * (size_t)-1.  SB_ERR_UNSUPPORTED otherwise, SB_ERR_INVALID_ARG
 * for odd h or w, SB_FUSE_RELU, NULL pointers or overlapping outputs.
 * With SB_PACKED_FILTERS, w is the forward packing (SB_PASS_FWD). */
sb_status sb_conv3x3_fwd_pool(const sb_conv3x3_desc *desc, const void *x,
                              const void *w, const float *bias, void *y,
                              uint8_t *idx, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Data gradient (sec. 2.2 backward propagation):
 *   dx[n,c,i,j] = sum_{k,r,s} dy[n,k,i-r+1,j-s+1] * w[k,c,r,s]
 * over in-image output positions.  When relu_mask_src is non-NULL (shape of
 * dx: the activation of the layer below, whose ReLU this gradient crosses),
 * dx is set to 0 wherever relu_mask_src <= 0.  desc->flags must be 0 or
 * SB_PACKED_FILTERS (w then the data-gradient packing, SB_PASS_BWD_DATA). */
sb_status sb_conv3x3_bwd_data(const sb_conv3x3_desc *desc, const void *dy,
                              const void *w, const void *relu_mask_src,
                              void *dx, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Weight gradient (sec. 2.2 backward propagation; sec. 3.1 Modulo Layer:
 * the conv parameters are updated from the gradient of the whole local
 * batch):
 *   dw[k,c,r,s] = sum_{n,h,w} x[n,c,h+r-1,w+s-1] * dy[n,k,h,w]   (fp32)
 *   db[k]       = sum_{n,h,w} dy[n,k,h,w]                        (fp32)
 * dw and db are overwritten; db may be NULL.  The summation order is fixed
 * (no atomics): repeated calls give bit-identical results. */
sb_status sb_conv3x3_bwd_weight(const sb_conv3x3_desc *desc, const void *x,
                                const void *dy, float *dw, float *db,
                                void *workspace, size_t workspace_bytes,
                                void *stream);

/* Weight gradients of `count` layers (1..SB_MANY_MAX) in one call, each as
 * sb_conv3x3_bwd_weight computes it (bit-identical results).  The weight
 * gradient of a step reads nothing a later layer's backward writes, so a
 * caller may defer several layers' weight gradients and issue them
 * together; consecutive layers whose plans run the same kernel then share
 * one launch (one round of blocks ramping up and draining instead of one
 * per layer).
 *  * descs[i], x[i], dy[i], dw[i] as for sb_conv3x3_bwd_weight; db may be
 *    NULL (no bias gradients) or an array whose entries may be NULL.  The
 *    arrays are host memory, read during the call only.
 *  * workspace: sb_conv3x3_bwd_weight_many_workspace_bytes(count, descs)
 *    bytes, layer i's split partials in its own region; needs no
 *    initialisation.
 *  * SB_ERR_INVALID_ARG for a count out of range, null arrays or pointers,
 *    an invalid descriptor, an output overlapping any layer's input or any
 *    other output, or a workspace overlapping any operand;
 *    SB_ERR_WORKSPACE for a short workspace.  Nothing is enqueued then. */
#define SB_MANY_MAX 64
size_t sb_conv3x3_bwd_weight_many_workspace_bytes(int count,
                                                  const sb_conv3x3_desc *descs);
sb_status sb_conv3x3_bwd_weight_many(int count, const sb_conv3x3_desc *descs,
                                     const void *const *x,
                                     const void *const *dy, float *const *dw,
                                     float *const *db, void *workspace,
                                     size_t workspace_bytes, void *stream);

/* Weight gradient for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.
 * Computes exactly what sb_conv3x3_bwd_weight computes, with the same kernels
 * and the same summation order (bit-identical results), but takes no
 * workspace: the split partial sums go to a scratch array of
 * SB_NOALLOC_SCRATCH_BYTES that the library keeps in device memory, one per
 * device, reserved when the library's device code is first loaded on that
 * device and held until the process ends.  The call itself allocates and
 * frees nothing.
 *  * The stream must belong to the current device (the scratch array used is
 *    the current device's).
 *  * Every call on a device shares that device's array, and its contents
 *    after a call are dead.  Calls on one device that may overlap in time
 *    (different streams without ordering between them) race on it: the
 *    caller serialises them.
 *  * SB_ERR_WORKSPACE when sb_conv3x3_workspace_bytes(desc,
 *    SB_PASS_BWD_WEIGHT) exceeds SB_NOALLOC_SCRATCH_BYTES (nothing enqueued);
 *    other errors as for sb_conv3x3_bwd_weight. */
#define SB_NOALLOC_SCRATCH_BYTES (40u << 20)
sb_status sb_conv3x3_bwd_weight_noalloc(const sb_conv3x3_desc *desc,
                                        const void *x, const void *dy,
                                        float *dw, float *db, void *stream);

/* Describes the launch plan `pass` would use for `desc`: the name of the
 * main kernel as a profiler reports it, the grid and whether a split
 * reduction follows.  Writes at most `len` bytes (NUL-terminated) into buf
 * and returns the length of the full string plus one; returns 0 for an
 * invalid or unsupported descriptor.  Enqueues nothing. */
size_t sb_conv3x3_plan_string(const sb_conv3x3_desc *desc, int pass, char *buf,
                              size_t len);

/* ------------------------------------------------------------------------
 * Fused ReLU + 2x2 max pooling, stride 2 (sec. 2.2: pooling layers
 * subsample; sec. 3.1 Layer Partitioning: pooling is never partitioned).
 *
 *   x   [n][c][h][w]       h and w even and > 0
 *   y   [n][c][h/2][w/2]   y = max(0, max of the window)
 *   idx [n][c][h/2][w/2]   uint8 code per window: bits 0-1 = row-major
 *                          position of the first maximum (0:(0,0) 1:(0,1)
 *                          2:(1,0) 3:(1,1)); bit 7 set when that maximum
 *                          is <= 0 (the ReLU blocks the gradient); bits
 *                          2-6 zero.
 * Backward: dx (un-pooled shape) is zero except dx[window position] = dy
 * for windows whose bit 7 is clear.  dx is fully overwritten.
 * layout (sb_layout) applies to x, y, dy, dx and idx alike (idx one byte per
 * element of y); SB_NCHW8C needs c a multiple of 8 (SB_ERR_INVALID_ARG
 * otherwise).
 * ---------------------------------------------------------------------- */
sb_status sb_relu_maxpool_fwd(int n, int c, int h, int w, int dtype, int layout,
                              const void *x, void *y, uint8_t *idx,
                              void *stream);
sb_status sb_relu_maxpool_bwd(int n, int c, int h, int w, int dtype, int layout,
                              const void *dy, const uint8_t *idx, void *dx,
                              void *stream);

/* ------------------------------------------------------------------------
 * FC column shard (sec. 3.1 Layer Partitioning: a LINEAR layer is split to
 * 1/K of its outputs; Modulo Layer: it runs on the batch gathered from the
 * K workers; Shard Layer: its backward yields gradients over the full
 * input, which are reduced across workers later).
 *
 *   x        [m][k_in]      gathered activations, row stride ldx
 *   w_shard  [k_in][n_shard] this worker's columns of W, dense
 *   y, dy    [m][n_shard]   row stride ldy
 * ---------------------------------------------------------------------- */
typedef struct {
    int m, k_in, n_shard;  /* gathered rows, input features, shard columns */
    int dtype;             /* sb_dtype: SB_F32, or SB_BF16 (x, w_shard, y,
                              dy, relu_mask_src, dx_partial bfloat16; b_shard,
                              dw_shard, db_shard fp32; products exact on the
                              bf16 MFMA, summed in fp32, y and dx_partial
                              rounded to nearest-even)                     */
    int ldx;               /* row stride of x and dx_partial (>= k_in)     */
    int ldy;               /* row stride of y, dy, relu_mask_src (>= n_shard) */
    unsigned flags;        /* SB_FUSE_RELU (forward only)                  */
} sb_fc_desc;

enum { SB_FC_FWD = 0, SB_FC_BWD = 1 };

/* Workspace bytes for `pass`; (size_t)-1 for an invalid descriptor. */
size_t sb_fc_workspace_bytes(const sb_fc_desc *desc, int pass);

/* y = x * w_shard + b_shard, then max(y, 0) with SB_FUSE_RELU.  b_shard
 * [n_shard] may be NULL. */
sb_status sb_fc_shard_fwd(const sb_fc_desc *desc, const void *x,
                          const void *w_shard, const float *b_shard, void *y,
                          void *workspace, size_t workspace_bytes, void *stream);

/* With g = dy, or g = dy * [relu_mask_src > 0] when relu_mask_src (shape
 * and stride of dy: this shard's ReLU output) is non-NULL:
 *   dx_partial[i,k] = sum_j g[i,j] * w_shard[k,j]   (may be NULL: skipped)
 *   dw_shard[k,j]   = (accumulate ? dw_shard[k,j] : 0) + sum_i x[i,k] g[i,j]
 *   db_shard[j]     = (accumulate ? db_shard[j]   : 0) + sum_i g[i,j]
 * dw_shard and db_shard are fp32; db_shard may be NULL.  accumulate = 1
 * adds the gradient of the K successive modulo iterations in place.  The
 * division by K that the paper applies to FC gradients is the optimiser's
 * and is not done here. */
sb_status sb_fc_shard_bwd(const sb_fc_desc *desc, const void *x,
                          const void *w_shard, const void *dy,
                          const void *relu_mask_src, void *dx_partial,
                          float *dw_shard, float *db_shard, int accumulate,
                          void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------
 * Gated FC column shard: a dense layer with a gate in place of the ReLU (one
 * projection of the input, through an activation, multiplies another), split
 * along its outputs like the FC shard above and run on the same gathered
 * batch:
 *   a = x * w_gate + b_gate,  u = x * w_up + b_up,  y = act(a) * u
 *
 *   x               [m][k_in]      gathered activations, row stride ldx
 *   w_gate, w_up    [k_in][n_shard] this worker's columns, dense
 *   b_gate, b_up    [n_shard]       fp32, each may be NULL (zero)
 *   y, dy           [m][n_shard]    row stride ldy
 *   pre             [2][m][n_shard] fp32, dense: a, then u
 * Types as for the FC shard: SB_F32, or SB_BF16 (x, the weights, y, dy and
 * dx_partial bfloat16; biases, pre and the parameters' gradients fp32).  a, u,
 * the activation and its product with u are fp32 in both.
 * ---------------------------------------------------------------------- */
typedef enum {
    SB_ACT_SIGMOID = 0,    /* 1 / (1 + exp(-a))                              */
    SB_ACT_SILU = 1,       /* a / (1 + exp(-a))                              */
    SB_ACT_GELU = 2,       /* a * (1 + erf(a / sqrt(2))) / 2                 */
    SB_ACT_GELU_TANH = 3,  /* a * (1 + tanh(sqrt(2/pi) (a + 0.044715 a^3))) / 2 */
    SB_ACT_RELU = 4        /* max(a, 0); its derivative at 0 is 0            */
} sb_act;

typedef struct {
    int m, k_in, n_shard;  /* gathered rows, input features, shard columns */
    int dtype;             /* sb_dtype                                     */
    int act;               /* sb_act                                       */
    int ldx;               /* row stride of x and dx_partial (>= k_in)     */
    int ldy;               /* row stride of y and dy (>= n_shard)          */
    unsigned flags;        /* SB_UNALIGNED (workspace query)               */
} sb_gated_desc;

/* Workspace bytes for `pass` (SB_FC_FWD, SB_FC_BWD); (size_t)-1 for an invalid
 * descriptor, and for one whose x, y or weights, or 32 rows of x or of a weight, reach
 * 2^31 bytes (the calls return SB_ERR_UNSUPPORTED).  The workspace starts at a multiple
 * of 16; where its size is 0 it may be NULL.
 * Operands that no 16-byte access fits are laid out anew in it: those of odd sizes
 * or strides always have their room; for x or weights whose addresses are not
 * multiples of 16 the query is asked with SB_UNALIGNED (a call with less returns
 * SB_ERR_WORKSPACE). */
size_t sb_gated_workspace_bytes(const sb_gated_desc *desc, int pass);

/* y as above.  pre may be NULL (inference); the backward needs it. */
sb_status sb_gated_shard_fwd(const sb_gated_desc *desc, const void *x,
                             const void *w_gate, const void *w_up,
                             const float *b_gate, const float *b_up, void *y,
                             float *pre, void *workspace,
                             size_t workspace_bytes, void *stream);

/* From the forward's pre and the gradient dy of y, with
 *   da = dy * u * act'(a),  du = dy * act(a)   (fp32):
 *   dx_partial[i,k] = sum_j da[i,j] w_gate[k,j] + du[i,j] w_up[k,j]
 *                                              (may be NULL: skipped)
 *   dw_gate[k,j]    = (accumulate ? dw_gate[k,j] : 0) + sum_i x[i,k] da[i,j]
 *   db_gate[j]      = (accumulate ? db_gate[j]   : 0) + sum_i da[i,j]
 * and dw_up, db_up likewise with du (db_gate, db_up may each be NULL).  The
 * parameters' gradients are fp32 and carry da and du in full; SB_BF16's
 * dx_partial, itself rounded to bf16, is summed from 16 bits of them or
 * more.  An infinity in x makes its row of the weights' gradients infinite, by
 * the signs of da and du (NaN where two of them disagree).  As for the FC shard
 * the division by K is the optimiser's.
 * The summation order is fixed: repeated calls give bit-identical results. */
sb_status sb_gated_shard_bwd(const sb_gated_desc *desc, const void *x,
                             const void *w_gate, const void *w_up,
                             const float *pre, const void *dy, void *dx_partial,
                             float *dw_gate, float *dw_up, float *db_gate,
                             float *db_up, int accumulate, void *workspace,
                             size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------
 * Modulo and shard layers on one device (sec. 3.1, Modulo Layer and Shard
 * Layer; sec. 3.2, Group MP Extension).
 *
 * The buffers of `workers` emulated workers sit on this device, worker w's
 * slot at w * stride elements from the base pointer (the layout an
 * exchange between devices would fill, one slot per peer).  Workers form MP
 * groups of `mp` consecutive ids (group of worker i: first id
 * g = (i / mp) * mp); inside a group the paper's K is mp, so mp = 1 is plain
 * data parallelism and mp = workers a single group.  A call serves the
 * group of worker `iproc`: all workers of a group gather the same data, and
 * a backward call writes the results of every worker of the group.  All
 * tensors are fp32, row-major; sums run over the group's workers in
 * increasing id (the result does not depend on the launch).  Strides are
 * in elements and at least one slot's size; input and output slots of the
 * group must not overlap.  Invalid arguments return SB_ERR_INVALID_ARG with
 * nothing enqueued.
 * ---------------------------------------------------------------------- */
typedef struct {
    int workers;   /* N, a multiple of mp                                  */
    int mp;        /* MP group size (the paper's K), >= 1                  */
    int batch;     /* B: examples per local batch, a multiple of mp        */
    int features;  /* F: elements per example                              */
} sb_modulo_desc;

/* Modulo layer forward, iteration k (the counter modulo mp, 0 <= k < mp).
 * Gathered example b comes from worker g + b / s (the paper's b / size
 * within the group, s = B / mp), block k of its local batch:
 *   gathered[b][f] = local[(g + b/s) * local_stride + (k*s + b%s) * F + f]
 * local: `workers` slots of [B][F]; gathered: [B][F]. */
sb_status sb_modulo_fwd(const sb_modulo_desc *desc, int iproc, int k,
                        const float *local, size_t local_stride,
                        float *gathered, void *stream);

/* Modulo layer backward, iteration k.  dgathered: `workers` slots of [B][F],
 * each worker's gradient with respect to its gathered batch (a partial sum:
 * its FC shard covers 1/mp of the layer's outputs).  For each worker g + r
 * of the group, rows k*s .. k*s + s - 1 of its dlocal slot receive the
 * group's sum at the gathered examples it supplied:
 *   dlocal[(g + r) * dl_stride + (k*s + j) * F + f]
 *       = sum_{w = 0 .. mp-1} dgathered[(g + w) * dg_stride + (r*s + j) * F + f]
 * Other rows of dlocal are left as they are (the mp iterations fill them in
 * turn). */
sb_status sb_modulo_bwd(const sb_modulo_desc *desc, int iproc, int k,
                        const float *dgathered, size_t dg_stride,
                        float *dlocal, size_t dl_stride, void *stream);

typedef struct {
    int workers;   /* N, a multiple of mp                                  */
    int mp;        /* MP group size, >= 1                                  */
    int rows;      /* M: rows of the batch                                 */
    int shard;     /* Ns: output columns of one worker's partition         */
} sb_shard_desc;

/* Shard layer forward: the next layer's full input [M][mp*Ns] from the
 * group's partitioned outputs (`workers` slots of [M][Ns]):
 *   full[m][r*Ns + c] = parts[(g + r) * parts_stride + m*Ns + c] */
sb_status sb_shard_fwd(const sb_shard_desc *desc, int iproc,
                       const float *parts, size_t parts_stride, float *full,
                       void *stream);

/* Shard layer backward: dfull holds `workers` slots of [M][mp*Ns], each
 * worker's gradient with respect to the full input (partial sums from its
 * shard of the layer above).  Worker g + r receives its column slice,
 * summed over the group:
 *   dparts[(g + r) * dp_stride + m*Ns + c]
 *       = sum_{w = 0 .. mp-1} dfull[(g + w) * df_stride + m*mp*Ns + r*Ns + c] */
sb_status sb_shard_bwd(const sb_shard_desc *desc, int iproc,
                       const float *dfull, size_t df_stride, float *dparts,
                       size_t dp_stride, void *stream);

/* Model averaging (sec. 2: data-parallel replicas reach a global model by
 * averaging; sec. 4: every worker exchanges its parameters up to the modulo
 * layer every few batches, and the FC model shards are averaged across the
 * MP groups).  params holds `workers` slots of n fp32 elements (worker w at
 * w * stride elements, stride >= n).  Worker g * mp + r holds shard r of
 * group g (sec. 3.2), so each slot is replaced, in place, by the mean over
 * the workers holding the same parameters:
 *   mp = 1: all workers (the conv layers' replicas);
 *   mp > 1: the workers r, mp + r, 2 mp + r, ... (FC shard r across groups).
 * Each mean is the sum in increasing worker id, divided once by the count.
 * workers must be a multiple of mp; slots must not overlap (stride >= n).
 * n = 0 does nothing. */
sb_status sb_model_average(int workers, int mp, size_t n, float *params,
                           size_t stride, void *stream);

/* Model averaging of replicas in separate buffers (the same reduce as
 * sb_model_average, sec. 2 and sec. 4, for replicas that do not share one
 * slotted allocation: one call per parameter tensor, with the tensor of
 * every replica, e.g. a conv layer's filters in every MP group, or FC shard
 * r of every group).  params is a HOST array of `replicas` device pointers,
 * each to n fp32 elements; every one is replaced, in place, by the mean
 * over the replicas (the sum in increasing replica index, divided once by
 * the count).  1 <= replicas <= SB_MAX_REPLICAS; the pointers must be
 * non-NULL and their ranges must not overlap (SB_ERR_INVALID_ARG).  n = 0
 * or a single replica does nothing. */
#define SB_MAX_REPLICAS 64
sb_status sb_model_average_replicas(int replicas, size_t n, float *const *params,
                                    void *stream);

/* ------------------------------------------------------------------------
 * Loss and parameter update (NEXT after the worker's forward and backward).
 *
 * Log-softmax and negative log-likelihood on the complete model output
 * (sec. 3.1 Layer Partitioning: when the last FC layer is partitioned, a
 * shard layer before the LOG_SOFTMAX layer hands every worker the full
 * output, so the output error is evaluated as for a complete local model).
 * Per row i of the logits z [m][classes] (row stride ldz, fp32):
 *   logp[i][c] = z[i][c] - log(sum_j exp(z[i][j]))
 *   loss[i]    = -logp[i][labels[i]]
 *   dz[i][c]   = scale * (exp(logp[i][c]) - [c == labels[i]])
 * i.e. dz is the gradient of scale * sum_i loss[i] (scale = 1/m for the
 * batch mean).  labels [m] are int32 device values; the kernel never
 * indexes memory with them: a label outside [0, classes) gives loss[i] =
 * NaN and a NaN row of dz.  logp, loss and dz may each be NULL (not
 * written); logp and dz use row stride ldz.  Outputs must not overlap z or
 * labels.  Sums run in a fixed order (bitwise reproducible).
 * ---------------------------------------------------------------------- */
sb_status sb_log_softmax_nll(int m, int classes, int ldz, const float *z,
                             const int32_t *labels, float scale, float *logp,
                             float *loss, float *dz, void *stream);

/* Plain SGD step on `count` fp32 tensors (sec. 4: SGD on mini-batches;
 * sec. 3.1 Modulo Layer: the FC layers, updated K times per local batch,
 * divide their gradients by K):
 *   w[t][i] = w[t][i] - (lr * scale[t]) * g[t][i],  i < n[t]
 * with the product lr * scale[t] formed once (fp32) and one fused
 * multiply-add per element.  w, g, n and scale are HOST arrays of `count`
 * entries (1 <= count <= SB_SGD_MAX_TENSORS); w[t] and g[t] are device
 * pointers, n[t] may be 0 (nothing to do; pointers may then be NULL).  A
 * gradient must not overlap any parameter tensor of the call, and the
 * parameter tensors must not overlap each other. */
enum { SB_SGD_MAX_TENSORS = 64 };
sb_status sb_sgd_update(int count, float *const *w, const float *const *g,
                        const size_t *n, const float *scale, float lr,
                        void *stream);

/* AdamW step on many tensors (Adam with decoupled weight decay: in place of the SGD
 * step).  For every element, with g = grad_scale * gradient and t the number of this
 * update:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   w = (1 - lr decay) w - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32 (the root, and the reciprocal of its sum with eps, may be the hardware's, a step
 * of fp32 off each); m and v of the update are those before they become bytes.
 *
 * Moments:
 *   32  fp32, zero before the first update;
 *   8   bytes.  The rank of a value is its fp32 pattern's exponent and upper
 *       three mantissa bits, as a whole number: 8 ranks an octave.  Each block
 *       of 256 consecutive elements of a tensor has a reference, the largest
 *       rank in it (m_top, v_top: ceil(n / 256) int16 values).  The byte of v is
 *       255 - (reference - rank), at least 1 unless v is 0; that of m has the
 *       sign in its highest bit and 127 - (reference - rank) below it, 0 where
 *       that is negative: 31 octaves below the block's largest v, 15 below its
 *       largest m.  A value is rounded to one of its two neighbours at random,
 *       up with the probability that makes its mean right (a moment that a
 *       step changes by less than half a rank would otherwise stay as it is),
 *       from 16 bits of a hash of seed, t and the element's number `first` + i;
 *       results are the same in every run.  All bytes zero before the first
 *       update, the references too.  Infinities and NaN stay what they are, the
 *       other values of their block are lost.
 *
 * Tensors: w, g (and m, v of 32 bits) fp32; copy, if not NULL, gets w's new value
 * in bfloat16.  first: the number of the tensor's first element among the random
 * numbers; tensors of one model take ranges of their own (unused with 32).  n may
 * be 0 (nothing to do). */
enum { SB_ADAMW_MAX_TENSORS = 512, SB_ADAMW_BLOCK = 256 };
typedef struct {
    float *w;
    void *copy;            /* bfloat16, or NULL                            */
    const float *g;
    void *m, *v;           /* fp32, or bytes                               */
    int16_t *m_top, *v_top; /* references (8), unused (32)                 */
    uint64_t first;
    size_t n;
    float grad_scale;      /* 1/K for FC shards                            */
    float decay;
} sb_adamw_tensor;
typedef struct { int tensors, moments, groups, blocks; } sb_adamw_plan;

/* The tensors of an update are written into a plan in device memory once, so that
 * every update is one launch however many there are.  plan: device memory of the
 * caller's, sb_adamw_plan_bytes(count) bytes (0 for a count outside 1 ..
 * SB_ADAMW_MAX_TENSORS), a multiple of 16, alive and unchanged as long as it is
 * used (a kernel on the stream writes it: an update on another stream has to be
 * ordered behind that); info: host memory, filled by the call and handed to every update.
 * moments: 32 or 8.  The tensor array is host memory, read before the call returns.
 * SB_ERR_INVALID_ARG for bad counts or moments, scales or decays that are not
 * finite, NULL pointers, pointers that are not multiples of their elements' size, and
 * for an output (w, copy, moments, references, the plan) that overlaps any other
 * tensor of the call; gradients may overlap each other.  SB_ERR_WORKSPACE for a
 * short plan, SB_ERR_UNSUPPORTED for 2^33 elements and more.  Nothing is enqueued
 * then. */
size_t sb_adamw_plan_bytes(int count);
sb_status sb_adamw_make_plan(int moments, int count,
                             const sb_adamw_tensor *tensors, void *plan,
                             size_t plan_bytes, sb_adamw_plan *info,
                             void *stream);

/* One update of a plan's tensors.  Its number is step + *steps_done, where steps_done
 * is a device counter (int32, 0 at the start) for callers that replay the call from
 * a graph and advance it there with sb_adamw_advance, or NULL: then it is step (sums
 * below 1 count as 1).  The counter must not be part of an output.  SB_ERR_INVALID_ARG for NULL pointers, an
 * info that no plan has, betas outside [0, 1), values that are not finite, a negative
 * eps, step < 1. */
typedef struct {
    double lr, beta1, beta2, eps;
    int step;              /* >= 1                                         */
    uint32_t seed;
} sb_adamw_desc;
sb_status sb_adamw_update(const sb_adamw_desc *desc, const sb_adamw_plan *info,
                          const void *plan, const int32_t *steps_done,
                          void *stream);

/* *steps_done += 1, on the stream. */
sb_status sb_adamw_advance(int32_t *steps_done, void *stream);

/* The values that n moments in bytes stand for, in fp32 (to store, inspect or go
 * on with in 32 bits).  m_out and v_out may each be NULL (with its inputs). */
sb_status sb_adamw_unpack(size_t n, const uint8_t *m, const int16_t *m_top,
                          const uint8_t *v, const int16_t *v_top, float *m_out,
                          float *v_out, void *stream);

/* ------------------------------------------------------------------------
 * Embedding: rows of a vocabulary's table for token ids.  The table is split
 * along the vocabulary as an FC layer is along its outputs: a worker has the
 * rows of the ids first .. first + vocab - 1, and its outputs are partial, to
 * be summed over the workers.
 *
 *   ids     [tokens]         int32, on the device.  An id outside the shard's
 *                            range, a negative one (padding) among them, is
 *                            no row of it: a zero row of y, no gradient.
 *   table   [vocab][width]   dense
 *   y, dy   [tokens][width]  row stride ldy
 * SB_F32, or SB_BF16 (table, y and dy bfloat16, dtable fp32).  tokens may be 0.
 * ---------------------------------------------------------------------- */
typedef struct {
    int tokens, vocab, width;
    int first;             /* id of the table's first row (>= 0)           */
    int dtype;             /* sb_dtype                                     */
    int ldy;               /* row stride of y and dy (>= width)            */
    float scale;           /* of y; finite                                 */
} sb_embed_desc;

/* y[i] = scale * table[ids[i] - first], in fp32 and rounded once (with a scale
 * of 1 the row as it is).  SB_ERR_INVALID_ARG for NULL pointers, pointers that
 * are not multiples of their elements' size, and a y that overlaps an input. */
sb_status sb_embed_fwd(const sb_embed_desc *desc, const void *table,
                       const int32_t *ids, void *y, void *stream);

/* dtable[v] = (accumulate ? dtable[v] : 0) + scale * sum_i dy[i] over the tokens
 * with ids[i] = first + v.  Sums are fp32 and their order is fixed: repeated
 * calls give bit-identical results.  With accumulate rows without a token are
 * not touched.  The workspace starts at a multiple of 16.  Arguments are checked
 * as above, the workspace must not overlap a tensor.  SB_ERR_UNSUPPORTED (the query:
 * (size_t)-1) for 2^29 rows of the table, 2^30 tokens, rows of 2^23 elements and more
 * of each, and where the rows come to 2^32 lanes (a row has 8 or a larger power of two,
 * from 64 on multiples of it, for one or two of its 16-byte pieces each). */
size_t sb_embed_workspace_bytes(const sb_embed_desc *desc);
sb_status sb_embed_bwd(const sb_embed_desc *desc, const int32_t *ids,
                       const void *dy, float *dtable, int accumulate,
                       void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------
 * Expert rows: each token goes to `top` experts (dense or gated layers), whose
 * rows have to lie together, and their outputs come back as one row.  What the
 * modulo layer does by a fixed rule is done here by the router's choice.  A
 * worker has the experts first .. first + experts - 1; y and dx are partial,
 * to be summed over the workers.
 *
 *   ids      [tokens][top]   int32: the experts of each token.  One outside the
 *                            worker's range is not its: no row.
 *   place    [tokens][top]   int32: the row of each slot among the rows sorted
 *                            by expert (tokens in their order within one), -1
 *                            for none.  Made by sb_expert_sort.
 *   offsets  [experts + 1]   int32: expert e's rows are offsets[e] ..
 *                            offsets[e + 1] - 1, offsets[experts] their number.
 *   x, y, dy [tokens][width]         row stride ldx
 *   xs, ys, dys [tokens * top][width] row stride ldr; rows from
 *                            offsets[experts] on are neither read nor written
 *   weights, dweights [tokens][top]  fp32
 * SB_F32, or SB_BF16 (the rows bfloat16; products and sums fp32, rounded once).
 * tokens may be 0.  The calls below return SB_ERR_INVALID_ARG for bad
 * descriptors, NULL pointers, pointers that are not multiples of their elements'
 * size and outputs that overlap inputs or each other, SB_ERR_UNSUPPORTED for 2^30 slots
 * and more, rows of 2^24 and more, and tokens whose rows come to 2^32 lanes (a row has 8
 * or a larger power of two, from 64 on multiples of it, for one or two of its 16-byte
 * pieces each).  Places outside the rows count as none.
 * ---------------------------------------------------------------------- */
enum { SB_MAX_EXPERTS = 512 };
typedef struct {
    int tokens, top, experts;
    int first;             /* the worker's first expert (>= 0)             */
    int width;
    int dtype;             /* sb_dtype                                     */
    int ldx;               /* row stride of the tokens' rows (>= width)    */
    int ldr;               /* row stride of the sorted rows (>= width)     */
} sb_expert_desc;

/* place and offsets from ids.  The workspace (sb_expert_workspace_bytes, often 0;
 * (size_t)-1 for a descriptor the calls refuse) starts at a multiple of 16. */
size_t sb_expert_workspace_bytes(const sb_expert_desc *desc);
sb_status sb_expert_sort(const sb_expert_desc *desc, const int32_t *ids,
                         int32_t *place, int32_t *offsets, void *workspace,
                         size_t workspace_bytes, void *stream);

/* xs[place[t][j]] = x[t]. */
sb_status sb_expert_gather(const sb_expert_desc *desc, const void *x,
                           const int32_t *place, void *xs, void *stream);

/* y[t] = add[t] + sum_j weights[t][j] * ys[place[t][j]], in the order of j; weights may
 * be NULL (1 each), and so may add (0; rows as y's, or y itself: added to in place).  A
 * token without a row gets add's.  Without weights, on the gradient of xs, this is the
 * gather's backward: dx[t] = sum_j dxs[place[t][j]]. */
sb_status sb_expert_combine(const sb_expert_desc *desc, const void *ys,
                            const int32_t *place, const float *weights,
                            const void *add, void *y, void *stream);

/* The gradients of sb_expert_combine (that of add is dy):
 *   dys[place[t][j]] = weights[t][j] * dy[t]   (weights NULL: dy[t])
 *   dweights[t][j]   = sum_c dy[t][c] * ys[place[t][j]][c], 0 where there is no row
 * dweights may be NULL (ys is then not read and may be NULL). */
sb_status sb_expert_combine_bwd(const sb_expert_desc *desc, const void *dy,
                                const void *ys, const int32_t *place,
                                const float *weights, void *dys,
                                float *dweights, void *stream);

/* ------------------------------------------------------------------------
 * Log-probabilities of given tokens on the complete model output (as
 * sb_log_softmax_nll, for vocabularies: the log-probabilities themselves are
 * not written), the entropy of each row and its most likely classes, with the
 * logits' gradient through all of them.  On the rows of a router, with
 * SB_TOP_PROBS, the alternatives are the experts and their probabilities.
 *
 *   z, dz       [m][classes]   row stride ldz; SB_F32, or SB_BF16
 *   targets     [m]            int32: the token of each row.  Negative: none
 *                              (padding): logp 0, no gradient.  One >= classes
 *                              gives logp = NaN and a row of dz of NaN.
 *   logp        [m]            z[target] - log(sum_c exp(z[c]))
 *   entropy     [m]            -sum_c p[c] log p[c]
 *   stats       [m][2]         the largest logit, and the logarithm of
 *                              sum_c exp(z[c] - largest): for the backward
 *   top_ids     [m][top]       int32: the `top` most likely classes, most likely
 *                              first, of equal logits the lower class first
 *   top_values  [m][top]       their log-probabilities, with SB_TOP_PROBS their
 *                              probabilities
 * All but z and dz fp32.  A logit of -inf is ruled out: probability 0, log-
 * probability -inf; its dz is 0, or the gradient on its own log-probability where it
 * has one.  A row of -inf alone has stats (-inf, -inf), entropy 0,
 * log-probabilities -inf, and dz 0.  A NaN or +inf in a row makes its
 * results NaN; NaN ranks above all classes.  m may be 0.
 * Sums run in a fixed order: repeated calls give bit-identical results.
 * ---------------------------------------------------------------------- */
enum { SB_LOGP_MAX_TOP = 32 };
typedef struct {
    int m, classes, ldz;
    int dtype;             /* sb_dtype                                     */
    int top;               /* 0 .. min(SB_LOGP_MAX_TOP, classes)           */
    unsigned flags;        /* SB_TOP_PROBS                                 */
} sb_token_logp_desc;

/* Workspace bytes of the forward (0 for short rows; the backward needs none);
 * (size_t)-1 for a descriptor that the calls refuse.  It starts at a multiple
 * of 16. */
size_t sb_token_logp_workspace_bytes(const sb_token_logp_desc *desc);

/* logp (and targets with it) and entropy may each be NULL; top_ids and top_values
 * are needed where top > 0.  SB_ERR_INVALID_ARG for bad descriptors, NULL
 * pointers, pointers that are not multiples of their elements' size and
 * outputs or a workspace that overlap an input or each other; SB_ERR_UNSUPPORTED for more
 * than 2^20 classes, 2^30 rows and more, or rows that come to 2^32 lanes (one has a lane
 * for 16 classes at most, 8 lanes at least). */
sb_status sb_token_logp_fwd(const sb_token_logp_desc *desc, const void *z,
                            const int32_t *targets, float *logp, float *entropy,
                            float *stats, int32_t *top_ids, float *top_values,
                            void *workspace, size_t workspace_bytes,
                            void *stream);

/* dz = the gradient of sum_i dlogp[i] logp[i] + dentropy[i] entropy[i] +
 * sum_k dtop[i][k] top_values[i][k], from the forward's stats and, where they are
 * used, entropy (with dentropy), top_ids (with dtop) and top_values (with dtop and
 * SB_TOP_PROBS).  dlogp (with targets), dentropy and dtop may each be NULL (0).
 * The sum is formed in fp32 and rounded once.  dz may be z itself (written in
 * place); it must not overlap otherwise.  Refusals as above. */
sb_status sb_token_logp_bwd(const sb_token_logp_desc *desc, const void *z,
                            const float *stats, const int32_t *targets,
                            const float *dlogp, const float *entropy,
                            const float *dentropy, const int32_t *top_ids,
                            const float *top_values, const float *dtop,
                            void *dz, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SB_H */
