/*
 * dynconv.h -- C ABI of the MI355X (gfx950) library for spatially gated
 * MobileNetV2 inverted-residual blocks: the inference path of Verelst &
 * Tuytelaars, "Dynamic Convolutions: Exploiting Spatial Sparsity for Faster
 * Inference" (CVPR 2020), Sec. 3.1.1 (block and mask unit), Sec. 3.1.2 (hard
 * decision) and Sec. 3.2 (gather / modified depthwise / scatter execution).
 *
 * Conventions shared by every call
 * --------------------------------
 * * Feature maps are NHWC, dense, channel fastest: element (n, h, w, c) sits
 *   at ((n*H + h)*W + w)*C + c.  Flat positions are raster ordered,
 *   i = (n*H + h)*W + w, image-major; the paper's "p-th active position of the
 *   flattened mask" uses this order (Sec. 3.2, masked gather).
 * * Pointers marked (device) must be device memory of the current HIP device;
 *   (host) pointers are read during the call only.  The library allocates and
 *   frees nothing: every buffer, including the workspace, belongs to the
 *   caller.  Its only global state is a cache of device occupancy figures
 *   (workgroups the device holds at once, per kernel; written once, read
 *   atomically) and the static scratch array of
 *   dynconv_stack_forward_noalloc, so calls on different streams may run
 *   concurrently as long as their buffers are disjoint (for that call: as
 *   long as they run on different devices).
 * * Every call validates all of its arguments on the host first.  On any
 *   error it returns a nonzero status and enqueues nothing.  Otherwise the
 *   work is enqueued asynchronously on `stream` (a hipStream_t; NULL is the
 *   null stream) and DYNCONV_OK is returned; a failed kernel launch is
 *   reported as DYNCONV_ERR_HIP (the call clears HIP's last-error state
 *   before launching).  Nothing synchronises with the host, nothing is
 *   printed, no exception leaves the library.  No call enqueues a memset or
 *   a host synchronisation, so the calls may be captured into a HIP graph.
 * * Sizes that the mask decides (the active count P and the dilated count
 *   P_d) stay on the device; kernels are sized for the capacity N*H*W and
 *   read the counts there.
 * * Data types: fp32, fp16 and bf16 storage.  Arithmetic is fp32 (fp32
 *   accumulation in the matrix-core products); the expanded and depthwise
 *   intermediates are rounded to the storage type.
 * * Supported channel counts: c_in == c_out (the identity path of Eq. 3),
 *   8 <= c_in <= 256 with c_in % 8 == 0, 16 <= c_hidden <= 1536 with
 *   c_hidden % 16 == 0.  Other valid shapes return DYNCONV_ERR_UNSUPPORTED.
 *   N*H*W must stay below 2^31 / 9.  Data pointers must be 16-byte aligned.
 */
#ifndef DYNCONV_H_
#define DYNCONV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* The enumerations are 32-bit integers on both sides of the ABI.  C++ gets a
 * fixed underlying type, so that a caller's out-of-range code (rejected with
 * DYNCONV_ERR_DTYPE) is a defined value there too. */
#ifdef __cplusplus
#define DYNCONV_ENUM(tag) enum tag : int32_t
#else
#define DYNCONV_ENUM(tag) enum tag
#endif

typedef DYNCONV_ENUM(dynconv_dtype_e) {
    DYNCONV_F32 = 0,
    DYNCONV_F16 = 1,
    DYNCONV_BF16 = 2
} dynconv_dtype;

typedef DYNCONV_ENUM(dynconv_status_e) {
    DYNCONV_OK = 0,
    DYNCONV_ERR_NULL = 1,        /* a required pointer is NULL */
    DYNCONV_ERR_SHAPE = 2,       /* non-positive / overflowing sizes, overlapping buffers */
    DYNCONV_ERR_DTYPE = 3,       /* unknown dtype */
    DYNCONV_ERR_UNSUPPORTED = 4, /* well-formed but outside what the kernels implement */
    DYNCONV_ERR_CAPACITY = 5,    /* index buffers hold fewer than N*H*W entries */
    DYNCONV_ERR_ALIGN = 6,       /* a data pointer is not 16-byte aligned */
    DYNCONV_ERR_WORKSPACE = 7,   /* workspace NULL or smaller than required */
    DYNCONV_ERR_HIP = 8,         /* a HIP launch failed */
    DYNCONV_ERR_ARG = 9          /* another argument is out of range (dilation, activation, block count) */
} dynconv_status;

typedef DYNCONV_ENUM(dynconv_act_e) {
    DYNCONV_ACT_NONE = 0,
    DYNCONV_ACT_RELU = 1,
    DYNCONV_ACT_RELU6 = 2,
    /* token operators (dynconv_grouped_linear and below) only: */
    DYNCONV_ACT_SILU = 3, /* v / (1 + exp(-v)) */
    DYNCONV_ACT_GELU = 4  /* v * (1 + erf(v / sqrt 2)) / 2 */
} dynconv_act;

/* Shape of a feature map: n images of h x w positions and c channels. */
typedef struct {
    int32_t n, h, w, c;
} dynconv_shape;

/*
 * One inverted-residual block with batch norm folded into weights and biases
 * (Sec. 3.2: pointwise expansion, depthwise 3x3, linear pointwise
 * projection), plus its 1x1 mask unit (Sec. 3.1.1).  All pointers (device).
 * Weight layouts are PyTorch's convolution layouts, in the storage dtype:
 *   w_expand  [c_hidden][c_in]    (from [E, C, 1, 1])
 *   w_dw      [c_hidden][9]       (from [E, 1, 3, 3]; tap k = 3*(dh+1) + (dw+1))
 *   w_project [c_out][c_hidden]   (from [Co, E, 1, 1])
 * Biases are fp32.  The mask unit is an fp32 weight vector w_mask [c_in] and
 * a scalar b_mask; MobileNetV2 uses act_expand = act_dw = RELU6 and
 * act_project = NONE.
 */
typedef struct {
    int32_t c_in, c_hidden, c_out;
    const void *w_expand;
    const float *b_expand;
    const void *w_dw;
    const float *b_dw;
    const void *w_project;
    const float *b_project;
    int32_t act_expand, act_dw, act_project;
    const float *w_mask;
    float b_mask;
} dynconv_block;

/*
 * Index maps of one hard mask (Sec. 3.2).  All arrays (device), int32, each
 * with room for `capacity` >= N*H*W positions (nbr: 9*capacity entries):
 *   active [P]     ascending flat positions with G = 1
 *   dilated[P_d]   ascending flat positions with G_dilated = 1
 *   nbr    [P][9]  nbr[p*9 + 3*(dh+1) + (dw+1)] = row of `dilated` holding the
 *                  neighbour (h+dh, w+dw) of active[p], or -1 when it lies
 *                  outside the image or outside the dilated mask
 *   counts [2]     P, P_d
 * Entries past the counts are left unspecified.
 */
typedef struct {
    int32_t *active;
    int32_t *dilated;
    int32_t *nbr;
    int32_t *counts;
    int64_t capacity;
} dynconv_indices;

/* Text for a status code, a dynconv_status value passed as an integer so
 * that any code is accepted (static storage, never NULL; codes outside the
 * enumeration give "unknown status"). */
const char *dynconv_status_str(int32_t status);

/* Library identification string (static storage). */
const char *dynconv_version(void);

/*
 * Mask unit and hard decision (Sec. 3.1.1, Eq. 2; Sec. 3.1.2, Eq. 8 with the
 * Gumbel noise fixed to zero at inference):
 *   m[i] = (sum over c ascending of w_mask[c] * x[i, c], as an fp32 fused
 *           multiply-add chain starting from +0) + b_mask     (fp32)
 *   mask[i] = m[i] > 0 ? 1 : 0                                 (ties, NaN -> 0)
 *   x       (device) NHWC, dtype dt, shape s
 *   w_mask  (device) fp32 [s.c]
 *   mask    (device) uint8 [N*H*W], written
 *   logits  (device) fp32 [N*H*W] or NULL, written when non-NULL
 * The fp32 operation order is fixed, so masks are reproducible bit for bit.
 */
dynconv_status dynconv_mask(const void *x, dynconv_shape s, dynconv_dtype dt,
                            const float *w_mask, float b_mask,
                            uint8_t *mask, float *logits, void *stream);

/*
 * The same mask unit with the G-Softmax hard decision at inference
 * (Sec. 3.1.2, the variant of Table 1 that keeps the softmax and the
 * logarithms): with m as above (fp32),
 *   p1 = 1 / (1 + exp(-m)),  p2 = 1 - p1          (Eq. 6, Eq. 7)
 *   y1 = exp(log p1) / (exp(log p1) + exp(log p2))  (Eq. 5, zero noise, tau = 1)
 *   mask[i] = y1 > 1/2 ? 1 : 0
 * in fp32 with the device's expf and logf.  In exact arithmetic y1 = p1 and
 * the decision equals dynconv_mask's; in fp32 the two differ only where the
 * rounding of p1 near 1/2 decides, i.e. for |m| below about 1e-7.
 * Arguments, logits and errors as dynconv_mask.
 */
dynconv_status dynconv_mask_gsoftmax(const void *x, dynconv_shape s, dynconv_dtype dt,
                                     const float *w_mask, float b_mask, uint8_t *mask, float *logits,
                                     void *stream);

/* Workspace bytes that dynconv_build_indices needs for shape s. */
size_t dynconv_indices_workspace_bytes(dynconv_shape s);

/*
 * Mask dilation and index maps, the paper's "bookkeeping" (Sec. 3.2, mask
 * dilation and masked gather; Table 2): the (2*dilate+1)^2 square dilation
 * of the mask within each image, then the raster-ordered lists and the
 * neighbour table described at dynconv_indices.  Output is unique, so it is
 * bit-exact and deterministic.
 *   mask    (device) uint8 [N*H*W] (nonzero = active); s.c is ignored
 *   dilate  0..3; block execution needs 1 (the depthwise kernel is 3x3)
 *   idx     (host struct, device arrays) outputs, capacity >= N*H*W
 *   ws      (device) dynconv_indices_workspace_bytes(s) bytes of scratch
 */
dynconv_status dynconv_build_indices(const uint8_t *mask, dynconv_shape s, int32_t dilate,
                                     const dynconv_indices *idx, void *ws, size_t ws_bytes,
                                     void *stream);

/* Workspace bytes that dynconv_block_forward needs. */
size_t dynconv_block_workspace_bytes(dynconv_shape s, const dynconv_block *blk,
                                     dynconv_dtype dt);

/*
 * One gated residual block (Eq. 3 with r = identity), executed on the
 * gathered rows only (Sec. 3.2):
 *   y[i] = x[i] + F(x)[i]  where the mask is active, y[i] = x[i] elsewhere,
 * with F = project(act_dw(DW3x3(act_expand(expand(x))))).  The expansion runs
 * on the dilated positions, the depthwise and projection on the active ones.
 *   x    (device) NHWC input, shape s, dtype dt
 *   y    (device) NHWC output; y == x runs in place, any other overlap is
 *        DYNCONV_ERR_SHAPE; when y != x inactive positions are copied
 *   blk  (host struct, device weights)
 *   idx  (host struct, device arrays) built by dynconv_build_indices with
 *        dilate >= 1, or NULL for the dense block (Eq. 1) on all positions
 *   ws   (device) dynconv_block_workspace_bytes bytes of scratch
 */
dynconv_status dynconv_block_forward(const void *x, void *y, dynconv_shape s, dynconv_dtype dt,
                                     const dynconv_block *blk, const dynconv_indices *idx,
                                     void *ws, size_t ws_bytes, void *stream);

/* Flags of dynconv_stack_forward. */
#define DYNCONV_STACK_DENSE 1   /* every block on all positions (Eq. 1), no mask units */
#define DYNCONV_STACK_UNFUSED 2 /* force the multi-kernel chain (mask, index maps, block) */
#define DYNCONV_STACK_GSOFTMAX 4 /* mask units decide as dynconv_mask_gsoftmax (Sec. 3.1.2) */

/* Workspace bytes that dynconv_stack_forward needs for these blocks and flags. */
size_t dynconv_stack_workspace_bytes(dynconv_shape s, const dynconv_block *blks,
                                     int32_t n_blocks, dynconv_dtype dt, int32_t flags);

/*
 * A stack of gated blocks (Sec. 3.1.1: every residual block has its own mask
 * unit, applied to that block's input), one stream, no host synchronisation.
 * The result is that of
 *   x_0 = x
 *   for b in 0..n_blocks-1:
 *     mask_b  = dynconv_mask(x_b, blks[b].w_mask, blks[b].b_mask)
 *     idx_b   = dynconv_build_indices(mask_b, dilate = 1)
 *     x_{b+1} = dynconv_block_forward(x_b, blks[b], idx_b)
 *   y = x_{n_blocks}
 * With DYNCONV_STACK_DENSE the mask units are skipped and every block runs on
 * all positions (the baseline of Eq. 1).
 *
 * Execution: when s.c <= 64 (fp32), or s.c <= 128 (fp16, bf16), or s.c is 160
 * or 192 (fp16, bf16) at maps and batches where one kernel is the faster and
 * needs no more scratch, and DYNCONV_STACK_UNFUSED is not set, each block is
 * ONE kernel over small patches of the image (at most 256 positions, at most
 * 40 columns wide), each of which builds the active and halo lists of its patch on chip (ballot ranks in raster order), gathers,
 * expands, runs the depthwise and the projection, adds the identity path and
 * computes the next block's mask (the first block also runs its own mask
 * unit); blocks alternate between y and a workspace copy.  The per-block
 * counts P, P_d take one more small kernel, launched only when counts is not
 * NULL.  Otherwise the block runs the kernel chain of the per-block calls,
 * in place on y.  Both give identical masks, counts and outputs: the same
 * arithmetic in the same order.
 *   x      (device) NHWC input, shape s, dtype dt; read only unless y == x
 *   y      (device) NHWC output; y == x runs in place, other overlap is
 *          DYNCONV_ERR_SHAPE
 *   blks   (host array of n_blocks, device weights), 1 <= n_blocks <= 1024
 *   flags  0 or DYNCONV_STACK_DENSE / DYNCONV_STACK_UNFUSED / DYNCONV_STACK_GSOFTMAX
 *          (others: ERR_ARG)
 *   masks  (device) uint8 [n_blocks][N*H*W] or NULL: per-block hard masks
 *   counts (device) int32 [n_blocks][2] or NULL: per-block P, P_d
 *   ws     (device) dynconv_stack_workspace_bytes bytes of scratch
 */
dynconv_status dynconv_stack_forward(const void *x, void *y, dynconv_shape s, dynconv_dtype dt,
                                     const dynconv_block *blks, int32_t n_blocks, int32_t flags,
                                     uint8_t *masks, int32_t *counts, void *ws, size_t ws_bytes,
                                     void *stream);

/*
 * Launch sequence of dynconv_stack_forward, for profiling: stores up to `cap`
 * names (static strings) in launch order into `names` (may be NULL when cap is
 * 0) and returns the number of launches, or -1 for invalid arguments.  A name
 * stands for a step and every kernel that runs it: "k_block_fused" is a block in
 * one launch on a patch kernel (a tracer shows k_block_fused or k_block_wide),
 * "k_conv1x1" and "k_conv3x3" of a network include k_conv1x1_tile and
 * k_conv3x3_mfma.  in_place says whether the call will have y == x.  The count
 * reduction (k_band_counts, last) is listed as if counts were requested; a
 * call without counts skips it and leaves its event pair unused.
 */
int32_t dynconv_stack_launch_names(dynconv_shape s, const dynconv_block *blks, int32_t n_blocks,
                                   dynconv_dtype dt, int32_t flags, int32_t in_place,
                                   const char **names, int32_t cap);

/*
 * dynconv_stack_forward with per-kernel timing: launch i of the sequence that
 * dynconv_stack_launch_names reports is issued with the event pair
 * (events[2i], events[2i+1]) (hipEvent_t, created by the caller), which the
 * runtime stamps when that kernel starts and ends, so
 * hipEventElapsedTime(events[2i], events[2i+1]) is the kernel's duration.
 * n_events must be at least 2 * count (else DYNCONV_ERR_ARG).  Results are
 * identical to dynconv_stack_forward.
 */
dynconv_status dynconv_stack_forward_profiled(const void *x, void *y, dynconv_shape s,
                                              dynconv_dtype dt, const dynconv_block *blks,
                                              int32_t n_blocks, int32_t flags, uint8_t *masks,
                                              int32_t *counts, void *ws, size_t ws_bytes,
                                              void *stream, void *const *events,
                                              int32_t n_events);

/*
 * dynconv_stack_forward for callers that cannot allocate device memory:
 * code under HIP graph capture that must not call hipMalloc, tight serving
 * loops, harnesses that forbid allocation.  It takes no workspace: the
 * library keeps one static scratch array of
 * dynconv_stack_noalloc_max_workspace_bytes() (16 MiB) in device memory on
 * every device it runs on, held until the process ends, and this call uses
 * the current device's copy.  Arguments, results and errors are those of
 * dynconv_stack_forward (the same kernels, bit-identical output), except:
 *   * a stack whose dynconv_stack_workspace_bytes exceeds the array returns
 *     DYNCONV_ERR_WORKSPACE and enqueues nothing;
 *   * the first call on a device looks the array up (hipGetSymbolAddress;
 *     a failure returns DYNCONV_ERR_HIP);
 *   * it calls no hipMalloc, hipFree or other allocating routine.
 * Every call on one device shares that device's array and leaves the last
 * call's contents in it (nothing in it needs to start at zero), so calls
 * that overlap in time on one device race: serialise them (one stream, or
 * events between streams).
 */
size_t dynconv_stack_noalloc_max_workspace_bytes(void);
dynconv_status dynconv_stack_forward_noalloc(const void *x, void *y, dynconv_shape s, dynconv_dtype dt,
                                             const dynconv_block *blks, int32_t n_blocks, int32_t flags,
                                             uint8_t *masks, int32_t *counts, void *stream);

/*
 * ShuffleNetV2 stride-1 units whose convolutional branch is a gated residual
 * block (Sec. 4.1.2: dynamic convolutions in the branch of the non-strided
 * units of ShuffleNetV2 with a residual connection; the branch is Eq. 3 with
 * r = identity).  With cb = s.c / 2, unit u maps its input x_u to
 *   x1 = x_u[..., 0 .. cb-1],  x2 = x_u[..., cb .. 2cb-1]
 *   mask_u = dynconv_mask(x2 zero-extended to cp channels, branches[u].w_mask,
 *                         branches[u].b_mask)
 *   b  = x2 + F(x2) where mask_u is 1, b = x2 elsewhere, with F the branch
 *        block (expand, depthwise 3x3, project with its activations;
 *        ShuffleNetV2: RELU, NONE, RELU) on x2 zero-extended to cp channels,
 *        of which the first cb outputs are kept
 *   x_{u+1}[..., 2k] = x1[k],  x_{u+1}[..., 2k+1] = b[k]    (k < cb)
 * i.e. channel_shuffle(concat(x1, b), 2), and y = x_{n_units}.
 * cp = branches[u].c_in, the same for every unit, with cb <= cp, cp a
 * multiple of 8 (so cb = 58 runs as cp = 64); the branch weights act on cp
 * channels (the caller zero-pads PyTorch's cb-channel weights; since the
 * padded input channels are zero, their weight columns do not matter, and
 * outputs cb .. cp-1 are discarded).  c_hidden is a multiple of 16 (pad
 * with zero weights).  Execution: when cp fits the one-launch unit
 * (cp <= 64 in fp32, cp <= 128 in fp16/bf16), cb * sizeof(dtype) is a
 * multiple of 4 and DYNCONV_STACK_UNFUSED is not set, each unit is ONE
 * launch on the unit's own rows: it stages the branch half (zero-extended
 * to cp channels) and the pass-through half, runs the gated block and
 * writes the shuffled rows.  Otherwise the branch input is copied into
 * compact cp-channel rows, the branch runs as one gated block (the
 * one-launch kernel or the kernel chain), and one kernel writes the
 * shuffled unit output together with the next unit's branch rows.
 *   x, y   (device) NHWC, shape s (s.c even), dtype dt; must not overlap
 *   branches (host array of n_units, device weights), 1 <= n_units <= 1024
 *   flags  0 or DYNCONV_STACK_DENSE (every branch on all positions, no mask
 *          units) / DYNCONV_STACK_UNFUSED / DYNCONV_STACK_GSOFTMAX; others: ERR_ARG
 *   masks  (device) uint8 [n_units][N*H*W] or NULL: per-unit hard masks
 *   counts (device) int32 [n_units][2] or NULL: per-unit P, P_d
 *   ws     (device) dynconv_shuffle_stack_workspace_bytes bytes of scratch
 * Errors as for dynconv_stack_forward; an odd s.c, cp < cb, or branch
 * blocks of different c_in are DYNCONV_ERR_SHAPE.
 */
size_t dynconv_shuffle_stack_workspace_bytes(dynconv_shape s, const dynconv_block *branches,
                                             int32_t n_units, dynconv_dtype dt, int32_t flags);

dynconv_status dynconv_shuffle_stack_forward(const void *x, void *y, dynconv_shape s, dynconv_dtype dt,
                                             const dynconv_block *branches, int32_t n_units,
                                             int32_t flags, uint8_t *masks, int32_t *counts, void *ws,
                                             size_t ws_bytes, void *stream);

/* Launch sequence of dynconv_shuffle_stack_forward (as for
 * dynconv_stack_launch_names; k_band_counts, when listed, is last). */
int32_t dynconv_shuffle_stack_launch_names(dynconv_shape s, const dynconv_block *branches,
                                           int32_t n_units, dynconv_dtype dt, int32_t flags,
                                           const char **names, int32_t cap);

/* dynconv_shuffle_stack_forward with per-kernel event pairs, as
 * dynconv_stack_forward_profiled. */
dynconv_status dynconv_shuffle_stack_forward_profiled(const void *x, void *y, dynconv_shape s,
                                                      dynconv_dtype dt, const dynconv_block *branches,
                                                      int32_t n_units, int32_t flags, uint8_t *masks,
                                                      int32_t *counts, void *ws, size_t ws_bytes,
                                                      void *stream, void *const *events,
                                                      int32_t n_events);

/*
 * Whole networks: a MobileNetV2 feature extractor whose stride-1 residual
 * blocks are gated (Sec. 3.1.1: every residual block gets its own mask unit;
 * Sec. 4.1.2: dynamic convolutions in MobileNetV2, with the stem, the strided
 * and the width-changing blocks evaluated at every position).
 */
typedef enum {
    DYNCONV_LAYER_CONV3X3 = 0, /* full 3x3 convolution, zero padding 1 (the stem) */
    DYNCONV_LAYER_BLOCK = 1,   /* inverted-residual block */
    DYNCONV_LAYER_CONV1X1 = 2  /* pointwise convolution */
} dynconv_layer_kind;

/*
 * One layer (host struct, device weights; PyTorch layouts in the storage
 * dtype, fp32 biases):
 *   CONV3X3  w [c_out][c_in][3][3], b [c_out], act, stride 1 or 2;
 *            y[o][i][j] = act(sum w[o][c][kh][kw] x[c][s*i+kh-1][s*j+kw-1] + b[o]),
 *            output (H-1)/stride+1 x (W-1)/stride+1; 1 <= c_in <= 16,
 *            c_out a multiple of 8, 9*c_in*c_out + c_out <= 16384
 *   CONV1X1  w [c_out][c_in], b [c_out], act; c_in, c_out multiples of 8,
 *            c_out <= 4096
 *   BLOCK    blk: expansion 1x1 (w_expand NULL for an expansion factor of 1,
 *            then c_hidden = c_in), depthwise 3x3 with `stride`, projection
 *            1x1, each with its activation; the block adds its input when
 *            stride is 1 and c_in == c_out (Eq. 1, r = identity).
 *            gated = 1 (stride 1, c_in == c_out, w_expand present): the gated
 *            block of Eq. 3 with blk's mask unit, executed as
 *            dynconv_stack_forward executes one block (constraints of
 *            dynconv_block apply); gated = 0: every position, channel
 *            counts multiples of 8, c_hidden <= 1792 (the depthwise weights
 *            are staged in 64 KB of LDS), c_out <= 4096.
 * c_in/c_out of BLOCK layers are blk.c_in/blk.c_out; the layer's own c_in,
 * c_out, w, b, act are for the convolutions.
 */
typedef struct {
    int32_t kind;
    int32_t stride;
    int32_t gated;
    int32_t c_in, c_out;
    const void *w;
    const float *b;
    int32_t act;
    dynconv_block blk;
} dynconv_layer;

/* Output shape of a layer list applied to `in` (its c = the first layer's
 * c_in); errors as dynconv_network_forward's validation. */
dynconv_status dynconv_network_output_shape(dynconv_shape in, const dynconv_layer *layers, int32_t n_layers,
                                            dynconv_shape *out);

/* Workspace bytes of dynconv_network_forward (0 for invalid arguments). */
size_t dynconv_network_workspace_bytes(dynconv_shape in, const dynconv_layer *layers, int32_t n_layers,
                                       dynconv_dtype dt, int32_t flags);

/*
 * y = layers(x), one stream, no host synchronisation.
 *   x      (device) NHWC input, shape `in`, dtype dt
 *   y      (device) NHWC output of dynconv_network_output_shape; must not
 *          overlap x
 *   layers (host array of n_layers, device weights), 1 <= n_layers <= 1024
 *   flags  0 / DYNCONV_STACK_DENSE (gated blocks on every position, no mask
 *          units) / DYNCONV_STACK_UNFUSED / DYNCONV_STACK_GSOFTMAX (as for
 *          dynconv_stack_forward; others: ERR_ARG)
 *   masks  (device) uint8 or NULL: the hard masks of the gated blocks in
 *          layer order, each N*H*W of that block's resolution, concatenated
 *   counts (device) int32 [number of gated blocks][2] or NULL: P, P_d
 *   ws     (device) dynconv_network_workspace_bytes bytes of scratch
 * Every layer is validated before anything is enqueued (ERR_SHAPE for a
 * width that does not chain, ERR_UNSUPPORTED for widths the kernels do not
 * take, ERR_ARG for a bad kind, stride or activation).
 */
dynconv_status dynconv_network_forward(const void *x, void *y, dynconv_shape in, dynconv_dtype dt,
                                       const dynconv_layer *layers, int32_t n_layers, int32_t flags,
                                       uint8_t *masks, int32_t *counts, void *ws, size_t ws_bytes,
                                       void *stream);

/* Launch sequence of dynconv_network_forward, as dynconv_stack_launch_names;
 * with_counts says whether the call will pass counts (each gated block then
 * ends with its count reduction). */
int32_t dynconv_network_launch_names(dynconv_shape in, const dynconv_layer *layers, int32_t n_layers,
                                     dynconv_dtype dt, int32_t flags, int32_t with_counts, const char **names,
                                     int32_t cap);

/* dynconv_network_forward with per-kernel event pairs, as
 * dynconv_stack_forward_profiled. */
dynconv_status dynconv_network_forward_profiled(const void *x, void *y, dynconv_shape in, dynconv_dtype dt,
                                                const dynconv_layer *layers, int32_t n_layers, int32_t flags,
                                                uint8_t *masks, int32_t *counts, void *ws, size_t ws_bytes,
                                                void *stream, void *const *events, int32_t n_events);

/*
 * Token operators: rows executed with weights chosen among many
 * --------------------------------------------------------------
 * The blocks above decide per position whether it runs.  These calls decide
 * which weights a row runs with: a router picks top_k of E experts per row and
 * lists the assignments by expert, products grouped by those lists read each
 * expert's weights for its rows only, and a shared projection takes low-rank
 * adapters per request beside it.  The conventions at the top of this file
 * hold (device pointers, host validation, one stream, no allocation, HIP graph
 * capture).  Rows are dense, channel fastest; fp32, fp16 and bf16 storage with
 * fp32 accumulation.  Widths (c_in, c_hidden, c_out) are multiples of 8 up to
 * 65536; data and weight pointers 16-byte aligned, lists 4-byte; row counts
 * below 2^31.  A call on no rows is valid: it enqueues nothing (the router
 * still writes its empty lists) and may have NULL row pointers.  Values in
 * device lists are checked by the kernels: an entry outside its range makes
 * its row (or assignment) one that is not computed, and nothing is read or
 * written for it.
 */

/* Routes of `tokens` rows (host struct, device arrays):
 *   expert [tokens][top_k]  chosen experts in falling order of their key, -1
 *                           in the slots without one
 *   weight [tokens][top_k]  fp32, 0 in the slots without an expert
 *   rows   [tokens*top_k]   assignments a = token*top_k + slot, grouped by
 *                           expert, ascending in each group; the entries
 *                           from starts[experts] on are -1
 *   starts [experts + 1]    group e is rows[starts[e]] .. rows[starts[e+1] - 1]
 *   capacity                entries that rows has room for
 */
typedef struct {
    int32_t *expert;
    float *weight;
    int32_t *rows;
    int32_t *starts;
    int64_t capacity;
} dynconv_routes;

#define DYNCONV_ROUTE_SIGMOID 1     /* weights by sigmoid instead of softmax */
#define DYNCONV_ROUTE_RENORMALIZE 2 /* weights of a row's chosen experts sum to `scale` */
#define DYNCONV_ROUTE_SCORE_BIAS 8  /* bias is added to the scores, not to the logits */

/* Workspace bytes of dynconv_route (0 for invalid sizes). */
size_t dynconv_route_workspace_bytes(int64_t tokens, int32_t experts, int32_t top_k);

/*
 * Top-k router.  key[t][e] = logits[t][e] + bias[e], one fp32 addition; row t
 * takes the top_k experts of the largest keys, ties to the lowest e (-0 and +0
 * tie).  Experts whose key is NaN or -inf are never chosen, and a row whose
 * mask is 0 chooses none.  With DYNCONV_ROUTE_SCORE_BIAS, the balancing bias of
 * routers that add it to what their weights come from, key[t][e] = s + bias[e],
 * s being the fp32 score 1 / (1 + exp(-l)) with DYNCONV_ROUTE_SIGMOID, else the
 * softmax over the row's experts (a logit of NaN or -inf still takes no part);
 * the two choices differ, as neither score is linear in the logits.  Without a
 * bias the flag changes nothing.  A bias counts in the choice alone: with l =
 * the unbiased logits in fp32,
 *   softmax:               w = exp(l) / sum of exp(l) over every expert of the
 *                          row that could be chosen; renormalised: over the
 *                          chosen ones (equal infinite maxima share alike)
 *   DYNCONV_ROUTE_SIGMOID: w = 1 / (1 + exp(-l)); renormalised: over the
 *                          chosen ones' sum, also where each of them underflows
 * and weight = scale * w.  The choice and the lists are exact and
 * deterministic.
 *   logits (device) [tokens][experts], dtype dt, aligned to its type
 *   bias   (device) fp32 [experts], finite, or NULL
 *   mask   (device) uint8 [tokens] (nonzero = routed) or NULL: all rows
 *   flags  any of DYNCONV_ROUTE_SIGMOID, DYNCONV_ROUTE_RENORMALIZE and
 *          DYNCONV_ROUTE_SCORE_BIAS (others: ERR_ARG)
 *   1 <= experts <= 1024, 1 <= top_k <= min(16, experts)
 */
dynconv_status dynconv_route(const void *logits, int64_t tokens, dynconv_dtype dt, int32_t experts, int32_t top_k,
                             const float *bias, const uint8_t *mask, int32_t flags, float scale,
                             const dynconv_routes *routes, void *ws, size_t ws_bytes, void *stream);

/* One pointwise product, or one per group: w [c_out][c_in] or
 * [groups][c_out][c_in] in the storage dtype, b fp32 [c_out] or
 * [groups][c_out] or NULL, and its activation (device pointers). */
typedef struct {
    int32_t c_in, c_out;
    const void *w;
    const float *b;
    int32_t act;
} dynconv_linear;

/*
 * Products grouped by weight, groups of any sizes: for every list position p
 * of group g, starts[g] <= p < starts[g + 1],
 *   y[dst ? dst[p] : p] = act(W_g x[src ? src[p] / src_div : p] + b_g)
 * With a router's lists, src = rows and src_div = top_k gather the rows of
 * each expert, and dst = rows puts results back at their assignments.
 *   x      (device) [x_rows][c_in];  y (device) [y_rows][c_out], not
 *          overlapping x; rows that no position names stay as they are
 *   starts (device) int32 [groups + 1], groups <= 1024, ascending (if they are
 *          not, nothing is computed); values are taken as if cut to 0 .. rows
 *   rows   list positions; src and dst (device) int32 [rows] or NULL (then
 *          x_rows or y_rows must be at least rows); the entries of dst are
 *          distinct; src_div >= 1, 1 without src
 */
dynconv_status dynconv_grouped_linear(const void *x, int64_t x_rows, void *y, int64_t y_rows, dynconv_dtype dt,
                                      const dynconv_linear *l, int32_t groups, const int32_t *starts, int64_t rows,
                                      const int32_t *src, int32_t src_div, const int32_t *dst, void *stream);

/*
 * An expert layer: per expert an expansion, optionally gated, and a
 * projection (device pointers; weights in the storage dtype, biases fp32 or
 * NULL):
 *   h = act(W_expand x + b_expand), or with w_gate
 *   h = act(W_gate x + b_gate) * (W_expand x + b_expand)
 *   F_e(x) = W_project h + b_project
 *   w_expand, w_gate [experts][c_hidden][c_in]; w_project [experts][c_out][c_hidden]
 * F_e(x) stays in fp32 until it is summed.  h is rounded to the storage type (fp16:
 * infinite past 65504), as the blocks' intermediates are; calls of one token, or of
 * so few that tokens * top_k * 2 <= experts, keep twice its bits, which costs little
 * there: a row's result is closer to the formula in such a call than in a longer one.
 */
typedef struct {
    int32_t c_in, c_hidden, c_out, experts;
    const void *w_expand;
    const float *b_expand;
    const void *w_gate;
    const float *b_gate;
    const void *w_project;
    const float *b_project;
    int32_t act;
} dynconv_experts;

#define DYNCONV_EXPERTS_RESIDUAL 1 /* add the layer's input (c_in == c_out) */

/* Workspace bytes of dynconv_experts_forward (0 for invalid arguments). */
size_t dynconv_experts_workspace_bytes(int64_t tokens, const dynconv_experts *e, dynconv_dtype dt, int32_t top_k);

/*
 * y[t] = (x[t] +) sum over the slots s of row t, in slot order, of
 *        weight[t][s] * F_{expert[t][s]}(x[t])
 * for routes that dynconv_route made.  A row without experts gives 0, or x[t].
 *   x (device) [tokens][c_in], y (device) [tokens][c_out]; y == x runs in
 *   place (c_in == c_out), any other overlap is DYNCONV_ERR_SHAPE
 */
dynconv_status dynconv_experts_forward(const void *x, void *y, int64_t tokens, dynconv_dtype dt,
                                       const dynconv_experts *e, int32_t top_k, const dynconv_routes *routes,
                                       int32_t flags, void *ws, size_t ws_bytes, void *stream);

/*
 * Low-rank adapters (device arrays), one per id:
 *   down [adapters][max_rank][c_in], up [adapters][c_out][max_rank] in the
 *   storage dtype, max_rank a multiple of 8 up to 256; ranks int32 [adapters]
 *   or NULL (all max_rank): rows of down and columns of up from ranks[i] on do
 *   not count, whatever they hold; scales fp32 [adapters] or NULL (1).  An
 *   infinity or NaN in an adapter stays in its own rows
 */
typedef struct {
    int32_t adapters, max_rank;
    const void *down;
    const void *up;
    const int32_t *ranks;
    const float *scales;
} dynconv_adapters;

/* Workspace bytes of dynconv_adapter_linear (0 for invalid arguments). */
size_t dynconv_adapter_workspace_bytes(int64_t rows, const dynconv_linear *l, const dynconv_adapters *adapters,
                                       dynconv_dtype dt);

/*
 * A projection shared by the rows of many requests, each with its own
 * adapter: with i = ids[r],
 *   y[r] = act(W x[r] + b + scales[i] * up_i (down_i x[r]))
 * and y[r] = act(W x[r] + b) where ids[r] is outside 0 .. adapters - 1.  The
 * rows may come in any order; those of one request side by side run fastest.
 * scales[i] * down_i x[r] is kept in twice the bits of a 16-bit storage type (where
 * it passes the type's largest value it is infinite).
 *   x (device) [rows][c_in], y (device) [rows][c_out], not overlapping
 *   ids (device) int32 [rows]
 */
dynconv_status dynconv_adapter_linear(const void *x, void *y, int64_t rows, dynconv_dtype dt, const dynconv_linear *l,
                                      const dynconv_adapters *adapters, const int32_t *ids, void *ws, size_t ws_bytes,
                                      void *stream);

#ifdef __cplusplus
}
#endif

#endif /* DYNCONV_H_ */
