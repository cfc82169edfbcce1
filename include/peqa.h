/*
 * peqa.h -- C-ABI of the MI355X (gfx950) PEQA quantized-linear library.
 *
 * PEQA (arXiv 2305.14152, Sec. 3.2) replaces a fully-connected weight
 * W0 in R^{N x K} by  What = (s0 + ds) . (Q - z0)  with frozen b-bit integer
 * codes Q (b = 3 or 4), zero-points z0 and scales s0 per output channel
 * (optionally per group of g input features, Sec. 4.2 and Table 5), and trains only ds.
 *
 * Conventions for every call
 *   - Every tensor argument is a DEVICE pointer owned by the caller, contiguous,
 *     row-major, 16-byte aligned (PEQA_ERR_ALIGN otherwise); outputs must not
 *     alias inputs.  Descriptor structs (peqa_layout, peqa_adamw) are HOST pointers.
 *   - `stream` is a hipStream_t passed opaquely (NULL = the default stream).
 *     Calls only enqueue work; they never synchronise and never allocate or free device
 *     memory.  All work of a call is ordered after what the stream held before the call and
 *     before what is enqueued after it; the library creates no streams and (outside peqa_trace_begin) no events,
 *     so every call may be recorded by stream capture.
 *   - Arguments are validated on the host before the device is touched, so the
 *     error paths work on a machine without a GPU.  Return value: peqa_status.
 *   - bf16 tensors are passed as uint16_t bit patterns.
 *   - G = number of groups per channel = K / group_size, or 1 when group_size = 0.
 *     Scale-shaped arrays (s0, ds, d_ds, m, v, z0) are [N, G] row-major.
 *
 * Shape limits: N % 128 == 0, K % 128 == 0 (every LLaMA-family linear satisfies
 * this).  group_size is 0 or a multiple of 64 that divides K.
 *
 * Options.  The library reads nothing from the process environment.  Three switches exist for tests and
 * comparisons, set explicitly with peqa_set_option (process-wide, not thread-safe; none is needed):
 * PEQA_OPT_GEMM_WAVES = 4 | 8 forces one of the two forms of the tiled contraction kernel (0, the default:
 * a launch of one contraction with more tiles, or pieces of tiles, than compute units runs four-wave
 * workgroups, two per compute unit, one with fewer eight-wave ones; a forced form is never cut into
 * pieces); PEQA_OPT_BWD_PAIR = 0 makes a per-channel backward that is asked for both gradients run its two
 * contractions as launches of their own, 1 as one launch of four-wave workgroups (-1, the default: one
 * launch unless PEQA_OPT_GEMM_WAVES is 8); PEQA_OPT_GROUPED_DDS = 1 selects the older of two routes to the
 * scale gradient of group-wise layers (0, the default: the contraction over tokens).  Results agree within
 * rounding.
 *
 * Stacking.  The packed array is stored by rows of 128-channel tiles and the scale-shaped
 * arrays by channel, so layers with equal K, bits and group_size that read the same input
 * (the query, key and value projections; gate and up) can be laid one after the other in
 * memory -- each quantized by its own peqa_quantize call into its slice of packed, s0, z0 --
 * and then run as ONE layer with N = the sum of theirs: Y and dY are [T, sum N] with every
 * member a column range, d_ds is the members' gradients one after the other, and dX is the
 * gradient of the shared input (the sum of the members' dX) from a single contraction.
 * Results per member are those of running it alone -- bit for bit when both runs take the same
 * form of the contraction kernel (see Options; the forms add the same products in a different
 * order) and the same number of pieces (see Workspaces), else to the last bf16 bit; only dX, a sum, is new.
 *
 * Workspaces.  Where a launch's tiles would leave the machine idle (T > 16, but few tokens or a few tiles of a long
 * contraction), contractions are split along their length into pieces whose fp32 sums meet in the workspace.  The size
 * queries include that room.  A workspace that has room for everything but the pieces (what the queries return while
 * PEQA_OPT_GEMM_WAVES or PEQA_OPT_BWD_PAIR forces a form) is served too, with whole contractions (a group-wise backward
 * of many tiles: in launches of its own, with their pieces where there is room for those): the same products
 * in another order; so is, at T <= 16, one that holds the partial sums of the fewest slices the layers need, with those.
 * For a given shape, T, workspace size and set of gradients asked for results are always the same bits.
 */
#ifndef PEQA_H
#define PEQA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PEQA_OK = 0,
    PEQA_ERR_NULL = 1,      /* a required pointer is NULL                       */
    PEQA_ERR_SHAPE = 2,     /* N, K or T out of the supported range             */
    PEQA_ERR_BITS = 3,      /* bits is not 3 or 4                               */
    PEQA_ERR_GROUP = 4,     /* group_size invalid for this K                    */
    PEQA_ERR_ALIGN = 5,     /* a device pointer is not 16-byte aligned          */
    PEQA_ERR_WORKSPACE = 6, /* workspace missing or smaller than required       */
    PEQA_ERR_DEVICE = 7,    /* the HIP runtime reported a launch error          */
    PEQA_ERR_PARAM = 8      /* an optimizer or other scalar parameter is invalid */
} peqa_status;

typedef struct {
    int32_t n_out;      /* N: output channels = rows of W0 (the paper's n)             */
    int32_t k_in;       /* K: input features = columns of W0 (the paper's m)           */
    int32_t bits;       /* b: 3 or 4                                                    */
    int32_t group_size; /* 0 = one (s, z) per channel; else g with g % 64 == 0, K % g == 0   */
} peqa_layout;

typedef enum {
    PEQA_OP_FWD = 0,      /* peqa_linear_fwd        */
    PEQA_OP_BWD = 1,      /* peqa_linear_bwd        */
    PEQA_OP_FWD_KEEP = 2, /* peqa_linear_fwd_keep   */
    PEQA_OP_BWD_KEPT = 3, /* peqa_linear_bwd_kept   */
    PEQA_OP_FWD_Z = 4,    /* peqa_linear_fwd_z      */
    PEQA_OP_BWD_Z = 5     /* peqa_linear_bwd_z      */
} peqa_op;

/* Host-only helpers (no device access). */
peqa_status peqa_check_layout(const peqa_layout *L);
size_t peqa_packed_words(const peqa_layout *L);   /* N*K*bits/32 uint32 words; 0 if invalid */
size_t peqa_num_scales(const peqa_layout *L);     /* N*G; 0 if invalid                      */
/* Bytes of scratch the given call asks for with T tokens (0 if invalid; see Workspaces).  This and the other size queries are
 * for a whole MI355X (256 compute units); a call on a partition of one plans for its units, within what it was given. */
size_t peqa_workspace_bytes(const peqa_layout *L, int32_t T, int32_t op);
const char *peqa_status_string(int32_t status);

/* Test and comparison switches (see Options above).  peqa_set_option returns PEQA_ERR_PARAM for an unknown
 * option or a value outside those listed; peqa_get_option returns the current value (INT32_MIN if unknown). */
typedef enum {
    PEQA_OPT_GEMM_WAVES = 0,   /* 0 (default), 4, 8 */
    PEQA_OPT_BWD_PAIR = 1,     /* -1 (default), 0, 1 */
    PEQA_OPT_GROUPED_DDS = 2   /* 0 (default), 1 */
} peqa_option;
peqa_status peqa_set_option(int32_t option, int32_t value);
int32_t peqa_get_option(int32_t option);

/*
 * Word and bit (0..31) that hold bit `t` of the code of channel i, feature k in the
 * packed array.  The paper fixes only the density (exactly b bits per weight,
 * Table 4); the placement is this library's and is part of its contract:
 * 8x8 blocks of (channel, feature) of 2b words each, stored tile by tile so that every
 * kernel streams contiguous memory: a tile is 128 channels x 32 features (16 x 4 blocks,
 * 256 b bytes), tile (i/128, k/32) has number (i/128) * (K/32) + k/32, and block
 * (i/8, k/8) is block ((i/8)%16) * 4 + (k/8)%4 of its tile, i.e. it starts at word
 * (64 * tile + block) * 2b; inside a block r = i%8, c = k%8 and
 *   b = 4: word r, bits [4p, 4p+4) with p = c/2 + 4*(c%2);
 *   b = 3: u = 4*(r/2) + c/2; u < 15: word 2*(u/5) + r%2, bits [16*(c%2) + 3*(u%5), +3);
 *          u = 15: code bit t is bit 15 + 16*(c%2) of word 2t + r%2.
 * Host-only.  Returns PEQA_ERR_SHAPE for indices out of range.
 */
peqa_status peqa_bit_location(const peqa_layout *L, int32_t i, int32_t k, int32_t t,
                              size_t *word, int32_t *bit);

/*
 * Eq. 1, round-to-nearest with a min-max range, then dense packing.
 * Per channel i and group g:  xmin = min(min w, 0), xmax = max(max w, 0),
 * s0 = (xmax - xmin) / (2^b - 1), z0 = rint(-xmin / s0),
 * Q = clamp(rint(w / s0) + z0, 0, 2^b - 1); rint rounds half to even; every step is one
 * IEEE fp32 operation.  A group whose s0 evaluates to 0 gets s0 = 1, z0 = 0.
 *   W0      [N, K] fp32, in
 *   packed  peqa_packed_words() uint32, out
 *   s0      [N, G] fp32, out;   z0  [N, G] uint8, out
 */
peqa_status peqa_quantize(const peqa_layout *L, const float *W0, uint32_t *packed,
                          float *s0, uint8_t *z0, void *stream);

/*
 * Error-minimising initialisation.  Sec. 3.2 wants s0, z0 chosen so that the Frobenius norm of W0 - What0 is
 * smallest, and gives no procedure (the experiments use the plain range of Eq. 1); this is the usual grid
 * over clipped ranges.
 * For j = 0 .. n_ratios-1 with r_j = 1 - j * (1 - min_ratio) / (n_ratios - 1)  (r_0 = 1: Eq. 1 itself),
 * every (channel, group) is quantized with the range [r_j xmin, r_j xmax] exactly as in peqa_quantize,
 * and the candidate with the smallest sum_k (w - s (Q - z))^2 is kept (the first of equal ones).
 * Residuals are formed in fp32 and their squares summed in fp64.  n_ratios = 1 equals peqa_quantize.
 *   1 <= n_ratios <= 1024, 0 < min_ratio <= 1 (PEQA_ERR_PARAM otherwise);
 *   supported where a row block fits on chip: K <= 12288 and 384 G + 9 K <= 153600 (PEQA_ERR_SHAPE).
 *   Arguments as peqa_quantize.
 */
peqa_status peqa_quantize_search(const peqa_layout *L, const float *W0, int32_t n_ratios,
                                 float min_ratio, uint32_t *packed, float *s0, uint8_t *z0,
                                 void *stream);

/*
 * Eq. 2 forward:  Y[t,i] = sum_k X[t,k] * (s0+ds)[i,g(k)] * (Q[i,k] - z0[i,g(k)]).
 *   ds may be NULL (= 0).  X [T, K] bf16 in, Y [T, N] bf16 out, T >= 1.
 *   bf16 operands, fp32 accumulation.  T <= 16 takes the bandwidth-bound
 *   matrix-vector path of Sec. 3.1 ("Inference Latency").
 *   Per-channel layers and the T <= 16 path contract over the exact integer codes and
 *   apply scale and zero-point in fp32 afterwards; group-wise layers with T > 16 (and
 *   their dX) form every weight (s0+ds)(Q - z0) in fp32 and round it once to bf16 before
 *   the contraction.
 *   workspace: peqa_workspace_bytes(L, T, PEQA_OP_FWD) bytes, contents undefined on return.
 */
peqa_status peqa_linear_fwd(const peqa_layout *L, const uint32_t *packed, const float *s0,
                            const float *ds, const uint8_t *z0, const uint16_t *X, int32_t T,
                            uint16_t *Y, void *workspace, size_t workspace_bytes, void *stream);

/*
 * peqa_linear_fwd for callers that cannot allocate device memory and have no workspace to pass: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and the same
 * result bit for bit as peqa_linear_fwd; the scratch a forward needs (row sums of X, the group table, or the
 * partial sums of the T <= 16 path) lives in an array of PEQA_STATIC_SCRATCH_BYTES that is part of the library's
 * device image (every GPU the library runs on holds its own copy until the process ends).  The call allocates
 * nothing and frees nothing.  A forward that needs more scratch than that even with whole contractions or the fewest
 * slices (see Workspaces) is refused with PEQA_ERR_WORKSPACE before anything is enqueued; one that does not is planned
 * within it by both calls.
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two streams, two
 * threads) race on it; calls on one stream are ordered and safe.  Nothing in the array needs to start at zero.
 * The array's device address is looked up once per device, at the first call on that device (not a stream
 * operation: make that first call outside a capture).
 */
#define PEQA_STATIC_SCRATCH_BYTES (16u << 20)
peqa_status peqa_linear_fwd_static(const peqa_layout *L, const uint32_t *packed, const float *s0,
                                   const float *ds, const uint8_t *z0, const uint16_t *X, int32_t T,
                                   uint16_t *Y, void *stream);

/*
 * The same forward for 1..PEQA_MAX_FUSED layers that read the same X (the query / key / value
 * projections of an attention block; the gate and up projections of its MLP): equal to calling
 * peqa_linear_fwd once per item, every item writing its own Y.  All items must share k_in, bits
 * and group_size (PEQA_ERR_PARAM otherwise).  With T <= 16 (Sec. 3.1, "Inference Latency": bound by
 * the weight bytes streamed) the layers run side by side in one launch, which matters because
 * a single LLaMA-size layer at such T is too short to fill the machine; larger T runs them one
 * after the other.  `items` is a HOST array; workspace: peqa_workspace_bytes_fused() bytes.
 */
#define PEQA_MAX_FUSED 4
typedef struct {
    peqa_layout layout;
    const uint32_t *packed;
    const float *s0;
    const float *ds;     /* may be NULL */
    const uint8_t *z0;
    uint16_t *Y;         /* [T, layout.n_out] bf16 out */
} peqa_fwd_item;

size_t peqa_workspace_bytes_fused(int32_t n, const peqa_fwd_item *items, int32_t T);
peqa_status peqa_linear_fwd_fused(int32_t n, const peqa_fwd_item *items, const uint16_t *X, int32_t T,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * The linears of a decoder block behind one call (Sec. 3.1 motivates PEQA by the cost of the fully-connected
 * layers of a block: the query / key / value / output projections and the gate / up / down projections of
 * LLaMA; Eq. 2 is applied to each).  An item is one layer with its own input: peqa_block_fwd equals
 * peqa_linear_fwd per item, peqa_block_bwd equals peqa_linear_bwd per item, up to the order of floating-point
 * additions.  Items are independent of each other: no item's input may be another item's output of the same
 * call.  Layers that read one input are best passed stacked as one item (see Stacking); items may also
 * simply share an X pointer.  All items share T and the bit width (PEQA_ERR_PARAM otherwise); shapes and
 * group sizes may differ.
 *   T <= 16 (the deployment path of Sec. 3.1): every layer of the call runs in ONE launch, whose workgroups
 *     get equal shares of the packed bytes, plus one short launch that adds up the feature slices of the
 *     layers that were sliced.
 *   T > 16, per-channel layers: forward = the row sums of all distinct inputs in one launch, then all
 *     items' contractions in one launch of four-wave tiles, longest contraction first.  Backward = all scale-gradient
 *     contractions in one launch whose grid also carries the scaling of dY for every item, then all dX
 *     contractions in one launch whose grid also carries the fixed-order sums of the scale-gradient partials.
 *     Group-wise layers: forward = the scale tables of all items in one launch, then all contractions in one
 *     launch.  Backward of few tiles (8 per compute unit) or of at most 1536 tokens, both gradients = the tables and
 *     the transposed copies of X (once per distinct X) and dY in one launch, then all dX contractions and the token
 *     contractions of all scale gradients in one launch.  Otherwise, and where dX is a few long contractions that a
 *     launch of its own would cut up or that would outlast what is asked for beside it, and (more tiles) with less
 *     workspace than the query says = the tables, then all dX contractions in one launch whose grid also writes the
 *     copies, then the token contractions in one launch.  (Always the token-contraction route:
 *     PEQA_OPT_GROUPED_DDS = 1 only keeps the two in launches of their own.)
 *     Contractions of few tokens are cut into pieces, whose sums, like those of the chunks of groups past 128
 *     features, are added up by one launch more.
 *   row_sums (optional, [T, 2] fp32 per distinct X, caller-owned): when not NULL, peqa_block_fwd stores the row
 *     sums of the item's X there (see peqa_row_sums) and peqa_block_bwd reads them instead of taking them again;
 *     items that share X may share the array.  Ignored by T <= 16 and by group-wise layers.
 *   `items` is a HOST array of 1..PEQA_MAX_BLOCK entries; workspace: peqa_block_workspace_bytes(n, items, T, op)
 *   with op = PEQA_OP_FWD or PEQA_OP_BWD, contents undefined on return.  dX and d_ds may be NULL per item (skipped).
 */
#define PEQA_MAX_BLOCK 8
typedef struct {
    peqa_layout layout;
    const uint32_t *packed;
    const float *s0;
    const float *ds;       /* may be NULL */
    const uint8_t *z0;
    const uint16_t *X;     /* [T, layout.k_in] bf16, in (both calls; may be NULL in the backward when d_ds is) */
    uint16_t *Y;           /* [T, layout.n_out] bf16, out of peqa_block_fwd (unused by the backward)           */
    const uint16_t *dY;    /* [T, layout.n_out] bf16, in of peqa_block_bwd (unused by the forward)             */
    uint16_t *dX;          /* [T, layout.k_in] bf16, out of peqa_block_bwd, or NULL                            */
    float *d_ds;           /* [N, G] fp32, out of peqa_block_bwd (overwritten), or NULL                        */
    float *row_sums;       /* optional, see above                                                              */
} peqa_block_item;

size_t peqa_block_workspace_bytes(int32_t n, const peqa_block_item *items, int32_t T, int32_t op);
peqa_status peqa_block_fwd(int32_t n, const peqa_block_item *items, int32_t T, void *workspace,
                           size_t workspace_bytes, void *stream);
peqa_status peqa_block_bwd(int32_t n, const peqa_block_item *items, int32_t T, void *workspace,
                           size_t workspace_bytes, void *stream);

/*
 * Backward of Eq. 2 by the chain rule (only the scales are trained, Sec. 3.2):
 *   dX[t,k]   = sum_i dY[t,i] * (s0+ds)[i,g(k)] * (Q[i,k] - z0[i,g(k)])
 *   d_ds[i,g] = sum_t dY[t,i] * sum_{k in g} X[t,k] * (Q[i,k] - z0[i,g])
 *   dX [T, K] bf16 out, or NULL to skip; d_ds [N, G] fp32 out (overwritten, not
 *   accumulated), or NULL to skip.  X may be NULL when d_ds is NULL.
 *   The result is deterministic (fixed reduction order, no atomics): the same call gives the
 *   same bits.  A call that skips one gradient may run the other's contraction in another form of
 *   the kernel than a call that asks for both (see Options): the same products added in
 *   another order, so the two agree to the last bf16 bit of dX / 1e-5 of |d_ds|, not bit for bit.
 *   Group-wise layers take d_ds by the other order of the two sums,
 *   d_ds[i,g] = sum_{k in g} (sum_t dY[t,i] X[t,k]) (Q[i,k] - z0[i,g]); their backward workspace
 *   therefore also holds transposed copies of X and dY (2 (K + N) T' bytes, T' = T rounded up to 64).
 */
peqa_status peqa_linear_bwd(const peqa_layout *L, const uint32_t *packed, const float *s0,
                            const float *ds, const uint8_t *z0, const uint16_t *X,
                            const uint16_t *dY, int32_t T, uint16_t *dX, float *d_ds,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * Row sums shared between calls.  The per-channel contractions for T > 16 take the code offset and the
 * zero-point out of the contraction through the sums of every row of X over the two halves of K,
 *   row_sums[t] = ( sum_{k < ks} X[t,k],  sum_{k >= ks} X[t,k] ),   ks = (K / 2) rounded down to 64,
 * which peqa_linear_fwd(_fused) and peqa_linear_bwd otherwise take themselves at every call (a launch of
 * several microseconds each).  A training step can take them once per activation with peqa_row_sums
 * ([T, 2] fp32: 8 T bytes to keep until the backward) and hand them to the forward of the layers that read
 * that X and, later, to their backward.  row_sums = NULL makes these calls equal to the plain ones; calls
 * that do not use such sums (T <= 16, group-wise layers) ignore the argument.
 */
peqa_status peqa_row_sums(const uint16_t *X, int32_t T, int32_t K, float *row_sums, void *stream);
peqa_status peqa_linear_fwd_fused_rs(int32_t n, const peqa_fwd_item *items, const uint16_t *X,
                                     const float *row_sums, int32_t T, void *workspace,
                                     size_t workspace_bytes, void *stream);
peqa_status peqa_linear_bwd_rs(const peqa_layout *L, const uint32_t *packed, const float *s0,
                               const float *ds, const uint8_t *z0, const uint16_t *X,
                               const float *row_sums, const uint16_t *dY, int32_t T, uint16_t *dX,
                               float *d_ds, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Optional trade of activation memory for arithmetic, per-channel layers only (PEQA_ERR_GROUP for
 * group-wise ones).  In the scale gradient of Eq. 2,  d_ds[i] = sum_t dY[t,i] * P[t,i]  with
 *   P[t,i] = sum_k X[t,k] * (Q[i,k] - z0[i]),
 * and Y[t,i] = (s0+ds)[i] * P[t,i]: the forward already forms P.  peqa_linear_fwd_keep writes it
 * (fp32, [T, N], caller-owned: 4 T N bytes per layer, against the memory motive of Sec. 3.1) next to
 * the same Y as peqa_linear_fwd; peqa_linear_bwd_kept then takes d_ds from dY and P with one pass
 * over both instead of the contraction over X, so that forward + backward cost 4 T N K flops, not
 * 6 T N K.  dX, NULL arguments and determinism as in peqa_linear_bwd; P may be NULL when d_ds is.
 *   any T >= 1 (the forward always runs the tiled contraction);
 *   workspace: peqa_workspace_bytes(L, T, PEQA_OP_FWD_KEEP / PEQA_OP_BWD_KEPT).
 */
peqa_status peqa_linear_fwd_keep(const peqa_layout *L, const uint32_t *packed, const float *s0,
                                 const float *ds, const uint8_t *z0, const uint16_t *X, int32_t T,
                                 uint16_t *Y, float *P, void *workspace, size_t workspace_bytes,
                                 void *stream);
peqa_status peqa_linear_bwd_kept(const peqa_layout *L, const uint32_t *packed, const float *s0,
                                 const float *ds, const uint8_t *z0, const float *P,
                                 const uint16_t *dY, int32_t T, uint16_t *dX, float *d_ds,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Trainable zero-points (Appendix K, "Choice of Updating Quantization Scales or Zero-Points": zero-points
 * only, or zero-points and scales together).  The zero-point becomes the real number z = z0 + dz with
 * dz [N, G] fp32 (NULL = 0); the codes stay frozen and Eq. 2 reads What = (s0+ds) (Q - z).
 *   peqa_linear_fwd_z:  Y as peqa_linear_fwd with z in place of z0 (every T, per-channel and group-wise).
 *   peqa_linear_bwd_z:  dX and d_ds as peqa_linear_bwd with z in place of z0, and
 *     d_dz[i,g] = -(s0+ds)[i,g] * sum_t dY[t,i] * sum_{k in g} X[t,k]      [N, G] fp32 out, or NULL to skip
 *   (z enters What only through -s z).  X may be NULL when d_ds and d_dz both are.
 *   dz is updated with peqa_scale_update(n, dz, d_dz, m, v, s0, opt): with opt->weight_decay = 0 the
 *   s0 argument is read but has no effect (pass the scales).
 *   workspace: peqa_workspace_bytes(L, T, PEQA_OP_FWD_Z / PEQA_OP_BWD_Z).
 */
peqa_status peqa_linear_fwd_z(const peqa_layout *L, const uint32_t *packed, const float *s0,
                              const float *ds, const uint8_t *z0, const float *dz, const uint16_t *X,
                              int32_t T, uint16_t *Y, void *workspace, size_t workspace_bytes,
                              void *stream);
peqa_status peqa_linear_bwd_z(const peqa_layout *L, const uint32_t *packed, const float *s0,
                              const float *ds, const uint8_t *z0, const float *dz, const uint16_t *X,
                              const uint16_t *dY, int32_t T, uint16_t *dX, float *d_ds, float *d_dz,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * One AdamW step on ds (Appendix A names AdamW with a linearly decaying learning rate;
 * the schedule is the caller's, who passes the current lr).  step is 1-based.
 *   m <- b1 m + (1-b1) g;  v <- b2 v + (1-b2) g^2
 *   ds <- ds - lr * ( (m / (1-b1^step)) / (sqrt(v / (1-b2^step)) + eps) + wd * (s0 + ds) )
 * ds, m, v [n] fp32 in/out (m, v zero-initialised by the caller); d_ds, s0 [n] fp32 in.
 */
typedef struct {
    float lr, beta1, beta2, eps, weight_decay;
    int32_t step;
} peqa_adamw;

peqa_status peqa_scale_update(size_t n_scales, float *ds, const float *d_ds, float *m, float *v,
                              const float *s0, const peqa_adamw *opt, void *stream);

/*
 * The same step on the scales of 1..PEQA_MAX_UPDATE layers in one launch (a decoder block's seven
 * updates are each a few microseconds of work behind a launch): equal to calling peqa_scale_update
 * once per item with the same `opt`.  `items` is a HOST array.
 */
#define PEQA_MAX_UPDATE 16
typedef struct {
    size_t n_scales;
    float *ds;           /* in/out */
    const float *d_ds;
    float *m, *v;        /* in/out */
    const float *s0;
} peqa_update_item;

peqa_status peqa_scale_update_multi(int32_t n, const peqa_update_item *items, const peqa_adamw *opt,
                                    void *stream);

/*
 * Decoding over a paged key-value cache.  What a decoder layer does between the query, key and value projections and
 * the output projection when it answers one token at a time (Sec. 3.1's deployment): the new tokens' queries and keys are
 * rotated by their positions, their keys and values stored, and every new query attends over its sequence's cache.
 *
 * The cache is two pools of pages, one of keys and one of values.  A page holds page_size consecutive positions of one
 * sequence for all kv_heads heads; the page of positions [b page_size, (b+1) page_size) of sequence s is table[s][b].
 * Element d of head h at position p lies at
 *   page * page_stride + h * head_stride + (p % page_size) * slot_stride + d      (elements, in both pools)
 * so pools of any order of heads and slots, and pools that hold keys and values side by side, can be described.
 *   dtype PEQA_CACHE_BF16: bf16.  PEQA_CACHE_FP8: 8-bit floats with 4 exponent and 3 mantissa bits, no infinities, largest
 *   finite value 448 ("e4m3fn"); a stored value stands for itself times k_scale[h] or v_scale[h] (normal fp32 numbers,
 *   device; NULL = 1).
 *   k, v and the strides are multiples of 16 bytes (PEQA_ERR_ALIGN); page_size is a power of two, 8 .. 1024; head_dim is
 *   64, 128 or 256; page_size * slot_stride is under 2^30, n_blocks * page_size at most 2^30.  A table entry outside
 *   [0, n_pages) stands for a page that is not there: nothing is stored to it and its positions are not attended to.
 * The struct is a HOST descriptor, read during the call; the table and the pools are read when the work runs.
 */
typedef enum { PEQA_CACHE_BF16 = 0, PEQA_CACHE_FP8 = 1 } peqa_cache_dtype;
typedef struct {
    void *k, *v;                                      /* pools                                         */
    const int32_t *table;                             /* [n_seqs, n_blocks], rows table_stride apart   */
    const float *k_scale, *v_scale;                   /* [kv_heads] or NULL; PEQA_CACHE_FP8 only       */
    int64_t page_stride, head_stride, slot_stride;    /* in elements                                   */
    int64_t table_stride;                             /* in entries                                    */
    int32_t n_pages, page_size, kv_heads, head_dim;
    int32_t n_seqs, n_blocks;
    int32_t dtype;                                    /* peqa_cache_dtype                              */
    int32_t reserved;                                 /* 0 */
} peqa_kv_cache;

/* PEQA_OK, or what is wrong with the descriptor (host-only). */
peqa_status peqa_check_cache(const peqa_kv_cache *C);

/*
 * Rotates and stores T new tokens.  Token t is position pos[t] of sequence seq[t] (seq NULL: of sequence t).
 *   q_out[t, h] = R(pos[t]) q[t, h];   cache[seq[t], pos[t], h] = R(pos[t]) k[t, h],  v[t, h]
 * R turns pair i of the first `rot` elements of a head, (x[i], x[i + rot/2]), or (x[2i], x[2i+1]) where `interleaved`, by
 * the angle whose cosine and sine are cos_table[pos, i] and sin_table[pos, i] (fp32 [n_pos, rot/2]); the other elements
 * stay.  rot is a multiple of 16, at most head_dim; rot = 0 (tables NULL, n_pos not read): no rotation.
 *   q [T, heads, head_dim] bf16, rows q_stride elements apart, or NULL (with q_out): keys and values only
 *   k, v [T, kv_heads, head_dim] bf16, rows k_stride, v_stride apart;  q_out as q (may be q itself), rows q_out_stride apart
 *   pointers and row strides multiples of 16 bytes: the members of a stacked query/key/value output can be passed as they lie
 * The rotation is fp32 and rounds once to what is stored (nearest even; 8-bit: of x / scale, values past 448 become 448).
 * A token with pos < 0, pos >= n_pos (where rotated), seq outside [0, n_seqs), a position past the table or a page that
 * is not there is skipped: its row of q_out is zeros and nothing is stored.  The places of one call have to be different: of
 * tokens with the same sequence and position, every 16 elements are one of theirs, not all of them the same one's.
 */
peqa_status peqa_rope_append(const peqa_kv_cache *C, int32_t T, const int32_t *pos, const int32_t *seq,
                             const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                             int32_t interleaved, int32_t heads, const uint16_t *q, int64_t q_stride, const uint16_t *k,
                             int64_t k_stride, const uint16_t *v, int64_t v_stride, uint16_t *q_out,
                             int64_t q_out_stride, void *stream);

/*
 * peqa_rope_append for decoders that normalise the heads of queries and keys before the rotation, and for caches that positions have left
 * (peqa_cache_evict), where a token's place is not its position.  Of every head of q and k
 *   r = (mean_d x_d^2 + eps)^(-1/2),   y_d = r x_d w_d,
 * y is rotated by pos[t] and goes to q_out, or to place[t] of the sequence; v is stored as it is.
 *   place [T] int32, or NULL: pos;  q_weight, k_weight [head_dim] fp32 (16-byte aligned), each or NULL: ones;  eps > 0 (PEQA_ERR_PARAM)
 * Sums and rotation are fp32 and what is stored is rounded once.  A head whose sum of squares passes fp32's range is zeros.
 * Everything else as in peqa_rope_append: tokens with place < 0 or past the table are skipped too, and the places of a call are
 * different.
 */
peqa_status peqa_norm_rope_append(const peqa_kv_cache *C, int32_t T, const int32_t *pos, const int32_t *place, const int32_t *seq,
                                  const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot, int32_t interleaved,
                                  const float *q_weight, const float *k_weight, float eps, int32_t heads, const uint16_t *q,
                                  int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                                  uint16_t *q_out, int64_t q_out_stride, void *stream);

/*
 * The same norms and rotation without a cache, for training, and their gradients.
 *   y = R(pos[t]) (r x w);   with g = R^T dy, z = r x, u = g w:   dx = r (u - z mean_d(u z)),   dw_d = sum over tokens and heads of g_d z_d
 *   q, q_out, d_q_out, dq [T, heads, head_dim], k, k_out, d_k_out, dk [T, kv_heads, head_dim] bf16, rows strides apart (multiples of 8,
 *   pointers 16-byte aligned: members of a stacked query/key/value output, and of its gradient, can be passed as they lie)
 *   head_dim 64, 128 or 256;  q_out may be q itself, dq d_q_out itself (with the same stride), k likewise
 *   d_q_weight, d_k_weight [head_dim] fp32 out (overwritten), each or NULL (PEQA's training leaves norms as they are: with both NULL no
 *   workspace is needed)
 *   workspace: peqa_norm_rope_bwd_workspace_bytes(T, heads, kv_heads, head_dim).
 * A token with pos < 0, or pos >= n_pos (where rotated), has zeros for outputs and gradients and no part in dw.  Sums are fp32 in a fixed
 * order: the same call gives the same bits.
 */
peqa_status peqa_norm_rope(int32_t T, const int32_t *pos, const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                           int32_t interleaved, const float *q_weight, const float *k_weight, float eps, int32_t head_dim, int32_t heads,
                           int32_t kv_heads, const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, uint16_t *q_out,
                           int64_t q_out_stride, uint16_t *k_out, int64_t k_out_stride, void *stream);
size_t peqa_norm_rope_bwd_workspace_bytes(int32_t T, int32_t heads, int32_t kv_heads, int32_t head_dim);
peqa_status peqa_norm_rope_bwd(int32_t T, const int32_t *pos, const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                               int32_t interleaved, const float *q_weight, const float *k_weight, float eps, int32_t head_dim, int32_t heads,
                               int32_t kv_heads, const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride,
                               const uint16_t *d_q_out, int64_t d_q_out_stride, const uint16_t *d_k_out, int64_t d_k_out_stride,
                               uint16_t *dq, int64_t dq_stride, uint16_t *dk, int64_t dk_stride, float *d_q_weight, float *d_k_weight,
                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention of one query token per row over its sequence's cache: for row r (sequence seq[r]; NULL: r), head h and
 * its key head h / (heads / kv_heads), over the positions j in [max(0, len - window), len), len = lens[r] (window 0: all)
 *   x_j = scale * <q[r,h], k_j>;   out[r,h] = sum_j exp(x_j) v_j / sum_j exp(x_j);   lse[r,h] = log sum_j exp(x_j)
 * A row with no position (len <= 0, seq outside [0, n_seqs), no page there) gives zeros and lse = -inf.  Positions outside
 * the range may hold anything, NaN included.  Several new tokens of one sequence are rows with the same seq.
 *   q, out [rows, heads, head_dim] bf16, rows q_stride, out_stride elements apart (multiples of 8, pointers 16-byte aligned)
 *   lens [rows] int32;  lse [rows, heads] fp32 or NULL
 *   max_len: the host's bound of lens, at most n_blocks * page_size (PEQA_ERR_SHAPE); longer rows are cut to it.  The work
 *            is split for it, so a tight bound is faster.  heads: a multiple of kv_heads.
 *   workspace: peqa_paged_attention_workspace_bytes(C, rows, heads, max_len, window).
 * Products and sums are fp32.  The softmax weights are rounded for the matrix instructions: against bf16 values in two bf16 parts (16
 * bits), against 8-bit values in two fp16 parts (22 bits) where up to eight heads share a key head, else to fp16 (11 bits; of weights
 * under 2^-28 of the row's largest to 2^-39 of it).
 * The same call gives the same bits; the order in which a row's positions are added depends on max_len, window, the number of rows and,
 * with many long rows, their lengths.
 */
size_t peqa_paged_attention_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len,
                                            int32_t window);
peqa_status peqa_paged_attention(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                 const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t window, float scale,
                                 uint16_t *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes,
                                 void *stream);

/*
 * peqa_paged_attention for rows whose sequences begin with the same positions (samples of one prompt, questions about one document, a system
 * prompt): the first `shared` positions of every row are those of sequence `prefix`, which are read once for all rows; those behind
 * them are the row's own sequence's.  With K_r = positions [0, shared) of sequence `prefix`, then [shared, lens[r]) of sequence seq[r]
 * (NULL: r), out and lse are those of peqa_paged_attention over K_r; a row with lens[r] < shared sees the first lens[r] of the
 * shared positions, and reads them by itself (slow where they are many: it is divided as the rows' own positions are).  The table's entries of a row's blocks before position `shared` are not used: a page in which the
 * shared positions end is there twice, in `prefix` and, with the row's own positions behind, in the row's.
 *   max_len: the host's bound of lens, shared positions included;  shared, max_len at most n_blocks * page_size (PEQA_ERR_SHAPE)
 *   prefix: 0 .. n_seqs - 1;  the other arguments as in peqa_paged_attention
 *   workspace: peqa_shared_attention_workspace_bytes(C, rows, heads, max_len, shared).
 * Products and sums are fp32; weights are rounded to two bf16 parts (16 bits) against bf16 values, to fp16 (11 bits; of weights under 2^-20
 * of the row's largest to 2^-31 of it) against 8-bit ones.  The same call gives the same bits.
 */
size_t peqa_shared_attention_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t shared);
peqa_status peqa_shared_attention(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                  const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t prefix, int32_t shared,
                                  float scale, uint16_t *out, int64_t out_stride, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream);

/*
 * peqa_paged_attention that also says what every position was given, for caches that are cut to what is looked at (peqa_cache_evict): for every
 * row r, its sequence s, key head h and position j < lens[r]
 *   weights_out[s, h, j] = weights[s, h, j] + sum over the sequence's rows and the heads i of h of exp(x_j - lse[r, i])
 * (0 of positions outside the window and of pages that are not there; nothing else of weights_out is written).  out and lse are
 * peqa_paged_attention's, bit for bit.
 *   weights [n_seqs, kv_heads, max_len or more] fp32, sequences and heads strides apart (multiples of 4; 16-byte aligned; either of them the outer
 *   one, and max_len of one never over those of another: PEQA_ERR_SHAPE), or NULL: zeros;  weights_out the same, may be weights itself
 *   workspace: peqa_paged_attention_weights_workspace_bytes(C, rows, heads, max_len, window): 4 bytes a row, head and position beside
 *   the attention's own.  A long prompt, whose rows are one sequence's, is best passed in calls of 256 rows or so that add to the same weights: all
 *   at once its scores take 538 MB for 2048 tokens of 32 heads, in blocks 67 MB and no more time.
 * Sums are fp32 in a fixed order: rows of one sequence after one another.  A weight is found from the row's maximum and sum, not from lse.
 */
size_t peqa_paged_attention_weights_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len,
                                                    int32_t window);
peqa_status peqa_paged_attention_weights(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                         const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t window, float scale,
                                         uint16_t *out, int64_t out_stride, float *lse, const float *weights, float *weights_out,
                                         int64_t weights_seq_stride, int64_t weights_head_stride, void *workspace,
                                         size_t workspace_bytes, void *stream);

/*
 * Eviction.  Of each of n sequences (entry i: sequence seq[i], lens[i] positions long; seq NULL: sequence i) and each key head by itself: where
 * there are more than `keep` positions, the first `sinks`, the last `recent` and, of those between, the keep - sinks - recent with the
 * largest weights stay (equal ones: the lowest positions; NaN is less than everything), in order, at places 0 .. keep - 1: keys, values and
 * weights.  Every head then has its own positions at a sequence's places, so that a token's place is no longer its position: the tokens that follow are
 * stored by peqa_norm_rope_append, which takes both.  (peqa_rope_append does not: a decoder without head norms cannot go on behind an eviction, unless
 * nothing is rotated and `pos` is the place.)  Shorter sequences keep everything.
 *   to: the cache that keys and values go to, at the same sequences' places: of as many sequences, the same heads, head_dim, dtype and scales,
 *   any page size; its pages of these places are none that C's sequences have.  NULL, or one with C's own pools and table: in place.  In
 *   place a sequence's pages are its own: what another sequence shares with it would change.
 *   lens [n] int32, cut to max_len (as in the attention);  1 <= keep,  0 <= sinks, recent,  sinks + recent <= keep (PEQA_ERR_PARAM)
 *   weights, weights_out as in peqa_paged_attention_weights; places behind what stays, up to max_len, become 0 (those of
 *   a sequence without positions are left as they are)
 *   kept [n, kv_heads, keep] int32 out or NULL: the position that each place's was, -1 behind what stays
 *   new_lens [n] int32 out or NULL: min(lens[i], keep); not lens itself, nor in part (the layers of a model have the same lens)
 * A sequence outside [0, n_seqs) has none; one that an earlier entry has is left out (kept -1, that entry's length).  What lies on a page that is
 * not there arrives as zeros; nothing is stored to one.  Weights are compared as they are: every choice is exact.
 *   workspace: peqa_cache_evict_workspace_bytes(C, n, max_len, keep).
 */
size_t peqa_cache_evict_workspace_bytes(const peqa_kv_cache *C, int32_t n, int32_t max_len, int32_t keep);
peqa_status peqa_cache_evict(const peqa_kv_cache *C, const peqa_kv_cache *to, int32_t n, const int32_t *seq, const int32_t *lens,
                             int32_t max_len, const float *weights, float *weights_out, int64_t weights_seq_stride,
                             int64_t weights_head_stride, int32_t keep, int32_t sinks, int32_t recent, int32_t *kept,
                             int32_t *new_lens, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Log probabilities.  Of every row x = logits[t, 0 .. vocab-1] (bf16 or fp32, rows `stride` elements apart), in fp32:
 *   lse[t] = log sum_j exp(x_j);  logp[t] = x[targets[t]] - lse[t];  entropy[t] = -sum_j p_j log p_j,  p_j = exp(x_j - lse[t])
 *   top_ids[t, i], top_logp[t, i], i < top: the `top` largest x_j in falling order (equal ones: the lowest index first) and
 *   their log probabilities
 * A target outside [0, vocab) is ignored: logp = 0.  Words may be masked with -inf or the type's lowest value; a row of -inf
 * only has lse = logp = top_logp = -inf and entropy 0.  A row with a NaN, or with +inf, gives NaN for all but the ids.
 *   logits: rows at any element (16-byte aligned rows are faster), stride >= vocab;  targets [T] int32 or NULL (with logp NULL)
 *   logp, entropy, lse [T] fp32, each or NULL;  top 0 .. PEQA_MAX_TOP, at most vocab;  top_logp, top_ids [T, top] (NULL if top = 0)
 *   workspace: peqa_token_logprobs_workspace_bytes(T, vocab, top).
 */
#define PEQA_MAX_TOP 32
typedef enum { PEQA_LOGITS_BF16 = 0, PEQA_LOGITS_F32 = 1 } peqa_logits_dtype;
size_t peqa_token_logprobs_workspace_bytes(int32_t T, int32_t vocab, int32_t top);
peqa_status peqa_token_logprobs(const void *logits, int32_t dtype, int32_t T, int32_t vocab, int64_t stride,
                                const int32_t *targets, int32_t top, float *logp, float *entropy, float *lse,
                                float *top_logp, int32_t *top_ids, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The gradient of sum_t d_logp[t] logp[t] + d_entropy[t] entropy[t] with respect to the logits, in the logits' type:
 *   d_logits[t, j] = d_logp[t] ([j = targets[t]] - p_j) - d_entropy[t] p_j (log p_j + entropy[t]),   p_j = exp(x_j - lse[t])
 * (an ignored target: without the first term; p_j = 0 has no second).  The mean cross entropy of n tokens is d_logp = -1/n.
 *   lse, and entropy where d_entropy is given, as peqa_token_logprobs left them;  d_logp or d_entropy may be NULL (= 0)
 *   d_logits: rows d_stride elements apart, may be logits itself with the same stride; only the first `vocab` elements of
 *   a row are written.  Rows whose two factors are 0 (logits not read), or whose lse is -inf, are zeros.
 * An fp32 lse is rounded, to 2^-24 of itself: p_j is off by 2^-17 of itself at most for |lse| < 256.  Of rows whose lse is larger, those of
 * the type's lowest value only among them, the rest is found from the row first (they take two to three times as long), unless lse differs
 * from the row's own by more than 2^-22 of itself: it is then taken to be of more words than these, and used as it is.
 */
peqa_status peqa_token_logprobs_bwd(const void *logits, int32_t dtype, int32_t T, int32_t vocab, int64_t stride,
                                    const int32_t *targets, const float *lse, const float *entropy, const float *d_logp,
                                    const float *d_entropy, void *d_logits, int64_t d_stride, void *stream);

/* Compute units and peak engine clock (kHz) of the current device, as the HIP runtime reports them
 * (for benchmark reports: the denominators of roofline fractions). */
peqa_status peqa_device_info(int32_t *compute_units, int32_t *clock_khz);

/*
 * Per-kernel timing for benchmarks.  peqa_trace_begin() makes every kernel the library
 * launches afterwards be bracketed by HIP events on its stream (it creates the events:
 * call it outside any region that must not allocate).  peqa_trace_end() synchronises those
 * events, stops tracing and fills, for up to `max_kernels` distinct kernels, a name
 * (static string), the number of launches and the summed duration in milliseconds;
 * it returns the number of distinct kernels seen.  Not thread-safe.
 */
peqa_status peqa_trace_begin(int32_t max_launches);
/* Restricts tracing to the kernels whose reported name starts with `prefix` (NULL or "": all kernels, the
 * default).  Bracketing only the kernel of interest leaves the other launches of a timed region back to back,
 * as they are without tracing.  Names are at most 31 characters (PEQA_ERR_PARAM otherwise). */
peqa_status peqa_trace_select(const char *prefix);
int32_t peqa_trace_end(int32_t max_kernels, const char **names, int32_t *launches, float *total_ms);

#ifdef __cplusplus
}
#endif
#endif /* PEQA_H */
