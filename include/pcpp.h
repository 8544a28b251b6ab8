/*
 * pcpp -- convolution on native points (PointCNN++) as MVMR, MI355X (gfx950) only.
 *
 * C ABI of libpcpp.so.  Plain pointers and sizes; every pointer is a DEVICE pointer unless the
 * comment says HOST.  The caller owns every buffer (inputs, outputs, plan, workspace).  The calls
 * below allocate no device or host memory and keep no data between calls; the only thing the
 * library remembers is, per kernel and device, that it has raised that kernel's dynamic LDS limit
 * (an idempotent attribute of the loaded code).  pcpp_build_triplets creates one event and destroys
 * it before it returns.
 *
 * Notation (paper -> here): output index i -> o, input index j -> i, kernel cell k;
 * t = kernel resolution per axis, K = t^3; T = the triplet set {(o, i, k)}.
 *
 * Conventions shared by all calls
 *   - return value: PCPP_OK or a negative PCPP_ERR_* code; pcpp_last_error() gives a message for
 *     the calling thread.  Nothing is printed, nothing throws.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Calls are asynchronous on it, except
 *     pcpp_build_triplets, which waits once for the triplet count.
 *   - outputs are overwritten, never accumulated into; rows without a triplet are zero.
 *   - indices are int32 (n_in, n_out, |T| < 2^31), segment offsets int64, coordinates fp32.
 *   - feature tensors are row-major, 16-byte aligned; dtype codes below.
 *   - feature tensors (x, dy, w) must hold finite values.  The matrix-core kernels form the sum of the
 *     source rows of a (cell, output) run as a product with a 0/1 selection matrix or stage it beside other
 *     rows, so an Inf or NaN in one source row can reach destination rows that have no triplet with it
 *     (within the same group of up to 128 consecutive centres).  Coordinates must be finite too.
 */
#ifndef PCPP_H_
#define PCPP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define PCPP_API __attribute__((visibility("default")))
#else
#define PCPP_API
#endif

#define PCPP_OK                 0
#define PCPP_ERR_INVALID_ARG   -1  /* null pointer, negative size, t < 1, bad radius, misaligned    */
#define PCPP_ERR_CAPACITY      -2  /* triplet buffers too small; *n_triplets holds the needed count */
#define PCPP_ERR_WORKSPACE     -3  /* workspace or plan buffer smaller than the matching *_bytes()  */
#define PCPP_ERR_UNSUPPORTED   -4  /* dtype / shape outside what the library handles                */
#define PCPP_ERR_HIP           -5  /* a HIP runtime call failed, or a device-side wait ran out      */

#define PCPP_F32   0   /* IEEE binary32                    */
#define PCPP_BF16  1   /* bfloat16, round-to-nearest-even  */

/* plan_flags: which parts of a plan pcpp_build_triplets writes, and how.  The same value must be passed
 * to every compute call that reads the plan. */
#define PCPP_PLAN_FWD        1   /* what pcpp_mvmr_fwd and pcpp_mvmr_bwd_weight read */
#define PCPP_PLAN_BWD_INPUT  2   /* what pcpp_mvmr_bwd_input reads (only together with PCPP_PLAN_FWD) */
#define PCPP_PLAN_SPATIAL    4   /* the plan groups the centres along a space-filling curve computed by the
                                    library instead of in index order: the centres a kernel block owns are then
                                    neighbours in space whatever the caller's point order, which wide layers need
                                    (they share source rows and weight slices through the caches).  The public
                                    triplet arrays, every result and every tolerance are unchanged; the build
                                    takes about twice as long. */
/* testing aids, accepted in plan_flags by pcpp_build_triplets only; results are identical with or without */
#define PCPP_BUILD_TEST_SHORT_LISTS  0x100  /* order at most 40 neighbours at a time on chip: tiles in many parts, and
                                               centres with more are ranked by scanning the candidates again */
#define PCPP_BUILD_TEST_WIDE_KEYS    0x200  /* treat cell and index as too wide to share one 32-bit word, as for
                                               clouds of 2^24 points or more                                  */

#define PCPP_BUILD_VOXEL             0x400  /* accepted in plan_flags by pcpp_build_triplets[_batched]: build the triplets
                                               of the degraded operator of Sec. 3.2 ("Voxel Convolution as a Special
                                               Case"; "Ours (degraded)" in Sec. 4.2), i.e. sparse voxel convolution:
                                               `radius` is then the pitch v of a global voxelisation, t must be odd,
                                               voxel of a coordinate = floor((double)p / (double)v); input i is a
                                               neighbour of output o iff their voxels differ by at most h = (t-1)/2
                                               along every axis, and k = ((dx+h)*t + dy+h)*t + dz+h with (dx, dy, dz) the
                                               voxel offset input minus output.  Everything else (order of T, plan,
                                               compute calls) is unchanged. */

#define PCPP_MAX_T  6            /* K = t^3 <= 216 */

/* Message for the last error returned on the calling thread (never NULL). HOST. */
PCPP_API const char *pcpp_last_error(void);

/* Library version, major*100 + minor. */
PCPP_API int pcpp_version(void);

/* ---------------------------------------------------------------------------------------------
 * Triplet construction: Sec. 3.2 "Definition" with the fixed radius search of Sec. 4.1, followed
 * by the reordering of Sec. 3.3.2 (sort by kernel cell; here by (k, o, i)).
 *
 * (o, i, k) is in T iff |in_xyz[i] - out_xyz[o]|^2 <= r^2, the test being evaluated in binary64
 * on the binary32 coordinates as (dx*dx + dy*dy) + dz*dz <= (double)r*(double)r without fused
 * multiply-add.  k is the cell of d = in - out in the t x t x t grid tiling [-r, r]^3 around the
 * output point: c_a = clamp(floor((d_a + r) * (t / (2r))), 0, t-1), k = (c_x*t + c_y)*t + c_z.
 *
 * Outputs
 *   tri_o, tri_i, tri_k  [capacity] int32: T in ascending (k, o, i) order.  All three NULL =>
 *                        count only (capacity, seg_offsets and plan are ignored).
 *   seg_offsets          [K+1] int64: start of each cell's run; seg_offsets[K] = |T|.
 *   n_triplets           HOST int64: |T|, also set when PCPP_ERR_CAPACITY is returned.  If it points into
 *                        pinned host memory (hipHostMalloc) the device writes the count straight into it
 *                        and the second pass is queued without waiting for the host; with pageable memory
 *                        the call copies the count synchronously first (same results, the GPU idles for one
 *                        round trip).
 *   plan                 optional opaque buffer of pcpp_plan_bytes(...) bytes that the three
 *                        compute calls need: per-(cell, centre) neighbour runs and tile offsets
 *                        for the forward / weight-gradient pass (PCPP_PLAN_FWD) and the same
 *                        triplets regrouped by (k, i, o) for the input gradient
 *                        (PCPP_PLAN_BWD_INPUT).  plan_flags selects the parts; NULL => none.
 *   workspace            scratch of pcpp_build_triplets_workspace_bytes(...) bytes, 256-byte
 *                        aligned; contents are undefined afterwards.  With
 *                        pcpp_build_triplets_workspace_bytes_for(..., capacity) bytes every centre's
 *                        neighbours are searched once and kept, and all later passes read those lists.
 *                        That takes, per side, lists of 4 bytes times twice the mean of the capacity's
 *                        triplets per centre (128 bytes to 2 KB a centre; 2 KB from a mean of 128 on) and
 *                        room for longer ones, 4.5 bytes per triplet of the capacity; clouds of up to 8192
 *                        points and 2^23 pairs, which are searched without a grid, 4 bytes per pair.  So a
 *                        generous capacity costs memory.  With less room the lists are shorter; in the
 *                        smallest workspace a call either finds room for them among its tables or searches
 *                        again in each pass (same results).
 * in_xyz [n_in,3] and out_xyz [n_out,3] may alias (outputs at the inputs).
 * Errors: INVALID_ARG (null xyz with n > 0, radius not finite or <= 0, t outside 1..PCPP_MAX_T,
 * some but not all tri_* NULL, unknown flag bits), CAPACITY, WORKSPACE, UNSUPPORTED (|T| >= 2^31), HIP.
 * Non-finite coordinates are not supported (undefined triplets, no fault).
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_build_triplets_workspace_bytes(int64_t n_in, int64_t n_out, int t);
PCPP_API size_t pcpp_build_triplets_workspace_bytes_for(int64_t n_in, int64_t n_out, int t, int64_t capacity);
PCPP_API size_t pcpp_plan_bytes(int64_t n_in, int64_t n_out, int t, int64_t n_triplets, int plan_flags);

PCPP_API int pcpp_build_triplets(const float *in_xyz, int64_t n_in,
                                 const float *out_xyz, int64_t n_out,
                                 float radius, int t,
                                 int32_t *tri_o, int32_t *tri_i, int32_t *tri_k, int64_t capacity,
                                 int64_t *seg_offsets,
                                 int64_t *n_triplets,
                                 void *plan, size_t plan_bytes, int plan_flags,
                                 void *workspace, size_t workspace_bytes,
                                 void *stream);

/* ---------------------------------------------------------------------------------------------
 * Triplet construction over a batch of clouds held as concatenated arrays plus offsets (the jagged batch
 * representation of Sec. 4.1, implementation details): cloud b owns inputs [in_batch_offsets[b],
 * in_batch_offsets[b+1]) and outputs [out_batch_offsets[b], out_batch_offsets[b+1]); a triplet pairs points of the same
 * cloud only, whatever their coordinates.  Both offset arrays are DEVICE int32 [n_batches + 1], ascending, first
 * entry 0, last entry n_in / n_out; both NULL (with n_batches = 1) is pcpp_build_triplets.  Triplet indices refer to
 * the concatenated arrays, so the compute calls take the whole batch as one cloud.  1 <= n_batches <= 65536.
 * Everything else as pcpp_build_triplets.
 * ------------------------------------------------------------------------------------------- */
PCPP_API int pcpp_build_triplets_batched(const float *in_xyz, int64_t n_in,
                                         const float *out_xyz, int64_t n_out,
                                         const int32_t *in_batch_offsets, const int32_t *out_batch_offsets,
                                         int n_batches,
                                         float radius, int t,
                                         int32_t *tri_o, int32_t *tri_i, int32_t *tri_k, int64_t capacity,
                                         int64_t *seg_offsets,
                                         int64_t *n_triplets,
                                         void *plan, size_t plan_bytes, int plan_flags,
                                         void *workspace, size_t workspace_bytes,
                                         void *stream);

/* ---------------------------------------------------------------------------------------------
 * Voxel-grid down-sampling that keeps original coordinates (Sec. 4.1, implementation details): the output points
 * of a strided layer.  For every occupied voxel of pitch `pitch` (voxel of a coordinate = floor((double)p /
 * (double)pitch)) the point with the lowest index is kept.
 *   kept    [n] int32 (room for all points): indices of the kept points, ascending
 *   n_kept  HOST int64: their number (pinned host memory is written by the device, as in pcpp_build_triplets)
 *   workspace: pcpp_voxel_subsample_workspace_bytes(n) bytes, 256-byte aligned
 * The call waits for its result.  A strided layer is then pcpp_build_triplets with out_xyz = the kept points'
 * coordinates; the up-sampling layer of a decoder is the same call with the roles of the two point sets swapped
 * (more outputs than inputs is an ordinary case).
 * Errors: INVALID_ARG, WORKSPACE, UNSUPPORTED (n >= 2^31), HIP.  Coordinates beyond 2^20 voxels from the origin fall
 * into the outermost voxel.
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_voxel_subsample_workspace_bytes(int64_t n);
PCPP_API int pcpp_voxel_subsample(const float *xyz, int64_t n, float pitch, int32_t *kept, int64_t *n_kept,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * MVMR forward, Eq. (1) of Sec. 3.1.1:  out[o, :] = sum_{(o,i,k) in T} W[k] x[i, :].
 *   x   [n_in , c_in ]  in_dtype        w  [K, c_out, c_in] in_dtype (the paper's layout, Sec. 3.3.2)
 *   out [n_out, c_out]  out_dtype (PCPP_F32, or PCPP_BF16 when in_dtype is PCPP_BF16)
 * Products are accumulated in fp32.  tri_* / seg_offsets / plan must be exactly what one
 * pcpp_build_triplets call produced for these n_in, n_out, K with these plan_flags (which must include
 * PCPP_PLAN_FWD); anything else is undefined behaviour.  plan_bytes is the size of the plan buffer.
 * workspace: pcpp_mvmr_workspace_bytes(...) bytes, 256-byte aligned.
 * Errors: INVALID_ARG (also: plan_flags lack the part this call reads), WORKSPACE (also: plan_bytes smaller
 * than pcpp_plan_bytes for these sizes and flags), UNSUPPORTED (c_in or c_out < 1 or > 1024, dtype combination).
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_mvmr_workspace_bytes(int op /*0 fwd, 1 bwd_input, 2 bwd_weight*/, int64_t n_in, int64_t n_out,
                                          int64_t n_triplets, int c_in, int c_out, int K, int in_dtype);

PCPP_API int pcpp_mvmr_fwd(const void *x, const void *w, void *out, int in_dtype, int out_dtype,
                           int64_t n_in, int64_t n_out, int c_in, int c_out, int K,
                           const int32_t *tri_o, const int32_t *tri_i, const int32_t *tri_k,
                           const int64_t *seg_offsets, int64_t n_triplets,
                           const void *plan, size_t plan_bytes, int plan_flags,
                           void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * MVMR backward w.r.t. the input features, first gradient equation of Sec. 3.3.3:
 *   dx[i, :] = sum_{(o,i,k) in T} W[k]^T dy[o, :].
 *   dy [n_out, c_out] in_dtype,  w [K, c_out, c_in] in_dtype,  dx [n_in, c_in] out_dtype.
 * Needs a plan built with PCPP_PLAN_BWD_INPUT.  Otherwise as pcpp_mvmr_fwd.
 * ------------------------------------------------------------------------------------------- */
PCPP_API int pcpp_mvmr_bwd_input(const void *dy, const void *w, void *dx, int in_dtype, int out_dtype,
                                 int64_t n_in, int64_t n_out, int c_in, int c_out, int K,
                                 const int32_t *tri_o, const int32_t *tri_i, const int32_t *tri_k,
                                 const int64_t *seg_offsets, int64_t n_triplets,
                                 const void *plan, size_t plan_bytes, int plan_flags,
                                 void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Backward w.r.t. the weights (VVOR), Eq. (5) of Sec. 3.3.3:
 *   dw[k] = sum_{(o,i,k) in T} dy[o, :] (outer) x[i, :],   dw [K, c_out, c_in] always fp32.
 * Cells with no triplet get exact zeros.  Needs a plan built with PCPP_PLAN_FWD.
 * ------------------------------------------------------------------------------------------- */
PCPP_API int pcpp_mvmr_bwd_weight(const void *x, const void *dy, float *dw, int in_dtype,
                                  int64_t n_in, int64_t n_out, int c_in, int c_out, int K,
                                  const int32_t *tri_o, const int32_t *tri_i, const int32_t *tri_k,
                                  const int64_t *seg_offsets, int64_t n_triplets,
                                  const void *plan, size_t plan_bytes, int plan_flags,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * pcpp_mvmr_fwd for callers that cannot provide scratch memory or let the library allocate it: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same operation, same arguments
 * and same results as pcpp_mvmr_fwd without the workspace: the packed weights go to a device array that is part
 * of the loaded library, one copy per GPU (48 MiB), held until the process ends.  The call allocates nothing and
 * creates nothing.
 * Limits: K * c_out * c_in * (2 bytes for bf16, 6 for fp32) must not exceed pcpp_static_scratch_bytes() (24 MiB; the
 * array is larger because weights are padded in it), otherwise UNSUPPORTED is returned and nothing is launched.  Every call on a GPU uses that GPU's one array, so two calls that overlap
 * in time on one GPU (different streams or threads) race; calls on one stream are ordered and safe.
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_static_scratch_bytes(void);
PCPP_API int pcpp_mvmr_fwd_static(const void *x, const void *w, void *out, int in_dtype, int out_dtype,
                                  int64_t n_in, int64_t n_out, int c_in, int c_out, int K,
                                  const int32_t *tri_o, const int32_t *tri_i, const int32_t *tri_k,
                                  const int64_t *seg_offsets, int64_t n_triplets,
                                  const void *plan, size_t plan_bytes, int plan_flags, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Choice of the processing order by measurement.  Sec. 3.3.2 ends with the remark that for configurations outside
 * its analysis the order in which the triplets are processed can be selected by auto-tuning before the massive
 * executions.  Here the public arrays are always in (k, o, i) order; what can differ is which centres share a tile
 * of the plan: index order, or positions along a Z-order curve (PCPP_PLAN_SPATIAL).  The call builds both plans for
 * this cloud, times pcpp_mvmr_fwd (and pcpp_mvmr_bwd_input when ops holds PCPP_PLAN_BWD_INPUT) on zero-filled
 * features of this layer shape, three passes each after a warm-up, and reports
 *   best_plan_flags  HOST int: ops, with PCPP_PLAN_SPATIAL added when that order was faster
 *   ms_index_order, ms_spatial_order  HOST float, optional: the time of one pass in either order
 * n_triplets must be |T| of this cloud (from a counting call of pcpp_build_triplets); build_flags is 0 or
 * PCPP_BUILD_VOXEL; ops is PCPP_PLAN_FWD or PCPP_PLAN_FWD | PCPP_PLAN_BWD_INPUT.  workspace:
 * pcpp_tune_workspace_bytes(...) bytes (device, 256-byte aligned; room for the triplets, the larger plan, the build's
 * workspace and the layer's tensors).  The call waits for its result and creates two events for the timing; it is
 * meant to run once per layer configuration, not per step.
 * Errors: INVALID_ARG, WORKSPACE, and whatever the calls it makes return.
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_tune_workspace_bytes(int64_t n_in, int64_t n_out, int t, int64_t n_triplets, int c_in, int c_out,
                                          int in_dtype, int ops);
PCPP_API int pcpp_tune_plan_order(const float *in_xyz, int64_t n_in, const float *out_xyz, int64_t n_out, float radius,
                                  int t, int build_flags, int64_t n_triplets, int c_in, int c_out, int in_dtype, int ops,
                                  void *workspace, size_t workspace_bytes, int *best_plan_flags, float *ms_index_order,
                                  float *ms_spatial_order, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Activations in 8 bits, for a backward pass that needs them later.  A row of c channels becomes
 *   q      [n, c] int8
 *   codes  [n, pcpp_act_code_bytes(c)] uint8: one code for 32 channels of the row, in order; the rest of the row's
 *          whole 32-bit words is zero
 * and stands for the values q * 2^(code - 127).  code is the smallest with which no channel of the 32 rounds past
 * +-127, at least 1 and at most 248; q is the channel over that power of two, rounded to nearest even, and +-127 where it
 * would pass that (finite magnitudes from 127.5 * 2^121 = 3.39e38 on).  The values are bf16 numbers exactly.  Code 255 (q = 0) marks channels of which one is Inf or NaN: they are read as NaN.
 *   x  [n, c] dtype (PCPP_F32 or PCPP_BF16), row-major, 16-byte aligned, as is q; codes 4-byte aligned.
 * Errors: INVALID_ARG, UNSUPPORTED (c outside 1..1024, n >= 2^31, dtype).
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_act_code_bytes(int c);      /* per row: 4 * ceil(c / 128); 0 if c is outside 1..1024 */
PCPP_API int pcpp_act_pack(const void *x, int dtype, int64_t n, int c, int8_t *q, uint8_t *codes, void *stream);
PCPP_API int pcpp_act_unpack(const int8_t *q, const uint8_t *codes, int64_t n, int c, void *x, int dtype, void *stream);

/* ---------------------------------------------------------------------------------------------
 * pcpp_mvmr_bwd_weight with the layer's input kept in 8 bits (pcpp_act_pack):
 *   dw[k] = sum_{(o,i,k) in T} dy[o, :] (outer) values(xq, xcodes)[i, :],   dw [K, c_out, c_in] always fp32.
 *   dy [n_out, c_out] dy_dtype.  The 8-bit values enter the products as they are, dy as in pcpp_mvmr_bwd_weight.
 * tri_* / seg_offsets as there.  plan may be NULL (with plan_bytes = 0 and plan_flags = 0) unless x in dy's type
 * (n_in * c_in elements: xq from 1 GiB with PCPP_F32, 2 GiB with PCPP_BF16), dy or tri_i takes more than 4 GiB less 4 KiB;
 * 256 -> 256 channels in PCPP_BF16 never need one.  Such x, those 256 -> 256 channels, and rows of one channel whose codes are
 * as large go by way of a copy of x in dy's type, which is part of the workspace.  A code of 255 is a non-finite feature (see the conventions above).
 * workspace: pcpp_mvmr_packed_workspace_bytes(...) bytes, 256-byte aligned.
 * Errors: as pcpp_mvmr_bwd_weight.
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_mvmr_packed_workspace_bytes(int64_t n_in, int64_t n_out, int64_t n_triplets, int c_in, int c_out, int K,
                                                 int dy_dtype);
PCPP_API int pcpp_mvmr_bwd_weight_packed(const int8_t *xq, const uint8_t *xcodes, const void *dy, float *dw, int dy_dtype,
                                         int64_t n_in, int64_t n_out, int c_in, int c_out, int K,
                                         const int32_t *tri_o, const int32_t *tri_i, const int32_t *tri_k,
                                         const int64_t *seg_offsets, int64_t n_triplets,
                                         const void *plan, size_t plan_bytes, int plan_flags,
                                         void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * What lies between two blocks of a residual network, in one pass: the norm behind a block, its gate, the residual,
 * and the norm in front of the next block.  Row by row, over c channels, with
 *   n(v) = v (PCPP_NORM_NONE), v * rstd (PCPP_NORM_RMS) or (v - mean(v)) * rstd (PCPP_NORM_LAYER),
 *   rstd = 1 / sqrt(mean((v - mean(v))^2) + eps), without the mean for PCPP_NORM_RMS:
 *
 *   r = residual_scale * x + sigmoid(gate) * (w_post * n_post(f))
 *   h = w_pre * n_pre(r)
 *
 *   x, r     [n, c] stream_dtype: the residual stream before and behind the block
 *   f        [n, c] dtype, row pitch ld_f elements: the block's output.  NULL: no block in front, r is x and is not
 *            written (r NULL); only h is formed
 *   gate     logits, dtype, row pitch ld_gate elements; gate_cols = 0 (NULL: factor 1), 1 (one for the row) or c
 *   w_post, w_pre  [c] fp32, NULL: ones
 *   h        [n, c] dtype: input of the next block; NULL exactly if pre_norm is PCPP_NORM_NONE
 *   fq, fcodes / hq, hcodes   optional 8-bit copies of f and h (pcpp_act_pack) for the backward pass
 * stream_dtype is dtype, or PCPP_F32 with dtype PCPP_BF16.  All arithmetic is fp32, each output is rounded once (h
 * and its 8-bit copy from the unrounded r).  x, r, h and hq, fq are contiguous and 16-byte aligned; f and gate need
 * only the alignment of an element.  Outputs may not overlap inputs.  A row with an Inf or NaN gives NaN in that row only; one
 * whose sum of squares passes fp32's range has n(v) = 0.
 *
 * Gradients.  dr is what flows to r from behind (NULL: nothing), dh what flows to h:
 *   y = w_pre * dh,  d = dr + rstd * (y - [mean(y)] - n(r) * mean(y * n(r)))          ([..]: PCPP_NORM_LAYER)
 *   dx = residual_scale * d,  du = sigmoid(gate) * d,  dgate = du * (1 - sigmoid(gate)) * w_post * n(f), summed over
 *   the row for gate_cols = 1,  df = gradient of n_post for w_post * du, as for h,
 *   dw_pre = sum over rows of dh * n(r),  dw_post = sum over rows of du * n(f)
 *   r        as the forward pass wrote it (x where f was NULL); NULL if pre_norm is PCPP_NORM_NONE, like dh
 *   f, or fq with fcodes (then f is NULL); both may be NULL if there was no block (df NULL) or neither a post norm
 *            nor a gate
 *   dx [n, c] stream_dtype; NULL: not wanted.  df [n, c] dtype, dgate [n, gate_cols] dtype: contiguous
 *   dw_post (needs f; without a post norm the gradient of a scale for every channel of f), dw_pre  [c] fp32; NULL: not wanted
 *   workspace: pcpp_block_norm_workspace_bytes(n, c) bytes, 256-byte aligned (backward only)
 * The sums over rows are taken in a fixed order: the same result each time.
 * Errors: INVALID_ARG, WORKSPACE, UNSUPPORTED (c outside 1..1024, n >= 2^31, pitch >= 2^24, dtype combination).
 * ------------------------------------------------------------------------------------------- */
#define PCPP_NORM_NONE   0
#define PCPP_NORM_RMS    1
#define PCPP_NORM_LAYER  2

PCPP_API int pcpp_block_norm_fwd(const void *x, const void *f, int64_t ld_f, const void *gate, int64_t ld_gate, int gate_cols,
                                 const float *w_post, const float *w_pre, int post_norm, int pre_norm,
                                 float residual_scale, float eps, int64_t n, int c, int stream_dtype, int dtype,
                                 void *r, void *h, int8_t *fq, uint8_t *fcodes, int8_t *hq, uint8_t *hcodes, void *stream);
PCPP_API size_t pcpp_block_norm_workspace_bytes(int64_t n, int c);
PCPP_API int pcpp_block_norm_bwd(const void *dr, const void *dh, const void *r,
                                 const void *f, int64_t ld_f, const int8_t *fq, const uint8_t *fcodes,
                                 const void *gate, int64_t ld_gate, int gate_cols,
                                 const float *w_post, const float *w_pre, int post_norm, int pre_norm,
                                 float residual_scale, float eps, int64_t n, int c, int stream_dtype, int dtype,
                                 void *dx, void *df, void *dgate, float *dw_post, float *dw_pre,
                                 void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Log probabilities of a head's classes (tokens of a vocabulary, labels of points), row by row over v classes:
 *   lse = log(sum_j exp(x_j)),  log_prob = x_label - lse,  entropy = -sum_j p_j log(p_j),  p_j = exp(x_j - lse),
 *   and the n_top most probable classes in descending order, of equal logits the lowest index first.
 *   logits  [n, v] dtype, row pitch ld elements, aligned to an element
 *   labels  [n] int32; a label outside 0 .. v - 1 is none: log_prob is 0 and has no gradient.  NULL: no labels
 *   log_prob, entropy  [n] fp32, max_log_sum [n, 2] fp32: max_j x_j and log(sum_j exp(x_j - max)), whose sum is lse;
 *            each NULL if not wanted (the gradient needs max_log_sum, and entropy for d_entropy)
 *   top_log_prob, top_index  [n, n_top] fp32, int32; 0 <= n_top <= min(v, PCPP_MAX_ALTERNATIVES)
 * A class is masked by a logit of -Inf: its probability is 0.  A row in which all are has max_log_sum = (-Inf, 0),
 * log_prob and top_log_prob -Inf, entropy 0, and no gradient.  A row with a NaN or +Inf has NaN in all floating outputs
 * (but the maximum); among the classes a NaN ranks as -Inf.
 *   workspace: pcpp_log_probs_workspace_bytes(...) bytes, 256-byte aligned (may be NULL if that is 0)
 * Gradient of the logits, from what flows to log_prob and to entropy ([n] fp32, NULL: nothing):
 *   d_logits_j = d_log_prob * (1[j = label] - p_j) - d_entropy * p_j * (log(p_j) + entropy)
 *   d_logits  [n, v] dtype, row pitch ld_d; it may be the logits themselves (same pitch), otherwise no overlap.
 * Errors: INVALID_ARG (also: pitch < v, n_top out of range), WORKSPACE, UNSUPPORTED (n or v >= 2^31, dtype).
 * ------------------------------------------------------------------------------------------- */
#define PCPP_MAX_ALTERNATIVES 64

PCPP_API size_t pcpp_log_probs_workspace_bytes(int64_t n, int64_t v, int n_top);
PCPP_API int pcpp_log_probs_fwd(const void *logits, int dtype, int64_t n, int64_t v, int64_t ld, const int32_t *labels,
                                int n_top, float *log_prob, float *entropy, float *max_log_sum,
                                float *top_log_prob, int32_t *top_index, void *workspace, size_t workspace_bytes, void *stream);
PCPP_API int pcpp_log_probs_bwd(const void *logits, int dtype, int64_t n, int64_t v, int64_t ld, const int32_t *labels,
                                const float *max_log_sum, const float *entropy, const float *d_log_prob,
                                const float *d_entropy, void *d_logits, int64_t ld_d, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Random numbers of the calls below.  `random` is a DEVICE array int64 [2], (seed, step), read when the kernel runs: a captured graph
 * whose caller adds to the step between replays draws other numbers each time.  `site` tells a program's operators apart.  The sixteen
 * bits of the element in row i, channel j of c come from ten rounds of Philox 4x32 (Salmon et al., "Parallel random
 * numbers: as easy as 1, 2, 3", 2011) with the seed's low and high words as key and the counter
 *   (i * ceil(c / 8) + j / 8, site, low word of step, high word of step):
 * of its four words, channel j has the low (j even) or high (j odd) half of word (j % 8) / 2.  So equal arguments give equal
 * numbers, whatever the type or pitch, and a backward pass draws the forward pass's.  n * ceil(c / 8) must be below 2^32 - 65536.
 *
 * Clouds of the calls below: rows [offsets[b], offsets[b + 1]) are cloud b's, offsets DEVICE int32 [n_clouds + 1], ascending, within 0 .. n;
 * NULL (with n_clouds = 1): all rows are one cloud's.  1 <= n_clouds <= 65536.  Clouds may be empty; what a call would write
 * for a row that belongs to none is not written.  (Entries outside 0 .. n count as the nearer end; no order of them makes a call leave its
 * tensors.)
 * ------------------------------------------------------------------------------------------- */

/* ---------------------------------------------------------------------------------------------
 * Dropout of a branch, with the residual behind it:  y = residual + k * x * 65536 / (65536 - t),  t = round(65536 p), where k is 1 if the
 * sixteen bits of the element are t or more, else 0 (also where x is Inf or NaN).  p = 1 leaves the residual.
 *   x         [n, c] dtype, row pitch ld_x elements, aligned to an element
 *   residual  [n, c] stream_dtype, contiguous; NULL: none
 *   y         [n, c] stream_dtype, contiguous
 *   scope     what stays or goes as one: PCPP_DROP_ELEMENTS, PCPP_DROP_ROWS (row i draws as element (i, 0) of one channel) or
 *             PCPP_DROP_CLOUDS (cloud b draws as row b); offsets and n_clouds belong to the last one and are NULL and 1 otherwise
 * stream_dtype is dtype, or PCPP_F32 with dtype PCPP_BF16.  Gradient: dx = k * dy * 65536 / (65536 - t) with dy [n, c] stream_dtype,
 * dx [n, c] dtype, both contiguous; dy itself flows on to the residual.  Tensors are aligned to an element; outputs may not overlap inputs.
 * Errors: INVALID_ARG (also: p outside 0 .. 1, y in place of x or the residual), UNSUPPORTED (c outside 1..65536, n >= 2^31, pitch >= 2^24,
 * dtype combination, too many random numbers).
 * ------------------------------------------------------------------------------------------- */
#define PCPP_DROP_ELEMENTS  0
#define PCPP_DROP_ROWS      1
#define PCPP_DROP_CLOUDS    2

PCPP_API int pcpp_dropout_fwd(const void *x, int64_t ld_x, const void *residual, const int64_t *random, uint32_t site, float p,
                              int scope, const int32_t *offsets, int n_clouds, int64_t n, int c, int dtype, int stream_dtype,
                              void *y, void *stream);
PCPP_API int pcpp_dropout_bwd(const void *dy, const int64_t *random, uint32_t site, float p, int scope, const int32_t *offsets,
                              int n_clouds, int64_t n, int c, int dtype, int stream_dtype, void *dx, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Group norm with an activation and dropout behind it, channels last.  Over the rows of each cloud and the c / groups neighbouring
 * channels of each group:
 *   v = (x - mean) * rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps),  z = w * v + b,  y = drop(act(z))
 *   act: PCPP_ACT_NONE, PCPP_ACT_RELU, PCPP_ACT_SILU (z / (1 + exp(-z))), PCPP_ACT_GELU (z (1 + erf(z / sqrt 2)) / 2)
 *   x          [n, c] dtype, row pitch ld_x elements, aligned to an element
 *   w, b       [c] fp32; NULL: ones, zeros
 *   random, site, p   dropout of the elements as in pcpp_dropout_fwd; p = 0: none (random may be NULL)
 *   y          [n, c] dtype, contiguous, 16-byte aligned, as are dy and dx
 *   mean_rstd  [n_clouds, groups, 2] fp32, 8-byte aligned, for the gradient (NULL: not wanted); (0, 0) for an empty cloud
 *   workspace  pcpp_group_norm_workspace_bytes(n, c, n_clouds, groups, 0) bytes, 256-byte aligned (may be NULL if that is 0)
 * An Inf or NaN makes its cloud's group NaN, and no other.  Squares are summed in fp32: where the sum passes its range (deviations of 2^60) rstd is 0 or NaN.
 *
 * Gradients, from dy [n, c] dtype, contiguous, and the forward pass's mean_rstd:
 *   dz = drop(dy) * act'(z),  dx = rstd * (w * dz - m1 - v * m2),  m1, m2 = means of w * dz and of w * dz * v over the cloud and group,
 *   dw = sum over rows of dz * v,  db = sum over rows of dz               (act'(0) = 0 for PCPP_ACT_RELU)
 *   dx  [n, c] dtype, contiguous; dw, db  [c] fp32; each NULL if not wanted
 *   workspace  pcpp_group_norm_workspace_bytes(n, c, n_clouds, groups, 1) bytes
 * Arithmetic is fp32, each output is rounded once; sums have one order: the same result each time.  Outputs may not overlap inputs.
 * Errors: INVALID_ARG (also: groups do not divide c, eps not finite or below 2^-126, p outside 0 .. 1), WORKSPACE, UNSUPPORTED (c
 * outside 1..1024, n >= 2^31, pitch >= 2^22, dtype, too many random numbers).
 * ------------------------------------------------------------------------------------------- */
#define PCPP_ACT_NONE  0
#define PCPP_ACT_RELU  1
#define PCPP_ACT_SILU  2
#define PCPP_ACT_GELU  3

PCPP_API size_t pcpp_group_norm_workspace_bytes(int64_t n, int c, int n_clouds, int groups, int backward);
PCPP_API int pcpp_group_norm_fwd(const void *x, int64_t ld_x, const float *w, const float *b, const int32_t *offsets, int n_clouds,
                                 int groups, int act, float eps, const int64_t *random, uint32_t site, float p,
                                 int64_t n, int c, int dtype, void *y, float *mean_rstd,
                                 void *workspace, size_t workspace_bytes, void *stream);
PCPP_API int pcpp_group_norm_bwd(const void *dy, const void *x, int64_t ld_x, const float *mean_rstd, const float *w, const float *b,
                                 const int32_t *offsets, int n_clouds, int groups, int act,
                                 const int64_t *random, uint32_t site, float p, int64_t n, int c, int dtype,
                                 void *dx, float *dw, float *db, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Rows in microscaled 4-bit floating point (sign, two bits of exponent, one of fraction; 32 elements share a power of two), for
 * linear layers.  A row of c channels becomes
 *   q       pcpp_mx_row_bytes(c) = 16 * ceil(c / 32) bytes: two elements a byte, the even channel's in the low half; codes 0 .. 7 are
 *           0, 0.5, 1, 1.5, 2, 3, 4, 6, with 8 added their negatives; past the last channel 0
 *   scales  pcpp_mx_scale_bytes(c) = 4 * ceil(c / 128) bytes: one code s for 32 channels, in order, for 2^(s - 127); the rest is zero
 * s is the smallest with which no channel of the 32 rounds past 6, at least 1 and at most 252; larger numbers than fit then become 6.  Code 255
 * (q = 0) marks channels of which one is Inf or NaN: they are read as NaN.  To nearest (random NULL): ties go to the even fraction.
 * At random (random, site; row i and channel j of x): with m the magnitude in steps of where it lies (0.5 below 2, 1 below 4, then 2, times 2^(s - 127)), up
 * if floor(65536 (m - floor(m))) + its sixteen bits reach 65536; s is then such that nothing passes 6.
 *   x            [n, c] dtype, row pitch ld_x elements, aligned to an element
 *   q, scales    the rows; both NULL: not wanted
 *   qt, scales_t the columns: the same form of x transposed, [c] rows of n elements; both NULL: not wanted
 * q and qt are 16-byte aligned, scales 4-byte.  pcpp_mx_unpack writes the values, [n, c] dtype, contiguous; they are bf16 numbers exactly.
 * Outputs may not overlap inputs.  Errors: INVALID_ARG, UNSUPPORTED (c >= 2^24, n >= 2^31, with columns n >= 2^24, pitch >= 2^25, dtype, too many random numbers).
 *
 * Products of such rows, out[i, j] = act(sum_l a[i, l] * b[j, l] + bias[j]) with a [n, k], b [m, k], bias [m] fp32 (NULL: none), out [n, m] out_dtype,
 * contiguous, aligned to an element.  Products and sums are fp32, rounded once.  A linear layer y = x W^T and its gradients dx = dy W, dW = dy^T x are
 * this call on rows of x and W; rows of dy and columns of W; columns of dy and of x.  What flows back through act and into bias (act'(z) dy, for
 * which z has to be kept or formed again, and its sums over the rows) is the caller's.
 * pcpp_mx_linear takes a as x [n, k] x_dtype, row pitch ld_x, and rounds it to 4 bits to nearest on the way.  Outputs may not overlap inputs.
 *   workspace  pcpp_mx_product_workspace_bytes / pcpp_mx_linear_workspace_bytes(n, m, k) bytes, 256-byte aligned (may be NULL if that is 0)
 * Errors: INVALID_ARG (also: m or k < 1; the gradient of a batch without rows, zeros, is the caller's to write), WORKSPACE, UNSUPPORTED (k or m >= 2^24, n >= 2^31, pitch >= 2^25, dtype).
 * ------------------------------------------------------------------------------------------- */
PCPP_API size_t pcpp_mx_row_bytes(int64_t c);    /* 0 if c is outside 1 .. 2^24 - 1 */
PCPP_API size_t pcpp_mx_scale_bytes(int64_t c);
PCPP_API int pcpp_mx_pack(const void *x, int64_t ld_x, int dtype, int64_t n, int64_t c, const int64_t *random, uint32_t site,
                          uint8_t *q, uint8_t *scales, uint8_t *qt, uint8_t *scales_t, void *stream);
PCPP_API int pcpp_mx_unpack(const uint8_t *q, const uint8_t *scales, int64_t n, int64_t c, void *x, int dtype, void *stream);
PCPP_API size_t pcpp_mx_product_workspace_bytes(int64_t n, int64_t m, int64_t k);
PCPP_API int pcpp_mx_product(const uint8_t *a, const uint8_t *a_scales, const uint8_t *b, const uint8_t *b_scales, const float *bias, int act,
                             int64_t n, int64_t m, int64_t k, void *out, int out_dtype, void *workspace, size_t workspace_bytes, void *stream);
PCPP_API size_t pcpp_mx_linear_workspace_bytes(int64_t n, int64_t m, int64_t k);
PCPP_API int pcpp_mx_linear(const void *x, int64_t ld_x, int x_dtype, const uint8_t *w, const uint8_t *w_scales, const float *bias, int act,
                            int64_t n, int64_t m, int64_t k, void *out, int out_dtype, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PCPP_H_ */
