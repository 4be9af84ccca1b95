/*
 * dp_bk.h -- C ABI of the Book-Keeping (BK) per-sample clipped-gradient path for
 * linear layers on AMD MI355X (gfx950).
 *
 * The path is the "DP back-propagation" of the paper's section 3 for one
 * micro-batch on one worker, before any ZeRO communication:
 *
 *     per-layer, per-sample squared gradient norms   (appendix A.1, mixed ghost norm)
 *  -> sum over layers, clip factor C_i               (section 2.1, eq. (1), M = 1 group)
 *  -> clipped weighted gradient  a^T diag(C) g       (section 3, "DP gradient")
 *  -> + sigma * R * N(0, I) on a contiguous shard    (eq. (1); ZeRO gradient partition, section 2.2)
 *
 * Notation (section 3): layer input a [B, T, d_in], output gradient g = dL/ds
 * [B, T, d_out], weight gradient [d_in, d_out]; B samples, T tokens per sample.
 *
 * General conventions
 *  - Every data pointer is a DEVICE pointer unless marked "host".  The library
 *    never dereferences a device pointer on the host.
 *  - Tensors are dense and row-major with the last index contiguous.  bf16
 *    tensors must be 16-byte aligned, fp32 tensors 16-byte aligned.
 *  - The caller owns every buffer.  The library allocates no device memory and
 *    never synchronises: work is enqueued on `stream` (a hipStream_t passed as
 *    void*; NULL is the default stream) and the call returns at once.  Calls on
 *    one stream execute in order.  The only state the library keeps between calls
 *    is a per-device table of flags recording which kernels have been allowed
 *    their large LDS allocation (set once, atomically; calls from several host
 *    threads are safe).
 *  - Results are deterministic: no floating-point atomics are used and every sum
 *    is taken in a fixed order, so the same inputs give the same bits on every run.
 *  - Errors are return codes.  Arguments are validated on the host before
 *    anything is launched: a validation error (DP_ERR_INVALID_ARG,
 *    DP_ERR_UNSUPPORTED, DP_ERR_WORKSPACE) means nothing has been enqueued.  A
 *    launch the runtime refuses gives DP_ERR_HIP; the multi-layer calls consist of
 *    several launches, so earlier ones may already be queued then.
 *  - DP_F32 layers run on the fp32 matrix instructions (fp32 operands and sums),
 *    one workgroup per layer and sample in the norm kernel: they are meant for
 *    layers of a few thousand elements.  A norm that
 *    needs more than 2^28 multiply-adds per sample (T^2 (d_in + d_out) / 2 for the
 *    ghost norm, T d_in d_out for the instantiated one) is refused with
 *    DP_ERR_UNSUPPORTED; store such layers in a 16-bit type.
 */
#ifndef DP_BK_H
#define DP_BK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DP_OK = 0,
  DP_ERR_INVALID_ARG = 1,  /* NULL pointer, non-positive size, bad enum, misalignment, bad R/sigma */
  DP_ERR_UNSUPPORTED = 2,  /* valid request this build has no kernel for */
  DP_ERR_WORKSPACE = 3,    /* workspace missing or smaller than dp_norm_workspace_bytes() */
  DP_ERR_HIP = 4           /* the HIP runtime refused a launch */
} dp_status;

/* Storage type of a and g.  The 16-bit types are multiplied on the matrix cores and summed in
 * fp32; every output is fp32.  DP_F16 is IEEE binary16 with subnormals honoured.  No loss scale
 * is applied or expected anywhere (section 3.4, "Mixed-precision training with DP": the clip
 * factor already does the scaling; and with fp32 sums the Gram entries and per-sample norms
 * of the loss-scaling table cannot overflow).  For 16-bit types d_in and d_out must be multiples
 * of 8. */
typedef enum { DP_F32 = 0, DP_BF16 = 1, DP_F16 = 2 } dp_dtype;
typedef enum { DP_CLIP_STANDARD = 0, DP_CLIP_AUTOMATIC = 1 } dp_clip_mode;
typedef enum { DP_PATH_GHOST = 0, DP_PATH_PEREX = 1 } dp_path;

/* One linear layer's book-kept tensors (appendix A.2: activations and output gradients of
 * every layer stay resident until the clip factors are known). */
typedef struct {
  const void* a;   /* device, [B, T, d_in]  */
  const void* g;   /* device, [B, T, d_out] */
  int32_t T;       /* tokens per sample at this layer */
  int32_t d_in;
  int32_t d_out;
  int32_t path;    /* dp_path used for this layer's norm (ignored by dp_clipped_grad_multi) */
} dp_layer;

const char* dp_status_string(dp_status s);

/* Library/ABI version: major*10000 + minor*100 + patch. */
int dp_version(void);

/*
 * Mixed ghost norm selection (appendix A.1: "the cheaper of two techniques at each layer").
 * Pure host function.  Rule: ghost norm iff 2*T^2 <= d_in*d_out (the two T x T Gram
 * matrices take no more room than one instantiated d_in x d_out gradient); ties go to
 * the ghost norm.  Returns DP_PATH_GHOST for non-positive arguments.
 */
dp_path dp_choose_path(int64_t T, int64_t d_in, int64_t d_out);

/*
 * Bytes of device workspace that dp_ghost_norm / dp_perex_norm need for one layer
 * (per-workgroup partial sums that are then added in a fixed order).  Returns 0 for
 * invalid arguments.
 */
size_t dp_norm_workspace_bytes(dp_path path, dp_dtype dt, int B, int T, int d_in, int d_out);

/*
 * Ghost norm (appendix A.1, eq. "mixed ghost norm", right-hand side):
 *   sqnorm_out[i] = sum_{t,t'} (a[i,t,:] . a[i,t',:]) * (g[i,t,:] . g[i,t',:]),   i < B.
 * The two T x T Gram matrices are never written to memory.  bf16 inputs are multiplied
 * exactly and accumulated in fp32.
 *   a, g        device inputs, [B,T,d_in] and [B,T,d_out] of type dt
 *   sqnorm_out  device, [B] fp32, overwritten
 *   ws          device scratch of at least dp_norm_workspace_bytes(DP_PATH_GHOST, ...) bytes,
 *               16-byte aligned; contents undefined afterwards
 * bf16 requires d_in and d_out to be multiples of 8 (16-byte rows).
 */
dp_status dp_ghost_norm(const void* a, const void* g, dp_dtype dt, int B, int T, int d_in,
                        int d_out, float* sqnorm_out, void* ws, size_t ws_bytes, void* stream);

/*
 * Per-sample gradient instantiation norm (appendix A.1, left-hand side):
 *   sqnorm_out[i] = || a[i]^T g[i] ||_F^2,   a[i]^T g[i] in R^{d_in x d_out}.
 * The per-sample gradients live only in accumulator registers.  Same arguments,
 * alignment rules and workspace protocol as dp_ghost_norm (with DP_PATH_PEREX).
 */
dp_status dp_perex_norm(const void* a, const void* g, dp_dtype dt, int B, int T, int d_in,
                        int d_out, float* sqnorm_out, void* ws, size_t ws_bytes, void* stream);

/*
 * Cross-layer accumulation and clip factor (section 2.1; all-layer clipping, one group):
 *   norm_i = sqrt(max(0, sum_l sqnorm[l*B + i]))            (layers added in a fixed order)
 *   DP_CLIP_STANDARD :  C_i = min(R / norm_i, 1)            (norm_i = 0 gives C_i = 1)
 *   DP_CLIP_AUTOMATIC:  C_i = R / (norm_i + stability)      (the paper prints R = 1, stability 0.01;
 *                                                            norm_i + stability = 0 gives C_i = 0)
 * A sum that is NaN gives norm_i = C_i = NaN in both modes (the sample's gradient is not a
 * number and the weighted gradient will show it); an infinite norm gives C_i = 0.
 *   sqnorm    device, [L, B] fp32 row-major
 *   C_out     device, [B] fp32
 *   norm_out  device, [B] fp32, or NULL
 * R must be > 0 (+infinity allowed: standard clipping then gives C = 1); stability >= 0.
 * Layer-wise clipping is this call with L = 1 per layer.
 */
dp_status dp_clip_factors(const float* sqnorm, int L, int B, dp_clip_mode mode, float R,
                          float stability, float* C_out, float* norm_out, void* stream);

/*
 * Clip-weighted gradient (section 3, "DP gradient" without the noise term):
 *   grad[j, k] (+)= sum_i C[i] * sum_t a[i,t,j] * g[i,t,k],   j < d_in, k < d_out.
 * C[i] is applied in fp32 to exact products, never to the 16-bit inputs: nothing of it is rounded
 * to 16 bits.  Samples with C[i] == 0 are not counted, whatever they hold.  Short samples and narrow
 * layers take any finite weights.  The other 16-bit kernels keep one accumulator, expressed in
 * units of the current sample's weight, and multiply it by C[i] / C[i+1] between samples: any
 * finite weights work whose ratios C[i] / C[j] (j the next sample with a non-zero weight) times
 * the largest partial sum stay inside fp32 range -- in particular every set of clip factors of
 * section 2.1, which lie in (0, 1] or in (0, R / stability]; ratios up to 1e10 either way are
 * tested.  Beyond that range (for instance a subnormal weight next to a normal one) the result
 * overflows to inf or NaN rather than being silently wrong.  A NaN weight gives a NaN gradient.
 *   C           device, [B] fp32
 *   grad        device, [d_in, d_out] fp32 row-major
 *   accumulate  0: overwrite grad; 1: add to it (gradient accumulation over micro-batches)
 * bf16 requires d_in and d_out to be multiples of 8.
 */
dp_status dp_clipped_grad(const void* a, const void* g, dp_dtype dt, int B, int T, int d_in,
                          int d_out, const float* C, float* grad, int accumulate, void* stream);

/*
 * Gaussian mechanism on one rank's contiguous gradient shard (eq. (1) with one group):
 *   grad_slice[e - global_offset] += sigma * R * z_e,   e in [global_offset, global_offset+count)
 * z_e ~ N(0,1) is a pure function of (seed, step, e): Philox4x32-10 block k = e >> 2 with
 * counter (k_lo, k_hi, step_lo, step_hi) and key (seed_lo, seed_hi) gives (x0,x1,x2,x3);
 * u = ((x >> 9) + 0.5) * 2^-23; (z_{4k}, z_{4k+1}) = sqrt(-2 ln u(x0)) * (cos, sin)(2 pi u(x1)),
 * (z_{4k+2}, z_{4k+3}) likewise from (x2, x3).  Any sharding of the flattened gradient
 * therefore draws the same noise.  A (seed, step) pair must not be reused.
 *   grad_slice     device, fp32, points at element global_offset; 4-byte aligned
 *   sigma          noise multiplier, >= 0; sigma == 0 enqueues nothing (R may be +inf then)
 *   R              clipping threshold, > 0 and finite when sigma > 0
 */
dp_status dp_add_noise(float* grad_slice, uint64_t global_offset, uint64_t count, float sigma,
                       float R, uint64_t seed, uint64_t step, void* stream);

/*
 * Raw generator stream, for verification: out[4*j .. 4*j+3] = Philox4x32-10 output of block
 * first_block + j under the counter/key layout documented at dp_add_noise.
 *   out  device, uint32 [4*n_blocks], 16-byte aligned
 */
dp_status dp_philox_blocks(uint32_t* out, uint64_t first_block, uint64_t n_blocks, uint64_t seed,
                           uint64_t step, void* stream);

/*
 * Grouped forms over a stack of layers: one launch covers every layer, so small layers
 * (GPT-2-sized: tens of tiles each) still fill the 256 compute units.  Semantics are exactly
 * L calls of the per-layer function.
 *
 * dp_norms_multi: sqnorm_out[l*B + i] for every layer l, by layers[l].path.
 *   layers    HOST array of L descriptors (copied before the call returns)
 *   ws        device scratch, >= dp_norms_multi_workspace_bytes(...), 16-byte aligned
 *             (fp32 layers need none: ws may be NULL when dt == DP_F32)
 * dp_clipped_grad_multi: grads[l] as dp_clipped_grad for every layer.
 *   grads     HOST array of L device pointers, grads[l] -> [d_in_l, d_out_l] fp32, 16-byte aligned
 * Layer descriptors travel in kernel arguments (at most 48 layers per launch; longer stacks
 * take several launches), so both calls are safe under stream capture.
 */
size_t dp_norms_multi_workspace_bytes(const dp_layer* layers, int L, dp_dtype dt, int B);
dp_status dp_norms_multi(const dp_layer* layers, int L, dp_dtype dt, int B, float* sqnorm_out,
                         void* ws, size_t ws_bytes, void* stream);
dp_status dp_clipped_grad_multi(const dp_layer* layers, int L, dp_dtype dt, int B, const float* C,
                                float* const* grads, int accumulate, void* stream);

/*
 * dp_norms_multi without a workspace argument, for callers that cannot allocate device memory
 * where they call it: code under HIP stream capture, tight serving loops, harnesses that forbid
 * hipMalloc.  The per-tile partial sums go to a fixed 1 MiB array that is part of the library's
 * device image (one copy per GPU, held until the process ends); the call allocates and frees
 * nothing, on the device or on the host, and gives bit for bit the results of dp_norms_multi.
 *   DP_ERR_WORKSPACE  the stack needs more than 1 MiB of partial sums (more than 262144 tiles
 *                     times samples; dp_norms_multi_workspace_bytes tells) or has more than 1024
 *                     layers: use dp_norms_multi with a workspace of your own
 * The first call on each device looks up the array's device address (no allocation, but do it
 * once outside stream capture).  All calls on one GPU share the array: calls that may overlap
 * in time on one GPU (different streams, several host threads) race on it and must be
 * serialised by the caller; calls on one stream are ordered and safe.
 */
dp_status dp_norms_multi_static(const dp_layer* layers, int L, dp_dtype dt, int B, float* sqnorm_out,
                                void* stream);

/*
 * dp_clipped_grad_multi with the noise of eq. (1) added in the same pass ("DP gradient" of
 * section 3 in one step): the result is what dp_clipped_grad_multi followed by dp_add_noise on
 * the same elements gives, value for value, without the second pass over the gradient.  For
 * callers whose clipped sums are already final when they are formed: one device, or each rank
 * adding its own share of the noise before the reduction (the appendix on the user interface).
 *
 * Element j of layer l's gradient has global index grad_offset[l] + j; it receives
 * sigma * R * z_index when shard_offset <= index < shard_offset + shard_count (z as documented
 * at dp_add_noise: the same generator, seed, step and indexing), and no noise otherwise.
 *   grad_offset  HOST array of L global element offsets (the layers' places in the flattened
 *                model; they need not be contiguous or ordered, but must not overlap)
 *   sigma, R     as dp_add_noise (sigma >= 0, finite; R > 0; sigma == 0 adds nothing)
 * fp32 layers get the noise in the gradient kernel's epilogue, 16-bit ones where every layer of their launch (up to
 * 48 layers that take the same kernel) has a grad_offset that is a multiple of 4; for the launches with another
 * offset, and for samples whose a or g has 2 GiB and more, the noise pass runs on the layers' slices
 * after their gradients.  Errors as dp_clipped_grad_multi and dp_add_noise.
 */
dp_status dp_clipped_grad_noise_multi(const dp_layer* layers, int L, dp_dtype dt, int B, const float* C,
                                      float* const* grads, const uint64_t* grad_offset, int accumulate,
                                      uint64_t shard_offset, uint64_t shard_count, float sigma, float R,
                                      uint64_t seed, uint64_t step, void* stream);

/*
 * dp_clipped_grad_noise_multi with the gradient stored in 16 bits, in the storage type of a and g
 * (mixed-precision training keeps parameters, activations and gradients in half precision:
 * section 2.3): the fp32 value that dp_clipped_grad_noise_multi would store -- weighted sum, plus
 * the old value widened to fp32 when accumulate == 1, plus the noise -- is rounded once, to nearest
 * even, to bf16 (dt == DP_BF16) or IEEE binary16 (dt == DP_F16).
 *   grads16   HOST array of L device pointers, grads16[l] -> [d_in_l, d_out_l] of type dt, 16-byte aligned
 * Only the large-tile kernels write 16-bit gradients: every layer needs d_in, d_out >= 128, T a
 * multiple of 32, a sample's a and g below 2 GiB each, and (when sigma > 0) a grad_offset that is a
 * multiple of 4; otherwise, and for dt == DP_F32, DP_ERR_UNSUPPORTED (nothing is enqueued).
 */
dp_status dp_clipped_grad_noise_multi_h16(const dp_layer* layers, int L, dp_dtype dt, int B, const float* C,
                                          void* const* grads16, const uint64_t* grad_offset, int accumulate,
                                          uint64_t shard_offset, uint64_t shard_count, float sigma, float R,
                                          uint64_t seed, uint64_t step, void* stream);

/*
 * Group-wise clipping (eq. (1) with M groups; section 2.1, "Mathematical gradient partition":
 * all-layer clipping is one group, layer-wise clipping one group per layer, the paper's default).
 * The rows of sqnorm (one per layer weight, plus one per bias when biases are trained) are
 * partitioned into M contiguous groups: group m owns rows [group_begin[m], group_begin[m+1]) and
 * has its own threshold R[m]:
 *   norm_{m,i} = sqrt(max(0, sum of the group's rows at sample i)),  C_{m,i} = clip(norm_{m,i}; R[m]).
 *   sqnorm       device, [L, B] fp32
 *   group_begin  HOST, [M+1] ascending, group_begin[0] = 0, group_begin[M] = L (empty groups allowed)
 *   R            HOST, [M], each > 0
 *   C_out        device, [M, B] fp32;  norm_out device [M, B] or NULL
 * dp_clipped_grad_grouped is dp_clipped_grad_multi with layer l weighted by row group_of_layer[l]
 * (HOST, [L], values in [0, M)) of C [M, B].
 * The noise of eq. (1) has standard deviation sigma * ||[R_1..R_M]||_2: pass
 * dp_group_noise_threshold(R, M) as the R of dp_add_noise.
 */
dp_status dp_clip_factors_grouped(const float* sqnorm, int L, int B, const int32_t* group_begin, int M,
                                  const float* R, dp_clip_mode mode, float stability, float* C_out,
                                  float* norm_out, void* stream);
dp_status dp_clipped_grad_grouped(const dp_layer* layers, int L, dp_dtype dt, int B, const float* C,
                                  const int32_t* group_of_layer, int M, float* const* grads,
                                  int accumulate, void* stream);
float dp_group_noise_threshold(const float* R, int M);

/*
 * Book-keeping for layers on the instantiated path (appendix A.2 applied to the left side of
 * appendix A.1's equation): the norm kernel already forms every per-sample gradient
 * G_{l,i} = a_{l,i}^T g_{l,i}; when the caller gives it room, it keeps them, and the
 * clip-weighted gradient is then sum_i C_i G_{l,i} -- a stream over B arrays of d_in * d_out floats
 * instead of a second contraction over the T tokens of a and g.  The rule that puts a layer on
 * this path (2 T^2 > d_in * d_out) also makes the kept gradients smaller than the layer's two
 * Gram matrices would be.
 * dp_norms_multi_keep: dp_norms_multi, and for every layer with kept[l] != NULL also
 *   kept[l][i, j, k] = sum_t a[i,t,j] g[i,t,k]   (fp32, [B, d_in, d_out], overwritten).
 *   kept   HOST array of L device pointers (16-byte aligned) or NULLs; NULL array = keep nothing.
 *          A non-NULL entry needs path == DP_PATH_PEREX and 16-bit storage (else
 *          DP_ERR_INVALID_ARG / DP_ERR_UNSUPPORTED).
 * dp_clipped_grad_kept_multi: dp_clipped_grad_noise_multi, with the layers that have kept[l] != NULL
 *   computed from kept[l] (a and g of those layers are not read; their descriptors still give
 *   the shapes).  Samples are added in index order in fp32; samples with C[i] == 0 do not enter.
 *   grad_offset may be NULL when sigma == 0 or shard_count == 0.
 */
dp_status dp_norms_multi_keep(const dp_layer* layers, int L, dp_dtype dt, int B, float* sqnorm_out,
                              float* const* kept, void* ws, size_t ws_bytes, void* stream);
dp_status dp_clipped_grad_kept_multi(const dp_layer* layers, int L, dp_dtype dt, int B, const float* C,
                                     float* const* kept, float* const* grads, const uint64_t* grad_offset,
                                     int accumulate, uint64_t shard_offset, uint64_t shard_count, float sigma,
                                     float R, uint64_t seed, uint64_t step, void* stream);

/*
 * One step of all-layer clipping with one call: dp_norms_multi_keep (kept == NULL: dp_norms_multi), dp_clip_factors and
 * dp_clipped_grad_kept_multi (kept == NULL: dp_clipped_grad_noise_multi) on the same arguments, with the same results
 * and fewer launches; what any of the three would refuse is refused before anything is enqueued.  norm_out may be NULL.
 *   counter  device, 4 bytes, 4-byte aligned, that are zero when the call's work begins and are left zero (one such cell may
 *            serve any calls whose work does not overlap on the GPU, as sqnorm_out and ws may); or NULL, which costs small
 *            stacks a launch.  Clear it on the stream of the calls, or before them: a call that finds another value there
 *            may leave C_out and norm_out unwritten, and so may each one after it.
 */
dp_status dp_private_step_multi(const dp_layer* layers, int L, dp_dtype dt, int B, dp_clip_mode mode, float R,
                                float stability, float* const* kept, float* const* grads, const uint64_t* grad_offset,
                                int accumulate, uint64_t shard_offset, uint64_t shard_count, float sigma, uint64_t seed,
                                uint64_t step, float* sqnorm_out, float* C_out, float* norm_out, void* ws,
                                size_t ws_bytes, void* counter, void* stream);

/*
 * Layer-wise clipping without book-keeping (section 3.3 (II), and the per-layer formula of the
 * appendix on the hook-free implementation).  With one clipping group per layer, C_{l,i} depends
 * on layer l alone, so nothing forces "all norms first, then all gradients": the stack is walked
 * in passes of consecutive layers, and each pass runs norms -> clip factors -> weighted
 * gradients (+ noise) before the next is touched, so a pass's a and g are still in the
 * memory-side cache when the gradient kernels read them again.  A layer on the instantiated
 * path (path == DP_PATH_PEREX, 16-bit storage) whose whole gradient fits one workgroup tile (up to
 * 128 x 128, 512 x 32 or 32 x 512) is done, where that is estimated to be faster for the stack, in ONE
 * kernel that reads a and g once: per sample it
 * forms G_i = a_i^T g_i in registers, takes ||G_i||, C_i = clip(||G_i||; R_l) and adds C_i G_i.
 * Squared norms and factors are the same bits either way, and those of dp_norms_multi; the order in which
 * samples are added to a gradient is not.
 * Any other layer on the instantiated path keeps its G_i ([B, d_in, d_out] fp32) in the workspace
 * between its norm kernel and a weighted sum, as dp_norms_multi_keep + dp_clipped_grad_kept_multi
 * do, so its a and g are read once as well; layers are given room in stack order up to 2 GiB in
 * total, the rest contract a and g a second time.
 * The result is that of dp_norms_multi + dp_clip_factors_grouped (one group per layer)
 * + dp_clipped_grad_grouped + dp_add_noise with R = dp_group_noise_threshold(R, L):
 *   grads[l] (+)= sum_i C[l,i] a_{l,i}^T g_{l,i} + sigma ||(R_1..R_L)||_2 z   on the shard's elements.
 *   R            HOST, [L], each > 0 (finite when sigma > 0)
 *   grads        HOST array of L device pointers, as dp_clipped_grad_multi
 *   grad_offset  HOST, [L] global element offsets as dp_clipped_grad_noise_multi (may be NULL when
 *                sigma == 0 or shard_count == 0)
 *   sqnorm_out, C_out   device, [L, B] fp32, overwritten
 *   ws           device scratch >= dp_layerwise_workspace_bytes(...), 16-byte aligned
 *   layers_per_pass   0: a pass ends once it holds 128 MiB of a and g and 1024 gradient tiles,
 *                     unless fewer than 512 tiles are left;
 *                     > 0: that many layers per pass
 */
size_t dp_layerwise_workspace_bytes(const dp_layer* layers, int L, dp_dtype dt, int B);
dp_status dp_layerwise_clipped_grad(const dp_layer* layers, int L, dp_dtype dt, int B, const float* R,
                                    dp_clip_mode mode, float stability, float* const* grads,
                                    const uint64_t* grad_offset, int accumulate, uint64_t shard_offset,
                                    uint64_t shard_count, float sigma, uint64_t seed, uint64_t step,
                                    float* sqnorm_out, float* C_out, void* ws, size_t ws_bytes,
                                    int layers_per_pass, void* stream);

/*
 * Bias gradients (appendix A.1, last paragraph): the per-sample bias gradient is 1^T dL/ds_i, the
 * sum of sample i's T rows of g; its norm is taken by instantiation.
 * dp_bias_norm:  colsum[i, k] = sum_t g[i, t, k]  and  sqnorm_out[i] = sum_k colsum[i, k]^2.
 *   g           device, [B, T, d_out] of type dt (bf16: d_out a multiple of 8), 16-byte aligned
 *   colsum      device, [B, d_out] fp32, overwritten; keep it for dp_clipped_bias_grad
 *   sqnorm_out  device, [B] fp32, overwritten (use it as one more row of sqnorm)
 * dp_clipped_bias_grad:  grad_b[k] (+)= sum_i C[i] * colsum[i, k]   (g is not read again).
 *   C device [B];  grad_b device [d_out] fp32;  accumulate 0 or 1
 */
dp_status dp_bias_norm(const void* g, dp_dtype dt, int B, int T, int d_out, float* colsum,
                       float* sqnorm_out, void* stream);
dp_status dp_clipped_bias_grad(const float* colsum, int B, int d_out, const float* C, float* grad_b,
                               int accumulate, void* stream);

/*
 * Order in which the large-tile matrix-core kernels visit their output tiles, replayed on the
 * host (pure functions; nothing is launched).  They exist so that a test without a GPU can check
 * that every tile of a layer is computed exactly once for any shape; the arrays may be NULL.
 * dp_clipped_grad_tile_order: tile b of a one-layer launch of the clip-weighted gradient
 *   (section 3, "DP gradient") starts at row tile_row0[b], column tile_col0[b] of the
 *   [d_in, d_out] gradient, for a contraction over more than 512 rows and, unless d_in and d_out are both
 *   multiples of 64, up to 2048 (over longer ragged rows a launch may cut other tiles); tiles are 256 x 256.  Tiles that
 *   the launch cuts into sub-tiles (its last ones, or all) come after the others, by the workgroup
 *   of their first sub-tile; -1 if a sub-tile were computed twice.
 * dp_ghost_tile_order: workgroup b of a one-layer ghost-norm launch (appendix A.1) computes, for
 *   sample[b], the 256 x 128 block of the two Gram matrices at token rows token_row0[b], token
 *   columns token_col0[b] (always on or above the diagonal), and writes partial sum slot[b].
 * Both return the number of tiles (at most `capacity` entries are written), or -1 for invalid
 * arguments.  All pointers are HOST pointers.
 */
int64_t dp_clipped_grad_tile_order(int d_in, int d_out, int32_t* tile_row0, int32_t* tile_col0,
                                   int64_t capacity);
/*
 * How the gradient (section 3) of up to 48 16-bit layers that take these tiles is launched, so that a test can pin the kernels that
 * it means to run; a pure host function, which reads only T, d_in and d_out of the layers.  launches[0 .. 5]: 256 x 256 tiles;
 * their workgroups (fewer: each goes from tile to tile); 1 where samples take whole 32-row k-blocks, else 0; tiles that are cut
 * after them; into side x side sub-tiles of 256 / side; 1 where those are the three-stage ones of short contractions.
 * DP_ERR_UNSUPPORTED: a layer takes another kernel, or there are more of them than one launch takes.
 */
dp_status dp_clipped_grad_launches(const dp_layer* layers, int n_layers, dp_dtype dt, int B, int out16, int32_t* launches);
int64_t dp_ghost_tile_order(int T, int B, int32_t* sample, int32_t* token_row0, int32_t* token_col0,
                            int32_t* slot, int64_t capacity);

/*
 * What stands around the linear layers in a private training step: layer norms, whose gain and bias are clipped per sample as the
 * linear layers' weights are; attention; and the optimizer that takes the private gradient.  Sums and statistics are fp32; what is
 * stored in 16 bits is rounded once, to nearest even.
 */

/*
 * Layer norm over the last axis:  y = (s - mean) * rstd * gain + bias,  rstd = 1 / sqrt(var + eps),  with s = x + add where a
 * residual stream goes through (its sum is written, and normalised as written), else s = x.
 *   x, y       device, [B, T, d] of type dt; any d from 1 to 32768 (wider: DP_ERR_UNSUPPORTED)
 *   add, sum   device, [B, T, d] of type dt, both or neither NULL; sum may be x or add
 *   gain, bias device, [d] fp32, or NULL: ones, zeros
 *   mean, rstd device, [B * T] fp32, kept for the backward pass, or NULL
 * The [B, T, d] arrays are 16-byte aligned; eps >= 0.
 */
dp_status dp_layer_norm(const void* x, const void* add, dp_dtype dt, int B, int T, int d, const float* gain, const float* bias,
                        float eps, void* sum, void* y, float* mean, float* rstd, void* stream);

/*
 * Backward pass of dp_layer_norm, with h = (x - mean) * rstd and u = dy * gain:
 *   dx = (u - mean_d(u) - h * mean_d(u h)) * rstd  (+ add: the gradient that reaches x beside the norm),
 *   kept[i] = (sum_t dy h, sum_t dy): sample i's gradients of gain and bias, [B, 2, d] fp32,
 *   sqnorm_out[i] = ||kept[i]||^2, one more row of sqnorm.
 * Once the clip factors are known, dp_clipped_bias_grad(kept, B, 2 * d, C, grad, ...) adds the clipped gradients up, gain's
 * and bias's one behind the other, as for biases.  (Without clipping: B = 1 and T = all rows give the plain sum in kept.)
 *   x          what was normalised (dp_layer_norm's sum, where there was one)
 *   dx         may be dy or add; NULL: not wanted (then add is NULL too)
 *   kept, sqnorm_out   both or neither NULL
 *   ws         device scratch, >= dp_layer_norm_workspace_bytes(...), 16-byte aligned; not used without kept
 */
size_t dp_layer_norm_workspace_bytes(dp_dtype dt, int B, int T, int d);
dp_status dp_layer_norm_backward(const void* x, const void* dy, const void* add, dp_dtype dt, int B, int T, int d, const float* gain,
                                 const float* mean, const float* rstd, void* dx, float* kept, float* sqnorm_out, void* ws,
                                 size_t ws_bytes, void* stream);

/*
 * Attention of Tq queries over Tk keys, H heads of width D:  o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - lse_i)
 * over the keys j that row i sees, lse_i = log sum_j exp(scale q_i . k_j).
 *   Heads: H_kv divides H; query heads h share key head h / (H / H_kv).
 *   Layout: element strides of sample, token and head, for q, k, v and o; columns are adjacent.  Packed projections
 *     ([B, T, 3 * H * D] and the like) need no copies.  Strides are >= 0 and, for 16-bit types, multiples of 8; a token stride is
 *     from D to 2^23 (of one token: whatever).  What is read may be broadcast (stride 0); what is written may not overlap
 *     itself: by growing stride, each axis steps over all that the ones before span (DP_ERR_INVALID_ARG else; the gradients have
 *     the strides of q, k and v).
 *   Lengths: q_len[b] queries and k_len[b] keys of sample b are there (device, [B] int32; NULL: all; values are held to 0 .. T).
 *     What lies behind them is not read.
 *   causal = 1: the ends are aligned; row i sees keys up to i + (keys there) - (queries there).
 * Rows that see no key, and rows that are not there, are zeros, with lse = -infinity.  What a row does not see does not reach
 * it, infinities and NaN included.
 * D is at most 128 and, for 16-bit types, a multiple of 8.  All types run on the matrix cores, 16-bit ones with
 * probabilities rounded to the type before their product with v; DP_F32 whose D or strides are not multiples of 4, or whose
 * arrays are not 16-byte aligned, runs on the vector units, for small networks.  scale is positive and finite.
 */
typedef struct {
  int32_t B, H, H_kv, Tq, Tk, D;
  int32_t causal;
  float scale;
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];   /* sample, token, head */
  const int32_t* q_len;
  const int32_t* k_len;
} dp_attention_shape;

/*
 *   shape     HOST
 *   q, k, v, o   device, of type dt, 16-byte aligned (DP_F32: 4-byte; the matrix cores want 16)
 *   lse       device, [B, H, Tq] fp32, kept for the backward pass
 *   ws        device scratch, >= dp_attention_workspace_bytes(...), 16-byte aligned, with which few queries (single tokens) on many keys are
 *             spread over the device; or NULL: slower there, otherwise the same to rounding.  The size is 0 where it is not used.
 */
size_t dp_attention_workspace_bytes(const dp_attention_shape* shape, dp_dtype dt);
dp_status dp_attention(const dp_attention_shape* shape, dp_dtype dt, const void* q, const void* k, const void* v, void* o, float* lse,
                       void* ws, size_t ws_bytes, void* stream);

/*
 * Backward pass, which forms the probabilities again from lse:
 *   dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - do_i . o_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,
 * dk and dv summed over the query heads that share a key head.  Every element of dq, dk and dv that the shape reaches is written (zeros
 * where a row is not there); p and ds are rounded to the type before their products (16-bit types; in fp16 ds times a power of two that keeps it
 * from over- and underflowing, taken out in fp32).
 *   o, lse    dp_attention's;  dout  the gradient of o, in o's strides
 *   dq, dk, dv   in the strides of q, k and v; they do not overlap each other nor an input
 *   ws        device scratch, >= dp_attention_backward_workspace_bytes(...), 16-byte aligned
 */
size_t dp_attention_backward_workspace_bytes(const dp_attention_shape* shape, dp_dtype dt);
dp_status dp_attention_backward(const dp_attention_shape* shape, dp_dtype dt, const void* q, const void* k, const void* v,
                                const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv, void* ws,
                                size_t ws_bytes, void* stream);

/*
 * Host query (no GPU): the rows of keys and values that a tile of the forward pass and of the query gradients' kernel holds, and those of queries and
 * their output gradients in the key gradients' kernel; 1 where rows are taken one by one.  Arrays are taken to be 16-byte aligned.  Where few
 * rows face many, tiles are larger, as far as rows that lie the token stride apart allow: rows * stride * size <= 2^31 bytes always.
 *   rows      HOST, [3]
 */
dp_status dp_attention_tile_rows(const dp_attention_shape* shape, dp_dtype dt, int32_t* rows);

/*
 * One AdamW step over many tensors (for a rank that holds one shard of the flattened gradient: one tensor), in place:
 *   g = grad_scale * grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2;
 *   param = param (1 - lr * weight_decay) - lr * m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps).
 * grad_scale is what the sum over samples of the private gradient lacks: 1 over the (expected) batch size.
 *   tensors     HOST array; param fp32 [n]; grad [n] of type grad_dt; n = 0: nothing to do.  Elements need no more than their own
 *               alignment; where all of a tensor's arrays are aligned to four elements they are moved four at a time.
 *   state_bits  32: m and v are fp32 [n].
 *               8: m and the root of v are e4m3 numbers (sign, 4 bits of exponent, 3 of fraction; largest 448), one byte each [n], in
 *               units of m_scale and v_scale, fp32 [ceil(n / 256)]: the largest magnitude of each 256 values, over 448.  A value is
 *               rounded up where its place between its neighbours (v's: between their squares) is at least 1 - f, f the fractional
 *               part of e (sqrt(2) - 1) + step (golden ratio - 1) for element e (in 32-bit integers: (e * 0x6A09E667 + step *
 *               0x9E3779B1) >> 8, over 2^24), so that slow averages do move; one above zero is not rounded to zero.  All-zero bytes
 *               and scales are zero states.
 *               An infinite or undefined state makes those of its 256 undefined.
 *   copy_dt     DP_BF16 or DP_F16: the new param is also written to copy [n], rounded to nearest even; DP_F32: copy is not used
 *   step        counts from 1
 * Tensors travel in kernel arguments, up to 128 to a launch.
 */
typedef struct {
  float* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  uint64_t n;
  float weight_decay;
  int32_t reserved;
} dp_adamw_tensor;
dp_status dp_adamw_multi(const dp_adamw_tensor* tensors, int n_tensors, dp_dtype grad_dt, int state_bits, dp_dtype copy_dt, double lr,
                         double beta1, double beta2, double eps, double grad_scale, uint64_t step, void* stream);

/*
 * What gated transformer blocks run besides: the position rotation of queries and keys, with or without a norm of each head before it,
 * the gated feed-forward layer's products, and an optimizer that orthogonalises the update.  Sums and statistics are fp32 at least; what is
 * stored in 16 bits is rounded once, to nearest even.
 */

/*
 * Heads of queries and keys, between their projection and attention.
 *   B, T      samples (at most 2^21) and tokens;  H, H_kv: heads of the queries and of the keys (H_kv = 0: queries alone, the keys' pointers and strides are
 *             not looked at);  D: a head's width, at most 256 and, for 16-bit types, a multiple of 8
 *   rotary    the first `rotary` columns of a head turn (even, from 0 to D); the others pass
 *   interleaved   1: columns 2 i and 2 i + 1 are a pair; 0: columns i and i + rotary / 2
 *   amplitude multiplies both of a pair (contexts longer than a model was made for: some ask for more than 1)
 *   q_stride .. k_out_stride   element strides of sample, token and head, as of dp_attention_shape; columns are adjacent.  For 16-bit types
 *             multiples of 8.  What is read may be broadcast (stride 0), what is written may not overlap itself.
 *   turns     device fp64 [rotary / 2], 8-byte aligned: of pair i, whole turns from one position to the next (dp_rotary_turns makes them)
 *   position  device int32 [B, T], or NULL: token t is at position t
 *   len       device int32 [B], or NULL: all tokens are there.  Rows from len[b] on (held to 0 .. T) are neither read nor written.
 * Angles are taken modulo whole turns in 64 bits: far positions lose nothing.  Results may lie where their own input does, in the same strides;
 * otherwise what is written overlaps nothing else.
 */
typedef struct {
  int32_t B, T, H, H_kv, D;
  int32_t rotary, interleaved;
  float amplitude;
  int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3];   /* sample, token, head */
  const double* turns;
  const int32_t* position;
  const int32_t* len;
} dp_heads_shape;

/*
 * Turns for `rotary` columns (host function): pair i has base^(-2 i / rotary) / (2 pi), changed for longer contexts by
 *   DP_ROTARY_LINEAR   all divided by `factor`
 *   DP_ROTARY_BASE     base times factor^(rotary / (rotary - 2)) (one pair alone: as it is)
 *   DP_ROTARY_PARTS    those that make `fast` turns or more within the `original` context stay, those of `slow` or fewer are divided by
 *                      `factor`, in between both are mixed by the turns' place between slow and fast
 *   turns     HOST fp64 [rotary / 2]
 */
typedef enum { DP_ROTARY_PLAIN = 0, DP_ROTARY_LINEAR = 1, DP_ROTARY_BASE = 2, DP_ROTARY_PARTS = 3 } dp_rotary_scaling;
dp_status dp_rotary_turns(double* turns, int rotary, double base, dp_rotary_scaling scaling, double factor, double original, double slow,
                          double fast);

/*
 * Rotation:  (x1, x2) -> amplitude (x1 cos - x2 sin, x2 cos + x1 sin)  of each pair, by position * turns[i] turns; and its gradient, the
 * same with the angle's sign changed.
 *   shape     HOST
 *   q, k, q_out, k_out   device, of type dt, 16-byte aligned (DP_F32: 4-byte)
 *   dq_out, dk_out   in the strides of q_out and k_out;  dq, dk  in those of q and k
 */
dp_status dp_rotary(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, void* q_out, void* k_out, void* stream);
dp_status dp_rotary_backward(const dp_heads_shape* shape, dp_dtype dt, const void* dq_out, const void* dk_out, void* dq, void* dk,
                             void* stream);

/*
 * Norm of each head, then the rotation:  y = R(h gain),  h = x r,  r = 1 / sqrt(mean_D(x^2) + eps).  rotary = 0: the norm alone.
 *   q_gain, k_gain   device fp32 [D], shared by all heads of their side, or NULL: ones
 */
dp_status dp_head_norm(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, const float* q_gain, const float* k_gain,
                       float eps, void* q_out, void* k_out, void* stream);

/*
 * Its backward pass, with g = R'(dy), u = g gain:  dx = r (u - h mean_D(u h)),
 *   kept[i] = sum_{t, heads} g h: sample i's gradients of q_gain and, behind it, k_gain: [B, 2, D] fp32 (H_kv = 0: [B, 1, D]);
 *   sqnorm_out[i] = ||kept[i]||^2, one more row of sqnorm.  dp_clipped_bias_grad(kept, B, 2 * D, C, grad, ...) then adds the clipped gradients up.
 *   q, k      what dp_head_norm was given;  dq_out, dk_out  in the strides of q_out, k_out;  dq, dk  in those of q, k; each may be its dq_out
 *             or its q where strides are the same
 *   kept, sqnorm_out   both or neither NULL
 *   ws        device scratch, >= dp_head_norm_workspace_bytes(...), 16-byte aligned; not used without kept
 */
size_t dp_head_norm_workspace_bytes(const dp_heads_shape* shape, dp_dtype dt);
dp_status dp_head_norm_backward(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, const void* dq_out,
                                const void* dk_out, const float* q_gain, const float* k_gain, float eps, void* dq, void* dk, float* kept,
                                float* sqnorm_out, void* ws, size_t ws_bytes, void* stream);

/*
 * Gated feed-forward layer, from its input to what its last projection reads, in one pass:
 *   gate = x w_gate + b_gate,  up = x w_up + b_up,  h = act(gate) up.
 * gate and up are formed in fp32 and rounded where they are stored; h comes from the unrounded ones.
 *   x         device, [rows, d] of type dt (rows = B T)
 *   w_gate, w_up   device, [d, f] of type dt;  b_gate, b_up  device, [f] of type dt, each or NULL
 *   gate, up  device, [rows, f] of type dt, kept for the backward pass; both or neither NULL
 *   h         device, [rows, f] of type dt
 *   ws        device scratch, >= dp_gated_workspace_bytes(...), 16-byte aligned; not used where the size is 0
 * For 16-bit types d and f are multiples of 8 and arrays 16-byte aligned (DP_F32: 4-byte).  d and f are at most 2^20.  Results overlap nothing.
 * act: silu x s(x), s the logistic function; gelu x Phi(x); gelu_tanh its form by tanh; relu; sigmoid s(x).  For 16-bit types Phi(x) is within 1.5e-7
 * (where it is below 1e-10 itself, at x < -6.5, from 0.5 % of it on), s(x) within 2^-22.
 */
typedef enum { DP_ACT_SILU = 0, DP_ACT_GELU = 1, DP_ACT_GELU_TANH = 2, DP_ACT_RELU = 3, DP_ACT_SIGMOID = 4 } dp_activation;
size_t dp_gated_workspace_bytes(dp_dtype dt, int rows, int d, int f);
dp_status dp_gated(const void* x, dp_dtype dt, int rows, int d, int f, const void* w_gate, const void* w_up, const void* b_gate,
                   const void* b_up, dp_activation act, void* gate, void* up, void* h, void* ws, size_t ws_bytes, void* stream);

/*
 * Its backward pass.  dgate and dup are the output gradients of the two projections, book-kept as the `g` of two linear layers whose input
 * is x (dp_layer); the last projection's are (h, dy).
 *   dh = dy w_down' (or given),  dgate = dh up act'(gate),  dup = dh act(gate),  dx = dgate w_gate' + dup w_up'  (of dgate and dup as stored)
 *   dy        device, [rows, d_out] of type dt, with w_down device [f, d_out];  or, w_down NULL, dh itself, [rows, f] (d_out is not looked at)
 *   gate, up  dp_gated's;  dgate, dup  device, [rows, f] of type dt; they may be gate and up, or one of them dh
 *   dx        device, [rows, d] of type dt, or NULL: not wanted (then the weights may be NULL); like dgate and dup otherwise it overlaps nothing
 *   ws        device scratch, >= dp_gated_backward_workspace_bytes(...), 16-byte aligned; not used where the size is 0.  The size is for calls with
 *             dx or without; d_out = 0: with no w_down
 */
size_t dp_gated_backward_workspace_bytes(dp_dtype dt, int rows, int d, int f, int d_out);
dp_status dp_gated_backward(const void* dy, const void* w_down, int d_out, const void* gate, const void* up, dp_dtype dt, int rows, int d,
                            int f, const void* w_gate, const void* w_up, dp_activation act, void* dgate, void* dup, void* dx, void* ws,
                            size_t ws_bytes, void* stream);

/*
 * Host query (no GPU): how a pass of a gated layer is launched, so that a test can pin the kernels that it means to run.
 *   pass      0: forward; 1: dgate and dup from dy and w_down (d_out is looked at here alone); 2: dx
 *   launches  HOST, [6]: the kernel (0: tiles of 16-bit types, 256 x 256 and 128 x 128; 1: few rows; 2: tiles of fp32, 128 x 128 and 64 x 64); large tiles
 *             of one workgroup each; small ones (where there are large ones too, of what those leave); tiles whose contraction several workgroups
 *             share; how many; the side of these
 */
dp_status dp_gated_launches(dp_dtype dt, int rows, int d, int f, int d_out, int pass, int32_t* launches);

/*
 * One step of an optimizer that orthogonalises its update, over many matrices, in place:
 *   g = grad_scale grad;  m = beta m + g;  u = g + beta m (nesterov = 1) or m;  X = u / (||u||_F + eps);
 *   `iterations` times  X <- a X + b A X + c A^2 X,  A = X X'  (on the shorter side);
 *   param = param (1 - lr weight_decay) - lr scale X.
 * Products are of values in two fp16 halves (within 2^-23 of a value, or 2^-37 of 1 below 2^-15), without that of the two lower halves, added
 * up in fp32.  X is then 0.6 to 0.8 times as far from its 64-bit value as fp32 products leave it for random matrices, up to 2.3 times where
 * singular values span four decades (768 x 2304: 8.4e-6 of its norm, and 5.4e-6).  Matrices that one workgroup holds (dp_muon_launches) are
 * fp32 throughout.
 *   tensors      HOST array; param, m fp32 [rows, cols]; grad of type grad_dt; copy of type copy_dt (DP_F32: not used), the new param rounded;
 *                elements need no more than their own alignment.  rows and cols are at most 2^20, the shorter at most 2^16.
 *   coefficients HOST fp64 [iterations, 3]: a, b, c of each iteration, 1 to 32 of them.  Singular values, which start in [0, 1], may not leave
 *                |x| <= 15 on the way, nor A's polynomial (DP_ERR_UNSUPPORTED).
 *   ws           device scratch, >= dp_muon_workspace_bytes(...), 16-byte aligned: some 8 bytes an element of up to 64 matrices at a time, 8 of
 *                each shorter side squared, and up to 32 MiB where they are few
 * What is written, workspace included, overlaps nothing else: no matrix is named twice.
 * Matrices go in runs of up to 64, each of them a few launches whatever the number of its matrices.
 */
typedef struct {
  float* param;
  const void* grad;
  float* m;
  void* copy;
  int32_t rows, cols;
  float weight_decay, scale;
} dp_muon_tensor;
size_t dp_muon_workspace_bytes(const dp_muon_tensor* tensors, int n_tensors);
/*
 * Host query (no GPU): how such a step is launched, so that a test can pin the kernels that it means to run; rows and cols are looked at alone.
 *   launches  HOST, [7]: matrices that one workgroup holds each; of the first run of others, for A, its polynomial and the update, the side of tiles
 *             and the workgroups that share one (0: there are none)
 */
dp_status dp_muon_launches(const dp_muon_tensor* tensors, int n_tensors, int32_t* launches);
dp_status dp_muon_multi(const dp_muon_tensor* tensors, int n_tensors, dp_dtype grad_dt, dp_dtype copy_dt, double lr, double beta, int nesterov,
                        double grad_scale, double eps, const double* coefficients, int iterations, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DP_BK_H */
