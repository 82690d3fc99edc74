/* libbns -- sampled batch normalisation for AMD MI355X (gfx950).
 *
 * Training-mode batch normalisation, forward and backward, in which the
 * per-channel mean and variance are estimated from a sampled subset S of the
 * activations ("Batch Normalization Sampling", Chen, Deng, Li et al.,
 * arXiv 1810.10962).  Citations below are to that paper.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Layout     x, y, dy, dx are dense tensors, element type given by
 *            bns_shape.dtype, in the layout bns_shape.layout names: N x C x H x W
 *            (channel planes of H*W contiguous elements; the default) or
 *            N x H x W x C (channels contiguous, the layout the paper's notation
 *            uses, Appendix A).  Either way the reduction axes are N, H, W, the
 *            paper's E_{0,1,2} / Var_{0,1,2}, and the same (shape, spec, seed) give
 *            the same index and, up to rounding order, the same results.
 *            Per-channel vectors (gamma, beta, statistics, dgamma, dbeta) are
 *            float[C].
 * Memory     Unless an argument is marked HOST it is a DEVICE pointer owned by
 *            the caller, at least 16-byte aligned.  The library allocates and
 *            frees nothing and keeps no state between calls except the tuning
 *            overrides of bns_set_option.  `workspace` is caller-provided
 *            device scratch of at least bns_workspace_bytes() bytes; its
 *            contents need not be initialised.  Its first 256 bytes hold a launch
 *            counter that the single-launch kernels keep from call to call: a
 *            workspace may be overwritten between calls (the counter is set up
 *            again), but not while a call that uses it is running.
 * Streams    `stream` is a hipStream_t passed as void* (NULL = the default
 *            stream).  Work is enqueued on it and the call returns without
 *            synchronising.  Calls that share a workspace must be ordered on
 *            one stream.
 * Concurrency The single-launch ("fused") kernels size their grid to what the
 *            device holds at once and let the blocks that share a channel wait
 *            for each other.  Calls from several host threads and streams of one
 *            process are safe: the library chains such kernels with an event, so
 *            that two of them never share the device.  If work the library does not
 *            know of occupies the device at the same time (another process, a HIP
 *            graph that holds captured libbns calls and is replayed beside other
 *            libbns calls), a wait can last until that work ends; it is bounded
 *            (2^21 polls, then 2^15 for the rest of the launch), after which the
 *            results of that channel are NaN -- never a wrong finite value -- the
 *            moving averages keep their old values, the kernel ends normally, and
 *            bns_expired_waits() reports it, so nobody has to scan tensors.
 *            The N x H x W x C calls whose blocks would wait for each other take
 *            the streaming kernels while their stream is being captured; and so do
 *            calls of either layout while the stream that carried the last such
 *            kernel is being captured and is not their own (they cannot be ordered
 *            behind it without touching that capture).
 * Aliasing   Outputs must not overlap inputs or each other (x is needed again
 *            by the backward pass; dx is written while dy is read).  The host
 *            checks the tensors (y against x; dx against x and dy) and returns
 *            BNS_EINVAL when they overlap.  The per-channel vectors and the
 *            workspace are not checked against anything: keeping them apart
 *            from each other and from the tensors is the caller's duty.
 * Errors     Every call returns a bns_status.  Arguments are validated on the
 *            host before anything is enqueued: BNS_EINVAL for NULL pointers,
 *            non-positive extents, n_s outside [1, N] (Alg. 1), patch sizes
 *            outside [1, H] x [1, W] (Alg. 2), VDN with n_s >= N, unknown
 *            enums, misaligned pointers, an output tensor that overlaps an
 *            input tensor (see Aliasing);
 *            BNS_EUNSUPPORTED for extents beyond the limits listed at
 *            bns_shape; BNS_EWORKSPACE when the workspace is too small;
 *            BNS_EDEVICE when the HIP runtime reports a launch failure.
 *            Nothing is thrown across the boundary.
 * Determinism No floating-point atomics: per-channel sums are combined in a
 *            fixed order, so results are bit-identical from run to run (of the
 *            same kernels: a call inside or beside a capture can take others
 *            than outside, see Concurrency, and differ in the last bits).
 */
#ifndef BNS_H
#define BNS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BNS_OK = 0,
    BNS_EINVAL = 1,
    BNS_EUNSUPPORTED = 2,
    BNS_EWORKSPACE = 3,
    BNS_EDEVICE = 4
} bns_status;

/* Which activations feed the statistics. */
typedef enum {
    BNS_FULL = 0, /* all m = N*H*W points of a feature map (Eq. 2): plain BN                   */
    BNS_NS = 1,   /* Naive Sampling: samples 0 .. n_s-1 (Alg. 1 with begin = 0)                */
    BNS_BS = 2,   /* Batch Sampling: samples begin .. begin+n_s-1, begin = randint(0, N-n_s),
                     one draw per (layer, epoch), shared by all channels (Alg. 1, Sec. 4.1)    */
    BNS_FS = 3,   /* Feature Sampling: one patch_h x patch_w patch at (begin_h, begin_w) of
                     every sample (Alg. 2); one location per layer, or one per channel         */
    BNS_VDN = 4   /* Virtual Dataset Normalisation: the n_s virtual samples that the caller
                     concatenated in front of the batch, samples 0 .. n_s-1 (Alg. 3)           */
} bns_mode;

typedef enum { BNS_F32 = 0, BNS_BF16 = 1 } bns_dtype; /* storage of x, y, dy, dx; arithmetic is fp32 */

typedef enum { BNS_NCHW = 0, BNS_NHWC = 1 } bns_layout; /* memory order of x, y, dy, dx */

/* Tensor extents.  For VDN, N counts virtual + real samples (virtual first).
 * Limits: N <= 65535, C <= 2^24, H*W < 2^31, N*H*W < 2^31, C*H*W < 2^31.
 * BNS_NHWC: every channel shares one location set there, so Feature Sampling with
 * fs_per_channel = 1 returns BNS_EUNSUPPORTED; the other modes, the bns_*_mixed calls, both storage
 * types and every stage call are available. */
typedef struct {
    int32_t N, C, H, W;
    int32_t dtype;  /* bns_dtype */
    int32_t layout; /* bns_layout */
} bns_shape;

/* Sampling specification.  (seed, layer_id, epoch) select the random index: the paper
 * refreshes indices once per epoch and draws them independently per layer (Sec. 4.1). */
typedef struct {
    int32_t mode;             /* bns_mode */
    int32_t n_s;              /* NS/BS: samples kept; VDN: number of virtual samples; else ignored */
    int32_t patch_h, patch_w; /* FS: patch extent; else ignored */
    int32_t fs_per_channel;   /* FS: 0 = one patch location per layer (the paper's rule),
                                 1 = an independent location for each channel */
    uint32_t layer_id;
    uint32_t epoch;
} bns_spec;

/* The location set S of one channel: the box [n0, n0+n_cnt) x [h0, h0+h_cnt) x [w0, w0+w_cnt). */
typedef struct {
    int32_t n0, n_cnt, h0, h_cnt, w0, w_cnt;
} bns_box;

const char* bns_status_string(bns_status s);

/* Sampling index, computed on the host (Alg. 1-3; "randint" includes both ends).
 * boxes: HOST array of shape->C entries, written.  A pure integer function of
 * (shape, spec, seed): 64-bit SplitMix64-style mixing of seed, layer_id, epoch, the
 * coordinate being drawn and (per-channel FS only) the channel; the top 32 bits are
 * scaled to the number of outcomes.  No device is touched. */
bns_status bns_sample_index(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                            bns_box* boxes /* HOST, C entries */);

/* The same index evaluated by the generator the kernels use, on the device.
 * boxes: DEVICE array of shape->C entries, written on `stream`. */
bns_status bns_sample_index_device(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                                   bns_box* boxes /* DEVICE, C entries */, void* stream);

/* Bytes of device scratch that bns_forward / bns_backward and their stages need (depends on the
 * extents and the layout only). */
size_t bns_workspace_bytes(const bns_shape* shape, const bns_spec* spec);

/* Forward (Eq. 1 with the statistics of Eq. 3):
 *   save_mean[c]   = E    = mean of x over S_c
 *   save_invstd[c] = 1 / sqrt(Var + eps), Var = biased variance of x over S_c
 *   y = gamma * (x - E) * invstd + beta                       for all N*H*W points
 *   running_mean/var <- (1 - momentum) * running + momentum * (E | Var)     (Eq. 8; pass
 *   momentum = 1 for its first-iteration branch); either may be NULL = not kept.
 * in: x, gamma, beta.  out: y, save_mean, save_invstd.  in-out: running_*. */
bns_status bns_forward(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                       const void* x, const float* gamma, const float* beta,
                       float eps, float momentum,
                       void* y, float* save_mean, float* save_invstd,
                       float* running_mean, float* running_var,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Backward (Eq. 5 with the modification of Eq. 6).  With g = dl/dy, r = save_invstd,
 * x^ = (x - save_mean) * r and s = |S_c|:
 *   dbeta[c]  = sum over all m points of g
 *   dgamma[c] = sum over all m points of g * x^
 *   dx_i = gamma r g_i                                            for x_i outside S
 *   dx_i = gamma r (g_i - (dbeta + x^_i dgamma) / s)              for x_i in S
 * (Eq. 6 after substituting dl/dE and dl/dVar of Eq. 5).  The index is re-derived from
 * (spec, seed), which must equal the forward call's.
 * in: x, dy, gamma, save_mean, save_invstd.  out: dx, dgamma, dbeta. */
bns_status bns_backward(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                        const void* x, const void* dy, const float* gamma,
                        const float* save_mean, const float* save_invstd,
                        void* dx, float* dgamma, float* dbeta,
                        void* workspace, size_t workspace_bytes, void* stream);

/* bns_backward for callers that cannot hand over a workspace they allocated: code recorded into a HIP graph
 * whose buffers are fixed before the scratch size is known, tight serving or training loops, harnesses that
 * forbid hipMalloc.  Same arguments, results (bit for bit) and errors as bns_backward, without `workspace`:
 * the partial sums and exchange slots live in an array of 5 MiB + 256 bytes built into the library's device code, one copy
 * per GPU, held from the first use of the library on that GPU until the process ends.  The call allocates
 * and frees nothing.  BNS_EWORKSPACE if bns_workspace_bytes(shape, spec) exceeds that size (N x H x W x C) or
 * 4 MiB + 256 bytes of it (N x C x H x W: more than 3840 channels).  All such calls on one GPU share the one array, which keeps what the last call left in it
 * (nothing in it has to start at zero): they must be ordered on one stream, like calls that share a
 * workspace; calls that overlap on a GPU race.  Against the other calls of the library they are ordered like any call
 * (see Concurrency).  The first call on each GPU looks the array's address up and
 * should be made outside stream capture. */
bns_status bns_backward_builtin_workspace(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                                          const void* x, const void* dy, const float* gamma,
                                          const float* save_mean, const float* save_invstd,
                                          void* dx, float* dgamma, float* dbeta, void* stream);

/* How many waits between blocks of the single-launch kernels ran out (see Concurrency) in the calls that used
 * `workspace` since the last such query; 0 = every result is what the equations say.  Calls whose waits ran
 * out have written NaN to the outputs of the channels concerned.  Synchronises `stream` (the stream those calls
 * were issued to), reads the count from the workspace and clears it; not to be called while `stream` is being
 * captured.  workspace = NULL asks about the built-in scratch of bns_backward_builtin_workspace.
 * expired: HOST, written. */
bns_status bns_expired_waits(void* workspace, size_t workspace_bytes, void* stream, int32_t* expired /* HOST */);

/* The stages that the two calls above are made of, for callers that want to place
 * other work between them (and for per-kernel timing).  Same conventions.  A whole call
 * that took the streaming kernels ("last_path_forward" / "last_path_backward" = 1) carries the bits of its
 * stages; the single-launch kernels sum in another order and can differ from them in the last bits.  In
 * N x H x W x C these are the default up to 8192 rows (N*H*W) and, as far as they are the faster side, beyond 4 MB.
 * Beyond them bns_backward of that layout may write part of dx while it sums ("last_path_backward" = 4, "nhwc_split_ordered"), in an
 * order of its own, too (with "path" = 1 or "nhwc_split_dx" = 2 it does not).
 *
 * bns_forward_stats     Eq. 3 + Eq. 8: statistics of x over S and running averages.
 * bns_forward_normalize Eq. 1: y from x and the saved statistics, all points.
 * bns_backward_reduce   the two length-m sums of Eq. 5: dbeta and dgamma.
 * bns_backward_dx       Eq. 6: dx from dy, (x on S), the statistics and dgamma, dbeta. */
bns_status bns_forward_stats(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                             const void* x, float eps, float momentum,
                             float* save_mean, float* save_invstd,
                             float* running_mean, float* running_var,
                             void* workspace, size_t workspace_bytes, void* stream);
bns_status bns_forward_normalize(const bns_shape* shape, const void* x,
                                 const float* gamma, const float* beta,
                                 const float* save_mean, const float* save_invstd,
                                 void* y, void* stream);
bns_status bns_backward_reduce(const bns_shape* shape, const void* x, const void* dy,
                               const float* save_mean, const float* save_invstd,
                               float* dgamma, float* dbeta,
                               void* workspace, size_t workspace_bytes, void* stream);
bns_status bns_backward_dx(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                           const void* x, const void* dy, const float* gamma,
                           const float* save_mean, const float* save_invstd,
                           const float* dgamma, const float* dbeta,
                           void* dx, void* stream);

/* "VDN + sampling" (Sec. 4.2 step 3, Eq. 4).  The tensor holds n_v virtual samples in front of
 * N - n_v real ones (Alg. 3).  `spec` (mode FULL, NS, BS or FS) is the sampling strategy applied to
 * the REAL samples, exactly as Alg. 1 / Alg. 2 on a batch of N - n_v samples shifted by n_v.  With
 * x_v the virtual set and x_s the sampled real set, each statistic by Eq. 3 on its own set,
 *   E   = mix_beta * E[x_v]   + (1 - mix_beta) * E[x_s]
 *   Var = mix_beta * Var[x_v] + (1 - mix_beta) * Var[x_s]           (the paper uses mix_beta = 0.5)
 * save_mean / save_invstd hold the blended E and 1/sqrt(Var + eps); save_mean_parts (float[2*C])
 * holds E[x_v] for every channel, then E[x_s] for every channel: the backward pass centres the
 * variance terms on them.  Everything else as bns_forward.
 * Errors as bns_forward, plus BNS_EINVAL for n_v outside [1, N-1], mix_beta outside [0, 1],
 * mode VDN, or a spec that is invalid for N - n_v samples.  Like bns_forward / bns_backward the two calls
 * take the single-launch kernels when a channel fits on chip and the streaming kernels otherwise
 * ("path" option, "last_path_forward" / "last_path_backward"). */
bns_status bns_sample_index_mixed(const bns_shape* shape, const bns_spec* spec, uint64_t seed, int32_t n_v,
                                  bns_box* boxes /* HOST, C entries: the sampled REAL set */);
bns_status bns_forward_mixed(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                             int32_t n_v, float mix_beta,
                             const void* x, const float* gamma, const float* beta,
                             float eps, float momentum,
                             void* y, float* save_mean, float* save_invstd, float* save_mean_parts,
                             float* running_mean, float* running_var,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Backward of bns_forward_mixed.  The paper prints none for Eq. 4; by the chain rule, in the form
 * of Eq. 5 / Eq. 6, with g = dl/dy, r = save_invstd, x^ = (x - E) r and dbeta, dgamma the sums over
 * all points as in bns_backward:
 *   dx_i = gamma r g_i - gamma r w (dbeta + r dgamma (x_i - E_set))
 * with (w, E_set) = (mix_beta / s_v, E[x_v]) on the virtual set, ((1 - mix_beta) / s_s, E[x_s]) on
 * the sampled real set, and w = 0 elsewhere. */
bns_status bns_backward_mixed(const bns_shape* shape, const bns_spec* spec, uint64_t seed,
                              int32_t n_v, float mix_beta,
                              const void* x, const void* dy, const float* gamma,
                              const float* save_mean, const float* save_invstd, const float* save_mean_parts,
                              void* dx, float* dgamma, float* dbeta,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Inference-mode normalisation (App. D): the statistics are the recorded moving averages of Eq. 8,
 *   y = gamma * (x - running_mean) / sqrt(running_var + eps) + beta        for all points.
 * in: x, gamma, beta, running_mean, running_var.  out: y. */
bns_status bns_inference(const bns_shape* shape, const void* x, const float* gamma, const float* beta,
                         const float* running_mean, const float* running_var, float eps, void* y, void* stream);

/* Weight of the new statistics in Eq. 8 at training iteration `iteration` (counted from 1): 1 at the first
 * iteration, where the moving average starts as a copy of the statistics, alpha afterwards.  The value to
 * pass as `momentum` to bns_forward / bns_forward_mixed.  HOST function, no device is touched; iteration 0
 * is treated as the first.  (Appendix D reports a larger alpha than the customary 0.1 to work better for
 * the noisier sampled statistics, so alpha is the caller's choice.) */
float bns_moving_average_weight(uint64_t iteration, float alpha);

/* Plain device-to-device copy of `bytes` bytes (a multiple of 16) with 128-bit accesses:
 * the "achievable bandwidth" yardstick that the benchmark reports beside the BN kernels,
 * and the known-size kernel that hardware traffic counters are calibrated against. */
bns_status bns_copy_reference(void* dst, const void* src, size_t bytes, void* stream);

/* Process-wide overrides of launch choices, for benchmarking and tests; value 0 restores the
 * automatic choice.  name: HOST string.  Returns BNS_EINVAL for an unknown name or a value out of range.
 *   "path"           1: only the streaming kernels (statistics / normalise / reduce / dx, several
 *                    launches per direction); 2: only the fused single-launch kernels, which keep a
 *                    channel in registers between its reduction and its element-wise pass
 *                    (BNS_EUNSUPPORTED if a channel does not fit or the layout is N x H x W x C, which has
 *                    none of these); 0: whichever is faster for the shape
 *   "fused_variant"  1..7: block size / registers-per-thread variant of the fused kernels
 *   "fused_pipe"     the backward kernel that holds two channels per block, loading the next one while the
 *                    sums of the current one are exchanged: 1..6 that (block size, vectors) variant whatever
 *                    the shape, 16 never; 0: when the launch has three or more rounds (tensors below 4 GiB)
 *   "fused_team"     blocks that share a channel in that kernel, if they can hold it    (1..128)
 *   "grouped"        the single-launch kernels that take groups of adjacent channels (N x C x H x W, small planes): 2 never,
 *                    1 whenever a group fits a block, 3..6 that block size; 0: where they are faster
 *   "grouped_channels"  channels per group in those kernels, if they can hold them (1..64)
 *   "resident"       the single-launch kernels of one block per compute unit (N x C x H x W, large tensors): 2 never, 1 whenever a
 *                    channel fits, 3 / 4 backward with dy alone / with x beside it on chip; 0: where they are faster
 *   "fused_coop"     1: launch the fused kernels with hipLaunchCooperativeKernel
 *   "fused_patch_mask"  Feature Sampling forward: by default, when one block holds a channel, the statistics of
 *                    the patch come from the vectors already in registers, under a column mask (built for the
 *                    two largest variants and rows that are a whole number of vectors); 1: also when several
 *                    blocks share a channel; 2: the patch elements are always read on their own, ahead of
 *                    the vectors
 *   "fused_keep_x"   the fused backward kernel keeps x in registers beside dy instead of reading it again
 *                    on S: 1 always, 2 never; 0: when S is the whole tensor or a patch of every plane
 *   "split_statistics"  1: the streaming forward statistics always run as partial sums + finalize
 *                    (by default one 1024-thread block per channel does both when a channel has few
 *                    sampled points)
 *   "splits_stats"   blocks per channel in the statistics reduction (implies split_statistics) (1..64; with
 *                    3073 to 3840 channels 48 at most are used)
 *   "splits_reduce"  blocks per channel in the backward reduction                (1..64; as above)
 *   "channel_group"  the streaming path walks the channels in groups of this many, every stage on
 *                    one group before the next                                   (1..C)
 *   "nhwc_fused"     the single-launch N x H x W x C kernels: 1 whenever they can run, 2 never; 0: few rows, or tensors beyond
 *                    4 MB that fit the registers about once.  Kernels whose blocks wait for each other (see Concurrency) are
 *                    not used while the stream is being captured in this layout, nor with "path" = 1
 *   "nhwc_fused_lanes"  128-bit accesses per row of a block's column tile in them  (1..32)
 *   "nhwc_blocks"    blocks that an N x H x W x C reduction launch aims for      (1..8192)
 *   "nhwc_ew_rows"   rows per thread in the N x H x W x C element-wise kernels   (1..2^20)
 *   "nhwc_split_dx"  the N x H x W x C backward writes dx on the rows outside S from its reduction kernel (Eq. 6
 *                    needs no sum there) and the rows of S from a kernel of their own: 1 always, with the bits of the stage calls;
 *                    2 never; 0: see "nhwc_split_ordered"
 *   "nhwc_split_ordered"  with "nhwc_split_dx" = 0 and "path" other than 1, bns_backward does so front to back, which adds the rows in another
 *                    order: 1 whenever it can (16-byte accesses), 2 never; 0: where it is the faster side (S at most a
 *                    quarter of the rows, tensors from 16 MB whose channels fill one, two, four or eight column tiles)
 *                    and the single launch does not run
 *   "cache_reuse"    streaming kernels: a first pass (statistics; the sums of Eq. 5) loads what the pass after it
 *                    (Eq. 1; Eq. 6) reads again without the non-temporal hint, so that it stays in the device's
 *                    memory-side cache: 1 all of it, 2 none; 0: as much as fits there (224 MB).  Results do not
 *                    depend on it (nor does the "nhwc_split_ordered" backward, which loads by a rule of its own).
 *   "nhwc_small"     2: N x H x W x C tensors of every size take the streaming kernels, as with "nhwc_fused" = 2
 *   "norm_unroll", "dx_unroll", "reduce_unroll"   128-bit accesses per thread    (1, 2, 4)
 *   "norm_nt", "dx_nt"   non-temporal access mask + 1: bit 0 loads, bit 1 stores
 *   "reduce_nt"      the same for the backward reduction: bit 0 loads of x, bit 1 loads of dy, for the channels
 *                    that "cache_reuse" keeps (the others are loaded non-temporally)
 * The loss over the vocabulary (bns_head_*; the workspace depends on them, so they are set before it is asked for):
 *   "head_logits", "head_logits_backward"   kernels of the logits in the forward and in the backward pass, "head_gradients" those of the two
 *                    gradients: 1 few tokens (gradients: from 33 tokens in fp32, 65 in bf16 on the choice by size holds), 2 / 3 operands read as they
 *                    lie in memory, tiles of 64 / 128, 4 / 5 operands laid out first, tiles of 256 / 128; 0: by size.  (Logits of 4 and 5 in the
 *                    backward pass need gradients of 1, 4 or 5; with others 3 takes their place.)
 *   "head_groups"    tiles of 64 share the steps along the summed dimension out between groups of waves: 1 always four, 2 never, 3 logits between two; 0: by size
 * Three more exist for the library's own tests only; they make results wrong on purpose and a caller has no
 * use for them:
 *   "test_spin_limit"    polls a block of a fused kernel waits for a team-mate's sums before it gives up
 *                    (1..2^21, the default)
 *   "test_mute_exchange" 1: no block publishes its sums, so every such wait runs out -- the two together let
 *                    a test reach the give-up path (NaN sums, the kernel ends normally) from the host
 *   "test_mute_channel"  c + 1: no block of an N x H x W x C kernel publishes its sums of channel c
 * The options are atomics: setting one while another thread launches work is defined (that call sees the old
 * or the new value), but the launch choices of calls in flight are then anyone's guess -- set them first.
 * Notes on the fused kernels: blocks of a team exchange partial sums through the workspace and wait
 * for each other with a bounded spin (the grid never exceeds what the device holds at once); they
 * are bit-reproducible like the streaming kernels, and they can be captured into a HIP graph like any other
 * launch (the stamps that tell one exchange from the next are counted in the workspace, on the device). */
bns_status bns_set_option(const char* name, int32_t value);
/* Current value of an option (as set, 0 = automatic); also, kept per calling thread,
 * "last_path_forward" / "last_path_backward": 1 if this thread's last bns_forward / bns_backward took the streaming kernels, 2 if the fused one, 3 if a
 * one-launch N x H x W x C kernel whose blocks do not wait for each other (few rows), 4 (backward, N x H x W x C) the streaming kernels with dx split
 * between the reduction kernel and a kernel for the rows of S ("nhwc_split_dx", "nhwc_split_ordered"); "last_fused_backward": which fused backward kernel that was
 * (1 plain, 2 x kept in registers, 3 pipelined, 4 groups of channels, 5 one block per compute unit); "last_fused_forward": 3 if groups of
 * channels, 4 if one block per compute unit,
 * 2 if the fused forward kernel took the statistics of a patch from the registers (see "fused_patch_mask"), else 1; "last_team_forward" /
 * "last_team_backward": blocks that shared a channel, or a column tile of N x H x W x C, in this thread's last single-launch call, "last_variant_forward" /
 * "last_variant_backward": the block size that it took, as in "fused_variant" (0: kernels that are not chosen by it); "launch_count": kernels launched by the library since it was
 * loaded, modulo 2^31 (benchmarks report launches per call from its differences).
 * -1 for an unknown name. */
int32_t bns_get_option(const char* name);

/* ---------------------------------------------------------------------------------------------------------------------
 * The last layers of a language model: the root-mean-square norm of the residual stream, the loss over the vocabulary
 * without its logits, and the loss against a teacher's top logits.
 *
 * The conventions at the top hold (device pointers of at least 16-byte alignment, the caller's workspace, work enqueued on
 * `stream`, one status, fp32 arithmetic, no floating-point atomics: results are bit-identical from run to run), with these additions.
 * Matrices are row-major; the strides are in elements from row to row, 0 stands for dense rows, anything else is at least the row's length
 * (rows may begin at any element).  A matrix of no rows is allowed: its pointers may be NULL and sums over it are zero.
 * Kernels here never wait for other blocks, keep nothing in the workspace from call to call and can be captured into a graph.
 * In place: an output may be the very tensor (address and stride) of an input where a function says so; any other overlap of an
 * output matrix with an input matrix or another output matrix is BNS_EINVAL.  Vectors and the workspace are the caller's duty. */

typedef enum { BNS_OUT_SAME = 0, BNS_OUT_E4M3 = 1 } bns_rms_out;

/* Rows of `width` elements.  Limits: rows < 2^31, width <= 16384, strides < 2^31. */
typedef struct {
    int64_t rows;
    int64_t x_stride;        /* x */
    int64_t residual_stride; /* residual; backward: dsum */
    int64_t sum_stride;      /* sum; backward: dx */
    int64_t y_stride;        /* y; backward: dy */
    int32_t width;
    int32_t dtype;        /* bns_dtype of x, residual, sum, dx, dy, dsum and, with BNS_OUT_SAME, y */
    int32_t weight_dtype; /* bns_dtype of weight */
    int32_t out;          /* bns_rms_out: the type of y (forward only) */
    int32_t group;        /* BNS_OUT_E4M3: 32, 64 or 128 neighbouring elements share a scale (the last group of a row may be
                             shorter), 0: the whole row does; else 0 */
    int32_t pow2_scales;  /* BNS_OUT_E4M3: 1: scales are rounded up to a power of two; else 0 */
    float eps;            /* >= 0 */
} bns_rms;

/* Residual addition and root-mean-square norm of every row:
 *   s = x + residual (s = x where residual is NULL)      rstd = 1 / sqrt(mean(s^2) + eps)      v = weight * s * rstd
 * s is held in fp32 on its way to the norm; sum receives it rounded to dtype.  So are the squares: where elements beyond 1.8e19 make their mean overflow, rstd is 0, and
 * with eps = 0 a row whose squares all underflow has rstd = infinity.
 * y = v rounded to dtype, or in 8 bits (OCP e4m3: 4 exponent bits, 3 mantissa bits, largest value 448) with
 *   scales[group] = max(max |v| / 448, 2^-126)           y = e4m3(v / scales[group]), round to nearest even
 * so that v = y * scales up to that rounding.  scales is float[rows][ceil(width / group)], dense (float[rows] for group = 0).
 * Elements that are NaN stay NaN in y; scales are those of the others.  An infinite v makes its group's scale infinite, its own y NaN and the others 0.
 * in: x, residual (may be NULL), weight[width].  out: sum (may be NULL; must be without residual), y, scales (BNS_OUT_E4M3, else NULL),
 * rstd[rows] (may be NULL).  In place: sum on x or on residual; y on x (BNS_OUT_SAME, no sum on it). */
bns_status bns_rms_forward(const bns_rms* rms, const void* x, const void* residual, const void* weight,
                           void* sum, void* y, float* scales, float* rstd, void* stream);

/* Bytes of workspace of bns_rms_backward; 0 for an invalid description. */
size_t bns_rms_workspace_bytes(const bns_rms* rms);

/* Gradients, with x the normalised rows (the forward call's sum, or its x where it had no residual), x^ = x * rstd:
 *   dx = rstd * (weight * dy - x^ * mean(weight * dy * x^)) + dsum            dweight = sum over the rows of dy * x^
 * dx is the gradient of x and of residual alike; dsum (may be NULL) is the gradient that reaches sum by its other uses.
 * (With BNS_OUT_E4M3 this is the gradient of v: the rounding to 8 bits counts as the identity.)
 * in: x, weight, rstd, dy, dsum.  out: dx, dweight[width].  In place: dx on dy or on dsum. */
bns_status bns_rms_backward(const bns_rms* rms, const void* x, const void* weight, const float* rstd,
                            const void* dy, const void* dsum, void* dx, float* dweight,
                            void* workspace, size_t workspace_bytes, void* stream);

/* `tokens` hidden states against a vocabulary.  Limits: tokens <= 2^20, width <= 65536, vocab < 2^24, strides < 2^31. */
typedef struct {
    int64_t tokens;
    int64_t hidden_stride; /* hidden (the gradients are dense) */
    int64_t weight_stride; /* weight */
    int32_t width;
    int32_t vocab;
    int32_t dtype;         /* bns_dtype of hidden, weight, dhidden, dweight */
    int32_t piece;         /* rows of weight that the workspace holds something for at a time; 0: the library's choice */
} bns_head;

/* Bytes of workspace of bns_head_forward and bns_head_backward (the larger of the two); 0 for an invalid description.  The backward pass needs most of it: a program
 * that only scores takes a small piece, which costs the forward pass nothing where hidden and weight need no copies (bf16, width and strides multiples of 64 and 8). */
size_t bns_head_workspace_bytes(const bns_head* head);

/* Softmax cross entropy of the logits z = hidden weight^T, which are never stored whole:
 *   lse[t] = log sum over v of exp(z[t][v])              loss[t] = lse[t] - z[t][targets[t]]
 * A token whose target lies outside [0, vocab) is left out: its loss is 0 (its lse is not).
 * Logits of -infinity count for nothing in the sum (as the target of a token that counts they make its loss infinite); a token with a logit that is NaN or +infinity
 * has a loss that is NaN (or infinite).
 * Products of bf16 are summed in fp32; f32 operands enter the matrix units as three bf16 parts each, the six products
 * that reach an fp32 result's last bits.
 * in: hidden[tokens][width], weight[vocab][width], targets[tokens].  out: loss[tokens], lse[tokens]. */
bns_status bns_head_forward(const bns_head* head, const void* hidden, const void* weight, const int64_t* targets,
                            float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of sum over t of dloss[t] * loss[t], with the logits computed again piece by piece:
 *   g[t][v] = dloss[t] * (exp(z[t][v] - lse[t]) - [v = targets[t]])      (0 for tokens that are left out, whatever they hold)
 *   dhidden = g weight                                                   dweight = g^T hidden
 * With bf16 operands g is rounded to bf16 before the two products, whose sums are fp32.
 * in: hidden, weight, targets, lse (of the forward call), dloss[tokens].  out: dhidden, dweight (dense). */
bns_status bns_head_backward(const bns_head* head, const void* hidden, const void* weight, const int64_t* targets,
                             const float* lse, const float* dloss, void* dhidden, void* dweight,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Rows of logits and, for each, `k` logits of a teacher.  Limits: tokens < 2^31, vocab < 2^30, 1 <= k <= 1024, strides < 2^31. */
typedef struct {
    int64_t tokens;
    int64_t logits_stride;  /* logits */
    int64_t dlogits_stride; /* dlogits */
    int32_t vocab;
    int32_t k;
    int32_t dtype;          /* bns_dtype of logits, dlogits */
    float temperature;      /* > 0 */
} bns_distill;

/* Distillation from a teacher's top logits.  With tau = temperature, over the row's entries j whose id lies in [0, vocab):
 *   q = softmax(teacher / tau)        p = softmax(logits / tau) over the vocabulary        lse = log sum exp(logits / tau)
 *   loss[t] = tau^2 * sum over j of q_j (log q_j - log p[id_j])
 * A row without such an entry has loss 0 and gradient 0, whatever its logits hold.  An id may occur more than once: its q add up in the gradient.
 * A teacher's logit of -infinity is no entry; one that is NaN or +infinity makes its row NaN, loss and gradient, and so does a logit of the student that is.  A student's
 * logit of -infinity has p = 0; with q > 0 there the loss is infinite.
 * dlogits = tau * dloss[t] * (p - q), in the same pass over the logits, where dlogits is given (then dloss is needed too).
 * in: logits[tokens][vocab], ids[tokens][k], teacher[tokens][k] (dense), dloss[tokens] (NULL without dlogits).
 * out: loss[tokens], lse[tokens], dlogits (may be NULL).  In place: dlogits on logits. */
bns_status bns_distill_forward(const bns_distill* distill, const void* logits, const int64_t* ids, const float* teacher,
                               const float* dloss, float* loss, float* lse, void* dlogits, void* stream);

/* The gradient on its own, from the lse of the forward call (probabilities carry its rounding, 2^-24 of |lse|; the forward call's own gradient does not).
 * in: logits, ids, teacher, lse, dloss.  out: dlogits.  In place: dlogits on logits. */
bns_status bns_distill_backward(const bns_distill* distill, const void* logits, const int64_t* ids, const float* teacher,
                                const float* lse, const float* dloss, void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BNS_H */
