/*
 * mv.h -- C ABI of the majority-voting vote step for AMD MI355X (gfx950).
 *
 * One call of mv_vote_step() is one iteration of sparse SGD with majority
 * voting for N workers whose vectors are held as an N x d matrix on one GPU
 * (paper: Algorithm 1, from the error compensation to the error update):
 *
 *   a[n][j]      = g[n][j] + e[n][j]                      (error compensation)
 *   worker_idx[n] = supp S_top(|a[n]|, K)                 (local mask, the vote)
 *   votes[j]     = #{ n : j in worker_idx[n] }            (vote count, Sec. 2)
 *   mask_idx     = supp S_top(votes, K)                   (global mask, Sec. 2 mask equation)
 *   agg[k]       = (sum_n a[n][mask_idx[k]]) * (1/N)      (masked send + aggregate; mean of Sec. 2)
 *   e[n][j]      = 0 if j in mask_idx else a[n][j]        (error update)
 *
 * S_top(x, K) marks the K entries with the highest values; the paper does not
 * say how ties are broken.  Here ties go to the LOWEST index, both for the
 * magnitudes of a row and for the vote counts.  "Highest absolute value" is the
 * order of the fp32 bit pattern with the sign bit cleared (so -0 == +0,
 * denormals are ordered and never flushed, and an infinity of either sign is
 * above all finite values; equal infinities tie like any equal magnitudes).
 * Infinite values are handled exactly as long as no NaN arises from them
 * (Inf - Inf in g + e or in the sum over workers).  NaN, given or arising, is
 * outside the contract: the values written are then unspecified (a NaN's
 * payload after an addition is the processor's choice); the call still ends,
 * every index written is a coordinate below d, index lists stay ascending and
 * nothing outside the output arrays is touched.
 *
 * All tensor pointers are DEVICE pointers owned by the caller.  The library
 * keeps none of them after a call returns, except cfg.workspace, which must
 * outlive the context.  Nothing throws; every entry point returns a status.
 */
#ifndef MV_H
#define MV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct mv_ctx mv_ctx; /* opaque */

typedef enum {
    MV_OK = 0,
    MV_ERR_INVALID_ARG = 1, /* null pointer, size out of range, misalignment, bad struct_size */
    MV_ERR_UNSUPPORTED = 2,
    MV_ERR_ALLOC = 3,       /* device or host allocation failed */
    MV_ERR_DEVICE = 4,      /* a HIP call failed */
    MV_ERR_STATE = 5        /* context already ended, or an earlier step on it failed with MV_ERR_DEVICE */
} mv_status;

typedef enum { MV_F32 = 0, MV_BF16 = 1 } mv_dtype;          /* dtype of g only; e and agg are fp32 */
typedef enum { MV_REDUCE_MEAN = 0, MV_REDUCE_SUM = 1 } mv_reduce;
/* mv_config.flags: the context also carries the scratch of mv_ad_vote_step */
#define MV_FLAG_ADD_DROP 1

typedef struct {
    uint32_t struct_size;   /* = sizeof(mv_config) */
    int32_t  device;        /* HIP device ordinal */
    int32_t  n_workers;     /* N, 1..255 (a vote count fits one byte) */
    int32_t  grad_dtype;    /* mv_dtype */
    int64_t  d;             /* coordinates per worker, 1 .. 2^31-1 */
    int64_t  k;             /* K, 1 .. d */
    int32_t  reduce;        /* mv_reduce; MEAN is Sec. 2's definition, SUM is Algorithm 1's last line */
    int32_t  flags;         /* MV_FLAG_* bits; unknown bits are refused */
    void*    workspace;     /* optional device scratch of >= mv_workspace_bytes(); NULL: the context allocates it */
    size_t   workspace_bytes;
} mv_config;

/*
 * Bytes of device scratch a context for this configuration needs.  Pure host
 * arithmetic, no device call.  Returns 0 if the configuration is invalid.
 */
size_t mv_workspace_bytes(const mv_config* cfg);

/*
 * Creates a context: validates cfg on the host first (no device call is made
 * for an invalid configuration), then allocates and zeroes the scratch.
 * cfg.workspace, when given, must be 256-byte aligned device memory.
 * Errors: MV_ERR_INVALID_ARG (null, struct_size, N, d, k, dtype, reduce,
 * unknown flags, workspace too small or misaligned), MV_ERR_ALLOC, MV_ERR_DEVICE.
 */
mv_status mv_begin(const mv_config* cfg, mv_ctx** out_ctx);

/*
 * One vote step (Algorithm 1, error compensation .. error update), enqueued on
 * `stream`; returns without waiting for the GPU and allocates nothing.
 *
 *   grads      device, N rows of d elements (fp32 or bf16 per cfg), row stride ld_g elements
 *   err        device, N rows of d fp32, row stride ld_e; in: e_t, out: e_{t+1} (in place)
 *   worker_idx device, N x K uint32 out, row n = the coordinates worker n votes for,
 *              ascending; may be NULL
 *   votes      device, d bytes out, votes[j] in 0..N; may be NULL
 *   mask_idx   device, K uint32 out, ascending
 *   agg_vals   device, K fp32 out, agg_vals[k] belongs to coordinate mask_idx[k]
 *   stream     hipStream_t, NULL = the default stream
 *
 * Only the first d elements of each row are read or written.  Row starts must
 * be 16-byte aligned: base pointers 16-byte aligned, ld_g a multiple of 4
 * (fp32) or 8 (bf16), ld_e a multiple of 4; mask_idx, agg_vals and worker_idx
 * 4-byte aligned.  The buffers must not overlap each other.
 *
 * Argument errors are found on the host before anything is enqueued, so err is
 * untouched when the call fails with MV_ERR_INVALID_ARG or MV_ERR_STATE.
 * Calls on one context must not overlap in time (one stream at a time); distinct
 * contexts are independent.  The result does not depend on earlier calls.
 */
mv_status mv_vote_step(mv_ctx* ctx,
                       const void* grads, int64_t ld_g,
                       float* err, int64_t ld_e,
                       uint32_t* worker_idx,
                       uint8_t* votes,
                       uint32_t* mask_idx,
                       float* agg_vals,
                       void* stream);

/*
 * One iteration of majority voting with random selection (paper: Algorithm 1, the
 * line with S_rand-weighted; Sec. 2, paragraph after Algorithm 1; Sec. 4.2),
 * enqueued on `stream` like mv_vote_step and with the same arguments, outputs and
 * error behaviour, except for how the mask is chosen: winners are drawn at random,
 * a coordinate's chance growing in proportion to its votes, until K distinct ones
 * are selected.  The paper names no sampler; here every voted coordinate j gets the
 * time rand_exp[j] / votes[j] (one correctly rounded fp32 division) and the K
 * soonest win, equal times going to the lowest coordinate.  With rand_exp[j]
 * independent Exp(1) variates this is that law (successive sampling without
 * replacement); the random numbers are the caller's, so a step is reproducible.
 *
 *   rand_exp   device, d fp32, non-negative and finite, 4-byte aligned; in.  Only the
 *              entries of voted coordinates are read.  Use fresh numbers every step.
 *   mask_idx   device, K uint32, ascending; out.  Every coordinate in it has a vote.
 *
 * worker_idx and votes (both optional) are those of mv_vote_step.  MV_ERR_INVALID_ARG
 * also for a null or misaligned rand_exp.
 */
mv_status mv_rs_vote_step(mv_ctx* ctx,
                          const void* grads, int64_t ld_g,
                          float* err, int64_t ld_e,
                          const float* rand_exp,
                          uint32_t* worker_idx,
                          uint8_t* votes,
                          uint32_t* mask_idx,
                          float* agg_vals,
                          void* stream);

/*
 * One iteration of majority voting with add-drop (paper: Algorithm 2, Sec. 3),
 * enqueued on `stream` like mv_vote_step.  The context must have been begun with
 * MV_FLAG_ADD_DROP (else MV_ERR_STATE).  Every worker keeps a standing vote
 * M~_n; per step at most k_ad coordinates join it (the k_ad largest |a| among
 * the worker's current top-K that are not in it) and at most k_ad leave it (the
 * k_ad smallest |a| among its members that are not in the current top-K), ties to
 * the lowest coordinate in both; M^sum, the sum of the standing votes, moves
 * with them, and the mask is the K most voted coordinates of M^sum.  The state is
 * the caller's (zero it to start; a first step with k_ad = K then is a plain
 * majority vote):
 *
 *   vote_bits  device, N rows of ld_bits 32-bit words, bit (j % 32) of word j / 32 of
 *              row n = M~_n[j]; in/out.  ld_bits >= ceil(d/32) rounded up to a multiple
 *              of 4, itself a multiple of 4; 16-byte aligned; at most K bits per row
 *   msum       device, d bytes rounded up to a multiple of 16 (the padding stays
 *              zero), 16-byte aligned; in: M^sum_{t-1}, out: M^sum_t
 *   k_ad       1 .. K
 *   add_idx    device, N x k_ad uint32 out: row n = the coordinates added to M~_n,
 *              ascending, counts[2n] of them valid
 *   drop_idx   device, N x k_ad uint32 out: the coordinates removed, counts[2n+1] valid
 *   counts     device, 2N uint32 out
 *   grads, err, mask_idx, agg_vals: as in mv_vote_step (err is updated with the mask
 *              of this step)
 *
 * Errors as mv_vote_step, plus MV_ERR_INVALID_ARG for k_ad, ld_bits, alignment or a
 * null state / output pointer.
 */
mv_status mv_ad_vote_step(mv_ctx* ctx,
                          const void* grads, int64_t ld_g,
                          float* err, int64_t ld_e,
                          int64_t k_ad,
                          uint32_t* vote_bits, int64_t ld_bits,
                          uint8_t* msum,
                          uint32_t* add_idx, uint32_t* drop_idx, uint32_t* counts,
                          uint32_t* mask_idx, float* agg_vals,
                          void* stream);

/*
 * Ends the context: waits for the stream of the context's last step (steps are
 * serialized by the caller, so that is the only one with work of this context
 * still in flight), frees scratch the context allocated
 * (never cfg.workspace).  The handle stays a valid pointer so that a later
 * mv_vote_step / mv_end on it reports MV_ERR_STATE; mv_release frees it.
 */
mv_status mv_end(mv_ctx* ctx);

/* Frees the handle itself (ends the context first if needed). NULL is allowed. */
void mv_release(mv_ctx* ctx);

/* Static string for a status code; never NULL, never freed. */
const char* mv_status_string(mv_status s);

/* ---- measurement hooks (not part of the method) ------------------------- */

/* Number of kernels one vote step launches, and their names (static strings). */
int32_t     mv_kernel_count(void);
const char* mv_kernel_name(int32_t i);

/*
 * level 0: no events (default).  level 1: the step records a pair of HIP
 * events around its dominant kernel (the streaming error-compensation pass).
 * level 2: a pair around every kernel.
 */
mv_status mv_set_profiling(mv_ctx* ctx, int32_t level);

/*
 * Inside the streaming kernel the wavefronts of a row wait for the row's threshold
 * estimate, which other workgroups of the same launch publish; the wait is bounded by
 * `polls` looks at memory (default 2^20, about a second), after which the wavefront
 * gives up and the row is selected exactly from memory instead.  The same bound holds
 * for the one other wait between workgroups: a block of the mask kernel waits for the
 * counts of the blocks before it, and if it gives up the kernel behind it finds the
 * mask from the counts instead.  Results never depend on the bound.  A test hook: 0
 * makes every waiter that does not find what it needs at its first look give up, which
 * forces both alternative paths without any kernel waiting.
 */
mv_status mv_set_spin_limit(mv_ctx* ctx, uint32_t polls);

/*
 * Durations, in milliseconds, of the kernels of the step enqueued `steps_back`
 * steps ago on this context (0 = the last one; the last 64 steps are kept),
 * one per kernel in mv_kernel_name order, -1 for kernels that were not
 * bracketed at the level then in force.  Waits for that step's events.  `ms`
 * is a HOST array of n >= mv_kernel_count() floats.
 */
mv_status mv_step_kernel_ms(mv_ctx* ctx, int32_t steps_back, float* ms, int32_t n);

/*
 * Diagnostics of the LAST step (waits for the stream the step ran on): per
 * worker row, how many candidates the streaming pass kept (cand_count), the
 * magnitude bit pattern it compared against (threshold_bits) and how the row's
 * K-th magnitude was found (slow_path: 0 = from the candidates through their
 * fine histogram, 2 = the generic select over the candidates, 1 = the slow exact
 * path over the whole row in memory).  A cand_count with its top bit set marks a row
 * whose wavefronts did not all see the threshold in time (see mv_set_spin_limit).
 * Rows of at most 32,768 coordinates are selected without an estimate: d, 0 and 0.
 * HOST arrays of N uint32 each; any may be NULL.
 */
mv_status mv_last_step_row_stats(mv_ctx* ctx, uint32_t* cand_count,
                                 uint32_t* threshold_bits, uint32_t* slow_path);

/* ---- sparse position code (paper: Sec. 4.3.1) ------------------------------ */

/*
 * The code of an ascending list of n coordinates of a d-vector: the coordinates
 * are cut into blocks of block_len = 1/phi; per listed coordinate a 1 bit and the
 * position inside its block in B = ceil(log2(block_len)) bits, most significant
 * first; a 0 bit closes every block (also empty ones and the last, shorter one).
 * Bit k of a stream is bit k % 32 of its 32-bit word k / 32; unused bits of the
 * last word are 0.  A stream has n (1 + B) + ceil(d / block_len) bits, i.e.
 * log2(1/phi) + 2 bits per coordinate when n = phi d (Sec. 2.1).
 * Returns that length in bits (host arithmetic), 0 for invalid arguments.
 */
uint64_t mv_codec_stream_bits(int64_t n, int64_t d, int64_t block_len);

/* Bytes of device scratch mv_codec_decode needs for `rows` streams of up to max_bits bits. */
size_t mv_codec_scratch_bytes(uint64_t max_bits, int32_t rows);

/*
 * Encodes `rows` lists at once (for instance the N workers' votes), enqueued on
 * `stream`; allocates nothing.
 *   idx       device, row r = idx + r * ld_idx: ascending coordinates < d
 *   counts    device or NULL: the length of row r is counts[r * counts_stride]
 *             (a value above n is read as n); NULL: every row holds n coordinates
 *   streams   device out, row r = streams + r * ld_words; ld_words >=
 *             ceil(mv_codec_stream_bits(n, d, block_len) / 32); words beyond a
 *             row's stream are left untouched
 *   n_bits    device out, rows entries: the length of each stream in bits
 * Lists that are not ascending or reach beyond d give an unspecified stream (no
 * out-of-bounds access).  Errors: MV_ERR_INVALID_ARG, MV_ERR_DEVICE.
 */
mv_status mv_codec_encode(const uint32_t* idx, int64_t ld_idx, const uint32_t* counts, int64_t counts_stride,
                          int64_t n, int32_t rows, int64_t d, int64_t block_len, uint32_t* streams,
                          int64_t ld_words, uint64_t* n_bits, void* stream);

/*
 * Decodes `rows` streams as the receiver of Sec. 4.3.1 reads them (a 1 bit: the
 * next B bits are a position inside the current block; a 0 bit: next block).
 *   streams, ld_words   device, as written by mv_codec_encode
 *   n_bits    device, rows entries: the length of each stream in bits (a value above
 *             max_bits is read as max_bits)
 *   idx_out   device out, row r = idx_out + r * ld_idx, room for max_n coordinates
 *   counts_out device out, rows entries: coordinates found in each stream (those
 *             beyond max_n are counted but not written)
 *   scratch   device, >= mv_codec_scratch_bytes(max_bits, rows) bytes
 * Malformed streams give unspecified lists (no out-of-bounds access).
 */
mv_status mv_codec_decode(const uint32_t* streams, int64_t ld_words, const uint64_t* n_bits, uint64_t max_bits,
                          int32_t rows, int64_t d, int64_t block_len, uint32_t* idx_out, int64_t ld_idx,
                          int64_t max_n, uint32_t* counts_out, void* scratch, size_t scratch_bytes, void* stream);

/*
 * mv_codec_decode for callers that cannot allocate device memory and have no
 * scratch buffer to hand over: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, results and errors as
 * mv_codec_decode without `scratch` / `scratch_bytes`: the decoder's tables live
 * in an array of MV_CODEC_STATIC_SCRATCH_BYTES bytes that is part of the
 * library's device code (every GPU the library runs on holds its own copy from
 * the first call on it until the process ends).  The call allocates and frees
 * nothing, on the device or through any library.
 *   - mv_codec_scratch_bytes(max_bits, rows) must not exceed
 *     MV_CODEC_STATIC_SCRATCH_BYTES, else MV_ERR_UNSUPPORTED (nothing is enqueued);
 *     MV_ERR_UNSUPPORTED also for a device number of 64 or more.
 *   - The array is shared by every call on a GPU, whatever the stream: two calls
 *     that may overlap in time on one GPU race on it and must be ordered by the
 *     caller (same stream, or an event between them).  mv_codec_decode with
 *     buffers of its own has no such limit.
 *   - Runs on the CURRENT device, enqueued on `stream`.
 */
#define MV_CODEC_STATIC_SCRATCH_BYTES (16u << 20)
mv_status mv_codec_decode_static(const uint32_t* streams, int64_t ld_words, const uint64_t* n_bits,
                                 uint64_t max_bits, int32_t rows, int64_t d, int64_t block_len, uint32_t* idx_out,
                                 int64_t ld_idx, int64_t max_n, uint32_t* counts_out, void* stream);

/* ---- fractional quantisation (paper: Sec. 4.3.2) --------------------------- */

/*
 * q bits per value (2 <= q <= 8): q-1 bits name one of L = 2^(q-1) geometric
 * intervals of |v| between the row's largest and smallest non-zero magnitude,
 * I_l = [v_max / alpha^(l-1), v_max / alpha^l], alpha = (v_max / v_min)^(1/L); one
 * bit is the sign; L means of the magnitudes that fell into the intervals follow
 * and the receiver reproduces sign * mean.  The paper leaves the arithmetic of the
 * edges open; here they are fp64 numbers from correctly rounded operations only
 * (alpha by q-1 square roots of v_max / v_min, edge_l = edge_{l-1} / alpha), a value
 * on an edge goes to the interval of the smaller magnitudes and zeros to the last.
 *   vals      device, `rows` rows of n fp32 values, row stride ld_vals
 *   streams   device out, row stride ld_words >= ceil(n q / 32): value k occupies
 *             bits [k q, (k+1) q) of its row's stream (bit b = bit b % 32 of word
 *             b / 32), code = (interval - 1) | sign << (q - 1)
 *   means     device out, rows x L fp32 (0 for an empty interval)
 *   scratch   device, >= mv_quant_scratch_bytes(n, rows, q)
 * Enqueued on `stream`; allocates nothing.
 */
size_t    mv_quant_scratch_bytes(int64_t n, int32_t rows, int32_t q);
mv_status mv_quant_encode(const float* vals, int64_t ld_vals, int64_t n, int32_t rows, int32_t q,
                          uint32_t* streams, int64_t ld_words, float* means, void* scratch, size_t scratch_bytes,
                          void* stream);
/* out[r][k] = +-means[r][interval of value k], row stride ld_out >= n. */
mv_status mv_quant_decode(const uint32_t* streams, int64_t ld_words, int64_t n, int32_t rows, int32_t q,
                          const float* means, float* out, int64_t ld_out, void* stream);

/* ---- gradient norm over many tensors, and clipping ------------------------- */

/*
 * A program has every worker's gradients as a list of tensors; the vote step takes
 * them as rows of a matrix.  For each group g of tensors (a worker's, as a rule):
 *
 *   norm[g] = sqrt(sum of x^2) or max |x| over all elements of the group's tensors
 *   coef[g] = min(1, max_norm / (norm[g] + 1e-6))          (fp32)
 *   dst     = src * coef[g]                                (fp32, rounded once to dst's type)
 *
 * Sums of squares are formed in fp64, so no square leaves the range, in an order that
 * follows from the list (all groups' sizes and types) and never from timing: equal lists
 * of equal values give equal norms.  A NaN makes the group's norm, coef and every dst NaN; an infinity makes norm
 * infinite and coef 0 (dst: NaN where src is infinite or NaN, else 0), and so do finite
 * values whose norm is beyond fp32 (dst: 0): look at norm before the result is used, as
 * with any clipping.  A group without elements has norm 0.
 *
 * Tensors are contiguous and aligned to their own element; numel 0 (then the pointers may be NULL) is
 * allowed.  A list has fewer than 2^24 chunks: 32 KB of src each, every tensor's rounded up, and one
 * more for each group that has elements (2^37 fp32 or 2^38 bf16 values, less what rounding takes).
 * dst is a tensor of its own -- a part of a matrix row at any offset, for instance -- or src itself, if
 * the types agree; apart from that no dst overlaps another tensor.  dst NULL: the tensor only counts for
 * its group's norm; then all tensors' must be NULL, and mv_clip_grads reports MV_ERR_STATE.
 */
typedef struct mv_clip mv_clip; /* opaque */

typedef enum { MV_NORM_L2 = 0, MV_NORM_MAX = 1 } mv_norm;

typedef struct {
    const void* src;
    void*       dst;
    int64_t     numel;
    int32_t     group;      /* 0 .. n_groups-1; in any order */
    int16_t     src_dtype;  /* mv_dtype */
    int16_t     dst_dtype;  /* mv_dtype */
} mv_clip_tensor;

typedef struct {
    uint32_t struct_size;   /* = sizeof(mv_clip_config) */
    int32_t  device;        /* HIP device ordinal */
    int32_t  n_groups;      /* 1 .. 65535 */
    int32_t  norm;          /* mv_norm */
    void*    workspace;     /* optional device scratch of >= mv_clip_workspace_bytes(); NULL: the handle allocates it */
    size_t   workspace_bytes;
} mv_clip_config;

/* Bytes of device scratch for this list; host arithmetic, 0 if anything is invalid.  `tensors` is a HOST array. */
size_t mv_clip_workspace_bytes(const mv_clip_config* cfg, const mv_clip_tensor* tensors, int64_t n_tensors);

/*
 * Creates a handle for a list of 1 .. 2^24 tensors (a HOST array, copied).  The handle
 * holds the tensors' ADDRESSES: they have to stay where they are until mv_clip_bind
 * gives new ones or the handle ends.  What they hold is read by each call anew.
 * cfg.workspace, when given, must be 256-byte aligned device memory and outlive the
 * handle.  Waits for the upload of the list.
 * Errors: MV_ERR_INVALID_ARG (before any device call), MV_ERR_ALLOC, MV_ERR_DEVICE.
 */
mv_status mv_clip_begin(const mv_clip_config* cfg, const mv_clip_tensor* tensors, int64_t n_tensors, mv_clip** out);

/*
 * Gives the tensors new addresses (HOST arrays of n_tensors pointers, in the order of
 * mv_clip_begin; sizes, types and groups stay; dst NULL where the list had none),
 * enqueued on `stream`: calls enqueued before use the old ones.  Allocates nothing.
 */
mv_status mv_clip_bind(mv_clip* clip, const void* const* src, void* const* dst, void* stream);

/*
 * Enqueues the norms of all groups on `stream`: norms = device, n_groups fp32 out.
 * Calls on one handle must not overlap in time; like mv_vote_step they return without
 * waiting and allocate nothing.
 */
mv_status mv_clip_norms(mv_clip* clip, float* norms, void* stream);

/*
 * Enqueues norms and clipping.  max_norm: finite, >= 0.  norms: device, n_groups fp32 out.
 * coefs: the same, out, the factors that were applied; may be NULL.  Tensors clipped in place whose
 * factor is 1 are not written.
 */
mv_status mv_clip_grads(mv_clip* clip, float max_norm, float* norms, float* coefs, void* stream);

/*
 * Where a group fits the GPU's registers, its gradients are read once: workgroups of one
 * launch then wait for each other's sums, for at most `polls` looks at memory (default
 * 512, about 0.5 ms); what is not done then the launch behind does, which happens where
 * another stream's work holds part of the GPU meanwhile and costs a call up to that wait
 * for each group and a second reading.  Results never depend on it.  A test hook: 0 makes
 * everyone who does not find what it needs at once give up.
 */
mv_status mv_clip_set_spin_limit(mv_clip* clip, uint32_t polls);

/* As mv_end and mv_release: waits for the stream of the last call, frees the handle's scratch; frees the handle. */
mv_status mv_clip_end(mv_clip* clip);
void      mv_clip_release(mv_clip* clip);

/* ---- microscaled 4-bit floating point ---------------------------------------- */

/*
 * Every 32 consecutive values of a row (a block; the row's last one may be shorter)
 * share a power of two, 2^s with s = floor(log2(largest magnitude)) - 2, at least -127;
 * a scale byte holds s + 127.  A value is held as a 4-bit code, sign << 3 | place, for
 * +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}[place] * 2^s: the nearest one, ties to the even place,
 * magnitudes beyond 6 to 6.  A block of zeros has s = -127.  A block that holds an infinity or a NaN gets
 * the scale byte 255 and codes 0: all of it reads as NaN.
 *
 * Layout: value k of a row is bits [4 (k % 8), 4 (k % 8) + 4) of 32-bit word k / 8.  Rows are whole
 * blocks: mv_mx_row_words(n) = 4 ceil(n / 32) words, the codes past n are 0, and
 * mv_mx_row_scales(n) = ceil(n / 32) rounded up to 4 scale bytes, those past the last
 * block are neither written nor used.  Codes are 16-byte aligned, ld_words a multiple
 * of 4; scales 4-byte aligned, ld_scales a multiple of 4.
 * Values (vals, resid, out, x, y, ...) are fp32 or bf16, aligned to their element, with
 * any row stride >= the row; 1 <= rows, n < 2^31.  Besides, MV_ERR_INVALID_ARG is what a
 * call gets beyond
 *   2^34 - 2^14 values in whole blocks, where rows are quantised or read back;
 *   2^24 - 1 tiles of 128 rows by 64 columns (bf16: by 128), where columns are quantised;
 *   2^24 - 1 of such tiles of x, of dy, and of dy's blocks by 32 (bf16: by 128), all added
 *   up, in mv_mx_linear_grad;
 * and may get from 2^23 tiles of 128 x 128 results of a product on.
 * All of these calls run on the CURRENT device, are enqueued on `stream` and allocate
 * nothing.  Errors: MV_ERR_INVALID_ARG, MV_ERR_DEVICE.
 */
int64_t mv_mx_row_words(int64_t n);   /* 0 for n outside 1 .. 2^31-1 */
int64_t mv_mx_row_scales(int64_t n);

/*
 * codes, scales = the rows of vals.  resid (fp32, may be NULL; may be vals itself, with its
 * stride, if vals is fp32) = vals minus what the codes stand for, exact: what an error
 * buffer keeps.
 */
mv_status mv_mx_encode(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint32_t* codes,
                       int64_t ld_words, uint8_t* scales, int64_t ld_scales, float* resid, int64_t ld_resid,
                       void* stream);

/* codes, scales = the COLUMNS of vals (rows x n): n rows of codes of `rows` values each. */
mv_status mv_mx_encode_t(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint32_t* codes,
                         int64_t ld_words, uint8_t* scales, int64_t ld_scales, void* stream);

/* out (rows x n, fp32 or bf16) = what the codes stand for. */
mv_status mv_mx_decode(const uint32_t* codes, int64_t ld_words, const uint8_t* scales, int64_t ld_scales, int64_t rows,
                       int64_t n, void* out, int32_t dtype, int64_t ld_out, void* stream);

/*
 * What the receiver of the rows (the workers' values) forms, without writing them out:
 *   agg[k] = sum over rows r of weights[r] * value[r][k]    fp32, r ascending
 * weights: device, rows fp32; NULL: the mean, the plain sum times fp32 1 / rows.
 */
mv_status mv_mx_aggregate(const uint32_t* codes, int64_t ld_words, const uint8_t* scales, int64_t ld_scales,
                          int64_t rows, int64_t n, const float* weights, float* agg, void* stream);

/*
 * c[i][j] = sum over k of a[i][k] * b[j][k]: m rows of a, n rows of b, k values each,
 * all in 4 bits along k; fp32 sums; c fp32 or bf16.  Here and in a layer's calls the order
 * of the sums follows from the arguments (sizes, types, strides, which results are asked
 * for) and never from timing: equal calls give equal results, other ones equal sums up to
 * rounding.  scratch: device, 16-byte aligned, >= mv_mx_product_scratch_bytes(m, n, k) (0: may be NULL).
 */
size_t    mv_mx_product_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_mx_product(const uint32_t* a_codes, int64_t ld_aw, const uint8_t* a_scales, int64_t ld_as,
                        const uint32_t* b_codes, int64_t ld_bw, const uint8_t* b_scales, int64_t ld_bs, int64_t m,
                        int64_t n, int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* scratch,
                        size_t scratch_bytes, void* stream);

/*
 * A layer with weights w (n x k) held in 4 bits along k:
 *   y (m x n) = q(x) w^T,  q(x) = what mv_mx_encode makes of x (m x k).
 */
size_t    mv_mx_linear_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_mx_linear(const void* x, int32_t x_dtype, int64_t ld_x, const uint32_t* w_codes, int64_t ld_words,
                       const uint8_t* w_scales, int64_t ld_scales, int64_t m, int64_t n, int64_t k, void* y,
                       int32_t y_dtype, int64_t ld_y, void* scratch, size_t scratch_bytes, void* stream);

/*
 * Its gradients from dy (m x n), each product with both factors in 4 bits along its own
 * sum (rounding is passed straight through):
 *   dx (m x k) = q(dy) wt^T            wt: the weights' COLUMNS, k rows of n values (mv_mx_encode_t of w)
 *   dw (n x k) = qt(dy) qt(x)^T        qt: mv_mx_encode_t
 * dx or dw may be NULL (then x, or wt_codes and wt_scales, may be too); x and dy have the same type.
 */
size_t    mv_mx_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_mx_linear_grad(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype,
                            const uint32_t* wt_codes, int64_t ld_words, const uint8_t* wt_scales, int64_t ld_scales,
                            int64_t m, int64_t n, int64_t k, void* dx, int32_t dx_dtype, int64_t ld_dx, void* dw,
                            int32_t dw_dtype, int64_t ld_dw, void* scratch, size_t scratch_bytes, void* stream);

/* ---- 8-bit floating point by blocks of 128 ----------------------------------- */

/*
 * Every 128 consecutive values of a row (a block; the row's last one may be shorter)
 * share a power of two, 2^s with s the smallest whole number for which the largest
 * magnitude is at most 448 * 2^s, and at least -127; a scale byte holds s + 127.  A value
 * is held as an 8-bit code, sign << 7 | e << 3 | f, for +-(8 + f) 2^(e - 10) * 2^s, or where
 * e is 0 +-f 2^-9 * 2^s: the nearest one, ties to the even f; no code is 0x7F or 0xFF.  A
 * block of zeros has s = -127.  A block that holds an infinity or a NaN gets the scale
 * byte 255 and codes 0: all of it reads as NaN.
 *
 * Layout: value k of a row is its byte k.  Rows are whole blocks: mv_f8_row_bytes(n) =
 * 128 ceil(n / 128) bytes, the codes past n are 0, and mv_f8_row_scales(n) = ceil(n / 128)
 * rounded up to 4 scale bytes, those past the last block are neither written nor used.
 * Codes are 16-byte aligned, ld_bytes a multiple of 16; scales 4-byte aligned, ld_scales a
 * multiple of 4.  Codes that a program makes itself must not be 0x7F or 0xFF.
 * Values, strides, sizes, devices, streams and errors are those of the 4-bit calls.
 * MV_ERR_INVALID_ARG is also what a call gets beyond
 *   2^36 - 2^16 values in whole blocks, where rows are quantised or read back;
 *   2^24 - 1 tiles of 128 rows by 64 columns (bf16: by 128), where columns are quantised;
 *   2^24 - 1 of such tiles of x, of dy, and of dy's blocks by 32, all added up, in
 *   mv_f8_linear_grad;
 * and may get from 2^23 tiles of 128 x 128 results of a product on.
 */
int64_t mv_f8_row_bytes(int64_t n);    /* 0 for n outside 1 .. 2^31-1 */
int64_t mv_f8_row_scales(int64_t n);

/* codes, scales = the rows of vals. */
mv_status mv_f8_encode(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint8_t* codes,
                       int64_t ld_bytes, uint8_t* scales, int64_t ld_scales, void* stream);

/* codes, scales = the COLUMNS of vals (rows x n): n rows of codes of `rows` values each. */
mv_status mv_f8_encode_t(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint8_t* codes,
                         int64_t ld_bytes, uint8_t* scales, int64_t ld_scales, void* stream);

/* out (rows x n, fp32 or bf16) = what the codes stand for. */
mv_status mv_f8_decode(const uint8_t* codes, int64_t ld_bytes, const uint8_t* scales, int64_t ld_scales, int64_t rows,
                       int64_t n, void* out, int32_t dtype, int64_t ld_out, void* stream);

/*
 * c[i][j] = sum over k of a[i][k] * b[j][k], as mv_mx_product, in 8 bits along k; the order
 * of the sums follows from the arguments, as there.  An fp32 c is a sum in fp32 (a factor's
 * value counts to the nearest multiple of 2^-133, and from 2^128 on, which scale bytes from 247 on
 * reach and a quantised value from 248 * 2^120 on, as infinite: c is right or not finite then, in
 * bf16, too).  A bf16 c may come from matrix instructions that add eight neighbouring products at
 * a time on a grid of 2^-13 of the largest one, cut towards zero, and those sums in fp32: off by
 * at most 7 * 2^-13 of the magnitudes' sum before it is rounded to bf16.  Of normal values that is
 * 2^-17 (k = 8) to 2^-22 (k = 8192) of it in the root of the mean square, and has been up to 2^-12.7
 * and 2^-18.5.
 * scratch: device, 16-byte aligned, >= mv_f8_product_scratch_bytes(m, n, k) (0: may be NULL).
 * Here and below it is a call's alone until the call's work has ended: calls, or graphs that
 * hold them, that may run at the same time have one each.  No output overlaps another argument.
 */
size_t    mv_f8_product_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_f8_product(const uint8_t* a_codes, int64_t ld_ab, const uint8_t* a_scales, int64_t ld_as,
                        const uint8_t* b_codes, int64_t ld_bb, const uint8_t* b_scales, int64_t ld_bs, int64_t m,
                        int64_t n, int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* scratch,
                        size_t scratch_bytes, void* stream);

/* A layer with weights w (n x k) held in 8 bits along k:  y (m x n) = q(x) w^T,  q: mv_f8_encode. */
size_t    mv_f8_linear_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_f8_linear(const void* x, int32_t x_dtype, int64_t ld_x, const uint8_t* w_codes, int64_t ld_bytes,
                       const uint8_t* w_scales, int64_t ld_scales, int64_t m, int64_t n, int64_t k, void* y,
                       int32_t y_dtype, int64_t ld_y, void* scratch, size_t scratch_bytes, void* stream);

/*
 * Its gradients from dy (m x n), as mv_mx_linear_grad's:
 *   dx (m x k) = q(dy) wt^T            wt: the weights' COLUMNS, k rows of n values (mv_f8_encode_t of w)
 *   dw (n x k) = qt(dy) qt(x)^T        qt: mv_f8_encode_t
 * dx or dw may be NULL (then x, or wt_codes and wt_scales, may be too); x and dy have the same type.
 */
size_t    mv_f8_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k);
mv_status mv_f8_linear_grad(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype,
                            const uint8_t* wt_codes, int64_t ld_bytes, const uint8_t* wt_scales, int64_t ld_scales,
                            int64_t m, int64_t n, int64_t k, void* dx, int32_t dx_dtype, int64_t ld_dx, void* dw,
                            int32_t dw_dtype, int64_t ld_dw, void* scratch, size_t scratch_bytes, void* stream);

/* ---- layer norm ---------------------------------------------------------------- */

/*
 * For every row x of n values (fp32 or bf16, aligned to its element, any row stride >= n):
 *
 *   mean = sum(x) / n,  rstd = 1 / sqrt(sum((x - mean)^2) / n + eps)
 *   y    = (x - mean) rstd gamma + beta            rounded once to y's type
 *
 * gamma, beta: n values of one type, or NULL for 1 and 0 (either).  mean, rstd: rows fp32
 * out, what the backward pass takes; either may be NULL.  y may be x itself, with its type
 * and stride.  Sums are fp32; the squares are those of differences from the mean, so rows far from
 * zero keep their digits.  A row that holds an infinity or a NaN, or whose sums leave fp32, has no
 * finite y and rstd, and no other row's are touched by it.  eps >= 0 and finite; with eps 0 a row of
 * equal values has an infinite rstd, or one as large as its mean's rounding makes it, and so has a row
 * whose squared differences are too small for fp32.
 *
 * These calls run on the CURRENT device, are enqueued on `stream` and allocate nothing.
 * 1 <= rows, n < 2^31.  The order of all sums follows from sizes and types: equal calls
 * give equal results.  Errors: MV_ERR_INVALID_ARG, MV_ERR_DEVICE.
 */
mv_status mv_layernorm_forward(const void* x, int32_t x_dtype, int64_t ld_x, int64_t rows, int64_t n, const void* gamma,
                               const void* beta, int32_t weight_dtype, float eps, void* y, int32_t y_dtype, int64_t ld_y,
                               float* mean, float* rstd, void* stream);

/*
 * The gradients, with h = (x - mean) rstd and d = dy gamma:
 *
 *   dx     = rstd (d - sum(d) / n - h sum(d h) / n)     rounded once to dx's type
 *   dgamma = sum over rows of dy h,  dbeta = sum over rows of dy      (n fp32 each)
 *
 * x and dy have the same type; mean, rstd as the forward pass left them.  A row whose mean times
 * rstd is beyond fp32 (equal values, very large) may have no finite dx.  dx, dgamma and
 * dbeta may each be NULL, not all three; dx may be dy or x itself, with its type and stride.
 * Apart from that no output overlaps another argument, as in the forward pass.  scratch:
 * device, 16-byte aligned, >= mv_layernorm_scratch_bytes(rows, n), one for each call, or graph
 * that holds calls, that may run at the same time as others.
 */
size_t    mv_layernorm_scratch_bytes(int64_t rows, int64_t n);   /* 0 for sizes outside 1 .. 2^31-1 */
mv_status mv_layernorm_backward(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype, int64_t rows,
                                int64_t n, const void* gamma, int32_t weight_dtype, const float* mean, const float* rstd,
                                void* dx, int32_t dx_dtype, int64_t ld_dx, float* dgamma, float* dbeta, void* scratch,
                                size_t scratch_bytes, void* stream);

/* ---- distillation from a teacher's top logits ---------------------------------- */

/*
 * A worker that learns from a teacher gets, for each row of its own n logits z, the
 * teacher's best ones: `top` coordinates idx[j] and logits t[j].  With a temperature T > 0,
 *
 *   q = softmax(z / T),  s = softmax(z),  p = softmax(t / T) over the row's list
 *   loss  = soft T^2 sum_j p_j (log p_j - log q[idx_j])  +  hard (-log s[label])
 *   dz[v] = g ( soft T (P q[v] - sum_{j: idx_j = v} p_j)  +  hard (s[v] - [v = label]) )
 *
 * An entry whose idx is outside 0 .. n-1 is not in the list (so shorter lists are filled
 * with -1), one whose t is -infinity has p = 0 and no part in the sums; P is 1, or 0 for a
 * list with neither, which has no first term.  A coordinate listed twice counts twice.  A label
 * outside 0 .. n-1, or labels NULL, has no second term; neither has a term a weight of 0.
 * A row without terms has loss 0 and dz 0, whatever its logits are.  A logit of
 * -infinity has q = s = 0 (an infinite loss where the teacher lists it); NaN, +infinity or
 * nothing but -infinity among a row's logits, and NaN or +infinity in its list, make loss and
 * dz NaN, of this row only.
 *
 *   logits      rows x n, fp32 or bf16, any row stride >= n
 *   idx, t      rows x top; int32, and fp32 or bf16; any row strides >= top; top 0 .. 4096,
 *               with 0 (or soft 0) both may be NULL
 *   labels      rows int32 or NULL
 *   loss        rows fp32 out; may be NULL where dz is wanted
 *   stats       rows x 3 fp32 out or NULL: the largest z, sum exp((z - largest) / T) and
 *               sum exp(z - largest); 0 for a sum that no row needs (soft 0 or top 0; hard 0
 *               or labels NULL)
 *   grad        rows fp32 or NULL for 1: g, the gradient that arrives at each loss
 *   dz          rows x n out, fp32 or bf16, or NULL; may be logits itself, with its type
 *               and stride
 *
 * mv_distill_loss forms loss and, where dz is wanted, the gradient in the same call;
 * mv_distill_grad forms the gradient alone from the stats of a call with the same logits,
 * lists, labels and weights: q = exp((z - stats[0]) / T) / stats[1], s = exp(z - stats[0]) /
 * stats[2].  Sums are fp32 in an order that follows from sizes and types.  soft and hard are
 * finite, T is 2^-60 .. 2^60.  1 <= rows, n < 2^31.  Runs on the CURRENT device, enqueued on
 * `stream`; allocates nothing.  Apart from dz over logits no output overlaps another argument.
 * scratch: device, 16-byte aligned, >= mv_distill_scratch_bytes(rows, n) (0: may be NULL), one
 * for each call, or graph that holds calls, that may run at the same
 * time as others.
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_DEVICE.
 */
size_t    mv_distill_scratch_bytes(int64_t rows, int64_t n);
mv_status mv_distill_loss(const void* logits, int32_t dtype, int64_t ld_z, int64_t rows, int64_t n, const int32_t* idx,
                          int64_t ld_idx, const void* t, int32_t t_dtype, int64_t ld_t, int64_t top, const int32_t* labels,
                          float temperature, float soft, float hard, float* loss, float* stats, const float* grad, void* dz,
                          int32_t dz_dtype, int64_t ld_dz, void* scratch, size_t scratch_bytes, void* stream);
mv_status mv_distill_grad(const void* logits, int32_t dtype, int64_t ld_z, int64_t rows, int64_t n, const int32_t* idx,
                          int64_t ld_idx, const void* t, int32_t t_dtype, int64_t ld_t, int64_t top, const int32_t* labels,
                          float temperature, float soft, float hard, const float* stats, const float* grad, void* dz,
                          int32_t dz_dtype, int64_t ld_dz, void* stream);

/*
 * Measurement aid, not part of the method: enqueues a plain streaming copy of
 * `bytes` (a multiple of 16; dst and src 16-byte aligned DEVICE pointers, not
 * overlapping) on `stream` of the current device.  Its achieved bandwidth is
 * the yardstick for the streaming pass, and its known byte count calibrates the
 * profiler's memory counters.
 */
mv_status mv_probe_copy(void* dst, const void* src, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MV_H */
