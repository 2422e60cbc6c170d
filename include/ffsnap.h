/*
 * ffsnap.h -- C ABI of the MI355X snapshot library (libffsnap.so).
 *
 * The library implements the data-moving step of FFTrainer's state management on one GPU:
 *   - "fast snapshot" (section 4.2): every iteration the worker's unique training state, a list
 *     of tensors, is copied without serialisation into one pre-allocated contiguous buffer,
 *     whose size is known up front (12 bytes per parameter for Adam: fp32 master, m, v);
 *   - state loading on failover (section 3.1 steps 5-6, section 3.3): a newcomer receives that
 *     buffer and loads its tensors from it;
 *   - snapshot right after the optimizer update (section 6.2).
 * The paper copies device-to-host into an RDMA buffer and assumes fail-stop; this library keeps
 * the buffer on the device, cuts it into fixed-size chunks "ready to send", and adds a CRC32C
 * per chunk so the receiver can verify what it got.
 *
 * Definitions (N = total payload bytes, C = chunk_bytes):
 *   stream   T = seg_0 || seg_1 || ...        raw little-endian bytes, order of segs[], no padding
 *   buffer     = T || zeros up to n_chunks*C  n_chunks = ceil(N / C)
 *   crcs[j]    = CRC32C(buffer[jC, (j+1)C))   Castagnoli polynomial 0x1EDC6F41, reflected,
 *                                             init and final XOR 0xFFFFFFFF; zero tail included
 *
 * Conventions for every call:
 *   - Pointers marked DEVICE address GPU memory that the caller allocates, owns and keeps alive
 *     until the stream work has completed; pointers marked HOST are ordinary host memory that
 *     is only read during the call.  The library owns nothing but the plan.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).  Work is
 *     enqueued on it and the call returns without synchronising; results stay on the device.
 *   - Return value: FF_OK (0) or a negative ff_status.  Nothing throws, nothing aborts.
 *     Corruption found by ff_restore is reported through bad[] / n_bad, never as an error code.
 *   - A plan's tables do not change after ff_snapshot_plan has returned.  Calls on one plan may run
 *     concurrently, from several host threads and on several streams, as long as their output
 *     arrays (chunks, crcs, bad, n_bad, and for restore and the optimizer steps the plan's tensors)
 *     differ.  Intermediate results live in the output arrays themselves -- while a call is in flight
 *     crcs[] / bad[] hold partial sums -- or, for calls on the default stream (hip_stream NULL, not
 *     captured), in a small tally of the plan that every call leaves as it found it.  Those calls are
 *     one kernel where the others are two or three: a few microseconds on a small snapshot.
 *   - Segments must not overlap each other, the chunk buffer or the crc arrays.
 *   - ff_pack, ff_restore, ff_restore_chunks and the optimizer steps allocate nothing, copy nothing
 *     and only launch kernels; host arrays they are given (gradient pointers, chunk ids) are read
 *     during the call and travel to the device inside kernel arguments.  They can therefore be
 *     recorded into a HIP graph, which then replays with the pointers it was captured with.
 *   - A plan belongs to the device that was current when it was built; device calls made with
 *     another device current return FF_ERR_INVALID.
 */
#ifndef FFSNAP_H
#define FFSNAP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ff_plan ff_plan; /* opaque */

typedef enum {
    FF_OK = 0,
    FF_ERR_NULL = -1,    /* a required pointer is NULL                                          */
    FF_ERR_INVALID = -2, /* bad chunk size, misaligned pointer, nbytes not a multiple of the
                            element size, unknown dtype/kind/flag, incomplete parameter group   */
    FF_ERR_EMPTY = -3,   /* the segments hold no bytes at all                                   */
    FF_ERR_NOMEM = -4,   /* host or device allocation failed                                    */
    FF_ERR_HIP = -5,     /* a HIP runtime call or a kernel launch failed                        */
    FF_ERR_HOST_ONLY = -6, /* device work asked of a plan built with FF_PLAN_HOST_ONLY          */
    FF_ERR_TOO_LARGE = -7, /* input beyond the fixed capacity of an entry point that allocates
                              nothing                                                           */
    FF_ERR_LAYOUT = -8     /* the buffer was packed for another layout (ff_restore_checked)     */
} ff_status;

typedef enum { FF_BF16 = 1, FF_F32 = 2, FF_F16 = 3 } ff_dtype;

/* Role of a segment in the fused optimizer step; RAW segments are only ever copied. */
typedef enum {
    FF_KIND_RAW = 0,
    FF_KIND_W16 = 1,    /* 16-bit working weights: bf16, or fp16 (one format per plan) */
    FF_KIND_MASTER = 2, /* fp32 master weights             */
    FF_KIND_M = 3,      /* fp32 Adam first moment          */
    FF_KIND_V = 4       /* fp32 Adam second moment         */
} ff_kind;

typedef struct {
    void *ptr;         /* DEVICE; aligned to the element size (2 or 4), not necessarily to 16   */
    uint64_t nbytes;   /* multiple of the element size; 0 is allowed (the segment is skipped)   */
    uint32_t dtype;    /* ff_dtype                                                              */
    uint32_t kind;     /* ff_kind                                                               */
    uint32_t param_id; /* groups the W16/MASTER/M/V segments of one parameter; ignored for RAW  */
    uint32_t reserved; /* must be 0                                                             */
} ff_segment;

/* ff_snapshot_plan flags */
#define FF_PLAN_HOST_ONLY 1u /* build the layout only: no device memory is touched, queries work,
                                device calls return FF_ERR_HOST_ONLY (lets a sender or a test
                                compute sizes and the layout id without a GPU)                  */
/* Tuning fields of the plan flags; 0 selects the defaults, results never depend on them.
 *   bits 8..15   log2 of the tile size in bytes (the stream range one wavefront folds; clamped to
 *                [10, log2(chunk_bytes)]; default 15)
 *   bits 16..18  bit 18 set: bits 16..17 choose non-temporal accesses on the tensor side (bit 16)
 *                and on the chunk-buffer side (bit 17); default both
 *   bits 19..23  order in which workgroups take tiles: 0 = default, n in 1..29 = every XCD takes
 *                runs of 2^(n-1) consecutive workgroup tiles, 31 = plain launch order (30 is
 *                FF_ERR_INVALID: a round over the 8 XCDs would exceed the 32-bit launch index)    */
#define FF_PLAN_TILE_LOG2(n) (((uint32_t)(n) & 0xFFu) << 8)
#define FF_PLAN_CACHE_HINT(h) (0x40000u | (((uint32_t)(h) & 3u) << 16))
#define FF_PLAN_XCD_ORDER(n) (((uint32_t)(n) & 31u) << 19)

/* ff_restore flags */
#define FF_RESTORE_VERIFY_ONLY 1u /* recompute and compare CRCs, write bad[]/n_bad, scatter nothing */
#define FF_RESTORE_SKIP_BAD 2u    /* verify first, then scatter only the chunks whose CRC matched:
                                     tensor ranges covered by a bad chunk keep their old contents.
                                     The buffer is read once on the default stream, where the device
                                     has room for all of a chunk (16 or 32 MiB on a whole MI355X) and
                                     the plan is of a layout, size and flags that keep their tiles in
                                     registers (README); else twice, 3 B of traffic per payload byte:
                                     always on other streams, under capture and with bad == crcs   */

#define FF_MIN_CHUNK_BYTES 1024ull
#define FF_MAX_CHUNK_BYTES (1ull << 30)

/*
 * Lay out a snapshot (section 4.2: the engine walks the training configuration once and
 * computes the buffer size).  segs: HOST array of n_segs descriptors, copied.  chunk_bytes: a
 * power of two in [FF_MIN_CHUNK_BYTES, FF_MAX_CHUNK_BYTES].  The plan keeps small device
 * tables (segment pointers and offsets, a tile-to-segment index, CRC constants, the work list of
 * the optimizer steps) on the device that is current at the time of the call.
 * Errors: NULL -> FF_ERR_NULL; bad chunk size / alignment / dtype / kind / reserved / flags ->
 * FF_ERR_INVALID; N == 0 -> FF_ERR_EMPTY; allocation -> FF_ERR_NOMEM; HIP -> FF_ERR_HIP.
 * On error *out is set to NULL.
 */
int ff_snapshot_plan(const ff_segment *segs, uint64_t n_segs, uint64_t chunk_bytes, uint32_t flags,
                     ff_plan **out);

/* Frees the plan and its device tables.  NULL is ignored.  The caller must have synchronised
 * every stream that still uses the plan. */
void ff_plan_destroy(ff_plan *plan);

uint64_t ff_plan_payload_bytes(const ff_plan *plan); /* N                                   */
uint64_t ff_plan_num_chunks(const ff_plan *plan);    /* ceil(N / chunk_bytes)               */
uint64_t ff_plan_buffer_bytes(const ff_plan *plan);  /* num_chunks * chunk_bytes            */
uint64_t ff_plan_chunk_bytes(const ff_plan *plan);
uint64_t ff_plan_num_segments(const ff_plan *plan);  /* non-empty segments                  */
uint64_t ff_plan_num_params(const ff_plan *plan);    /* complete W16/MASTER/M/V groups      */
/* CRC32C over the little-endian uint64 sequence (chunk_bytes, nbytes of every non-empty segment
 * in order): equal ids on sender and receiver mean the two layouts agree. */
uint32_t ff_plan_layout_id(const ff_plan *plan);
/* Stream range [*begin, *end) of non-empty segment i; FF_ERR_INVALID if i is out of range. */
int ff_plan_segment_range(const ff_plan *plan, uint64_t i, uint64_t *begin, uint64_t *end);

/*
 * Checkpoint razor (section 4.2): which of a worker's segments are unique state, to be
 * snapshotted every iteration, and which are redundant across the data-parallel group, to be
 * saved only at recovery time by one healthy worker ("lazy backup").  The two rules:
 *   (1) data-parallel degree > 1                                  -> model weights are redundant;
 *   (2) data-parallel degree > 1 and no distributed optimizer     -> optimizer states are redundant.
 * FF_KIND_W16 segments are the model weights, FF_KIND_MASTER / M / V the optimizer states (the
 * 12 bytes per parameter of the paper's size law); FF_KIND_RAW segments have no known role and
 * always count as unique.  Host-only; no GPU is touched.
 */
typedef struct {
    uint32_t dp_degree;             /* d >= 1 */
    uint32_t distributed_optimizer; /* 0 / 1: optimizer states sharded over the DP group */
} ff_razor_config;

#define FF_RAZOR_UNIQUE 0u    /* the per-iteration snapshot list */
#define FF_RAZOR_REDUNDANT 1u /* the lazy-backup list (the complement) */

/*
 * Writes to out_indices (HOST, room for n_segs entries) the indices, ascending, of the segments
 * of segs[] (HOST) that fall into `which`, and their number to *n_out.  A plan for the selection
 * is then built from those segments in that order.  FF_ERR_NULL / FF_ERR_INVALID (dp_degree 0,
 * unknown `which`, kind or flag value) as usual.
 */
int ff_razor_select(const ff_segment *segs, uint64_t n_segs, const ff_razor_config *cfg,
                    uint32_t which, uint64_t *out_indices, uint64_t *n_out);

/*
 * Snapshot (section 4.2, "fast snapshot"): gather the segments into `chunks` and write one
 * CRC32C per chunk.  chunks: DEVICE, 16-byte aligned, ff_plan_buffer_bytes() bytes, every byte
 * of it is written (the tail of the last chunk with zeros).  crcs: DEVICE, num_chunks uint32.
 */
int ff_pack(const ff_plan *plan, void *chunks, uint32_t *crcs, void *hip_stream);

/*
 * Snapshot into host memory (section 4.2: the snapshot is copied device-to-host into a
 * pre-allocated buffer, from where it is streamed to the next worker).  The snapshot is packed
 * in slices of slice_chunks chunks on pack_stream; as soon as a slice and its CRCs are complete
 * they are copied to host_chunks / host_crcs on copy_stream, while the next slice is being
 * packed.  chunks / crcs: DEVICE staging of the full snapshot, as for ff_pack (it also holds the
 * snapshot afterwards).  host_chunks (buffer_bytes) and host_crcs (num_chunks uint32): HOST,
 * ideally pinned (hipHostMalloc); pageable memory works but the copies then do not overlap.
 * The two streams should differ (both default priority); the call returns without
 * synchronising: the host buffers are complete once copy_stream has been synchronised.  Keeping
 * the two most recent snapshots (section 4.2) is the caller alternating two host buffers.
 */
int ff_pack_to_host(const ff_plan *plan, void *chunks, uint32_t *crcs, void *host_chunks,
                    uint32_t *host_crcs, uint64_t slice_chunks, void *pack_stream,
                    void *copy_stream);

/*
 * State loading on failover (section 3.1 steps 5-6, section 3.3): recompute the CRC32C of every
 * chunk of `chunks`, set bad[j] = (recomputed != crcs[j]) and *n_bad = sum(bad), and copy every
 * segment's bytes out of the buffer into the plan's tensors -- from good and bad chunks alike:
 * the caller must treat tensor ranges that a bad chunk covers as invalid.  chunks: DEVICE,
 * 16-byte aligned, buffer_bytes.  crcs: DEVICE, num_chunks.  bad: DEVICE, num_chunks uint32,
 * each set to 0 or 1.  n_bad: DEVICE, one uint64.  flags: 0, FF_RESTORE_VERIFY_ONLY or
 * FF_RESTORE_SKIP_BAD.
 */
int ff_restore(const ff_plan *plan, const void *chunks, const uint32_t *crcs, uint32_t *bad,
               uint64_t *n_bad, uint32_t flags, void *hip_stream);

/*
 * ff_restore for a buffer that arrives from another worker (section 3.1 steps 5-6: the state
 * controller forwards a healthy worker's state to the newcomer): sender_layout_id is the sender's
 * ff_plan_layout_id(), shipped along with the buffer.  If it differs from this plan's id the two
 * workers disagree on chunk size or tensor sizes and the buffer's bytes would land in the wrong
 * tensors: FF_ERR_LAYOUT is returned, nothing is enqueued, no tensor, bad[] or n_bad is written.
 * Otherwise exactly ff_restore.
 */
int ff_restore_checked(const ff_plan *plan, uint32_t sender_layout_id, const void *chunks,
                       const uint32_t *crcs, uint32_t *bad, uint64_t *n_bad, uint32_t flags,
                       void *hip_stream);

/*
 * Selective state loading: the same as ff_restore for the n_ids chunks named in chunk_ids only
 * (HOST array, strictly ascending, each < num_chunks) -- the chunks a worker re-fetched after a
 * first restore flagged them, or the part of the state another source supplies (section 4.2:
 * state that instant checkpointing cannot supply comes from a fallback).  bad[j] is written for
 * the listed chunks alone, *n_bad counts the bad ones among them, tensor bytes outside the
 * listed chunks are not touched.  Flags as for ff_restore.  FF_ERR_INVALID for an id out of
 * range or a list that is not strictly ascending.  n_ids == 0 only sets *n_bad = 0.
 */
int ff_restore_chunks(const ff_plan *plan, const void *chunks, const uint32_t *crcs,
                      const uint64_t *chunk_ids, uint64_t n_ids, uint32_t *bad, uint64_t *n_bad,
                      uint32_t flags, void *hip_stream);

/* Which tensor ranges a chunk covers: [*begin, *end) is the chunk's payload range in stream
 * coordinates (clipped to N), and the non-empty segments *first_seg .. *first_seg + *n_seg - 1
 * intersect it (use ff_plan_segment_range for their stream ranges).  Host-only query. */
int ff_plan_chunk_span(const ff_plan *plan, uint64_t chunk, uint64_t *first_seg, uint64_t *n_seg,
                       uint64_t *begin, uint64_t *end);

typedef struct {
    float lr, beta1, beta2, eps, weight_decay;
    uint32_t step; /* t >= 1 of the bias corrections */
} ff_adam_hparams;

/*
 * Optimizer update with the snapshot taken in the same pass (section 6.2: the optimizer state
 * is checkpointed immediately after each update).  For every parameter group of the plan one
 * decoupled-weight-decay Adam step in fp32, each operation rounded separately, in this order:
 *     g = float(grad);  p = master*decay;  m' = b1*m + omb1*g;  v' = b2*v + (omb2*g)*g;
 *     d = sqrt(v')/bc2s + eps;  p' = p - step_size*(m'/d);  w' = bf16_rne(p')
 * with decay = 1 - lr*wd, omb1 = 1 - b1, omb2 = 1 - b2, step_size = lr/(1 - b1^t),
 * bc2s = sqrt(1 - b2^t) evaluated in double and rounded once to fp32.  master, m, v and the bf16
 * weights are overwritten in place and the same bytes are written at their stream offsets in
 * `chunks`; RAW segments are copied unchanged; crcs as in ff_pack.  The result equals ff_pack
 * run after an unfused update.  A new master, m or v that is NaN is stored as the canonical quiet
 * NaN 0x7FC00000 (IEEE 754 leaves sign and payload of a produced NaN open and processors differ;
 * the snapshot and its CRCs must not), and w' is rounded from the stored value: 0x7FC0.  grads: HOST array of ff_plan_num_params() DEVICE pointers to
 * bf16 gradients (2-byte aligned), indexed by param_id rank (ascending param_id); read only.
 * FF_ERR_INVALID if the plan has an incomplete group, mismatched element counts, or step == 0.
 */
int ff_adam_step_snapshot(const ff_plan *plan, const void *const *grads, const ff_adam_hparams *hp,
                          void *chunks, uint32_t *crcs, void *hip_stream);

/*
 * The same step for fp16 training with a loss scale (section 7.1: the evaluated models train in
 * fp16).  The plan's working weights are FF_F16; grads point to fp16 gradients of a loss that
 * was multiplied by S, and inv_loss_scale = 1/S:
 *     g = float(grad) * inv_loss_scale   (one rounded fp32 multiplication)
 * then the arithmetic of ff_adam_step_snapshot, and w' = fp16_rne(p') (overflow gives infinity;
 * the canonical NaN that a NaN result is stored as becomes 0x7E00).  n_nonfinite: DEVICE, one uint64,
 * 8-byte aligned, or NULL: receives the number of gradient elements that are infinite or NaN.
 * The update is applied to every element regardless; a caller that lowers S on overflow goes
 * back to the previous snapshot (the paper keeps the two most recent ones, section 4.2).
 * FF_ERR_INVALID also if the plan's working weights are bf16 (and ff_adam_step_snapshot
 * returns it for an fp16 plan).
 */
int ff_adam_step_snapshot_f16(const ff_plan *plan, const void *const *grads,
                              const ff_adam_hparams *hp, float inv_loss_scale,
                              uint64_t *n_nonfinite, void *chunks, uint32_t *crcs,
                              void *hip_stream);

/*
 * The same step with the optimizer state kept in the snapshots themselves.  The paper holds the
 * two most recent snapshots and alternates between them (section 4.2) and snapshots right after
 * every update (section 6.2); here the update of step t reads the old master, m and v of every
 * parameter group from `prev_chunks`, the snapshot of step t-1, at the segments' stream offsets,
 * and writes the new master, m, v and 16-bit weights into `chunks`.  The plan's MASTER, M and V
 * tensors are neither read nor written (they may be views into the snapshot buffers, or unused);
 * the W16 tensors receive the new working weights as in the other two steps; gradients and RAW
 * segments are read from their tensors.  Arithmetic, rounding, crcs and the zero tail are those
 * of ff_adam_step_snapshot (bf16 plan: inv_loss_scale must be 1 and n_nonfinite NULL) or of
 * ff_adam_step_snapshot_f16 (fp16 plan), so the result equals that step run on tensors holding
 * the state of `prev_chunks`.  The CRCs of `prev_chunks` are not checked here (ff_restore with
 * FF_RESTORE_VERIFY_ONLY does that).  Per element it moves 14 bytes in and 16 out, where the
 * in-place steps move 14 in and 28 out.
 * prev_chunks: DEVICE, 16-byte aligned, ff_plan_buffer_bytes() long, read only; it must not
 * overlap `chunks` (FF_ERR_INVALID).
 */
int ff_adam_step_chained(const ff_plan *plan, const void *const *grads, const ff_adam_hparams *hp,
                         float inv_loss_scale, uint64_t *n_nonfinite, const void *prev_chunks,
                         void *chunks, uint32_t *crcs, void *hip_stream);

/* ---- between the loss and the step: gradient norm, clipping, clipped step --------------------- */

/*
 * A list of gradient tensors: sizes, formats and addresses, laid out once.  segs: HOST array of n
 * descriptors, copied; FF_BF16, FF_F16 and FF_F32 tensors may be mixed, kind must be FF_KIND_RAW.
 * Empty tensors and an empty list are allowed.  flags: 0 or FF_PLAN_HOST_ONLY.  The list keeps small device tables
 * on the device that is current at the time of the call and does not change afterwards; the rules for
 * calls on one plan hold for calls on one list, every call that is in flight with a workspace of its own.
 * Addresses may be left out (NULL) if every call brings its own.
 * Errors as for ff_snapshot_plan, but an empty list is none.
 */
typedef struct ff_grad_list ff_grad_list; /* opaque */
int ff_grad_list_create(const ff_segment *segs, uint64_t n, uint32_t flags, ff_grad_list **out);
void ff_grad_list_destroy(ff_grad_list *list); /* as ff_plan_destroy */
uint64_t ff_grad_list_numel(const ff_grad_list *list);           /* elements of all tensors   */
uint64_t ff_grad_list_workspace_bytes(const ff_grad_list *list); /* what ff_grad_norm is given */

/* What is known about a list of gradients; DEVICE, 8-byte aligned.  Calls read it where it lies, so that
 * no host waits for a norm before the update can be enqueued. */
typedef struct {
    double sumsq;         /* sum of the squares of the elements as stored                      */
    uint64_t n_nonfinite; /* infinite or NaN elements                                          */
    double norm;          /* sqrt(sumsq) * inv_loss_scale                                      */
    float scale;          /* what clipping multiplies a stored element by:
                             inv_loss_scale * min(1, max_norm / norm); 0 if skip               */
    uint32_t skip;        /* n_nonfinite > 0: clipping and update are left out                 */
} ff_grad_stats;

/*
 * Global L2 norm over all tensors of the list, and what follows from it for clipping.  Squares and
 * sums are held in 64 bits: no finite element overflows or underflows; the order of the sums depends on the
 * list alone, so the same values give the same bits, wherever they lie.  grads: HOST array of n DEVICE pointers in the list's order, each
 * aligned to its element (entries of empty tensors are ignored), or NULL for the list's own addresses.
 * inv_loss_scale: finite and > 0 in fp32 as well (1 without a loss scale); max_norm: > 0, INFINITY for no clipping.
 * stats: DEVICE, 8-byte aligned.  workspace: DEVICE, 16-byte aligned, ff_grad_list_workspace_bytes() bytes,
 * ZERO before its first use; every call leaves it as the next one needs it.
 */
int ff_grad_norm(const ff_grad_list *list, const void *const *grads, double inv_loss_scale,
                 double max_norm, void *workspace, ff_grad_stats *stats, void *hip_stream);

/*
 * The same for gradients that are spread over several workers (or several lists): parts: DEVICE array of
 * n_parts >= 1 stats, one from each worker's ff_grad_norm, gathered in rank order; their sumsq and n_nonfinite
 * are summed up in that order, so every worker arrives at the same bits.  stats may be one of the
 * parts.
 */
int ff_grad_norm_join(const ff_grad_stats *parts, uint64_t n_parts, double inv_loss_scale,
                      double max_norm, ff_grad_stats *stats, void *hip_stream);

/*
 * Clipping in place, for an optimizer other than this library's step: every element g of the list becomes
 * g * stats->scale, one fp32 multiplication rounded to the tensor's format.  Nothing is touched if
 * stats->skip is set (what overflowed stays to be looked at) or the scale is exactly 1.  grads as for ff_grad_norm.
 */
int ff_grad_clip(const ff_grad_list *list, const void *const *grads, const ff_grad_stats *stats,
                 void *hip_stream);

/*
 * The optimizer step with the snapshot in the same pass on clipped gradients: ff_adam_step_snapshot, or for an fp16 plan
 * ff_adam_step_snapshot_f16, with g = float(grad) * stats->scale (one rounded fp32 multiplication, the
 * loss scale included); prev_chunks: NULL, or the previous snapshot as for ff_adam_step_chained.  If stats->skip is
 * set the update is left out: master, m and v keep their bits, the 16-bit weights are rounded from
 * the master (a NaN to the format's canonical one), and the snapshot holds that state.  hp->step is the caller's: a step that
 * was left out counts in the next one's bias correction if the caller counts it, and does not if the caller, who has
 * looked at stats->skip, hands the same step in again.  stats: DEVICE, read when the
 * stream gets there.  Gradients, hp, chunks, crcs and errors as for those steps.
 */
int ff_adam_step_clipped(const ff_plan *plan, const void *const *grads, const ff_adam_hparams *hp,
                         const ff_grad_stats *stats, const void *prev_chunks, void *chunks,
                         uint32_t *crcs, void *hip_stream);

/* ---- clipped policy loss with a KL term, and its gradient ------------------------------------- */

/*
 * One batch of tokens.  logits: n_tokens rows of `vocab` elements of `dtype`, row_stride >= vocab elements apart
 * (the last row need not be padded); aligned to the element.  All arrays DEVICE; targets int64, the others fp32,
 * n_tokens each.  weights: what a token counts in the loss, its share of the mean included; 0 leaves it
 * out (prompts, padding): its row is not read.
 */
typedef struct {
    const void *logits;
    uint64_t n_tokens, vocab, row_stride;
    uint32_t dtype;    /* FF_BF16, FF_F16 or FF_F32 */
    uint32_t reserved; /* must be 0 */
    const int64_t *targets;
    const float *old_logp;   /* log-probability under the policy that made the token */
    const float *ref_logp;   /* ... under the reference policy, or NULL: no KL term  */
    const float *advantages;
    const float *weights;
    float clip_low, clip_high; /* the ratio is clipped to [1 - clip_low, 1 + clip_high]; 0 <= clip_low <= 1,
                                  0 <= clip_high                                     */
    float beta;                /* >= 0, of the KL term; > 0 needs ref_logp           */
    float loss_scale;          /* finite, > 0: the gradient is that of loss * loss_scale */
} ff_policy_batch;

/* DEVICE, 8-byte aligned */
typedef struct {
    float loss, kl;      /* sums of weight * token loss, and of weight * KL                      */
    uint64_t n_tokens;   /* that count                                                            */
    uint64_t n_clipped;  /* of these: the clipped product was the smaller one                    */
    uint64_t n_invalid;  /* weight not 0 and yet left out: target outside the vocabulary, or every logit -inf */
} ff_policy_stats;

/* What ff_policy_loss is given.  Never falls with either argument: the workspace of the largest batch and
 * vocabulary serves every smaller call. */
uint64_t ff_policy_workspace_bytes(uint64_t n_tokens, uint64_t vocab);

/*
 * For every token with weight w != 0, target y, logits z, advantage A:
 *     logp  = z_y - log(sum_j exp(z_j))            r = exp(logp - old_logp)
 *     token = -min(r * A, clip(r) * A) + beta * kl, kl = exp(d) - d - 1 with d = ref_logp - logp
 *     loss  = sum of w * token
 *     dlogits_j = loss_scale * w * slope * ([j = y] - exp(z_j) / sum exp),
 *     slope = (the clipped product is the smaller ? 0 : -r * A) + beta * (1 - exp(d))
 * Sums over the vocabulary in fp32 against the row's largest logit and joined in fp64, what hangs on logp in
 * fp64; the gradient is rounded once.  Logits of -inf are probabilities of 0.  A row with a NaN or +inf gives NaN in its outputs and
 * its whole gradient row (which ff_grad_norm finds downstream).  A token that is left out (weight 0 or invalid) has logp and token
 * loss 0 and a gradient row of zeros.
 * logp, token_loss: DEVICE fp32[n_tokens], apart from each other and from every input.  dlogits: NULL (no gradient), or DEVICE, of `dtype`, rows grad_stride >= vocab elements apart; it may
 * be the logits themselves with the same stride, and elements between rows are not touched.
 * stats: DEVICE.  workspace: DEVICE, 16-byte aligned, ff_policy_workspace_bytes(), ZERO before its
 * first use; every call leaves it as the next one needs it.  Calls that are in flight at once need outputs, stats and workspaces of
 * their own.
 * n_tokens = 0 is allowed: the stats become zero.  FF_ERR_INVALID for vocab 0, and for vocab or n_tokens above 2^31 - 1.
 */
int ff_policy_loss(const ff_policy_batch *batch, float *logp, float *token_loss, void *dlogits,
                   uint64_t grad_stride, ff_policy_stats *stats, void *workspace, void *hip_stream);

/* Test helper: CRC32C of nbytes at dev_buf (DEVICE, 16-byte aligned) into *dev_out (DEVICE),
 * computed by the same tile and combine kernels as ff_pack.  Allocates and frees a small
 * scratch array, so it synchronises the stream before returning. */
int ff_crc32c(const void *dev_buf, uint64_t nbytes, uint32_t *dev_out, void *hip_stream);

/*
 * ff_crc32c for callers that cannot allocate or must not be synchronised: code that is being
 * captured into a HIP graph, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments and result as ff_crc32c, but the scratch memory (reduction tables and one CRC
 * register per 1 MiB of input) is a fixed array in the library's device image instead of an
 * allocation, and the call only enqueues kernels on hip_stream and returns: *dev_out is valid
 * once the stream has reached that point.  It never calls hipMalloc or hipFree.
 * Limits: nbytes <= FF_CRC32C_NOALLOC_MAX_BYTES, else FF_ERR_TOO_LARGE and nothing is enqueued.
 * The array (about 260 KiB) exists once per GPU and is shared by every call on that GPU: two
 * calls whose kernels may overlap in time (different streams) race on it and give wrong results;
 * calls on one stream are safe back to back.  The first call on a device looks up the array's
 * address and copies the tables into it with a blocking hipMemcpy, so make one eager call per
 * device before capturing it into a graph.
 */
#define FF_CRC32C_NOALLOC_MAX_BYTES (1ull << 36) /* 64 GiB */
int ff_crc32c_noalloc(const void *dev_buf, uint64_t nbytes, uint32_t *dev_out, void *hip_stream);

/* Bench helper: plain device copy of nbytes (both DEVICE, 16-byte aligned, nbytes a multiple of
 * 16, the ranges disjoint) in the access pattern of ff_pack but without the CRC: the measured
 * bandwidth ceiling printed beside the real kernels. */
int ff_copy_ceiling(void *dst, const void *src, uint64_t nbytes, void *hip_stream);

/* Bench helper: the memory traffic of the optimizer steps with nothing else -- for every
 * parameter group of the plan the same tiles, loads and stores as ff_adam_step_snapshot
 * (prev_chunks NULL: 14 bytes read, 28 written per element) or as ff_adam_step_chained
 * (prev_chunks set: 14 read, 16 written), but no arithmetic and no CRC: the new 16-bit weights are
 * the gradient's bits, master, m and v keep their values.  crcs, RAW segments and the zero tail
 * of `chunks` are not written.  The measured ceiling of this mix of streams, printed beside the
 * real steps.  Arguments as for those steps. */
int ff_mix_ceiling(const ff_plan *plan, const void *const *grads, const void *prev_chunks,
                   void *chunks, void *hip_stream);

/* Static string for a status code; for FF_ERR_HIP the text of the last HIP error seen by the
 * calling thread is appended. */
const char *ff_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* FFSNAP_H */
