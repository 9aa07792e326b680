/*
 * avmp.h -- C ABI of the B200-native AVMP hot path.
 *
 * AVMP (Asymmetric Virtual Memory Paging) keeps two physically different cache
 * stores for hybrid Mamba-Transformer inference -- fine-grained KV pages and
 * per-layer SSM state blocks -- behind one space of 32-bit virtual handles, and
 * moves capacity between them when an allocation would otherwise fail (paper
 * Sections 3.1 and 3.2).  This library holds all allocator state in device
 * memory and runs every step of the path as CUDA kernels on sm_100a:
 *
 *   avmp_step        batched admit / extend / finish in array order, including the
 *                    CapacityError handler, the migration (shrink donor, relocate
 *                    live units, remap handles, grow recipient) and the retry;
 *   avmp_translate   handle -> (pool, physical offset);
 *   avmp_gather_kv   paged gather of one attention layer into ragged batch buffers;
 *   avmp_gather_ssm  gather of one SSM layer's state blocks into batch buffers;
 *   avmp_scatter_*   the matching write side;
 *   avmp_attn_*      attention over the KV chains where they lie (whole prompts, single tokens, with and without a window);
 *                    norms, rotation and cache writes of new rows;
 *   avmp_ssm_*       the linear recurrence on the SSM blocks where they lie (prompts, single tokens);
 *   avmp_conv_*, avmp_scan_*   short convolution and selective scan on the SSM blocks where they lie.
 *
 * Conventions
 *   - "d_" arguments are DEVICE pointers, "h_" arguments are HOST pointers.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *     Every call is ordered on that stream.  Calls with only device arguments never
 *     synchronise with the host; calls that take or fill host memory do, and say so.
 *   - The library never allocates device memory: the caller owns the arena and the
 *     workspace (e.g. two torch tensors) and must keep them alive until avmp_destroy.
 *   - Return value: AVMP_OK or a negative AVMP_E* code for misuse the host can see.
 *     What only the device can see (an invalid handle, a dead request in a gather
 *     list, an output buffer too small) never traps: the item is skipped, a sticky
 *     error code and an error count are recorded in the statistics block.
 *   - One context must not be used from two streams at once.
 */
#ifndef AVMP_H
#define AVMP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define AVMP_API __attribute__((visibility("default")))
#else
#define AVMP_API
#endif

#define AVMP_INVALID 0xFFFFFFFFu              /* no handle / no slot */
#define AVMP_NONE64 0xFFFFFFFFFFFFFFFFull     /* no offset / "never" */

enum { AVMP_OK = 0, AVMP_EINVAL = -1, AVMP_ENOSPC = -2, AVMP_ECUDA = -3, AVMP_ETOOBIG = -4 };
enum { AVMP_POOL_KV = 0, AVMP_POOL_SSM = 1 };

/* Operation kinds and flags (avmp_op). */
enum { AVMP_OP_ADMIT = 1, AVMP_OP_EXTEND = 2, AVMP_OP_FINISH = 3 };
enum {
    AVMP_FLAG_KEEP_KV = 1, /* FINISH: free only the SSM blocks, keep the KV chain (slot becomes KV_ONLY) */
    AVMP_FLAG_RESUME = 2   /* ADMIT: the slot is KV_ONLY; allocate SSM blocks and extend the kept chain */
};
/* Per-operation result written by avmp_step. */
enum {
    AVMP_ST_OK = 0,
    AVMP_ST_OOM = 1,      /* did not fit, even after the migration attempt; nothing was taken */
    AVMP_ST_BAD_REQ = 2,  /* slot out of range or in the wrong state for this kind */
    AVMP_ST_TOO_LONG = 3, /* chain would pass max_pages_per_request */
    AVMP_ST_BAD_ARG = 4   /* unknown kind, or zero tokens on ADMIT / EXTEND */
};
enum { AVMP_REQ_EMPTY = 0, AVMP_REQ_LIVE = 1, AVMP_REQ_KV_ONLY = 2 };
/* Rebalancer state label (paper Figure 2). */
enum { AVMP_FSM_BALANCED = 0, AVMP_FSM_KV_PRESSURED = 1, AVMP_FSM_SSM_PRESSURED = 2, AVMP_FSM_REBALANCING = 3 };
/* Sticky device-side error codes (avmp_stats.error_code keeps the first one). */
enum {
    AVMP_DEV_OK = 0,
    AVMP_DEV_BAD_HANDLE = 1,     /* translate: handle does not resolve */
    AVMP_DEV_BAD_REQUEST = 2,    /* gather / scatter / attn / ssm: request slot out of range or holds nothing,
                                    or a row range that does not fit what it holds */
    AVMP_DEV_OUT_OVERFLOW = 3,   /* gather_kv: rows would pass out_capacity_tokens */
    AVMP_DEV_TIMEOUT = 4         /* a kernel gave up a bounded wait; what its call puts out is not to be used */
};

/* Model shape: what one KV page and one SSM block hold (paper Section 3.1).
 * KV page  = page_tokens tokens of {K, V} x kv_heads x head_dim x kv_elem_bytes for EVERY
 *            attention layer, laid out [layer][K|V][token][head][dim];
 * SSM block = one layer's ssm_state_elems then ssm_conv_elems elements of ssm_elem_bytes. */
typedef struct {
    uint32_t n_attn_layers, n_ssm_layers, page_tokens, kv_heads, head_dim, kv_elem_bytes;
    uint32_t ssm_state_elems, ssm_conv_elems, ssm_elem_bytes;
} avmp_model_spec;

/* Rebalancer and table-size options (paper Section 3.2; defaults from avmp_default_options). */
typedef struct {
    uint32_t threshold_low_ppm;           /* 50000: labels the PRESSURED states only */
    uint32_t threshold_high_ppm;          /* 300000: donor free fraction must exceed this */
    uint64_t min_rebalance_interval_ops;  /* 1000 logical operations between migrations; >= 1 */
    uint32_t migration_enabled;           /* 0 = static partition with AVMP handles */
    uint32_t max_requests;                /* request slots: op.req is in [0, max_requests) */
    uint32_t max_pages_per_request;       /* longest KV chain, in pages */
    uint32_t reclaim_gap;                 /* 0 (default): the paper's rule, recipient gains floor(n*U_donor /
                                             U_recipient) units and the remainder is lost to the gap between
                                             the pools.  1: a variant with no counterpart in the paper, the
                                             bytes already in the gap are offered again with the ceded ones:
                                             gain = floor((gap + n*U_donor) / U_recipient), gap = remainder,
                                             wasted_bytes stays 0 */
} avmp_options;

/* One allocator operation, 12 bytes. */
typedef struct {
    uint8_t kind, flags;
    uint16_t rsvd;
    uint32_t req;     /* caller-chosen dense slot id */
    uint32_t tokens;  /* ADMIT / EXTEND: tokens appended */
} avmp_op;

/* Sizes derived from the model and the pool (host-side arithmetic, no device access). */
typedef struct {
    uint64_t pool_bytes_aligned;  /* pool_bytes rounded down to 128 (slab alignment) */
    uint64_t unit_bytes[2];       /* KV page, SSM block; each rounded up to 16 */
    uint64_t vid_space[2];        /* virtual ids per pool = pool_bytes_aligned / unit */
    uint64_t cap0[2];             /* initial capacities in units */
    uint64_t gap0;                /* initial bytes in neither store */
    uint64_t kv_layer_bytes;      /* one attention layer inside a page (K then V) */
    uint64_t kv_row_bytes;        /* one token's K (or V) of one layer */
    uint64_t ssm_state_bytes, ssm_conv_bytes;
} avmp_layout;

/* All counters of a context (same order as uint64_t[AVMP_N_STATS]). */
typedef struct {
    uint64_t op_counter;          /* logical operations processed (Section 3.2) */
    uint64_t last_rebalance_op;   /* AVMP_NONE64 before the first migration */
    uint64_t n_oom;               /* operations that ended AVMP_ST_OOM (the paper's N_OOM) */
    uint64_t n_capacity_error;    /* CapacityError handler runs */
    uint64_t n_rebalance;         /* completed migrations */
    uint64_t migrated_bytes;      /* donor bytes ceded */
    uint64_t wasted_bytes;        /* sum of ceded bytes modulo the recipient unit */
    uint64_t relocated_blocks;    /* live units copied out of ceded regions */
    uint64_t relocated_bytes;
    uint64_t gap_bytes;
    uint64_t cap[2];
    uint64_t free_units[2];
    uint64_t fsm_state;
    uint64_t n_invalid;           /* operations rejected with BAD_REQ / TOO_LONG / BAD_ARG */
    uint64_t unit_bytes[2];
    uint64_t vid_space[2];
    uint64_t pool_bytes_aligned;
    uint64_t error_code;          /* first AVMP_DEV_* error seen, sticky */
    uint64_t error_count;         /* items skipped because of device-side errors */
    uint64_t relocation_ns_last;  /* device-clock duration of the last relocation copy (first CTA in, last out) */
    uint64_t relocation_ns_total; /* sum over all relocation copies: the time spent migrating payload */
    /* Time decomposition of the allocator kernel (paper Section 4.3), SM cycles at the nominal clock:
     * everything; the part spent handling CapacityErrors that ended OOM; the part spent planning
     * migrations.  The rest is service time. */
    uint64_t step_ns_total, step_ns_oom_retry, step_ns_migration_plan;
} avmp_stats;
#define AVMP_N_STATS (sizeof(avmp_stats) / sizeof(uint64_t))

/* Host copies of every table, for parity checks and snapshot / restore.  The caller
 * provides the arrays (sizes from avmp_layout and avmp_options); counts are filled by
 * export and read by import. */
typedef struct {
    uint32_t *slot_stack[2];  /* [vid_space[p]]  free physical slots, bottom first */
    uint32_t *vid_stack[2];   /* [vid_space[p]]  free virtual ids, bottom first */
    uint32_t *vt[2];          /* [vid_space[p]]  page table: vid -> slot or AVMP_INVALID */
    uint32_t *ow[2];          /* [vid_space[p]]  owner: slot -> vid or AVMP_INVALID */
    uint32_t *req_state;      /* [max_requests] */
    uint32_t *req_len;        /* [max_requests] tokens held */
    uint32_t *req_npages;     /* [max_requests] */
    uint32_t *req_chain;      /* [max_requests * max_pages_per_request] KV handles */
    uint32_t *req_ssm;        /* [max_requests * n_ssm_layers] SSM handles */
    uint32_t n_slot_stack[2], n_vid_stack[2];
    avmp_stats stats;
} avmp_tables;

typedef struct avmp_ctx avmp_ctx;

/* Fill *opt with the paper's defaults (thresholds 0.05 / 0.30, interval 1000, migration
 * on) and max_requests = 1024, max_pages_per_request = 4096. */
AVMP_API void avmp_default_options(avmp_options *opt);

/* Section 3.1 arithmetic.  initial_split is the fraction of the pool given to the SSM store
 * at start (the static systems' "mamba ratio").  Returns AVMP_EINVAL on zero units, a split
 * outside [0, 1], a pool too small for one unit, or an id space beyond 31 bits. */
AVMP_API int avmp_derive_layout(const avmp_model_spec *spec, uint64_t pool_bytes, double initial_split,
                       avmp_layout *out);

/* Bytes of workspace avmp_create needs (0 on invalid arguments). */
AVMP_API size_t avmp_workspace_bytes(const avmp_model_spec *spec, uint64_t pool_bytes, const avmp_options *opt);

/* Create a context over a caller-owned arena and workspace and initialise the tables on
 * `stream` (fresh pools hand out slot 0, 1, 2, ... and id 0, 1, 2, ...).
 *   d_arena      >= pool_bytes, 256-byte aligned.  KV slot i lives at byte i * U_kv; SSM slot j
 *                at pool_bytes_aligned - (j + 1) * U_ssm, so each store's high end faces the gap
 *                in the middle and ceded bytes are what the other store grows into.  The arena
 *                is never cleared.
 *   d_workspace  >= avmp_workspace_bytes(...), 256-byte aligned.
 *   migration_batch_size  B: upper bound, in donor units, on one migration (Section 3.1).
 *   opt          NULL = defaults.  threshold_low >= threshold_high is rejected (Section 4.6).
 *                max_requests * max_pages_per_request * max(page_tokens, copy pieces per page) must
 *                stay below 2^32: row offsets (cu_seqlens) and the gathers' piece counts are 32-bit.
 * Returns AVMP_EINVAL / AVMP_ENOSPC (workspace too small) / AVMP_ECUDA. */
AVMP_API int avmp_create(avmp_ctx **out, const avmp_model_spec *spec, void *d_arena, uint64_t pool_bytes,
                double initial_split, uint32_t migration_batch_size, const avmp_options *opt,
                void *d_workspace, size_t workspace_bytes, void *stream);
AVMP_API int avmp_destroy(avmp_ctx *ctx);

/* One engine step (Sections 3.1-3.2): process d_ops[0..n_ops) exactly as if they were applied
 * one at a time in array order -- each op advances the logical counter, allocations pop the
 * LIFO free lists, a shortage runs the CapacityError handler (SSM first, then KV), which may
 * migrate min(B, donor free) donor units when the donor's free fraction exceeds
 * threshold_high and the throttle allows, relocating live units out of the ceded range and
 * remapping their handles; the op is then retried once.  d_status[i] receives AVMP_ST_*.
 * Stream-ordered, no host synchronisation.  n_ops == 0 is a no-op. */
AVMP_API int avmp_step(avmp_ctx *ctx, const avmp_op *d_ops, uint32_t n_ops, uint32_t *d_status, void *stream);

/* avmp_step followed by avmp_translate of d_handles against the tables that step leaves (Sections 3.1-3.2
 * and Figure 1), with the translation riding on the step's relocation-copy launch: two launches per engine
 * step instead of three, which is most of what the allocator part of a step costs (lists of more than 32 768
 * handles, and contexts with migration disabled, take the wide translate kernel as a third launch).  Results
 * are exactly those of the two calls made one after the other.  n_handles == 0 is avmp_step; n_ops == 0 is avmp_translate. */
AVMP_API int avmp_step_translate(avmp_ctx *ctx, const avmp_op *d_ops, uint32_t n_ops, uint32_t *d_status,
                                 const uint32_t *d_handles, uint32_t n_handles, uint32_t *d_pool, uint64_t *d_offset,
                                 uint64_t *d_arena_offset, void *stream);

/* Same step, with the batch length read from device memory when the kernel runs (*d_n_ops, clamped
 * to max_ops): for batches that another kernel builds, so that a serving loop needs no host round
 * trip per step.  max_ops bounds the work the host queues (the number of migration rounds). */
AVMP_API int avmp_step_indirect(avmp_ctx *ctx, const avmp_op *d_ops, const uint32_t *d_n_ops, uint32_t max_ops,
                                uint32_t *d_status, void *stream);

/* Same step with HOST arrays: copies the ops in, runs the step, copies the statuses out
 * and waits for them.  n_ops is limited to 65536 per call. */
AVMP_API int avmp_step_host(avmp_ctx *ctx, const avmp_op *h_ops, uint32_t n_ops, uint32_t *h_status, void *stream);

/* Section 3.1 / Figure 1: resolve handles.  d_pool[i] = pool tag, d_offset[i] = slot * unit
 * bytes (offset inside that store), d_arena_offset[i] (may be NULL) = byte offset of the unit
 * from d_arena.  A handle that does not resolve gives AVMP_INVALID / AVMP_NONE64 and a sticky
 * AVMP_DEV_BAD_HANDLE. */
AVMP_API int avmp_translate(avmp_ctx *ctx, const uint32_t *d_handles, uint32_t n, uint32_t *d_pool,
                   uint64_t *d_offset, uint64_t *d_arena_offset, void *stream);

/* Paged KV gather (Section 2.2 "paged scatter-gather memory lookups") of attention layer
 * `attn_layer` for the request slots d_reqs[0..n_reqs), n_reqs <= max_requests.  Rows are one
 * token's kv_heads x head_dim elements; request k's rows start at d_cu_seqlens[k] (prefix sums
 * of the held lengths, n_reqs + 1 entries, always written).  Only valid tokens are copied
 * (the last page may be partial).  A slot that holds no chain contributes length 0 and a
 * sticky AVMP_DEV_BAD_REQUEST; a request whose rows would pass out_capacity_tokens copies
 * nothing (AVMP_DEV_OUT_OVERFLOW).  Output pointers must be 16-byte aligned.
 * Lists of up to 1024 requests are planned inside the copy kernel (one launch, no shared
 * scratch); longer lists are planned by a kernel of their own into the context's workspace, so
 * KV gathers / scatters with such lists must not overlap on the GPU (keep them on one stream). */
AVMP_API int avmp_gather_kv(avmp_ctx *ctx, uint32_t attn_layer, const uint32_t *d_reqs, uint32_t n_reqs,
                   void *d_out_k, void *d_out_v, uint64_t out_capacity_tokens,
                   uint32_t *d_cu_seqlens, void *stream);

/* SSM gather (Section 2.2 "contiguous read and write access") of SSM layer `ssm_layer`:
 * d_out_state[k] gets the state elements, d_out_conv[k] the convolution window of request
 * d_reqs[k].  Requests must be LIVE; others are skipped with AVMP_DEV_BAD_REQUEST. */
AVMP_API int avmp_gather_ssm(avmp_ctx *ctx, uint32_t ssm_layer, const uint32_t *d_reqs, uint32_t n_reqs,
                    void *d_out_state, void *d_out_conv, void *stream);

/* The two gathers for `n_layers` consecutive layers in ONE launch (same results as calling the
 * single-layer entry once per layer; one launch instead of n_layers removes the per-launch ramp
 * and tail, which is most of what separates a 250 MB gather from the HBM roofline).  Layer
 * first_layer + l writes to the given buffers advanced by l * stride bytes; strides are multiples
 * of 16 and at least one layer's worth (out_capacity_tokens rows for KV, n_reqs blocks for SSM).
 * d_cu_seqlens is shared by all layers. */
AVMP_API int avmp_gather_kv_layers(avmp_ctx *ctx, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs,
                                   uint32_t n_reqs, void *d_out_k, void *d_out_v, uint64_t layer_stride_bytes,
                                   uint64_t out_capacity_tokens, uint32_t *d_cu_seqlens, void *stream);
AVMP_API int avmp_gather_ssm_layers(avmp_ctx *ctx, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs,
                                    uint32_t n_reqs, void *d_out_state, uint64_t state_layer_stride_bytes,
                                    void *d_out_conv, uint64_t conv_layer_stride_bytes, void *stream);

/* Both gathers of an engine step in ONE launch (Section 2.2: the two access patterns, for the
 * same request list): attention layers [first_attn_layer, + n_attn_layers) exactly as
 * avmp_gather_kv_layers, then SSM layers [first_ssm_layer, + n_ssm_layers) exactly as
 * avmp_gather_ssm_layers -- same outputs, same error items (a slot that is KV_ONLY contributes
 * its rows to the KV part and one AVMP_DEV_BAD_REQUEST per SSM layer).  A step that moves only
 * tens of MB is bound by the ramp and tail of its launches; this pays them once.  Both layer
 * counts must be at least 1 (use the single-kind entry points otherwise). */
AVMP_API int avmp_gather_step(avmp_ctx *ctx, const uint32_t *d_reqs, uint32_t n_reqs,
                              uint32_t first_attn_layer, uint32_t n_attn_layers, void *d_out_k, void *d_out_v,
                              uint64_t kv_layer_stride_bytes, uint64_t out_capacity_tokens, uint32_t *d_cu_seqlens,
                              uint32_t first_ssm_layer, uint32_t n_ssm_layers, void *d_out_state,
                              uint64_t state_layer_stride_bytes, void *d_out_conv, uint64_t conv_layer_stride_bytes,
                              void *stream);

/* Write side of the two gathers (what the model's kernels do after a step).  Tokens
 * [d_tok_start[k], len_k) of request k are read from rows cu[k].. of d_in_k / d_in_v, cu being
 * the prefix sum of (len_k - d_tok_start[k]); d_tok_start == NULL means 0. */
AVMP_API int avmp_scatter_kv(avmp_ctx *ctx, uint32_t attn_layer, const uint32_t *d_reqs,
                    const uint32_t *d_tok_start, uint32_t n_reqs, const void *d_in_k,
                    const void *d_in_v, void *stream);
AVMP_API int avmp_scatter_ssm(avmp_ctx *ctx, uint32_t ssm_layer, const uint32_t *d_reqs, uint32_t n_reqs,
                     const void *d_in_state, const void *d_in_conv, void *stream);

/* (No counterpart in the paper: a deployment convenience.)  The same gather as avmp_gather_kv
 * for callers that can neither allocate device memory nor lend the library scratch of their
 * own -- e.g. code running after the process gave the whole card to a memory pool, or a
 * plug-in that is only ever handed device pointers.  Inputs and outputs are still the
 * caller's; the gather's planning arrays live in a fixed array inside the library
 * (about 33 KB per GPU, held until the process exits), which limits the request list to
 * AVMP_STATIC_GATHER_MAX_REQS entries: a longer list returns AVMP_ETOOBIG and does nothing
 * (and, as for avmp_gather_kv, a list longer than max_requests returns AVMP_EINVAL).
 * The context's device must be current.  The array's device address is resolved on the host,
 * once per device: by avmp_create (so that the driver loads the array onto the GPU while the
 * caller still has memory to spare), or else by the first call of this entry point on that
 * device -- make that call (n_reqs = 0 will do) before handing all memory away and before any
 * stream capture.  After a cudaDeviceReset create a new context before calling this again.
 * All calls on a device share the array: calls whose kernels may overlap on the GPU
 * (different streams) race -- keep them on one stream or order them with events.  Results,
 * error items and cu_seqlens are exactly those of avmp_gather_kv. */
#define AVMP_STATIC_GATHER_MAX_REQS 4096
AVMP_API int avmp_gather_kv_static(avmp_ctx *ctx, uint32_t attn_layer, const uint32_t *d_reqs, uint32_t n_reqs,
                                   void *d_out_k, void *d_out_v, uint64_t out_capacity_tokens,
                                   uint32_t *d_cu_seqlens, void *stream);

/* Write side for a range of layers in one launch (layer first_layer + l reads its rows from the
 * buffers advanced by l * stride bytes; rows of a layer are laid out as for the single-layer call). */
AVMP_API int avmp_scatter_kv_layers(avmp_ctx *ctx, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs,
                                    const uint32_t *d_tok_start, uint32_t n_reqs, const void *d_in_k,
                                    const void *d_in_v, uint64_t layer_stride_bytes, void *stream);
AVMP_API int avmp_scatter_ssm_layers(avmp_ctx *ctx, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs,
                                     uint32_t n_reqs, const void *d_in_state, uint64_t state_layer_stride_bytes,
                                     const void *d_in_conv, uint64_t conv_layer_stride_bytes, void *stream);

/* ---- compute on the caches in place (no counterpart in the paper, which stops at the memory) ----
 * The gathers above hand a model's kernels a dense copy of what they need; the entry points below
 * are those kernels, reading pages and blocks where they lie, so a step touches its cache once.
 * All rows ("tokens") of a batch are packed; a row stride of 0 in a descriptor means densely packed
 * rows.  Pointers to rows must be 16-byte aligned and row strides multiples of 16 bytes (decays: 4).
 * Outputs must not overlap inputs.  The context's device must be current.  Nothing is allocated: where
 * a call needs scratch it takes a caller's buffer, whose content need not be preserved and which two calls
 * may share if they cannot overlap on the GPU.  Calls can be captured into graphs; nothing is read on the host
 * but the arguments.  An item that only the device can see to be wrong (see each call) is skipped, its output
 * rows and its state are left as they were, and it counts one AVMP_DEV_BAD_REQUEST.
 * Numerics: sums, softmax statistics and states are held in 32 bits.  Besides the outputs, these are rounded to the rows' 16 bits:
 * the softmax weights that multiply V (their denominator is summed before), and in avmp_ssm_prompt the decayed scores and the
 * carried state where they enter an output (not where they enter the state that is kept).  One in eight of the exponentials of
 * avmp_attn_prompt and of a shared prefix is a polynomial with a relative error of 2.6e-6.  What a row does not see (later tokens,
 * tokens in front of a reset, other requests' rows and leftovers of pages) does not reach it, whatever it holds; NaN and
 * infinities that it does see do.  A row all of whose scores are -inf is NaN, its logarithm -inf. */
enum { AVMP_TYPE_BF16 = 0, AVMP_TYPE_F16 = 1 };   /* type of input and output rows (and of cached K and V) */

/* q and out rows are [q_heads][head_dim].  Query head h reads KV head h / (q_heads / kv_heads).
 * Supported: kv_elem_bytes 2, head_dim 64 or 128, page_tokens a multiple of 8, q_heads a multiple
 * of kv_heads with at most 64 query heads to a KV head; else AVMP_EINVAL. */
typedef struct {
    uint32_t type, q_heads;
    float scale;               /* scores are scale * <q, k>; finite */
    uint32_t rsvd;             /* 0 */
    uint64_t q_stride_bytes, out_stride_bytes;
} avmp_attn_desc;

/* Scratch bytes that any avmp_attn_* call of up to n_reqs list entries needs (0 on invalid arguments). */
AVMP_API size_t avmp_attn_workspace_bytes(const avmp_ctx *ctx, const avmp_attn_desc *desc, uint32_t n_reqs);

/* Causal attention of the newest tokens of a batch (a prompt, a turn appended to a kept chain, a chunk
 * of a prompt).  Rows d_cu_q[k] .. d_cu_q[k+1] of d_q are the LAST tokens of request d_reqs[k]'s chain,
 * whose K and V have been written to the cache; row i of n stands at position held - n + i and sees
 * the tokens up to and including its own position.  d_lse (may be NULL) receives the natural logarithm
 * of each row's softmax denominator, [total_q][q_heads].  total_q is the number of rows of the buffers;
 * rows that no list entry owns are not touched.  Skipped items: a slot that holds nothing, more rows
 * than held tokens, offsets that decrease or pass total_q.  n_reqs <= max_requests; q_heads * total_q < 2^31. */
AVMP_API int avmp_attn_prompt(avmp_ctx *ctx, uint32_t attn_layer, const avmp_attn_desc *desc, const uint32_t *d_reqs,
                              uint32_t n_reqs, const uint32_t *d_cu_q, uint32_t total_q, const void *d_q, void *d_out,
                              float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream);

/* Attention of one token per request over its whole chain: row k of d_q belongs to d_reqs[k] (slots may
 * repeat).  With prefix_req != AVMP_INVALID every request also sees all tokens of that slot's chain
 * (a shared prompt that is held once); the batch's products with it are computed together.  A prefix slot
 * out of range or holding nothing skips every item.  n_reqs <= max_requests; q_heads * n_reqs < 2^31. */
AVMP_API int avmp_attn_decode(avmp_ctx *ctx, uint32_t attn_layer, const avmp_attn_desc *desc, const uint32_t *d_reqs,
                              uint32_t n_reqs, uint32_t prefix_req, const void *d_q, void *d_out, float *d_lse,
                              void *d_workspace, size_t workspace_bytes, void *stream);

/* The same two calls through a window: the row at position p sees the tokens j <= p with j > p - window or j < sinks (its own token, the
 * window - 1 in front of it, and the first `sinks` tokens of the chain).  window >= 1; a window as long as the chain shows all of it.  The
 * work is that of the tokens that are seen; pages that no row sees are not read, but stay in the chain.  What the calls take, skip and need
 * as scratch is otherwise as above (there is no shared prefix). */
AVMP_API int avmp_attn_window_prompt(avmp_ctx *ctx, uint32_t attn_layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks,
                                     const uint32_t *d_reqs, uint32_t n_reqs, const uint32_t *d_cu_q, uint32_t total_q, const void *d_q,
                                     void *d_out, float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream);
AVMP_API int avmp_attn_window_decode(avmp_ctx *ctx, uint32_t attn_layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks,
                                     const uint32_t *d_reqs, uint32_t n_reqs, const void *d_q, void *d_out, float *d_lse,
                                     void *d_workspace, size_t workspace_bytes, void *stream);

/* What stands between a projection and attention, in one pass: query and key heads are normalised and rotated, keys and values go to
 * their pages, queries to d_out.  A head x of head_dim columns becomes
 *     y = x / sqrt(mean(x^2) + eps) * weight        (weight: fp32 [head_dim], one for queries and one for keys; NULL: y = x),
 * and its first rotary_dim columns are rotated in pairs (a, b) <- (a cos t - b sin t, b cos t + a sin t) with t = position * freq[i] for
 * pair i: columns i and i + rotary_dim / 2 (AVMP_ROTATE_HALVES) or 2 i and 2 i + 1 (AVMP_ROTATE_NEIGHBOURS).  Values are copied.
 * All of it is computed in 32 bits (angles in 64) and rounded once.  d_freq: fp32 [rotary_dim / 2], NULL if that is 0.  Positions are the
 * tokens' places in their chains, or d_pos (one per row) where that is not NULL, e.g. behind a shared prefix.
 * Supported: kv_elem_bytes 2, head_dim 64 or 128, rotary_dim a multiple of 8 up to head_dim; else AVMP_EINVAL. */
enum { AVMP_ROTATE_HALVES = 0, AVMP_ROTATE_NEIGHBOURS = 1 };
typedef struct {
    uint32_t type, q_heads, rotary_dim, pairing;
    float eps;                 /* >= 0 */
    uint32_t rsvd;             /* 0 */
    uint64_t q_stride_bytes, k_stride_bytes, v_stride_bytes, out_stride_bytes;
} avmp_rows_desc;

/* Rows d_cu[k] .. d_cu[k+1] are the LAST tokens of request d_reqs[k]'s chain, which already counts them (avmp_step); their K and V are
 * written to attention layer attn_layer of its pages.  Skipped items: a slot that holds nothing, a slot that an earlier entry of the
 * list names, more rows than held tokens, offsets that decrease or pass total_tokens.  n_reqs <= max_requests; total_tokens < 2^31. */
AVMP_API int avmp_attn_rows_prompt(avmp_ctx *ctx, uint32_t attn_layer, const avmp_rows_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                                   const uint32_t *d_cu, uint32_t total_tokens, const uint32_t *d_pos, const void *d_q, const void *d_k,
                                   const void *d_v, const float *d_q_weight, const float *d_k_weight, const float *d_freq, void *d_out,
                                   void *stream);
/* One token per request: row k is the last token of d_reqs[k]'s chain.  Skipped items as above. */
AVMP_API int avmp_attn_rows_step(avmp_ctx *ctx, uint32_t attn_layer, const avmp_rows_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                                 const uint32_t *d_pos, const void *d_q, const void *d_k, const void *d_v, const float *d_q_weight,
                                 const float *d_k_weight, const float *d_freq, void *d_out, void *stream);

/* Linear attention with a decay for each head (the recurrence of a state-space layer), on the state
 * elements of the SSM blocks, laid out [heads][dv][dk] in fp32 (ssm_elem_bytes 4, ssm_state_elems =
 * heads * dv * dk):   S <- exp(g) S + v k^T,   out = S q.
 * Rows: q and k [groups][dk], v and out [heads][dv], g (log decay, fp32, at most 0) [heads]; head h
 * reads group h / (heads / groups).  g of -inf clears the state, whatever it held; a state that is not finite is also gone once the
 * decays since then multiply to less than 2^-126.  There is one decay for a head's whole dv x dk elements (layers with a decay
 * of its own for every channel and state element: avmp_scan_prompt and avmp_scan_step).  Supported: dk 16, 32, 64 or 128, dv a
 * multiple of 32, heads a multiple of groups, at most 2^31 state elements; else AVMP_EINVAL.  The convolution window of the block is
 * not touched. */
typedef struct {
    uint32_t type, heads, groups, dk, dv;
    uint32_t rsvd;             /* 0 */
    uint64_t q_stride_bytes, k_stride_bytes, v_stride_bytes, decay_stride_bytes, out_stride_bytes;
} avmp_ssm_desc;

/* Scratch bytes that any avmp_ssm_prompt call of up to n_reqs list entries and total_tokens rows needs (under 5 MB; 0 on
 * invalid arguments).  Only calls whose few heads and long prompts would leave SMs idle use scratch: where this is 0, and for a
 * call of many requests or heads, the workspace may be NULL. */
AVMP_API size_t avmp_ssm_workspace_bytes(const avmp_ctx *ctx, const avmp_ssm_desc *desc, uint32_t n_reqs, uint32_t total_tokens);

/* Whole prompts: rows d_cu[k] .. d_cu[k+1] are consecutive tokens of request d_reqs[k]; the state after the last
 * of them is left in its block.  d_resume[k] != 0: start from the state in the block; 0, or d_resume NULL:
 * from zero (a fresh block holds leftovers), so that a request without rows gets a zero state.
 * Skipped items: a slot that is not LIVE, a slot that an earlier entry of the list names, offsets that
 * decrease or pass total_tokens.  n_reqs <= max_requests; total_tokens < 2^31. */
AVMP_API int avmp_ssm_prompt(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_ssm_desc *desc, const uint32_t *d_reqs,
                             uint32_t n_reqs, const uint32_t *d_cu, uint32_t total_tokens, const uint32_t *d_resume,
                             const void *d_q, const void *d_k, const void *d_v, const float *d_log_decay, void *d_out,
                             void *d_workspace, size_t workspace_bytes, void *stream);

/* One token per request: row k belongs to d_reqs[k].  Skipped items: a slot that is not LIVE, a slot that an
 * earlier entry of the list names.  n_reqs <= max_requests. */
AVMP_API int avmp_ssm_step(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_ssm_desc *desc, const uint32_t *d_reqs,
                           uint32_t n_reqs, const void *d_q, const void *d_k, const void *d_v, const float *d_log_decay,
                           void *d_out, void *stream);

/* Short causal convolution over a state layer's rows, each channel for itself:
 *     y_t = bias + sum_j weight[j] x_(t - width + 1 + j),   out_t = y_t, or y_t / (1 + exp(-y_t)) with silu 1.
 * Rows of x and out: [channels].  weight: fp32 [channels][width], 16-byte aligned; bias: fp32 [channels], 16-byte aligned, or NULL.  The
 * window elements of the SSM blocks are the last width - 1 rows of a request, oldest first, [width - 1][channels] in fp32.
 * Supported: ssm_elem_bytes 4, width 2, 3 or 4, channels a multiple of 8 up to 2^24, ssm_conv_elems = channels * (width - 1), ssm_state_elems a
 * multiple of 4; else AVMP_EINVAL.  The state elements of the block are not touched. */
typedef struct {
    uint32_t type, channels, width, silu;
    uint64_t x_stride_bytes, out_stride_bytes;
} avmp_conv_desc;

/* Whole prompts and single tokens; rows, requests, d_resume (here: whether the window is continued or counts as zeros) and skipped items
 * as for avmp_ssm_prompt and avmp_ssm_step.  The window after the last row is left in the block. */
AVMP_API int avmp_conv_prompt(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_conv_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                              const uint32_t *d_cu, uint32_t total_tokens, const uint32_t *d_resume, const void *d_x,
                              const float *d_weight, const float *d_bias, void *d_out, void *stream);
AVMP_API int avmp_conv_step(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_conv_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                            const void *d_x, const float *d_weight, const float *d_bias, void *d_out, void *stream);

/* Selective scan: the recurrence of a state layer whose channels and state elements have a decay each, on the state elements of the SSM
 * blocks, laid out [channels][states] in fp32:
 *     step = delta_t + delta_bias, with softplus 1: log(1 + exp(that));
 *     h <- exp(step * A) h + step * u_t * B_t,   y = <C_t, h> + D * u_t,   out_t = y * z_t / (1 + exp(-z_t)).
 * Rows: u, delta, z and out [channels], b and c [groups][states]; channel i reads group i / (channels / groups).
 * A decay exp(step * A) is off by 2^-22 (1 + |step * A|) of its value at most, and 0 below 2^-126.  In a state this adds up over the tokens that
 * it remembers: 3e-6 of it on the mean where they are a thousand, 2.2e-5 where they are twenty thousand; where steps are all alike as much
 * as 9e-5 and 1.6e-3 (exponentials exact but for their rounding to 32 bits: 4e-5 and 7e-4).
 * A: fp32 [channels][states], 16-byte aligned, finite (at most 0 where steps are positive, or states grow without bound); D and delta_bias: fp32
 * [channels] or NULL (without that term); z NULL: out_t = y.  A NaN or an infinity in a channel's rows or state stays in that channel's state; the decay of a
 * single token that is beyond the range of fp32 counts as an infinity (which makes NaN of a zero state).
 * Supported: ssm_elem_bytes 4, states 8, 16, 32 or 64, channels a multiple of 8 * groups up to 2^24, ssm_state_elems = channels *
 * states; else AVMP_EINVAL.  With softplus a delta of -inf or of the type's lowest value leaves the state as it was (u and b
 * of that token being finite: what is added is 0 times their product).  The convolution window of the block is not touched. */
typedef struct {
    uint32_t type, channels, groups, states, softplus;
    uint32_t rsvd;             /* 0 */
    uint64_t u_stride_bytes, delta_stride_bytes, z_stride_bytes, b_stride_bytes, c_stride_bytes, out_stride_bytes;
} avmp_scan_desc;

/* Scratch bytes that any avmp_scan_prompt call of up to n_reqs list entries and total_tokens rows needs (0 on invalid arguments).  Only calls
 * whose few channels and long prompts would leave SMs idle use scratch: where this is 0, and for a call of many requests or channels, the
 * workspace may be NULL. */
AVMP_API size_t avmp_scan_workspace_bytes(const avmp_ctx *ctx, const avmp_scan_desc *desc, uint32_t n_reqs, uint32_t total_tokens);

/* Whole prompts and single tokens; rows, requests, d_resume and skipped items as for avmp_ssm_prompt and avmp_ssm_step. */
AVMP_API int avmp_scan_prompt(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_scan_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                              const uint32_t *d_cu, uint32_t total_tokens, const uint32_t *d_resume, const void *d_u, const void *d_delta,
                              const void *d_b, const void *d_c, const void *d_z, const float *d_a, const float *d_d,
                              const float *d_delta_bias, void *d_out, void *d_workspace, size_t workspace_bytes, void *stream);
AVMP_API int avmp_scan_step(avmp_ctx *ctx, uint32_t ssm_layer, const avmp_scan_desc *desc, const uint32_t *d_reqs, uint32_t n_reqs,
                            const void *d_u, const void *d_delta, const void *d_b, const void *d_c, const void *d_z, const float *d_a,
                            const float *d_d, const float *d_delta_bias, void *d_out, void *stream);

/* Counters -> host.  Synchronises the stream. */
AVMP_API int avmp_get_stats(avmp_ctx *ctx, avmp_stats *h_out, void *stream);
/* Clear the sticky device error code and count.  Stream-ordered. */
AVMP_API int avmp_clear_error(avmp_ctx *ctx, void *stream);

/* Tables <-> host (parity checks, snapshot / restore).  Both synchronise the stream.
 * Import checks the snapshot on the host first (capacities and pool-byte conservation, free lists
 * distinct and inside their stores, page table and owner table mutually inverse, every handle of
 * every request resolvable and owned once) and returns AVMP_EINVAL, with the context untouched, if
 * it does not hang together: the kernels index these tables without bounds checks. */
AVMP_API int avmp_export_tables(avmp_ctx *ctx, avmp_tables *h_out, void *stream);
AVMP_API int avmp_import_tables(avmp_ctx *ctx, const avmp_tables *h_in, void *stream);

/* ---- on-device closed loop (the paper's harness drives its traces from the host, Section 4.1) ----
 * A device-resident scheduler for queue-type traces: every avmp_driver_step builds the next batch
 * on the GPU (FINISH for requests whose decode is complete, EXTEND by one token for the other
 * running requests, ADMITs from the queue head into the lowest free slots within the concurrency
 * and a slow-start window), runs it through the allocator (avmp_step_indirect) and folds the
 * statuses back into the request slots -- three stream-ordered launches and no host round trip, so
 * a serving loop can be queued (or graph-captured) many steps ahead.  d_prompt / d_output are
 * device arrays of n_requests token counts; the driver's slots are the context's request slots.
 * The workspace (avmp_driver_workspace_bytes(max_requests), 256-byte aligned) is the caller's. */
typedef struct avmp_driver avmp_driver;
typedef struct {
    uint64_t steps, completed, dropped, preempted, n_oom_admit, n_oom_extend;
    uint64_t queue_next;      /* requests taken from the arrays so far */
    uint64_t requeued;        /* entries waiting at the queue head (failed admits, pre-empted requests) */
    uint64_t window;          /* current admission window */
    uint64_t last_batch_ops;
    uint64_t overflow;        /* 1 if the re-queue buffer ever overflowed (entries were lost) */
} avmp_driver_stats;
AVMP_API size_t avmp_driver_workspace_bytes(uint32_t max_requests);
AVMP_API int avmp_driver_create(avmp_driver **out, avmp_ctx *ctx, const uint32_t *d_prompt, const uint32_t *d_output,
                                uint32_t n_requests, uint32_t concurrency, void *d_workspace, size_t workspace_bytes,
                                void *stream);
AVMP_API int avmp_driver_destroy(avmp_driver *drv);
AVMP_API int avmp_driver_step(avmp_driver *drv, void *stream);
/* Both synchronise the stream.  Export copies the per-slot arrays (state 0 free / 1 running, request
 * index, tokens held, decode tokens left), max_requests entries each. */
AVMP_API int avmp_driver_get_stats(avmp_driver *drv, avmp_driver_stats *h_out, void *stream);
AVMP_API int avmp_driver_export(avmp_driver *drv, uint32_t *h_state, uint32_t *h_uid, uint32_t *h_len,
                                uint32_t *h_remaining, void *stream);

/* ---- the same loop for multi-turn sessions (the agentic-burst workload; the paper gives that
 * workload one sentence in Section 4.1 and no scheduler, so the policy is this library's) ----
 * Sessions arrive at d_arrival_step[i] (ascending); turn t of session i appends d_turn_prompt[i *
 * max_turns + t] prompt tokens and decodes d_turn_output[...] tokens; between turns the request
 * parks (FINISH with KEEP_KV) for d_turn_think[i * max_turns + t] steps and then resumes on its own
 * slot (ADMIT with RESUME); after turn d_n_turns[i] - 1 it finishes for good.  Each step admits, in
 * this order, re-queued entries, parked sessions whose think time is over (by ready step, then by
 * parking order) and newly arrived sessions, within the concurrency and the slow-start window;
 * a step that saw an OOM or ran out of free slots evicts the longest-parked chain (that session re-enters with its whole
 * context as the prompt), a step without any success pre-empts the most recently admitted
 * request, an admit that fails with nothing running and nothing parked is dropped.
 * All five arrays are device arrays of uint32 owned by the caller and must outlive the driver;
 * concurrency <= 1024.  The workspace (avmp_session_driver_workspace_bytes, 256-byte aligned) is
 * the caller's.  Each step is one launch plus the relocation copy (a few launches when a batch may
 * hold more than one migration), with no host round trip. */
typedef struct avmp_session_driver avmp_session_driver;
typedef struct {
    uint64_t steps, completed, dropped, preempted, evicted, n_oom_admit, n_oom_extend;
    uint64_t arrived;         /* sessions whose arrival step has passed */
    uint64_t arrival_queue;   /* of those, still waiting for their first admission */
    uint64_t requeued;        /* entries at the queue head (failed admits, pre-empted, found no slot) */
    uint64_t waiting;         /* parked or evicted sessions waiting for their ready step */
    uint64_t window, last_batch_ops;
    uint64_t forced_slot;     /* slot the next step will pre-empt or evict, ~0 if none */
} avmp_session_stats;
AVMP_API size_t avmp_session_driver_workspace_bytes(uint32_t max_requests, uint32_t n_sessions);
AVMP_API int avmp_session_driver_create(avmp_session_driver **out, avmp_ctx *ctx, const uint32_t *d_arrival_step,
                                        const uint32_t *d_n_turns, const uint32_t *d_turn_prompt,
                                        const uint32_t *d_turn_output, const uint32_t *d_turn_think,
                                        uint32_t n_sessions, uint32_t max_turns, uint32_t concurrency,
                                        void *d_workspace, size_t workspace_bytes, void *stream);
AVMP_API int avmp_session_driver_destroy(avmp_session_driver *drv);
AVMP_API int avmp_session_driver_step(avmp_session_driver *drv, void *stream);
/* Both synchronise the stream.  Export copies the per-slot arrays (state 0 free / 1 running / 2
 * parked, session index, tokens held, decode tokens left, turn), max_requests entries each, and the
 * session indices in the re-queued and the waiting queue, in order (room for n_sessions each). */
AVMP_API int avmp_session_driver_get_stats(avmp_session_driver *drv, avmp_session_stats *h_out, void *stream);
AVMP_API int avmp_session_driver_export(avmp_session_driver *drv, uint32_t *h_state, uint32_t *h_uid, uint32_t *h_len,
                                        uint32_t *h_remaining, uint32_t *h_turn, uint32_t *h_requeued,
                                        uint32_t *h_waiting, void *stream);

/* How long a wait inside the kernels of later avmp_attn_* and avmp_ssm_prompt calls may last before they give up
 * (AVMP_DEV_TIMEOUT): 2 000 000 000 ns unless set, which is also the most. */
AVMP_API int avmp_set_wait_limit(avmp_ctx *ctx, uint64_t ns);

/* How many kernels this context has launched so far (host counter). */
AVMP_API uint64_t avmp_launch_count(const avmp_ctx *ctx);

AVMP_API const char *avmp_error_string(int code);

#ifdef __cplusplus
}
#endif
#endif
