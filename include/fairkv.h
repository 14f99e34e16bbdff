/*
 * fairkv.h - C ABI of the MI355X (gfx950) library for single-token grouped-query
 * decode attention over a KV cache compressed per head.
 *
 * Setting (paper: Introduction, "unfair head load"; Section 3.2; Section 4.2
 * Fair-Copying; Appendix A).  Per-head KV-cache compression leaves every
 * (sequence b, KV head h) pair with its own number len[b][h] of retained
 * tokens.  Decode attention is bandwidth bound and its cost is linear in the
 * retained tokens (Section 3.2), so unequal heads mean unequal work.  The
 * paper equalises per-GPU load by placing heads with care and by replicating
 * heavy heads so that each replica carries W/copies of the load (Algorithm 2;
 * objective eq. 4, cap on copies eq. 3, coverage eq. 2, efficiency eq. 5).
 * This library applies the same rule inside one GPU: the "devices" are
 * persistent workgroups, one per compute unit, and a heavy pair is shared by
 * several of them, each taking a token chunk.
 *
 * Conventions for every entry point
 *   - returns FAIRKV_OK (0) or a negative fairkv_status; never throws, aborts or prints;
 *   - "host" pointers are ordinary process memory, "device" pointers are HIP device
 *     memory of the current device; the library never allocates or frees device memory
 *     and keeps no state between calls (the only state, the arrival counters, lives in
 *     the caller's workspace); all buffers are owned by the caller;
 *   - on error nothing is launched and no output buffer is written.
 *
 * Packed ragged KV layout.  K and V are two row-major buffers [n_rows][D] of the
 * same element type; the tokens of pair (b, h) are rows off[b][h] ... off[b][h] +
 * len[b][h] - 1 of both.  off is in rows (int64), len in tokens (int32), both
 * [B][Hkv] row-major.  Ranges of different pairs must not overlap; gaps are allowed.
 * A row is D * sizeof(element) bytes and the K and V base addresses must be 16-byte
 * aligned.  Query heads [h*G, (h+1)*G), G = Hq / Hkv, attend over KV head h.
 */
#ifndef FAIRKV_H
#define FAIRKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FAIRKV_OK = 0,
    FAIRKV_EINVAL = -1,       /* null pointer, non-positive size, bad parameter combination */
    FAIRKV_ECAP = -2,         /* caller's output array is too small; the summary says how big */
    FAIRKV_EWORKSPACE = -3,   /* workspace smaller than fairkv_workspace_bytes() */
    FAIRKV_EUNSUPPORTED = -4, /* element type / head_dim / group size without a kernel */
    FAIRKV_EHIP = -5          /* a HIP call failed; the HIP error is left for hipGetLastError */
} fairkv_status;

enum { FAIRKV_BF16 = 0, FAIRKV_F32 = 1,
       FAIRKV_E4M3 = 2, /* one byte per element: fairkv_pack and fairkv_append only (they move bytes) */
       FAIRKV_BF16_VALU = 3 /* in_dtype of fairkv_decode_attn only: bf16 inputs through a vector-ALU kernel instead of
                               the matrix-core kernel; for A/B measurements of the two */ };
enum { FAIRKV_SHORT_PAIR_TOKENS = 96 }; /* a whole pair of at most this many tokens is a "short pair": the bf16 and 8-bit
                                           kernels let one wave run it alone (four such pairs stream side by side,
                                           no fold across waves), and the planner may charge it its own overhead */
enum { FAIRKV_MAX_SLOTS = 320 };   /* most workgroups fairkv_decode_attn launches; a plan with more slots is run with
                                      consecutive slots sharing a workgroup */

/* How the work list is built; the four mirror the paper's ablation (Section 5.2.1).
 *   NAIVE      pairs dealt to slots round-robin in (b, h) order, unsplit: the analogue of the
 *              paper's static head allocation baseline (Figure 3 (1), Section 5.1 Baseline).
 *   LPT        load-aware placement of whole pairs, longest first onto the least loaded slot:
 *              Best-effort Assignment only (Section 1.2, Technique I).
 *   LPT_SPLIT  Fair-Copying as the paper states it (Section 4.2, Algorithm 2): a heavy pair
 *              becomes r equal chunks, each carrying len/r (the W/copies rule), then LPT.
 *   FAIR       Fair-Copying taken to its limit on one GPU, where a replica may take any share:
 *              all pairs are laid end to end and the line is cut into n_slots pieces of equal
 *              cost, so a pair is shared only by the slots whose boundary falls inside it.
 *              Reaches the lower bound of eq. 4 up to min_chunk and the per-item overhead. */
enum { FAIRKV_POLICY_NAIVE = 0, FAIRKV_POLICY_LPT = 1, FAIRKV_POLICY_LPT_SPLIT = 2, FAIRKV_POLICY_FAIR = 3 };

/* One unit of work: rows row ... row + tok_count - 1 of K and V, a chunk of pair (b, h),
 * for all G query heads of the group.  The pair was cut into n_chunks items, of which this
 * is number `chunk` (in token order: the first token of the chunk is row - off[b][h]);
 * part is the index of this item's partial result, and the partials of a pair are
 * consecutive: part - chunk ... part - chunk + n_chunks - 1.  A pair without tokens has
 * one item with tok_count == 0, so that some slot writes its zero output. */
typedef struct {
    int64_t row;
    int32_t tok_count;
    int32_t b, h;
    int32_t chunk;
    int32_t n_chunks;
    int32_t part;
} fairkv_item;          /* 32 bytes */

typedef struct {
    int32_t n_slots;         /* persistent workgroup slots to balance over (one per compute unit) */
    int32_t tile;            /* cuts inside a pair fall on multiples of this many tokens (>= 1) */
    int32_t min_chunk;       /* no piece of a cut pair is smaller; positive multiple of tile */
    int32_t max_split;       /* most items one pair may be cut into: eq. 3's cap (>= 1) */
    int32_t oversub;         /* LPT_SPLIT aims for about n_slots * oversub chunks in total (>= 1) */
    int32_t overhead_tokens; /* fixed cost of an item in token units: the offset of the
                                linear latency model of Section 3.2 (>= 0) */
    int32_t policy;          /* FAIRKV_POLICY_* */
    int32_t short_overhead_tokens; /* the same for an item that is a short pair (a whole pair of at most
                                FAIRKV_SHORT_PAIR_TOKENS tokens, empty pairs included); 0: overhead_tokens (>= 0) */
} fairkv_plan_params;

typedef struct {
    int64_t total_tokens;    /* sum of len */
    int64_t max_slot_load;   /* largest and smallest predicted slot load, in token units, */
    int64_t min_slot_load;   /*   over ALL n_slots (an idle slot counts 0): eq. 4 / Algorithm 2 */
    int32_t n_items;         /* items the plan has (also when it did not fit items_cap) */
    int32_t n_parts;         /* partial-result slots the workspace must hold (== n_items) */
} fairkv_plan_summary;

/* Defaults: n_slots = n_compute_units, tile 16, min_chunk 32, max_split 256, oversub 2,
 * overhead_tokens 160 (measured on MI355X: an extra item in a slot costs about as much as
 * streaming 120-160 tokens; large layers are within 1 % from 96 to 192), short_overhead_tokens 48
 * (a short pair costs a slot about a third of that), policy FAIR.  n_compute_units must be >= 1.
 * The token-valued fields are those of a bf16 cache with D = 128.  Where a token is fewer or more bytes the same item is worth
 * more or fewer tokens: measured good are tile 32, min_chunk 64, overhead_tokens 256, short_overhead_tokens 128 for an 8-bit
 * cache and overhead_tokens 64, short_overhead_tokens 32 for an fp32 cache (up to 22 % less time than with the defaults).  On a
 * bf16 cache of few or short pairs overhead_tokens 96 and min_chunk 64 or 128 are better (256 pairs of 64 tokens 7.3 -> 4.9 us, one
 * sequence of eight pairs of 1024 9.4 -> 8.8), on large layers by at most 1 %. */
int fairkv_default_params(fairkv_plan_params *p /*host, out*/, int32_t n_compute_units);

/*
 * Host-side planner (integer arithmetic only; deterministic).  An item costs
 * tok_count + ov, ov = short_overhead_tokens for a short pair (if that is not 0) and overhead_tokens
 * otherwise; the load of a slot is the sum over its items (objective: eq. 4).
 *
 * FAIR       pairs in (b, h) order fill slot 0, 1, ...  A slot opened as number j gets the budget
 *            ceil((tokens not yet placed + the ov of every pair not yet finished, taken whole +
 *            overhead_tokens * slots unopened) / slots unopened).  With fit = the whole tiles that still fit the slot's room: a pair
 *            (or its rest) that fits is placed whole; else it is cut at `fit` if both pieces are
 *            >= min_chunk; else it is placed whole anyway if the excess is <= fit; else the slot
 *            is closed and the next one opened.  After a cut the rest goes on in the next slot.
 *            The last slot, and the max_split-th piece of a pair, take all that is left.
 * LPT_SPLIT  target = max(min_chunk, roundup_tile(ceil(sum len / (n_slots * oversub)))); a pair is
 *            cut into r = min(max_split, ceil(len / target)) shares of roundup_tile(ceil(len / r))
 *            tokens, the last one shorter (W / copies, Algorithm 2); shares are sorted by
 *            tok_count descending, then pair and chunk ascending, and each goes to the slot with
 *            the smallest load so far (lowest index on ties).
 * LPT        the same with whole pairs.  NAIVE: whole pairs, pair i to slot i mod n_slots.
 *
 * len, off   host [B*Hkv]: tokens and first row of every pair; len >= 0, off >= 0 where len > 0.
 * items      host [items_cap], out, grouped by slot, inside a slot in the order the slot runs
 *            them; may be NULL iff items_cap == 0.
 * slot_ptr   host [n_slots+1] or NULL, out: slot j runs items[slot_ptr[j] .. slot_ptr[j+1]).
 * part_base  host [B*Hkv+1] or NULL, out: items before each pair; pair p owns partial slots
 *            part_base[p] ... part_base[p+1]-1, in chunk order.
 * summary    host, out, required; filled whenever the arguments are valid.
 *
 * Returns FAIRKV_ECAP (after filling summary, slot_ptr and part_base, writing no item)
 * when the plan has more items than items_cap: call once with items_cap = 0 to size.
 */
int fairkv_plan(const int32_t *len, const int64_t *off, int32_t B, int32_t Hkv, const fairkv_plan_params *p,
                fairkv_item *items, int32_t items_cap, int32_t *slot_ptr, int32_t *part_base,
                fairkv_plan_summary *summary);

/* Bytes of device workspace fairkv_decode_attn needs: fp32 partial outputs and softmax
 * statistics for n_parts items, plus the arrival counters of the hand-over.  0 on bad arguments.
 * Layout: the counters first (fairkv_workspace_counter_bytes(n_pairs) bytes: one per pair and
 * one per group of 8 pieces of a pair cut 16 ways or more; their number depends on n_pairs alone),
 * then statistics and partial outputs.  The counter bytes must be zero before the first use;
 * every completed call leaves them zero again, whatever its plan, so calls that are ordered on
 * one stream may share one workspace (the counter region of a smaller B * Hkv is a prefix of a
 * larger one's).  After a launch that did not complete (an aborted process, a device reset) zero
 * the counter bytes again: nothing else in the workspace carries state from call to call. */
size_t fairkv_workspace_counter_bytes(int32_t n_pairs);
size_t fairkv_workspace_bytes(int32_t n_parts, int32_t n_pairs, int32_t G, int32_t D);

/* Sets the counter bytes of a device workspace (the first fairkv_workspace_counter_bytes(n_pairs) bytes) to zero
 * with a small kernel on hip_stream, without synchronising: for a fresh workspace, and for one that a launch which
 * did not complete may have left with non-zero counters.  workspace: device, 16-byte aligned, at least that many
 * bytes (FAIRKV_EWORKSPACE otherwise).  Order it on the stream before the next decode call. */
int fairkv_workspace_reset(void *workspace, size_t workspace_bytes, int32_t n_pairs, void *hip_stream);

/*
 * Decode attention for one layer: for every sequence b and query head hq (KV head
 * h = hq / G), out[b][hq] = softmax(scale * q[b][hq] . K_rows^T) V_rows over the
 * len[b][h] retained rows of pair (b, h), and lse[b][hq] = log sum exp of the scaled
 * scores.  Pairs with len == 0 give out = 0 and lse = -inf.  Accumulation is fp32.
 *
 * Enqueues ONE kernel on hip_stream and returns without synchronising: n_slots persistent
 * workgroups, workgroup j streaming the K/V rows of its items from HBM exactly once (shared
 * by the G query heads of the group).  An item that is a whole pair writes out directly; the
 * items of a cut pair leave partial results in the workspace and the one that finishes last
 * combines them (log-sum-exp merge), so no second launch is needed.
 *
 * q          device [B][Hq][D], element type in_dtype, 16-byte aligned
 * k, v       device [n_rows][D], element type in_dtype, 16-byte aligned; every item must lie inside:
 *            row + tok_count <= n_rows (else FAIRKV_EINVAL)
 * items      device [n_items]: the items of a plan made by fairkv_plan from this cache's len
 *            and off, copied to the device by the caller.  The kernels read exactly the rows
 *            the items name.
 * items_host HOST [n_items]: the same array as the planner wrote it, and
 * slot_ptr   HOST [n_slots+1]: the plan's slot pointer.  The slot pointer and the first item
 *            of every slot travel to the GPU inside the kernel arguments, so that a workgroup
 *            requests its first K/V rows without first fetching its item list (two memory
 *            round trips less at the start of a 20 us kernel); with more than
 *            FAIRKV_MAX_SLOTS slots, consecutive slots share a workgroup.  items_host is also
 *            checked: every item must name a pair of this problem, rows >= 0 and a partial slot
 *            below n_parts, and a cut pair must come with every one of its n_chunks pieces, each
 *            once, in consecutive partial slots (else FAIRKV_EINVAL).
 * workspace  device, at least fairkv_workspace_bytes(n_parts, B*Hkv, G, D) bytes, 16-byte
 *            aligned, its counter bytes zero before the first use (see fairkv_workspace_bytes)
 * out        device [B][Hq][D], element type out_dtype (FAIRKV_F32, or FAIRKV_BF16 rounded
 *            to nearest even), 16-byte aligned
 * lse        device [B][Hq] float, or NULL
 * scale      multiplies the scores (1/sqrt(D) in the usual models)
 * hip_stream a hipStream_t (NULL = the default stream)
 *
 * Supported: D in {64, 128}; in_dtype BF16 or F32 (or BF16_VALU); G = Hq/Hkv in {1, 2, 4, 8}
 * (else FAIRKV_EUNSUPPORTED).
 * Calls that share a workspace must be ordered on one stream.
 */
int fairkv_decode_attn(const void *q, const void *k, const void *v, int64_t n_rows,
                       const fairkv_item *items, const fairkv_item *items_host, int32_t n_items,
                       const int32_t *slot_ptr, int32_t n_slots,
                       int32_t n_parts, void *workspace, size_t workspace_bytes,
                       void *out, float *lse,
                       int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
                       int32_t in_dtype, int32_t out_dtype, float scale, void *hip_stream);

/* ---- placement over the GPUs of a tensor-parallel group (Section 4.3, Algorithms 1 and 2) -------
 *
 * Host only.  Which GPU holds which attention head of one layer, and which heads are replicated
 * so that their copies share the batch rows (Fair-Copying); with max_extra = 0 it is the
 * Best-effort Assignment (heads permuted over GPUs, no copies).  A copy of a head with c copies
 * weighs W / c (Algorithm 2's adjusted weights); the scheme kept is the first one, in the order of
 * the paper's two algorithms, with the smallest difference between the heaviest and the lightest
 * GPU (Algorithm 2's criterion).  Appendix A: every head is placed (eq. 2), at most max_copies
 * copies per head (eq. 3), efficiency = mean load / largest load (eq. 5).
 *
 * Readings: the extra copies of a scheme, sum over heads of (copies - 1), are at most max_extra
 * (Algorithm 1 declares such a bound and never uses it); the copies of a head sit on different
 * GPUs; GPUs may hold different numbers of heads; an idle GPU weighs 0; schemes are walked head
 * by head with 1 copy first, then 2, 3, ..., and splits in lexicographic order of the GPU of
 * (head 0 copy 0, head 0 copy 1, ..., head 1 copy 0, ...).
 *
 * FAIRKV_PLACE_EXACT walks all schemes (exponential: meant for the paper's handful of heads);
 * FAIRKV_PLACE_GREEDY places copies longest first on the least loaded GPU that does not hold
 * the head yet, then up to max_extra times gives one more copy to the heaviest copy on the
 * most loaded GPU while that lowers the largest load; FAIRKV_PLACE_AUTO is EXACT while
 * n_heads + max_extra <= 12, else GREEDY. */
enum { FAIRKV_PLACE_AUTO = 0, FAIRKV_PLACE_EXACT = 1, FAIRKV_PLACE_GREEDY = 2 };

typedef struct {
    int32_t tp;          /* GPUs of the group, >= 1 */
    int32_t max_extra;   /* m: extra copies in total, >= 0 */
    int32_t max_copies;  /* R_max of eq. 3: copies per head, 1..8 (and never more than tp) */
    int32_t mode;        /* FAIRKV_PLACE_* */
} fairkv_place_params;

/* One copy of a head: GPU `gpu` serves batch rows [row_begin, row_end) of head `head`.  The
 * copies of a head are numbered by ascending GPU and share the B rows contiguously; with c
 * copies the first B mod c of them take ceil(B / c) rows. */
typedef struct {
    int32_t head, gpu, copy, n_copies, row_begin, row_end;
} fairkv_share; /* 24 bytes */

typedef struct {
    int64_t den;           /* loads are in units of 1/den tokens, den = lcm(1..max_copies) */
    int64_t delta_num;     /* heaviest minus lightest GPU */
    int64_t max_load_num;
    int64_t min_load_num;
    double efficiency;     /* eq. 5 */
    int32_t n_shares;      /* copies in the scheme (also when they did not fit shares_cap) */
    int32_t exact;         /* 1: exhaustive walk, 0: greedy */
} fairkv_place_summary;

/* W         host [n_heads]: weight of every head (tokens it keeps, summed over the batch), 0..2^40
 * B         batch rows to share among the copies of a head, >= 1
 * shares    host [shares_cap], out, ordered by (head, copy); may be NULL iff shares_cap == 0
 * gpu_load  host [tp] or NULL, out: load of every GPU in units of 1/den
 * summary   host, out, required
 * Returns FAIRKV_ECAP (summary and gpu_load filled, no share written) when the scheme has more
 * copies than shares_cap; n_heads + max_extra always suffices. */
int fairkv_place(const int64_t *W, int32_t n_heads, int32_t B, const fairkv_place_params *p,
                 fairkv_share *shares, int32_t shares_cap, int64_t *gpu_load, fairkv_place_summary *summary);

/* Several new tokens per sequence in one call (a draft of q_len tokens being verified, or a short
 * chunk of prompt): not in the paper; the same path with the G heads of a group and the q_len new
 * tokens sharing the 16 columns of a matrix-core tile, so K and V are still streamed once.  The
 * caller has appended the new tokens' K/V first: they are the LAST q_len rows of every pair, and
 * new token i (0-based) attends rows [0, len - (q_len - 1 - i)) of the pair (causal among the new
 * tokens; nothing if that is not positive: out 0, lse -inf).  q and out are [B][q_len][Hq][D],
 * lse [B][q_len][Hq]; everything else as in fairkv_decode_attn, which is the case q_len = 1.
 * The workspace must hold fairkv_workspace_bytes(n_parts, B*Hkv, G * q_len, D) bytes.
 * The last chunk of a cut pair must hold at least q_len - 1 tokens (else FAIRKV_EINVAL): the rows
 * the new tokens hide from one another are masked inside that chunk only.  The FAIR policy makes
 * no chunk below min_chunk >= 16, so its plans always qualify.
 * Supported: bf16 inputs, G * q_len in {1, 2, 4, 8, 16} (else FAIRKV_EUNSUPPORTED). */
int fairkv_decode_attn_multi(const void *q, const void *k, const void *v, int64_t n_rows,
                             const fairkv_item *items, const fairkv_item *items_host, int32_t n_items,
                             const int32_t *slot_ptr, int32_t n_slots,
                             int32_t n_parts, void *workspace, size_t workspace_bytes,
                             void *out, float *lse,
                             int32_t B, int32_t q_len, int32_t Hq, int32_t Hkv, int32_t D,
                             int32_t in_dtype, int32_t out_dtype, float scale, void *hip_stream);

/* The same path over a cache stored as 8-bit floats: not in the paper (which fixes no storage
 * precision), an extension of its decode step.  Half the bytes per retained token, on a path bound
 * by HBM bandwidth.
 * k8, v8   device [n_rows][D] bytes: E4M3 in the finite-only encoding (1 sign, 4 exponent bits with
 *          bias 7, 3 mantissa bits; no infinities; S.1111.111 is NaN and must not occur).  A stored
 *          byte x stands for the value x * k_scale (x * v_scale): one scale per tensor.
 * q        device bf16 [B][q_len][Hq][D], D 64 or 128; out, lse, items, slot_ptr, workspace, n_rows,
 *          q_len as in fairkv_decode_attn_multi (q_len = 1: fairkv_decode_attn).
 * The bytes are widened to bf16 exactly and the products run as in the bf16 path, k_scale folded
 * into the softmax scale and v_scale into the final normalisation.
 * Returns FAIRKV_EINVAL for a scale that is not finite. */
int fairkv_decode_attn_kv8(const void *q, const void *k8, const void *v8, int64_t n_rows,
                           float k_scale, float v_scale,
                           const fairkv_item *items, const fairkv_item *items_host, int32_t n_items,
                           const int32_t *slot_ptr, int32_t n_slots,
                           int32_t n_parts, void *workspace, size_t workspace_bytes,
                           void *out, float *lse,
                           int32_t B, int32_t q_len, int32_t Hq, int32_t Hkv, int32_t D,
                           int32_t out_dtype, float scale, void *hip_stream);

/* The same with a scale per KV head: k_scale, v_scale host [Hkv], Hkv <= 8 (else FAIRKV_EUNSUPPORTED); a
 * stored byte of head h stands for byte * k_scale[h] (v_scale[h]).  The scales travel in the kernel
 * arguments; nothing else differs from fairkv_decode_attn_kv8. */
int fairkv_decode_attn_kv8_per_head(const void *q, const void *k8, const void *v8, int64_t n_rows,
                                    const float *k_scale, const float *v_scale,
                                    const fairkv_item *items, const fairkv_item *items_host, int32_t n_items,
                                    const int32_t *slot_ptr, int32_t n_slots,
                                    int32_t n_parts, void *workspace, size_t workspace_bytes,
                                    void *out, float *lse,
                                    int32_t B, int32_t q_len, int32_t Hq, int32_t Hkv, int32_t D,
                                    int32_t out_dtype, float scale, void *hip_stream);

/* For callers that cannot allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  fairkv_decode_attn_multi with the workspace inside the library: a device
 * array of FAIRKV_STATIC_WORKSPACE_BYTES that is part of the loaded library on every GPU (each GPU the library
 * runs on holds it until the process ends).  The call allocates and frees nothing, on the device or on the
 * host; inputs and outputs are the caller's as before.
 * Returns FAIRKV_EWORKSPACE when fairkv_workspace_bytes(n_parts, B*Hkv, G*q_len, D) exceeds
 * FAIRKV_STATIC_WORKSPACE_BYTES (8 MiB: about 1500 partial slots at G = 8, D = 128; the largest workload here,
 * 1024 pairs on 256 slots, needs 1279).  Everything else as fairkv_decode_attn_multi, same kernels.
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (different streams, or
 * different host threads without ordering) race; order them on one stream.  The array is zero when the
 * library is loaded; a call needs only the arrival counters at the array's start to be zero, and every
 * completed call leaves them zero, whatever its sizes (nothing else is read before it is written). */
enum { FAIRKV_STATIC_WORKSPACE_BYTES = 8 << 20 };
int fairkv_decode_attn_static(const void *q, const void *k, const void *v, int64_t n_rows,
                              const fairkv_item *items, const fairkv_item *items_host, int32_t n_items,
                              const int32_t *slot_ptr, int32_t n_slots, int32_t n_parts, void *out, float *lse,
                              int32_t B, int32_t q_len, int32_t Hq, int32_t Hkv, int32_t D,
                              int32_t in_dtype, int32_t out_dtype, float scale, void *hip_stream);

/* ---- building and growing the packed cache (the step before the path) ---------------------------
 *
 * fairkv_pack gathers the tokens a per-head compressor kept (Section 2: which entries a method
 * retains per head is its own business) out of a dense cache into the packed layout: for pair
 * p = b*Hkv + h and i < len, packed row off[p] + i = dense row keep_t[keep_ptr[p] + i] of
 * k_dense[b][h].  The rows to move are named by a work list in the format of fairkv_plan (made
 * from the same len and off: an item is a run of tok_count packed rows of pair (b, h) starting
 * at row; chunk fields are ignored), so that a ragged cache is gathered by evenly loaded
 * workgroups, one per slot.  Rows of no pair are left untouched.
 *
 * All pointers are DEVICE pointers.  k_dense, v_dense [B][Hkv][T][D] and k_out, v_out
 * [n_rows][D] of element type dtype, 16-byte aligned; keep_ptr int64 [B*Hkv+1]; keep_t int32;
 * off int64 [B*Hkv]; items [slot_ptr[n_slots]], slot_ptr int32 [n_slots+1]; bad: int32 counter or
 * NULL, incremented for every item or row that points outside its arrays (such rows are skipped,
 * nothing out of bounds is touched).  Supported: D * sizeof(element) in {128, 256, 512}.
 * Enqueues one kernel on hip_stream; no synchronisation. */
int fairkv_pack(const void *k_dense, const void *v_dense, int32_t B, int32_t Hkv, int32_t T, int32_t D,
                int32_t dtype, const int64_t *keep_ptr, const int32_t *keep_t, const int64_t *off,
                const fairkv_item *items, const int32_t *slot_ptr, int32_t n_slots, void *k_out, void *v_out,
                int64_t n_rows, int32_t *bad, void *hip_stream);

/* fairkv_append puts a decode step's new K and V row of every pair (k_new, v_new [B][Hkv][D])
 * behind the pair's last row, row off[p] + len[p], and adds one to len[p]; a pair with
 * len[p] >= cap[p] (its reserved rows are used up) is left alone and counted in *full.  All
 * pointers are DEVICE pointers; len is updated in place.  The caller re-plans (or grows the last
 * chunk of every pair in its plan) from the new lengths.  Enqueues one kernel; no synchronisation. */
int fairkv_append(const void *k_new, const void *v_new, int32_t B, int32_t Hkv, int32_t D, int32_t dtype,
                  const int64_t *off, int32_t *len, const int32_t *cap, void *k, void *v, int64_t n_rows,
                  int32_t *full, void *hip_stream);

/* Host mirror of fairkv_append for a plan that stays in use: the last chunk of every pair whose
 * len[p] < cap[p] covers one more row (tok_count + 1) and len[p] grows by one; pairs at capacity
 * are left alone.  items, len (in/out) and cap are HOST arrays; items must be a whole plan (one
 * last chunk per pair).  The plan stays valid and drifts from balance by at most one row per pair
 * and step; re-plan with fairkv_plan every few hundred steps. */
int fairkv_plan_grow(fairkv_item *items, int32_t n_items, int32_t B, int32_t Hkv, int32_t *len, const int32_t *cap);

/* ---- a step over a growing cache: append the new tokens, attend, keep what was accepted -----------
 *
 * The entry points above plan on the host, for lengths that stay as the compressor left them.  While a sequence is
 * decoded its lengths grow, by one token a step or by the accepted part of a draft, and they are known on the GPU first.
 * The three calls of such a step read lengths there and nowhere else: nothing is planned on the host, and a step captured
 * into a graph may be replayed while the cache grows.
 *
 *     fairkv_append_rotated       the new tokens' heads: norm, rotation by position, keys and values into the cache
 *     fairkv_decode_attn_tree     every new token attends over the cache and over the new tokens that are its ancestors
 *     fairkv_accept               the rows of the accepted path move to the front of the draft's, the others are dropped
 *
 * fairkv_cache says where a layer's rows are.  Pair p = b * Hkv + h, token t >= 0:
 *   packed (off given, pages null)   row off[p] + t
 *   paged (pages given, off null)    row pages[p * max_pages + t / page_rows] * page_rows + t % page_rows
 * A pair may hold cap[p] tokens (paged: and max_pages * page_rows).  Rows of different pairs must not overlap; pages that no
 * token lies in are not looked at.  A token whose page or row lies outside the n_rows rows has no such row:
 * it is not attended to, and nothing is appended or moved there.  A packed pair whose run of len rows does not lie inside the cache as a whole is
 * not attended to at all (its nodes see nothing); append and accept look at the rows that they read and write. */
enum { FAIRKV_MAX_DRAFT = 64,     /* most new tokens of a sequence in one call */
       FAIRKV_CACHE_SCALES = 32 };

typedef struct {
    void *k, *v;             /* device [n_rows][D] of type dtype, 16-byte aligned */
    int64_t n_rows;
    const int64_t *off;      /* device [B][Hkv], or NULL */
    const int32_t *pages;    /* device [B][Hkv][max_pages], or NULL */
    const int32_t *cap;      /* device [B][Hkv] */
    int32_t max_pages;       /* 0 for a packed cache */
    int32_t page_rows;       /* a power of two, 16 or more; 0 for a packed cache */
    int32_t B, Hkv, D;       /* D 64 or 128 */
    int32_t dtype;           /* FAIRKV_BF16, FAIRKV_E4M3 or (append, accept) FAIRKV_F32 */
    int32_t n_scales;        /* E4M3: 1, or Hkv (at most FAIRKV_CACHE_SCALES): a stored byte of head h stands for byte * k_scale[h]; else 0 */
    float k_scale[FAIRKV_CACHE_SCALES], v_scale[FAIRKV_CACHE_SCALES];   /* finite, not 0, their reciprocals finite */
    int64_t expected_rows;   /* rows that all pairs together are expected to have, 0: as many as there are.  Only what is fast, and the order of sums,
                              * depends on it: the attention deals its columns for so much work (and takes a workspace for that).  Worth giving where
                              * the cache is made for far more rows than the sequences have. */
} fairkv_cache;              /* a host struct; 344 bytes */

/* What is done to the heads of new queries and keys before they are used, all of it in fp32, rounded once at the end:
 *   x = x / sqrt(mean(x^2) + eps) * norm      over the D elements of a head; q_norm, k_norm device float [D], NULL: not done
 *   (x_a, x_b) = (x_a cos - x_b sin, x_b cos + x_a sin)   for the rot / 2 pairs of the first rot elements: a = i, b = i + rot / 2,
 *       or with `pairs` set a = 2 i, b = 2 i + 1.  table: device float [n_pos][rot], the cosines of the rot / 2 angles of a position
 *       and then their sines (made in as many bits as far positions want), 16-byte aligned; NULL: not done.
 *   pos        device int32 [B][q_len]: the new tokens' positions (the nodes of a tree at one depth share one). */
typedef struct {
    const float *q_norm, *k_norm;
    const float *table;
    const int32_t *pos;
    float eps;               /* >= 0 */
    int32_t n_pos, rot;      /* rot a multiple of 16, at most D */
    int32_t pairs;
} fairkv_rotation;

/* Norm and rotation of q_len new tokens per sequence; queries go to q_out, keys and values into the cache as tokens
 * len[p] .. len[p] + n - 1 of every pair, with len_out[p] = len[p] + n, n = n_new[b].
 * q, k_new, v_new   device, of type dtype (BF16, or F32 with an F32 cache): token (b, i) at element (b * q_len + i) * stride, its Hq (Hkv)
 *                   heads one behind the other; strides in elements, at least Hq * D (Hkv * D), so that all three may lie in one
 *                   projection's output.  16-byte aligned, strides multiples of 16 bytes.
 * q_out             device [B][q_len][Hq][D] of type dtype; may be q where q's tokens follow one another, else it must not meet what lies from
 *                   the first to the last token of q, k_new or v_new
 * n_new             device [B]: how many of the q_len tokens a sequence has (taken into 0 .. q_len), or NULL: all.  What is behind them is not
 *                   read, and the queries there are left as they are.
 * len_out           device [B][Hkv]; may be len
 * bad               device counter or NULL: plus one for every pair that is left alone (its length kept, none of its rows written), because
 *                   it has no room for all n, a row of them lies outside the cache or a position outside the table, and for every token whose
 *                   queries are left alone because its position lies outside the table.
 * An E4M3 cache takes x / scale, the quotient of two fp32 numbers, rounded to nearest even, what is beyond +-448 as +-448.
 * Enqueues one kernel; no synchronisation.  FAIRKV_EUNSUPPORTED: q_len > FAIRKV_MAX_DRAFT, types, D.  FAIRKV_EINVAL also: more than 2^24 - 1
 * workgroups, of 64 tokens' queries each and of one pair or more each. */
int fairkv_append_rotated(const fairkv_cache *cache, const fairkv_rotation *r, const void *q, int64_t q_stride, const void *k_new,
                          int64_t k_stride, const void *v_new, int64_t v_stride, void *q_out, int32_t q_len, int32_t Hq, int32_t dtype,
                          const int32_t *n_new, const int32_t *len, int32_t *len_out, int32_t *bad, void *hip_stream);

/* Attention of a draft tree.  The last n = n_new[b] of the len[p] rows of every pair are the draft's (fairkv_append_rotated has put
 * them there); node i < n of sequence b sees every row in front of them and draft row j < n iff bit j of tree[b][i] is set: its ancestors'
 * bits and, as a rule, its own.  tree == NULL: nodes 0 .. i, a chain; q_len = 1 is a plain decode step.
 * out = softmax(scale * q . K^T) V over the rows that are seen, in fp32, and lse = log sum exp of the scaled scores; a node that sees
 * nothing, or only rows whose scores are -inf, gets out = 0 and lse = -inf.  An infinite or NaN row counts for the nodes that see it only: an
 * infinite value gives an infinite output as long as its weight, next to the largest, is one of fp32's normal numbers (2^-126), below that an
 * infinite one or NaN, as 0 times infinity.  Softmax weights have all 24 bits for an fp32
 * output, 2^-16 of them are lost for a bf16 one.  Nodes i >= n are left as they are.
 * q          device bf16 [B][q_len][Hq][D], 16-byte aligned; Hq a multiple of Hkv, any Hq / Hkv up to 16
 * tree       device uint64 [B][q_len], or NULL
 * workspace  device, fairkv_tree_workspace_bytes(cache, Hq, q_len, n_slots) bytes, 16-byte aligned.  Its first fairkv_tree_counter_bytes(n_slots)
 *            bytes must be zero before the first use (fairkv_tree_workspace_reset); every completed call leaves them zero, and nothing else
 *            in it is kept from call to call, so calls of any shapes with one n_slots that are ordered on one stream may share it.  What
 *            it takes does not fall with q_len, Hq or expected_rows: a workspace for a cache's longest draft is one for all shorter ones.
 * n_slots    workgroups to balance over: the GPU's compute units
 * out        device [B][q_len][Hq][D] of out_dtype (FAIRKV_F32 or FAIRKV_BF16); lse device float [B][q_len][Hq] or NULL
 * Lengths below 0 count as 0, those beyond the cache's rows (paged: max_pages * page_rows) as that many.
 * Enqueues one kernel; no synchronisation.  FAIRKV_EUNSUPPORTED: q_len > FAIRKV_MAX_DRAFT, an F32 cache, D, Hq / Hkv > 16.  FAIRKV_EINVAL also:
 * more than 2^31 - 1 elements of q, a scale (times a k_scale) that is not finite in log2 units. */
size_t fairkv_tree_counter_bytes(int32_t n_slots);
size_t fairkv_tree_workspace_bytes(const fairkv_cache *cache, int32_t Hq, int32_t q_len, int32_t n_slots);
int fairkv_tree_workspace_reset(void *workspace, size_t workspace_bytes, int32_t n_slots, void *hip_stream);
int fairkv_decode_attn_tree(const fairkv_cache *cache, const void *q, const uint64_t *tree, const int32_t *n_new, const int32_t *len,
                            void *workspace, size_t workspace_bytes, int32_t n_slots, void *out, float *lse, int32_t q_len, int32_t Hq,
                            int32_t out_dtype, float scale, void *hip_stream);

/* Keeps n_path[b] of the n = n_new[b] draft rows at the end of every pair: draft row path[b][i] becomes draft row i for i < n_path[b], and
 * len_out[p] = len[p] - n + n_path[b].  path: device int32 [B][q_len], in any order, what is behind n_path[b] is not read; n_path device [B].
 * A pair is left alone (its length kept) and counted in *bad if n_path[b] is not in 0 .. n, an entry not in 0 .. n - 1, its length below n,
 * or a row outside the cache.  len_out may be len; bad may be NULL.  Enqueues one kernel; no synchronisation.  FAIRKV_EINVAL also: more
 * than 2^24 - 1 workgroups, of one pair or more each. */
int fairkv_accept(const fairkv_cache *cache, const int32_t *path, const int32_t *n_path, const int32_t *n_new, const int32_t *len,
                  int32_t *len_out, int32_t q_len, int32_t *bad, void *hip_stream);

/* The same, and the weights of the rows that move (fairkv_attn_weights, below) move with them: device float [n_rows], or NULL, which is fairkv_accept. */
int fairkv_accept_weights(const fairkv_cache *cache, float *weights, const int32_t *path, const int32_t *n_path, const int32_t *n_new,
                          const int32_t *len, int32_t *len_out, int32_t q_len, int32_t *bad, void *hip_stream);

/* ---- compression of a growing cache: which rows matter, which stay, and away with the others ---------
 *
 * What makes a cache one that is compressed per head (the setting above) and keeps it one while it grows.  Three calls, which read lengths and lists
 * on the GPU and may be captured:
 *
 *     fairkv_attn_weights    the attention weight that the last tokens' queries give every row, added to what it had
 *     fairkv_select          which rows of every pair stay, under a budget of the pair or of the sequence
 *     fairkv_evict           these rows move to the front of their pair, or into another cache
 *
 * Weights lie as the rows do: weights[row] belongs to row `row` of the cache, whichever pair and token that is, so what moves rows has to move them:
 * fairkv_evict does, and fairkv_accept_weights.
 * A draft is scored in one of two orders.  fairkv_accept, then fairkv_attn_weights with the queries and log-sum-exps of the accepted nodes, gathered in
 * the order of the path (from a root on), tree NULL and n_new = n_path: rows have what the accepted tokens gave them.  Or fairkv_attn_weights with the
 * draft's tree, then fairkv_accept_weights: rows keep what rejected nodes gave them, too.
 * A row that was appended and not scored has what its place in weights held before, a dropped token's weight maybe, and that counts (times decay) from
 * the next call on.  So every step is scored, or weights of rows that are appended without are set by the caller; a call with decay 0 sets those of
 * all tokens. */

/* For every token t of every pair, over the q_len queries of a sequence (its last n = n_new[b] tokens, whose rows are in the cache already):
 *     weights_out[row] = decay * weights[row] + sum over the nodes i < n that see t, and the heads g of the group, of exp(scale * q . k_t - lse)
 * in fp32; a row of the last n themselves starts from 0 instead of from decay * weights[row], and with decay 0 weights are not read.  Who sees what
 * is as in fairkv_decode_attn_tree, whose lse of the same queries it takes.
 * q            device bf16 [B][q_len][Hq][D], 16-byte aligned; Hq a multiple of Hkv, any Hq / Hkv up to 16
 * tree, n_new  as in fairkv_decode_attn_tree; queries and lse of nodes i >= n are not read
 * lse          device float [B][q_len][Hq]; -inf for a node that sees nothing, which gives no weight to any row, whatever is in it
 * weights      device float [n_rows]; weights_out may be weights, or must not meet it
 * n_slots      the GPU's compute units
 * Rows of no token are left as they are, and so are those of a packed pair whose run sticks out of the cache.  The sums are the same from call to
 * call.  A NaN or infinite row counts for the nodes that see it, in its own weight only; a node whose lse is +inf gives rows of finite scores no
 * weight, one whose lse is NaN gives NaN to all that it sees.
 * Enqueues one kernel; no synchronisation, no workspace.  FAIRKV_EUNSUPPORTED: q_len > FAIRKV_MAX_DRAFT, an F32 cache, D, Hq / Hkv > 16.
 * FAIRKV_EINVAL also: more than 2^31 - 1 elements of q, a decay, or a scale (times a k_scale) in log2 units, that is not finite. */
int fairkv_attn_weights(const fairkv_cache *cache, const void *q, const uint64_t *tree, const int32_t *n_new, const int32_t *len,
                        const float *lse, const float *weights, float *weights_out, float decay, int32_t n_slots, int32_t q_len,
                        int32_t Hq, float scale, void *hip_stream);

typedef struct {
    const int32_t *budget;   /* device [B][Hkv]: rows that a pair may keep; shared: [B], rows that the pairs of a sequence may keep together */
    int32_t shared;          /* 0 or 1 */
    int32_t pool;            /* odd, 1 .. 63 */
    int32_t sink, recent;    /* >= 0 */
} fairkv_selection;

/* The first `sink` and the last `recent` tokens of a pair are protected and stay, whatever the budget.  Of the others, the candidates, each has the value
 * max weights[row of u] over the candidates u of its pair with |u - t| <= pool / 2, and the largest values of a pair (shared: of a sequence) stay, as many
 * as the budget leaves room for behind the protected tokens.  Of equal values that of the lower head stays, then that of the lower token; -0 is
 * 0, and a NaN is as low as -inf.  A token that has no row in the cache does not stay and takes no part.  Lengths count as in fairkv_decode_attn_tree.
 * weights    device float [n_rows]
 * keep       device [B][Hkv][max_keep], out: the tokens that stay, ascending; what is behind them is left as it is
 * n_keep     device [B][Hkv], out: their number; -1, and the pair counted in *bad, for a pair with more than max_keep of them, whose list then says nothing.
 *            Pairs whose rows overlap, which they must not, may get it too
 * bad        device counter or NULL
 * workspace  device, fairkv_select_workspace_bytes(cache, shared, n_slots) bytes or more, 16-byte aligned.  Its first workspace_bytes / 3 bytes must be zero
 *            before the first use (fairkv_select_workspace_reset); every completed call leaves them zero, and nothing else in it is kept from call to
 *            call, so calls of any shapes that are ordered on one stream may share a workspace that is large enough for each, with one workspace_bytes
 * n_slots    the GPU's compute units
 * keep, n_keep, bad and workspace must not meet one another, or weights, len, budget or the cache's off or pages.
 * Enqueues one kernel, or four where the sizes of the cache allow a group of more than about 16000 rows (of a paged cache max_pages * page_rows is the most
 * that a pair has, of a packed one n_rows); no synchronisation.  Tokens without rows cost time where they make the pairs of a budget longer than the cache's rows: 0.2 to 3 ms for
 * 131072 of them a pair.  FAIRKV_EUNSUPPORTED: pool > 63.  FAIRKV_EINVAL also: more than 2^21 groups. */
size_t fairkv_select_workspace_bytes(const fairkv_cache *cache, int32_t shared, int32_t n_slots);
int fairkv_select_workspace_reset(void *workspace, size_t workspace_bytes, void *hip_stream);
int fairkv_select(const fairkv_cache *cache, const fairkv_selection *s, const float *weights, const int32_t *len, int32_t *keep,
                  int32_t max_keep, int32_t *n_keep, int32_t *bad, void *workspace, size_t workspace_bytes, int32_t n_slots,
                  void *hip_stream);

/* Row keep[p][i] of every pair becomes its row i for i < n_keep[p], K, V and, if given, its weight; len_out[p] = n_keep[p].
 * K and V of the cache that rows move in, or into, must not meet each other.
 * into         NULL: in place, a list has to ascend.  Else another cache of the same B, Hkv, D, type and scales: lists may be in any order and name a token
 *              twice.  Its k and v must not meet this one's, or be the same of as many rows (one pool); then its rows of the pairs are none that
 *              this one's tokens have, by pages or first rows of its own.
 * keep         device [B][Hkv][max_keep], n_keep device [B][Hkv], as fairkv_select leaves them
 * len_out      device [B][Hkv]; may be len
 * weights      device float [n_rows] and weights_out device float [n_rows of into], or both NULL; in place the same, in one pool the same or apart
 * A pair is left alone and counted in *bad, its length kept (into another cache: 0, and what is in its rows there says nothing), if n_keep[p] is not in
 * 0 .. max_keep (in place: or its length; else: or its room there), an entry not in 0 .. len - 1, not ascending (in place), or a row outside its cache.
 * len_out, bad and weights_out must not meet one another, or keep, n_keep or the caches' off or pages or into's cap.
 * Pages behind ceil(len_out / page_rows) hold no token of a pair any more.  Packed rows stay where the pair's run begins.
 * What n_keep says is known on the GPU only, so the host chooses how rows are dealt by max_keep: one not much larger than the lists are serves best.
 * Enqueues one kernel, and a second one if len_out is len; no synchronisation.  FAIRKV_EINVAL also: more than 2^20 pairs, max_keep
 * > 2^31 - 2^16. */
int fairkv_evict(const fairkv_cache *cache, const fairkv_cache *into, const int32_t *keep, int32_t max_keep, const int32_t *n_keep,
                 const int32_t *len, int32_t *len_out, const float *weights, float *weights_out, int32_t *bad, int32_t n_slots,
                 void *hip_stream);

/* The measurement aids (the decode kernel with wall-clock stamps, the reader that only streams) are declared in
 * fairkv_measure.h: they are in the library for the benchmark, not for callers of the method. */

const char *fairkv_strerror(int code);
int fairkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FAIRKV_H */
