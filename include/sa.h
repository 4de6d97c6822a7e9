/*
 * sa.h — C ABI of the segment re-prefill library (MI355X / gfx950).
 *
 * The library implements the data-parallel work behind lookahead context
 * engineering (SmoothAgent, arXiv 2607.00151): a context transformation
 * invalidates the KV cache and forces a re-prefill (paper Sec. 1, Sec. 3.1);
 * the lookahead stream builds the transformed segment's KV on top of the
 * already transformed prefix, in order (Sec. 3.2); at commit the transformed
 * prefix is spliced in place of the old one (Sec. 3.2, Listing of the agent
 * loop); keep-recent-K keeps the head of the context and its recent turns and
 * drops the run in between (Sec. 3.4).  The three data operations are:
 *
 *   sa_kv_assemble           commit splice: gather the surviving pages of a
 *                            cached context into fresh slots, in order, and
 *                            reserve room for the segment that follows
 *   sa_kv_append             write a new segment's K/V rows into the cache
 *   sa_segment_prefill_attn  causal grouped-query attention of the segment's
 *                            queries over the cached prefix plus, causally,
 *                            the segment itself (Sec. 4, prefill-attention
 *                            term: segment token i sees prefix + i + 1 keys)
 * and, fused from them, sa_kv_assemble_append (splice + append, one launch),
 * sa_segment_prefill_attn_append (append + attention, one launch) and the
 * copy-free splice sa_kv_splice_alias.  Several branches of one context are kept
 * by sa_kv_fork, sa_kv_retain, sa_kv_release and sa_kv_compact, written by
 * sa_kv_append_rope and attended by sa_shared_prefix_attn.  Contexts of text and
 * images are rotated by several axes' positions (sa_kv_append_rope_axes), and a
 * cache may be held in 4 bits (sa_kvq_append, sa_kvq_pack, sa_kvq_unpack,
 * sa_kvq_attn).
 *
 * Data layout (all device memory is owned by the caller):
 *   bf16 values are IEEE bfloat16 bit patterns (uint16).
 *   K pool, V pool  bf16 [num_layers][num_slots][num_kv_heads][page_size][head_dim]
 *                   (one slot holds page_size consecutive tokens of every KV head
 *                   of one layer; a slot id is the same in every layer)
 *   page table      CSR over sequences: the pages of sequence b are
 *                   indices[indptr[b] .. indptr[b+1]-1], logical token x of b is
 *                   row x % page_size of slot indices[indptr[b] + x / page_size]
 *   Q, O            bf16 [sum q_len][num_q_heads][head_dim], sequences back to back
 *   new K, V rows   bf16 [sum new_len][num_kv_heads][head_dim]
 *   LSE             fp32 [sum q_len][num_q_heads], natural log of the softmax
 *                   denominator of the scaled scores
 * Query head h reads KV head h / (num_q_heads / num_kv_heads).
 *
 * Conventions:
 *   - Lengths, spans and counts are small HOST int32 arrays, so grids are
 *     sized without a device round trip; page tables and free lists live on
 *     the device.
 *   - Every call validates its arguments on the host before touching HIP and
 *     returns a status; nothing throws across the ABI.  Validation order:
 *     layout and shapes, then pointers, then the context.
 *   - Calls enqueue work on `stream` (a hipStream_t; NULL is the default
 *     stream) and return without synchronising.  Buffers must stay valid until
 *     the stream has run the work.
 *   - A context keeps per-call plans (work lists) in device memory and reuses
 *     an uploaded plan when the next call of the same kind needs the same one.
 *     Calls on one context must therefore be ordered: use one stream per
 *     context (or one context per stream / thread).  Attention calls that
 *     overlap all the same may also leave the counters by which a launch split
 *     by key range merges its parts off, and then later split launches of the
 *     context give wrong outputs until sa_sync_check has reported and cleared
 *     them.
 *   - Page ids inside device tables are range-checked by the kernels: a page
 *     beyond a sequence's list or a slot outside [0, num_slots) is skipped
 *     (never dereferenced) and latched in a device flag that sa_sync_check
 *     reports.  Reads of such pages contribute zeros.  Nothing on the hot
 *     path checks that slots do not repeat; with the environment variable
 *     SA_DEBUG=1 (read once per process) every splice and append first copies
 *     the tables it will use back to the host (synchronising its stream) and
 *     refuses, before launching, slots outside the pool or pages a sequence
 *     lacks (SA_ERR_RANGE), a free list that repeats a slot or hands out a
 *     surviving source slot, and two sequences writing the same row of a slot
 *     (SA_ERR_OVERLAP); every fork and shared-prefix attention likewise (see there).
 *   - Plan buffers grow on demand (hipMalloc) and an outgrown one is kept
 *     until sa_destroy, since kernels already enqueued may still read it; no
 *     call synchronises the device.  sa_reserve sizes them ahead of time.
 *   - Pointers to pools, Q, O, K/V rows must be 16-byte aligned.
 */
#ifndef SA_H
#define SA_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum sa_status {
    SA_OK = 0,
    SA_ERR_NULL = 1,          /* a required pointer (or the context) is NULL            */
    SA_ERR_SHAPE = 2,         /* inconsistent sizes or lengths                          */
    SA_ERR_UNSUPPORTED = 3,   /* head_dim != 128, page_size not 16 or 32, ...          */
    SA_ERR_ALIGN = 4,         /* a data pointer is not 16-byte aligned                  */
    SA_ERR_RANGE = 5,         /* a span or page id is out of range                      */
    SA_ERR_NO_PAGES = 6,      /* free list or destination table too small               */
    SA_ERR_HIP = 7,           /* a HIP runtime call failed (see sa_last_error)          */
    SA_ERR_DEVICE = 8,        /* no usable gfx950 device                                 */
    SA_ERR_OVERLAP = 9        /* slot lists repeat where they must not (SA_DEBUG checks),
                                 or split launches overlapped (sa_sync_check)           */
} sa_status;

typedef struct sa_ctx sa_ctx;

/* Cache geometry shared by every call that touches the pools. */
typedef struct sa_layout {
    int32_t num_q_heads;      /* Hq, a multiple of num_kv_heads                         */
    int32_t num_kv_heads;     /* Hkv >= 1                                               */
    int32_t head_dim;         /* must be 128                                            */
    int32_t page_size;        /* tokens per slot: 16 or 32                              */
    int32_t num_layers;       /* layers held by each pool (>= 1)                        */
    int64_t num_slots;        /* slots per layer                                        */
} sa_layout;

/* Device page table in CSR form (see the layout notes above). */
typedef struct sa_pages {
    const int32_t *indptr;    /* device [batch + 1]                                     */
    const int32_t *indices;   /* device [indptr[batch]] slot ids                        */
} sa_pages;

/* Create a context on HIP device `device` (must be gfx950).  The context owns
 * only plan buffers, pinned staging, split-KV scratch and an error flag.
 * Returns SA_ERR_DEVICE if the device is missing or not gfx950. */
sa_status sa_create(int device, sa_ctx **out);

/* Release a context (waits for the device first).  NULL is ignored. */
void sa_destroy(sa_ctx *ctx);

/* Static description of a status code. */
const char *sa_status_string(sa_status status);

/* Message of the most recent failing call on this thread ("" if none). */
const char *sa_last_error(void);

/*
 * sa_reserve — size the context's buffers ahead of time, so that later calls
 * whose plans fit them allocate no device or pinned memory (for example
 * before a timed loop or a serving loop).  plan_bytes: capacity of each call
 * kind's device plan buffer and of each pinned staging buffer; an attention
 * call's plan takes about 40 bytes per work item (one per sequence, KV head
 * and 128 packed query rows, and per key-range part of a split item) plus
 * 16 bytes per sequence, 8 per key-range part and 768 of alignment; a splice's
 * about 24 bytes per surviving page plus 16 per sequence; a shared-prefix
 * attention's 40 bytes per work item and 36 per up to 32 query rows of a
 * sequence that are split, a rotated append's 12 bytes per sequence and 512 for
 * the frequencies, a fork's 32 bytes per child, each with 768 of alignment.  It
 * is also the capacity of the buffer in which sa_kv_release and sa_kv_compact
 * scan the slots: 4 bytes per 4096 slots, and 16 per slot and 8 per 4096.
 * split_bytes: capacity of the split-KV partials, 128 * 129 * 4 bytes per
 * key-range part (sa_shared_prefix_attn: 516 bytes per query row, head and part).
 * Buffers only grow; outgrown ones are kept until sa_destroy.
 * Errors: SA_ERR_NULL (context), SA_ERR_SHAPE (negative size), SA_ERR_HIP.
 */
sa_status sa_reserve(sa_ctx *ctx, int64_t plan_bytes, int64_t split_bytes);

/*
 * sa_attn_plan_stats — the shape of the attention launch sa_segment_prefill_attn
 * would make for these lengths on a GPU with num_cu compute units (host only:
 * no context, no GPU), for latency models of a batch (paper Sec. 4, Eq. 1
 * models a batch from its decode and prefill work; how the work falls onto
 * the chip's workgroup slots adds to that).  out[0]: workgroups; out[1]:
 * key-range parts of split items (whose partial results the launch itself merges);
 * out[2]: 64-key tiles over all items; out[3]: makespan in tiles when the
 * items are taken in launch order by whichever of the 2 x num_cu workgroup
 * slots frees first (a decode item's tiles count a quarter: its four waves
 * split them).  Errors: those of sa_segment_prefill_attn's shape checks;
 * SA_ERR_NULL for a NULL out; SA_ERR_SHAPE for num_cu < 1.
 */
sa_status sa_attn_plan_stats(const sa_layout *layout, int32_t batch, const int32_t *h_q_len,
                             const int32_t *h_kv_len, int32_t num_cu, int64_t *out);

/* Wait for `stream`, then report SA_ERR_RANGE if any kernel of this context
 * met an out-of-range page id or slot, or a slot's count that does not fit the
 * tables, since the last check (and clear it; the message says which and ends
 * with the flags: 1 an attention, 2 an append, 4 a splice, fork, count,
 * compaction or conversion, 8 a count), or
 * SA_ERR_OVERLAP if launches split by key range overlapped against the rules
 * above and left the context's arrival counters off (and clear them; only then,
 * or while a launch of the context still runs on another stream, it also waits
 * for the device). */
sa_status sa_sync_check(sa_ctx *ctx, void *stream);

/*
 * sa_kv_append — store a segment's new K/V rows in the cache (paper Sec. 3.2:
 * the lookahead transform builds KV on the transformed prefix).
 *
 * For each sequence b, new token t (0 <= t < h_new_len[b]) goes to logical
 * position h_start[b] + t of layer `layer`: slot
 * pages.indices[pages.indptr[b] + (h_start[b] + t) / page_size], row
 * (h_start[b] + t) % page_size.  Rows are copied bit for bit; nothing else in
 * the pools changes.  k_new / v_new hold the rows of all sequences back to
 * back ([sum new_len][Hkv][128]).  A sequence with h_new_len[b] == 0 is a
 * no-op.  The page list of b must cover the written positions.
 *
 * Errors: SA_ERR_SHAPE (batch < 1, negative start or length, layer outside
 * [0, num_layers)), SA_ERR_UNSUPPORTED, SA_ERR_NULL, SA_ERR_ALIGN, SA_ERR_HIP.
 */
sa_status sa_kv_append(sa_ctx *ctx, const sa_layout *layout, int32_t layer,
                       void *k_pool, void *v_pool,
                       const void *k_new, const void *v_new,
                       int32_t batch, const int32_t *h_start, const int32_t *h_new_len,
                       sa_pages pages, void *stream);

/*
 * sa_kv_assemble — commit splice into a replacement cache (paper Sec. 3.2
 * commit; Sec. 3.4 keep-recent-K drops an interior run of turns).
 *
 * Sequence b's source cache holds h_src_len[b] tokens on the pages of `src`.
 * Its surviving pages are the [begin, end) logical page spans
 * h_keep_spans[2*s], h_keep_spans[2*s+1] for s in h_keep_indptr[b] ..
 * h_keep_indptr[b+1]-1 (ascending, disjoint, non-empty, within the source
 * pages).  The replacement cache of b is those pages in order, renumbered
 * from 0, followed by enough new pages for h_reserve[b] more tokens:
 *   kept_b  = tokens on the surviving pages   (returned in h_dst_len[b])
 *   pages_b = ceil((kept_b + h_reserve[b]) / page_size)
 * Destination slots are taken from the front of the device free list
 * d_fresh[0 .. num_fresh), sequence after sequence.  Every surviving page is
 * copied whole (all page_size rows, every KV head, every layer) from its
 * source slot to its destination slot; reserved pages are left untouched.
 * The destination page table is written to d_dst_indptr[batch + 1] and
 * d_dst_indices[sum pages_b] (capacity dst_capacity entries).
 *
 * k_dst / v_dst may be the same pools as k_src / v_src.  Fresh slots must not
 * be surviving source slots of this call (the copy reads and writes in
 * parallel) and must not repeat; nothing checks this on the hot path
 * (SA_DEBUG=1 does, see the conventions above).
 *
 * Errors: SA_ERR_SHAPE, SA_ERR_RANGE (bad span), SA_ERR_NO_PAGES (free list
 * or dst_capacity too small), SA_ERR_UNSUPPORTED, SA_ERR_NULL, SA_ERR_ALIGN,
 * SA_ERR_HIP.
 */
sa_status sa_kv_assemble(sa_ctx *ctx, const sa_layout *layout,
                         const void *k_src, const void *v_src, void *k_dst, void *v_dst,
                         int32_t batch, const int32_t *h_src_len,
                         const int32_t *h_keep_indptr, const int32_t *h_keep_spans,
                         const int32_t *h_reserve,
                         sa_pages src, const int32_t *d_fresh, int32_t num_fresh,
                         int32_t *d_dst_indptr, int32_t *d_dst_indices, int32_t dst_capacity,
                         int32_t *h_dst_len, void *stream);

/*
 * sa_kv_assemble_append — sa_kv_assemble followed by the segment's
 * sa_kv_append, in one launch (paper Sec. 3.2: the transformed KV is the
 * spliced prefix plus the segment's rows).
 *
 * Arguments and results of sa_kv_assemble, plus: layer, the layer whose new
 * rows are written; k_new / v_new, bf16 [sum h_new_len][num_kv_heads][head_dim];
 * h_new_len[b] (host), the new tokens of sequence b, which go to logical
 * positions h_dst_len[b] .. h_dst_len[b] + h_new_len[b] - 1 of its
 * replacement cache (they must fit its pages: kept + new <= pages_b *
 * page_size).  The pools end exactly as after the two calls in sequence: the
 * rows of a partial last surviving page that the segment fills come from the
 * new rows, the rest of that page from its source.
 *
 * Errors: those of sa_kv_assemble, and SA_ERR_SHAPE for a bad layer or new
 * tokens that do not fit, SA_ERR_NULL for NULL new rows or h_new_len.
 */
sa_status sa_kv_assemble_append(sa_ctx *ctx, const sa_layout *layout,
                                const void *k_src, const void *v_src, void *k_dst, void *v_dst,
                                int32_t batch, const int32_t *h_src_len,
                                const int32_t *h_keep_indptr, const int32_t *h_keep_spans,
                                const int32_t *h_reserve,
                                sa_pages src, const int32_t *d_fresh, int32_t num_fresh,
                                int32_t *d_dst_indptr, int32_t *d_dst_indices, int32_t dst_capacity,
                                int32_t *h_dst_len, int32_t layer, const void *k_new,
                                const void *v_new, const int32_t *h_new_len, void *stream);

/*
 * sa_kv_splice_alias — zero-copy form of the commit splice (paper Sec. 3.2
 * commit, Sec. 3.4 keep-recent-K), for callers whose surviving pages may stay
 * where they are.
 *
 * Same spans, lengths, free list and outputs as sa_kv_assemble, but no page
 * is copied: the destination table of sequence b lists the SOURCE slots of its
 * surviving pages, in order, followed by fresh slots -- taken from the front of
 * d_fresh, sequence after sequence -- for the pages that h_reserve[b] more
 * tokens need beyond the surviving ones (so the free list is consumed only by
 * reserved pages).  The surviving pages are then shared between the source and
 * the destination tables: an append into the last surviving page (when it is
 * partial) writes into the source slot, past the source's own length.
 *
 * Errors: as sa_kv_assemble (d_fresh may be NULL when no page is reserved).
 * A missing source page or a source slot outside [0, num_slots) is latched in
 * the device flag that sa_sync_check reports (a missing page's entry is -1).
 */
sa_status sa_kv_splice_alias(sa_ctx *ctx, const sa_layout *layout, int32_t batch,
                             const int32_t *h_src_len, const int32_t *h_keep_indptr,
                             const int32_t *h_keep_spans, const int32_t *h_reserve,
                             sa_pages src, const int32_t *d_fresh, int32_t num_fresh,
                             int32_t *d_dst_indptr, int32_t *d_dst_indices, int32_t dst_capacity,
                             int32_t *h_dst_len, void *stream);

/*
 * sa_segment_prefill_attn — causal grouped-query attention of each
 * sequence's last h_q_len[b] tokens over its h_kv_len[b] cached tokens
 * (paper Sec. 4, prefill-attention term; decode rows are the q_len = 1 case of
 * the decode-attention term).
 *
 * With prefix_b = h_kv_len[b] - h_q_len[b], segment row i of query head h
 * attends keys 0 .. prefix_b + i of KV head h / (Hq / Hkv) in layer `layer`:
 *   O = softmax(softmax_scale * q . K^T) V,   LSE = log(sum exp(scale * q . k))
 * The segment's own K/V must already be in the cache (sa_kv_append).  Output
 * rows are bf16 (round to nearest even); `lse` may be NULL.  Sequences with
 * h_q_len[b] == 0 are skipped.  Arithmetic: bf16 MFMA products with fp32
 * accumulation, fp32 online softmax, probabilities rounded to bf16 before the
 * PV product.  The scale is applied to each fp32 score (with log2(e)) before
 * the exponential; a row's exponent offset moves only when its max grows by
 * more than 2^8, and the bf16 rounding of the probability of every key that
 * was its row's largest when it arrived is carried into the normaliser of the
 * output (not into the LSE), so a dominant key's weight comes out as its
 * exact share.  After sa_set_exact_scale(ctx, 0) the kernel instead
 * multiplies each query row by softmax_scale * log2(e) once and rounds it to
 * bf16 (faster; moves a row's scaled scores by up to
 * 2^-8 * sum_d |scale log2(e) q_d k_d| in log2 units).  A row that meets a
 * score of +infinity or NaN has a NaN output and a NaN LSE.  A masked key's
 * probability is 0 and its value is multiplied by that: an infinite or NaN value
 * of a segment's token reaches, besides the rows that see it, the earlier rows of
 * the segment in its work item (128 packed rows, num_q_heads / num_kv_heads to a
 * token), and no others.
 *
 * Errors: SA_ERR_SHAPE (0 <= q_len <= kv_len violated, bad batch or layer,
 * softmax_scale not finite and positive),
 * SA_ERR_UNSUPPORTED, SA_ERR_NULL, SA_ERR_ALIGN, SA_ERR_HIP.
 */
sa_status sa_segment_prefill_attn(sa_ctx *ctx, const sa_layout *layout, int32_t layer,
                                  const void *q, const void *k_pool, const void *v_pool,
                                  int32_t batch, const int32_t *h_q_len, const int32_t *h_kv_len,
                                  sa_pages pages, float softmax_scale,
                                  void *o, float *lse, void *stream);

/*
 * sa_segment_prefill_attn_noalloc — sa_segment_prefill_attn for callers that
 * cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, same results (bit
 * for bit as long as its split-KV partials fit, see below), but it calls no
 * hipMalloc, hipFree or other allocating HIP routine (the host planner uses
 * only ordinary C++ heap memory): the launch's plan and its split-KV partials
 * live in one fixed device array of 32 MiB per GPU, a file-scope
 * `static __device__` array that each GPU the library runs on holds until
 * the process ends; the plan reaches it through pinned staging the context
 * allocated at sa_create.  Limits: the plan (about 40 bytes per work item, a
 * work item per sequence, KV head and 128 packed query rows) must fit 2 MiB,
 * else SA_ERR_SHAPE before anything is enqueued; the partials get the other
 * 30 MiB (476 key-range parts of 128 rows), and a launch that would split
 * into more parts is split more coarsely instead.  Every call on one GPU uses
 * that GPU's array, whichever context makes it, and leaves the last call's
 * contents there: calls that overlap in time on one GPU (two streams, two
 * contexts) race, so order them; their outputs are undefined, and those of the
 * same contexts' later split launches until sa_sync_check (see there).  The
 * call may wait on the host for the previous plan copy of the same context to
 * finish.
 * Errors: those of sa_segment_prefill_attn.
 */
sa_status sa_segment_prefill_attn_noalloc(sa_ctx *ctx, const sa_layout *layout, int32_t layer,
                                          const void *q, const void *k_pool, const void *v_pool,
                                          int32_t batch, const int32_t *h_q_len, const int32_t *h_kv_len,
                                          sa_pages pages, float softmax_scale,
                                          void *o, float *lse, void *stream);

/*
 * sa_set_exact_scale — how later attention calls on this context apply
 * softmax_scale.  enable != 0 (the default) multiplies each fp32 score by it
 * (with log2(e)) before the exponential: the only roundings are those of the
 * probabilities to bf16 before the PV product and of the output.  enable == 0
 * is a fast mode that folds the scale into the query rows, rounded to bf16
 * once per row, which saves one fma per score and moves the scores by at most
 * 2^-8 * sum_d |scale log2(e) q_d k_d| (log2 units) -- of the order of the
 * error bf16 query and key rows already carry, but large when the logits
 * are.  Applies to the default kernel; SA_ATTN_VARIANT=1 always scales in
 * fp32, SA_ATTN_VARIANT=2 never.  Errors: SA_ERR_NULL for a NULL context.
 */
sa_status sa_set_exact_scale(sa_ctx *ctx, int32_t enable);

/*
 * sa_set_fused_append — how later sa_segment_prefill_attn_append calls on
 * this context write the segment's rows.  enable != 0: inside the attention
 * launch, which reads the segment's keys from k_new / v_new; enable == 0 (the
 * default): an append launch (sa_kv_append) and then the attention.  Both
 * forms leave the same pool; their outputs are equal bit for bit when every
 * prefix length is a multiple of 4 and no request has at most 32 query rows,
 * and otherwise both are held to the same tolerance.
 * Errors: SA_ERR_NULL for a NULL context.
 */
sa_status sa_set_fused_append(sa_ctx *ctx, int32_t enable);

/*
 * sa_set_kernel_events — timing hook for measurement.  While set for `which`,
 * every kernel of that kind this context launches is launched by
 * hipExtLaunchKernelGGL with start_event and stop_event (hipEvent_t handles
 * the caller created with timing enabled), which binds both events to that
 * kernel, so their elapsed time is the kernel's execution on the device
 * rather than that of the call (events recorded around a call also span the
 * dispatch gap, several microseconds).  Kinds:
 *   SA_TIMED_ATTN   the attention kernel of sa_segment_prefill_attn and
 *                   sa_segment_prefill_attn_append (which merges the parts of
 *                   a launch split by key range; not the merge kernel of
 *                   SA_ATTN_VARIANT 1 and 2)
 *   SA_TIMED_PAGES  the page kernel of sa_kv_append, sa_kv_assemble,
 *                   sa_kv_assemble_append, sa_kv_splice_alias and the append
 *                   launch of sa_segment_prefill_attn_append
 * A later launch of the same kind re-binds the same events.  Both NULL clears
 * the hook; the events stay owned by the caller and must outlive the launches.
 * Errors: SA_ERR_NULL for a NULL context or one event without the other,
 * SA_ERR_SHAPE for an unknown kind.
 */
#define SA_TIMED_ATTN 0
#define SA_TIMED_PAGES 1
sa_status sa_set_kernel_events(sa_ctx *ctx, int32_t which, void *start_event, void *stop_event);

/*
 * sa_set_block_clock — per-workgroup timestamps for measurement (which work of
 * a mixed decode + prefill launch ends when; paper Sec. 4 and Alg. 2 batch
 * decode requests with prefill chunks).  While set, each launch of the default
 * attention kernel writes, for every workgroup w, four uint64 words at
 * d_buf[4w]: the device's constant-rate wall clock (s_memrealtime) when w
 * started and when all its output stores were done; then its work item: word
 * 2 holds the sequence index in bits 0-31, the KV head in bits 32-47 and the
 * item's first key tile (of 64 keys) modulo 2^16 in bits 48-63; word 3 holds
 * that sequence's q_len in bits 0-31 (1: a decode row; 0 for a workgroup with
 * no work, which the planner adds to even out the XCDs) and the item's first
 * packed query row in bits 32-63.  The launch has one workgroup per
 * work item, at most max_blocks of them, else it fails with SA_ERR_SHAPE
 * before launching.  d_buf: device memory of 32 * max_blocks bytes, 8-byte
 * aligned, owned by the caller; the words of one launch are overwritten by
 * the next.  clock_khz (nullable, host): receives the clock's rate in kHz.
 * NULL, 0 clears.  The other attention kernels (SA_ATTN_VARIANT 1, 2) write
 * nothing.  Errors: SA_ERR_NULL (context), SA_ERR_SHAPE, SA_ERR_ALIGN,
 * SA_ERR_HIP.
 */
sa_status sa_set_block_clock(sa_ctx *ctx, void *d_buf, int64_t max_blocks, int64_t *clock_khz);

/*
 * sa_set_xcd_weights — relative speeds of the chip's 8 XCDs (workgroup i of a
 * launch runs on XCD i % 8) for the attention planner.  The XCDs of one
 * MI355X do not run equally fast under a long MFMA-bound launch (their clocks
 * differ by several percent), and a launch ends with its slowest XCD.  With
 * speeds set, the planner, when it places the work items of each KV head on
 * one XCD, evens out key tiles per unit of speed across the XCDs of a launch
 * of at most two rounds of workgroups: it pairs the XCDs by speed (slowest
 * with fastest, and so on) and, within each pair, swaps the longest item of
 * the XCD whose busiest CU is the more loaded for the shortest item of the
 * other (every XCD keeps its number of items; a moved item reads its KV
 * head's K/V through the other XCD's L2).  Launches of more rounds are placed
 * as without speeds.  Results are
 * unchanged bit for bit (a work item's arithmetic does not depend on where it
 * runs).  h_speed: host float[8], each finite and > 0 (only ratios matter),
 * e.g. the inverse of each XCD's mean workgroup time from sa_set_block_clock
 * on a launch with equal work per XCD; NULL resets to equal speeds.
 * Errors: SA_ERR_NULL (context), SA_ERR_SHAPE.
 */
sa_status sa_set_xcd_weights(sa_ctx *ctx, const float *h_speed);

/*
 * sa_segment_prefill_attn_append — the segment's append and its attention in
 * one call: each sequence's h_q_len[b] new K/V rows are written to its
 * logical positions h_kv_len[b] - h_q_len[b] .. h_kv_len[b] - 1 (as
 * sa_kv_append with start = kv_len - q_len), then the attention is computed
 * exactly as sa_segment_prefill_attn does over the cache that results (paper
 * Sec. 3.2: the lookahead builds the segment's KV on the transformed prefix).
 * k_new / v_new: bf16 [sum h_q_len][num_kv_heads][head_dim], token-major like
 * q; the pools are written.  The pages for the new rows must already be in
 * the table (sa_kv_assemble's reserve).  By default this is the append
 * kernel followed by the attention kernel on `stream`.  With fusion switched
 * on (sa_set_fused_append) it is one launch of the default attention kernel:
 * every workgroup reads the segment's keys and values from k_new / v_new, not
 * from their pages, and the first key-range part of each 128-row tile writes
 * the rows of the tokens whose first query row lies in that tile, so the rows
 * are written once and no workgroup waits on another (a request of at most
 * 32 query rows writes its own rows and reads them back).  The fused form
 * falls back to the two launches for the other kernel variants
 * (SA_ATTN_VARIANT), when a layer's pool spans 2^31 bytes or more, or when
 * k_new does.  The rows written must not be
 * rows that another sequence of the call reads as part of its prefix (as with
 * the two launches, whose order would otherwise decide what it reads).
 *
 * Errors: those of sa_segment_prefill_attn; SA_ERR_NULL for NULL new rows
 * (when any q_len > 0), SA_ERR_ALIGN for new rows not 16-byte aligned.  A
 * missing or out-of-range page of a new row raises the device error flag
 * (reported by sa_sync_check) and that row is not written.
 */
sa_status sa_segment_prefill_attn_append(sa_ctx *ctx, const sa_layout *layout, int32_t layer,
                                         const void *q, void *k_pool, void *v_pool,
                                         const void *k_new, const void *v_new, int32_t batch,
                                         const int32_t *h_q_len, const int32_t *h_kv_len,
                                         sa_pages pages, float softmax_scale, void *o, float *lse,
                                         void *stream);

/* ------------------------------------------------ branches of one context
 *
 * Several lookahead streams, or sub-agents isolated on one context (paper
 * Sec. 3.2, Sec. 3.5), keep branches of a cached context alive side by side.
 * The calls below fork a context without copying its full pages, write the
 * branches' rows, attend over them with the common part read once, and give
 * the pages of ended branches back.  They use the calling thread's device only
 * within the call.  Calls that plan on the host (sa_kv_append_rope, sa_kv_fork,
 * sa_shared_prefix_attn) return SA_ERR_UNSUPPORTED on a stream that is being
 * captured into a graph, since a replay would find another call's plan in the
 * context; sa_kv_retain, sa_kv_release and sa_kv_compact can be captured once
 * a call of the same pool size has run on the context or sa_reserve has made
 * room for it (they allocate nothing then), and their replays count as calls on it.  Slots of more than 2^30
 * elements and pools of 2^31 - 4096 slots or more are refused (SA_ERR_UNSUPPORTED).
 *
 * A pool whose slots are shared by several tables keeps one count per slot,
 * d_ref: device int32 [num_slots], the number of table entries that name the
 * slot, owned by the caller and zero for a slot that is not in use.
 * A count that does not fit its tables (a fork that takes a fresh slot with a
 * count, or shares a page without one; a release that finds a count at zero; a
 * compacted table that names a slot not in use) is latched like a bad page and
 * reported by sa_sync_check as SA_ERR_RANGE.
 */

/* Norms and rotation of a segment's new rows (sa_kv_append_rope). */
typedef struct sa_rope {
    int32_t rot_dim;          /* leading dims of each head that are rotated: a multiple
                                 of 16 from 0 to head_dim                               */
    int32_t interleaved;      /* 0: dims d and d + rot_dim/2 are a pair; else 2d and 2d+1 */
    const double *h_inv_freq; /* host [rot_dim / 2]: radians per position of each pair,
                                 0 to 1024                                              */
    const void *q_weight;     /* device bf16 [head_dim]; NULL: query heads are not normed */
    const void *k_weight;     /* the same for key heads                                 */
    float eps;                /* of the norms, at least 2^-126                           */
    float weight_offset;      /* added to every weight (1 where weights are stored less 1) */
} sa_rope;

/*
 * sa_kv_append_rope — sa_kv_append for rows straight out of a projection: the
 * norm of each query and key head, the rotation of both by position, and the
 * key and value rows into the cache, in one pass.
 *
 * Token t of sequence b has cache position h_start[b] + t, where its rows go
 * as by sa_kv_append, and rotation position h_pos[b] + t (h_pos NULL: h_start;
 * they differ where a splice renumbered the pages of a context whose keys keep
 * their angles).  Each query head row x, and each key head row, becomes
 *   y = x / sqrt(mean_d x_d^2 + eps) * (weight_d + weight_offset)   (with weights)
 *   (y_i, y_j) = (y_i cos a - y_j sin a, y_j cos a + y_i sin a),  a = position * inv_freq
 * for its pairs (i, j), computed in fp32 (the angle exactly, modulo a turn) and
 * rounded once to bf16; dims from rot_dim on are not rotated.  Query rows go to
 * q_out, bf16 [sum new_len][num_q_heads][128]; value rows are copied bit for bit.
 * q, k_new and v_new hold the rows of all sequences back to back; token t's
 * heads start at element t * q_stride (k_stride, v_stride), so the three may be
 * slices of one projection's output.  Strides are in elements, multiples of 8.
 * q_out may be q itself with q_stride = num_q_heads * 128, and must not overlap
 * it otherwise.
 *
 * Errors: those of sa_kv_append; SA_ERR_SHAPE for a negative position, a stride
 * too small, an inv_freq out of range or a bad eps, SA_ERR_UNSUPPORTED for a bad
 * rot_dim or a capturing stream, SA_ERR_ALIGN for a stride that is not a
 * multiple of 8.  A missing or out-of-range page is latched for sa_sync_check;
 * its rows are not written, q_out is.
 */
sa_status sa_kv_append_rope(sa_ctx *ctx, const sa_layout *layout, int32_t layer, const sa_rope *rope,
                            const void *q, int64_t q_stride, const void *k_new, int64_t k_stride,
                            const void *v_new, int64_t v_stride, void *q_out, void *k_pool, void *v_pool,
                            int32_t batch, const int32_t *h_start, const int32_t *h_new_len,
                            const int32_t *h_pos, sa_pages pages, void *stream);

/*
 * sa_kv_fork — open children of cached contexts.
 *
 * Child c continues sequence b = h_parent[c] of `src`, which holds h_src_len[b]
 * tokens, and has room for h_reserve[c] more: its table lists the parent's full
 * pages (the same slots), and fresh slots for the rest of its
 *   pages_c = ceil((h_src_len[b] + h_reserve[c]) / page_size)
 * pages, taken from the front of d_fresh, child after child.  Where the
 * parent's last page is partial its valid rows are copied, in every layer, to
 * the child's first fresh slot (whose other rows stay as they are), so the
 * child's appends never touch a shared page.  A sequence may have any number of
 * children; its own table stays as it is.  The children's table is written to
 * d_dst_indptr[num_children + 1] and d_dst_indices (capacity dst_capacity),
 * which must not be the source table.
 * d_ref (nullable): the count of every listed slot is raised by one per entry.
 * *h_fresh_used receives the number of fresh slots taken.  Fresh slots must not
 * repeat nor be pages of a source context (SA_DEBUG=1 checks).
 *
 * Errors: SA_ERR_SHAPE, SA_ERR_RANGE (a parent out of range), SA_ERR_NO_PAGES,
 * SA_ERR_UNSUPPORTED (capture), SA_ERR_NULL, SA_ERR_ALIGN, SA_ERR_HIP.
 */
sa_status sa_kv_fork(sa_ctx *ctx, const sa_layout *layout, void *k_pool, void *v_pool, int32_t batch,
                     const int32_t *h_src_len, int32_t num_children, const int32_t *h_parent,
                     const int32_t *h_reserve, sa_pages src, const int32_t *d_fresh, int32_t num_fresh,
                     int32_t *d_dst_indptr, int32_t *d_dst_indices, int32_t dst_capacity, int32_t *d_ref,
                     int32_t *h_fresh_used, void *stream);

/*
 * sa_kv_retain — raise the count of every slot that the batch's tables name, by
 * one per entry indptr[0] .. indptr[batch] - 1 (tables made by sa_kv_assemble
 * or sa_kv_splice_alias, which keep no counts).  max_entries: entries that
 * pages.indices holds; a table that runs beyond them is latched as an error and
 * nothing is counted.  Errors: SA_ERR_SHAPE, SA_ERR_NULL, SA_ERR_HIP.
 */
sa_status sa_kv_retain(sa_ctx *ctx, const sa_layout *layout, int32_t batch, sa_pages pages,
                       int64_t max_entries, int32_t *d_ref, void *stream);

/*
 * sa_kv_release — the batch's tables end: lower the count of every slot they
 * name, by one per entry (never below zero), and list the slots whose count is
 * then zero: d_free[0 .. *d_num_free) holds them in ascending order and the
 * rest of d_free (num_slots entries) is -1.  d_free and d_num_free may both be
 * NULL (counts only).  max_entries as in sa_kv_retain.
 * Errors: SA_ERR_SHAPE, SA_ERR_NULL, SA_ERR_HIP.
 */
sa_status sa_kv_release(sa_ctx *ctx, const sa_layout *layout, int32_t batch, sa_pages pages,
                        int64_t max_entries, int32_t *d_ref, int32_t *d_free, int32_t *d_num_free,
                        void *stream);

/*
 * sa_kv_compact — vacate the slots from `limit` on, so that the pool can shrink
 * or its tail serve something else: the pages in use (count > 0) in slots
 * >= limit move, in ascending order, to the slots < limit that are not in use,
 * in ascending order, in every layer of both pools.  Where there are more such
 * pages than free slots the last ones stay.
 *   d_moved[0], [1]   pages moved, pages left in slots >= limit
 *   d_slot_map[s]     (num_slots entries) where slot s's page is now; -1 if
 *                     slot s was not in use
 *   d_ref_out         the counts after the move (may be d_ref)
 *   d_indices_out     the num_entries table entries d_indices through the map
 *                     (may be d_indices); an entry outside the pool stays as it
 *                     is and is latched
 * Moved pages stay in their old slots too, as bits nobody names.  The outputs
 * other than d_ref_out and d_indices_out must not overlap the inputs.
 * Errors: SA_ERR_RANGE (limit outside [0, num_slots]), SA_ERR_SHAPE,
 * SA_ERR_NULL, SA_ERR_ALIGN, SA_ERR_HIP.
 */
sa_status sa_kv_compact(sa_ctx *ctx, const sa_layout *layout, void *k_pool, void *v_pool, int32_t limit,
                        const int32_t *d_ref, int32_t *d_ref_out, const int32_t *d_indices,
                        int32_t *d_indices_out, int64_t num_entries, int32_t *d_slot_map, int32_t *d_moved,
                        void *stream);

/*
 * sa_shared_prefix_attn — sa_segment_prefill_attn for a batch whose sequences
 * share prefixes, each read and multiplied once for all of its sequences.
 *
 * The members of group g are sequences h_group_indptr[g] .. h_group_indptr[g+1]-1;
 * every sequence is in one group (group_indptr runs from 0 to batch; a group
 * may have one member or none).  The caches of a group's members hold the same
 * keys and values for their first h_shared_len[g] tokens (the same pages, as
 * sa_kv_fork leaves them, or equal copies): whole 64-key tiles of them are read
 * through the page list of the group's first member that has query rows.
 * shared_len may be anything from 0 to the smallest h_kv_len - h_q_len of the
 * group.  One beyond what the members have in common gives the later members
 * wrong results; with SA_DEBUG=1 the call refuses it (SA_ERR_SHAPE), comparing
 * the pages that are not the same slots bit for bit, and pages of the shared
 * part that a table lacks or that lie outside the pool (SA_ERR_RANGE).
 *
 * The result is that of sa_segment_prefill_attn over the same tables, held to
 * the same tolerance: probabilities are rounded to bf16 before the PV product,
 * and parts are joined in fp32.  Scores and values that are not finite do what
 * they do there; those of one member's own tokens do not reach the others.
 * Where the members' rows fill the kernel's row tiles anyway (long segments)
 * the group is computed member by member, and a batch that would gain nothing
 * goes to the segment attention's launch (sa_shared_plan_stats tells).  The
 * softmax scale is always applied exactly; SA_ATTN_VARIANT and the block clock
 * apply only to such batches.  sa_set_kernel_events times the first kernel
 * (SA_TIMED_ATTN), and the partial results (516 bytes per query row, head and
 * key-range part) take the place of the split-KV partials that sa_reserve sizes.
 *
 * Errors: those of sa_segment_prefill_attn, SA_ERR_SHAPE for bad groups or
 * shared lengths, SA_ERR_UNSUPPORTED for a capturing stream.
 */
sa_status sa_shared_prefix_attn(sa_ctx *ctx, const sa_layout *layout, int32_t layer, const void *q,
                                const void *k_pool, const void *v_pool, int32_t batch,
                                const int32_t *h_q_len, const int32_t *h_kv_len, sa_pages pages,
                                int32_t num_groups, const int32_t *h_group_indptr,
                                const int32_t *h_shared_len, float softmax_scale, void *o, float *lse,
                                void *stream);

/*
 * sa_shared_plan_stats — what sa_shared_prefix_attn would make of these lengths
 * on a GPU with num_cu compute units (host only: no context, no GPU).  out[0]:
 * groups whose prefix is computed once for their members (0: the batch goes to
 * the segment attention's launch, and the other numbers are 0); out[1]:
 * workgroups; out[2]: rows of partial results, 516 bytes each; out[3]: the most
 * parts that a row is joined from.  h_once (nullable, [num_groups]): 1 for each
 * group whose prefix is computed once, else 0.
 * Errors: those of sa_shared_prefix_attn's shape checks; SA_ERR_NULL for a NULL
 * out; SA_ERR_SHAPE for num_cu < 1.
 */
sa_status sa_shared_plan_stats(const sa_layout *layout, int32_t batch, const int32_t *h_q_len,
                               const int32_t *h_kv_len, int32_t num_groups,
                               const int32_t *h_group_indptr, const int32_t *h_shared_len,
                               int32_t num_cu, int64_t *out, int32_t *h_once);

/* --------------------------------------- several axes, and a cache of 4 bits
 *
 * Contexts of agents that look at screens hold images and video beside text:
 * their tokens have a position on each of a few axes (time, height, width), and
 * their caches are long.  The calls below rotate by such positions, keep a cache
 * in 4.25 bits a value, and attend over it, with a causal mask or, over an
 * encoder's states, without one.
 *
 * Format of a 4-bit cache.  A head row of 128 is four blocks of 32 neighbouring
 * dims.  A block has a scale byte s, worth 2^(s - 127) (255: the block is NaN),
 * and 32 elements of 4 bits: the sign in bit 3, and 0, 0.5, 1, 1.5, 2, 3, 4, 6
 * for bits 2..0 = 0..7.  A row's codes take 64 bytes (dim 2 d in the low half of
 * byte d, 2 d + 1 in the high half) and its scales 4.  Pools:
 *   kq_pool, vq_pool  uint8 [num_layers][num_slots][num_kv_heads][page_size * 68]:
 *                     a head's page holds its rows' codes, page_size * 64 bytes, and
 *                     then their scales, page_size * 4
 * Rows are quantised block by block: s = e - 2 with e the exponent byte of the
 * block's largest magnitude in fp32, rounded half up to one bit behind the point,
 * held to 1..252; each value divided by 2^(s - 127) goes to the nearest element,
 * halves to the one with an even code, beyond 6 to 6.  A block that holds an
 * infinity or a NaN becomes 255 with codes of 0.  Page tables, slots and their
 * counts are those of a bf16 cache (sa_kv_splice_alias, sa_kv_retain and
 * sa_kv_release work on them as they are; sa_kv_assemble, sa_kv_fork and
 * sa_kv_compact move bf16 pages and do not take these pools).
 *
 * They use the calling thread's device only within the call.  The calls that plan
 * on the host (sa_kv_append_rope_axes, sa_kvq_append, sa_kvq_attn) return
 * SA_ERR_UNSUPPORTED on a stream that is being captured into a graph;
 * sa_kvq_pack and sa_kvq_unpack keep nothing in the context and can be captured.
 * Slots of more than 2^30 elements and pools of 2^31 - 4096 slots or more are
 * refused (SA_ERR_UNSUPPORTED).
 */

/* Positions on several axes (sa_kv_append_rope_axes, sa_kvq_append). */
typedef struct sa_axes {
    int32_t num_axes;         /* 1 to 8                                                 */
    const int32_t *h_axis;    /* host [rot_dim / 2]: the axis that turns each pair, from
                                 0 to num_axes - 1 (sections or mixed, as the model has it) */
    const int32_t *d_pos;     /* device [num_axes][pos_stride]: each new token's position
                                 on each axis, any int32                                */
    int64_t pos_stride;       /* at least the number of new tokens                      */
} sa_axes;

/*
 * sa_kv_append_rope_axes — sa_kv_append_rope with a position per token and axis:
 * pair j of new token t (counted over all sequences) turns by
 *   a = axes.d_pos[axes.h_axis[j] * axes.pos_stride + t] * inv_freq[j]
 * (negative positions turn back).  h_start gives the cache positions, as there.
 *
 * Errors: those of sa_kv_append_rope; SA_ERR_NULL for NULL axes, axis numbers
 * (with a rot_dim) or positions, SA_ERR_SHAPE for a number of axes or an axis
 * out of range or a pos_stride below the new tokens, SA_ERR_ALIGN for positions
 * that are not 4-byte aligned.
 */
sa_status sa_kv_append_rope_axes(sa_ctx *ctx, const sa_layout *layout, int32_t layer, const sa_rope *rope,
                                 const sa_axes *axes, const void *q, int64_t q_stride, const void *k_new,
                                 int64_t k_stride, const void *v_new, int64_t v_stride, void *q_out,
                                 void *k_pool, void *v_pool, int32_t batch, const int32_t *h_start,
                                 const int32_t *h_new_len, sa_pages pages, void *stream);

/*
 * sa_kvq_append — new rows into a 4-bit cache, normed and rotated on the way.
 *
 * rope NULL: the key and value rows are quantised as they are; q and q_out must be
 * NULL, h_pos and axes too, and q_stride is not read.  Otherwise the key heads, and
 * the query heads where q and q_out are given (both or neither), are normed and
 * rotated as by sa_kv_append_rope (axes NULL; positions from h_pos, or h_start) or
 * sa_kv_append_rope_axes (h_pos NULL); keys are computed in 64 bits and
 * quantised from that, query rows in fp32 and rounded to bf16.  Value rows are quantised as they are.  Rows go to the
 * positions sa_kv_append would give them; nothing else in the pools changes.
 *
 * Errors: as sa_kv_append_rope and sa_kv_append_rope_axes, for the arguments given;
 * SA_ERR_SHAPE for q without q_out, or queries, positions or axes without a rope,
 * or both h_pos and axes.  A missing or out-of-range page is latched for
 * sa_sync_check; its rows are not written, q_out is.
 */
sa_status sa_kvq_append(sa_ctx *ctx, const sa_layout *layout, int32_t layer, const sa_rope *rope,
                        const sa_axes *axes, const void *q, int64_t q_stride, const void *k_new,
                        int64_t k_stride, const void *v_new, int64_t v_stride, void *q_out, void *kq_pool,
                        void *vq_pool, int32_t batch, const int32_t *h_start, const int32_t *h_new_len,
                        const int32_t *h_pos, sa_pages pages, void *stream);

/*
 * sa_kvq_pack — quantise pages: for i in 0 .. num_pages - 1, slot d_slots[i] of the
 * bf16 pools (layout, whole pages, every head and layer) into slot d_slots4[i] of
 * the 4-bit pools, which hold num_slots4 slots a layer.  Both lists are on the
 * device; a slot may be packed more than once, and d_slots4 must not repeat.
 * sa_kvq_unpack — the way back: slot d_slots4[i] of the 4-bit pools into slot
 * d_slots[i] of the bf16 pools, exactly (every value is a bf16 number; an element
 * of 4 or 6 under a scale byte of 253, or of 2 and more under 254, which the
 * quantisation never makes, becomes an infinity).  There d_slots must not repeat.
 * A slot outside its pool is latched for sa_sync_check and its page skipped;
 * SA_DEBUG=1 refuses it (SA_ERR_RANGE), and repeated destinations (SA_ERR_OVERLAP),
 * before launching, except on a stream that is being captured.
 *
 * Errors: SA_ERR_SHAPE (num_pages < 0, num_slots4 < 1, more pages than a launch
 * takes: layers * pages up to 2^23), SA_ERR_UNSUPPORTED, SA_ERR_NULL, SA_ERR_ALIGN,
 * SA_ERR_HIP.
 */
sa_status sa_kvq_pack(sa_ctx *ctx, const sa_layout *layout, const void *k_pool, const void *v_pool,
                      const int32_t *d_slots, int64_t num_slots4, void *kq_pool, void *vq_pool,
                      const int32_t *d_slots4, int32_t num_pages, void *stream);
sa_status sa_kvq_unpack(sa_ctx *ctx, const sa_layout *layout, int64_t num_slots4, const void *kq_pool,
                        const void *vq_pool, const int32_t *d_slots4, void *k_pool, void *v_pool,
                        const int32_t *d_slots, int32_t num_pages, void *stream);

/*
 * sa_kvq_attn — grouped-query attention over a 4-bit cache.
 *
 * causal != 0: sa_segment_prefill_attn's rows and keys (0 <= q_len <= kv_len; row i
 * sees kv_len - q_len + i + 1 keys).  causal == 0: every query row of a sequence
 * sees all of its kv_len keys (cross attention to states of another length; any
 * q_len, kv_len >= 0); where kv_len is 0 the rows are zeros and their LSE is
 * -infinity.  Lengths of keys are at most 2^31 - 64.
 * O = softmax(softmax_scale * q . K^T) V with the values the cache stands for.
 * Scores are the products of the cached keys with the bf16 query rows, summed in fp32
 * and then scaled.  In work items of more than 32 packed rows (num_q_heads / num_kv_heads
 * to a token) query values below 2^-6 of the largest of their 32 dims may be off by 2^-14 of
 * that, if in no block of 32 dims of the item's rows this adds up to more than 2^-14 of the
 * magnitudes of all its dims but the largest; else, in smaller items, and where a part of a
 * launch is of 512 keys or fewer, products are exact.
 * Probabilities are rounded to bf16 before the PV product, the rest is fp32.  A row that
 * sees a key with a NaN block has a NaN output and a NaN LSE; a NaN block of a value it sees
 * makes those 32 dims of its output NaN, and an infinite element (see sa_kvq_unpack) makes its
 * dim infinite or NaN; an infinite element of a key may make its row NaN.  What a row does
 * not see does not reach it.  Sums of values below 2^110 do not overflow, over however many
 * keys; of larger ones they may.  A page that is missing or outside the pool reads
 * as zeros and is latched for sa_sync_check.  `lse` may be NULL; pages.indices may
 * be NULL where no sequence with queries has keys.  Parts of a launch split by key
 * range (516 bytes of the split-KV partials per query row, head and part) are joined
 * by the launch itself where a row tile has few of them, else by a second kernel.  Plans take 52 bytes per
 * work item and 36 per split row tile.  sa_set_kernel_events times the first kernel
 * (SA_TIMED_ATTN).
 *
 * Errors: those of sa_segment_prefill_attn, SA_ERR_UNSUPPORTED for a capturing stream.
 */
sa_status sa_kvq_attn(sa_ctx *ctx, const sa_layout *layout, int32_t layer, const void *q, const void *kq_pool,
                      const void *vq_pool, int32_t batch, const int32_t *h_q_len, const int32_t *h_kv_len,
                      sa_pages pages, int32_t causal, float softmax_scale, void *o, float *lse, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SA_H */
