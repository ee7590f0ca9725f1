/*
 * tkv.h -- C ABI of libtkv: TriAxialKV's decode / append hot path on AMD
 * MI355X (gfx950).
 *
 * The library quantises newly written bf16 keys / values at a per-token
 * bitwidth (INT2 or INT4, chosen upstream from the token's temporal x
 * modality x semantic-role tag) into a paged mixed-precision KV pool, and
 * runs decode attention over that pool with on-the-fly dequantisation.
 *
 * Conventions
 *  - Every function returns an int status (TKV_OK = 0, errors negative)
 *    unless its type says otherwise; nothing throws, aborts or prints.
 *  - "host" pointers are ordinary CPU memory; "device" pointers are HIP
 *    device memory on the current device.  The caller owns every buffer and
 *    the stream.  The library allocates no device memory, never synchronises
 *    a stream and keeps no global state: calls on different streams are
 *    independent.
 *  - Argument checks that are possible from host-visible values are done
 *    before anything is launched, so a bad call launches nothing.
 *  - Geometry is fixed in this version: head_dim 128, group_size 32,
 *    page_tokens 64; other values return TKV_ERR_BAD_SHAPE.
 *  - bf16 and fp16 values are raw 16-bit patterns.
 */
#ifndef TKV_H
#define TKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    TKV_OK = 0,
    TKV_ERR_INVALID_ARG = -1,        /* null pointer, negative count, misaligned buffer */
    TKV_ERR_BAD_BITS = -2,           /* a bitwidth other than 2 or 4                      */
    TKV_ERR_BAD_SHAPE = -3,          /* unsupported geometry / head counts                */
    TKV_ERR_PAGE_RANGE = -4,         /* page id outside its pool                          */
    TKV_ERR_POOL_EXHAUSTED = -5,     /* allocator has too few free pages (state unchanged) */
    TKV_ERR_WORKSPACE_TOO_SMALL = -6,
    TKV_ERR_HIP = -7,                /* a launch failed; see hipGetLastError               */
    TKV_ERR_CAPACITY = -8            /* an output array supplied by the caller is too small */
};

/* Bits the kernels may OR into the optional device status word. */
enum {
    TKV_STATUS_TAG_MISMATCH = 1,     /* append: tag_bits[token] differs from its page's pool width (token skipped);
                                        tkv_quantize_rows: it is none of 0, 2 and 4 (token skipped) */
    TKV_STATUS_BITMAP_MISMATCH = 2,  /* decode: bit_map[page] differs from the width its position implies (page skipped) */
    TKV_STATUS_PAGE_RANGE = 4,       /* a page id read on the device lies outside the pool (page skipped) */
    TKV_STATUS_DST_RANGE = 8,        /* tkv_gather_dequant: an output row index >= n_tokens (slot skipped) */
    TKV_STATUS_BLOCK_PARTIAL = 16,   /* append, per-channel INT2 keys: a 32-token block arrived incomplete (block skipped);
                                        tkv_quantize_rows: a block names a token outside the call or not at INT2 (block skipped) */
    TKV_STATUS_SCALE_SATURATED = 32, /* decode: a stored V scale above 255, or a per-channel INT2 key scale above 1023, was
                                        clamped: the output is finite but not the attention over the stored values */
    TKV_STATUS_BAD_ITEM = 64,        /* decode: a work item names a sequence outside the batch (it contributes nothing)
                                        or a partial slot outside the workspace (its partial is not stored); prefill: an
                                        item names tokens, rows or slots that the call does not have (it is skipped) */
    TKV_STATUS_TABLE_REFUSED = 128,  /* tkv_table_append: lengths, widths or a table that cannot be (nothing was changed) */
    TKV_STATUS_POOL_EXHAUSTED = 256, /* tkv_table_append: too few free pages (nothing was changed) */
    TKV_STATUS_CAPACITY = 512        /* tkv_table_append: max_pages or max_work is too small (nothing was changed) */
};

const char *tkv_strerror(int status);

/*
 * Pool geometry.  Pages [0, n_pages_int2) form the INT2 pool, pages
 * [n_pages_int2, n_pages_int2 + n_pages_int4) the INT4 pool: one address
 * space split by an offset, so a page's precision is one comparison
 * (paper Sec. 3.2.2, "Shared address space").
 */
typedef struct tkv_desc {
    int32_t n_kv_heads;
    int32_t head_dim;       /* 128 */
    int32_t group_size;     /* 32  */
    int32_t page_tokens;    /* 64  */
    int32_t n_pages_int2;
    int32_t n_pages_int4;
    int32_t int2_key_axis;  /* TKV_KEYS_PER_TOKEN or TKV_KEYS_PER_CHANNEL */
} tkv_desc;

/*
 * Quantisation axis of the keys in the INT2 pool (Sec. 3.2.1, "Bitwidths and
 * quantization axes").  Values and INT4 keys are always per token: a group is
 * 32 consecutive channels of one token.
 *   TKV_KEYS_PER_TOKEN    INT2 keys are grouped the same way.
 *   TKV_KEYS_PER_CHANNEL  the paper's scheme: the 32 tokens of a block (slots
 *       0..31 or 32..63 of an INT2 page) share one (scale, zero-point) pair
 *       per channel.  A block is quantised in one piece, so INT2 tokens arrive
 *       in whole blocks: the stream of a sequence's INT2 tokens always holds a
 *       multiple of 32 tokens, and tokens that do not fill a block are stored
 *       at INT4 (tkv_route_residual).  The record size is the same; the K
 *       scale / K zero planes hold fp16 [block][128 channel positions].
 */
enum { TKV_KEYS_PER_TOKEN = 0, TKV_KEYS_PER_CHANNEL = 1 };

/* Bytes of one (page, kv head) record: 6144 for bits = 2, 10240 for bits = 4, 0 otherwise
 * (codes of K and V plus fp16 scale and zero-point per group of 32 channels, Sec. 3.2.1). */
size_t tkv_record_bytes(int bits);
/* Bytes of one page of the INT2 (bits = 2) or INT4 (bits = 4) pool: n_kv_heads records, the unit the per-pool
 * allocators hand out (Sec. 3.2.2, "Memory allocation").  0 on a bad descriptor or width; host only. */
size_t tkv_page_bytes(const tkv_desc *desc, int bits);
/* Bytes of the mixed-precision pool: the INT2 pages followed by the INT4 pages in ONE buffer, so that a page id
 * below n_pages_int2 is an INT2 page and any other an INT4 page (Sec. 3.2.2, "Shared address space": the split
 * point is fixed when the pool is sized from the average bitwidth).  The caller allocates this much device
 * memory, 256-byte aligned, and owns it.  0 on a bad descriptor; host only. */
size_t tkv_pool_bytes(const tkv_desc *desc);
/* Byte offset of the record of (page, head) inside the pool, or (size_t)-1 if out of range. */
size_t tkv_record_offset(const tkv_desc *desc, int32_t page, int32_t head);

/* ------------------------------------------------------------------ */
/* Page allocators (host).  One free list per pool, no coordination     */
/* between them (Sec. 3.2.2, "Memory allocation").                      */
/* ------------------------------------------------------------------ */
typedef struct tkv_alloc tkv_alloc;

/* shuffle_seed = 0: pages are handed out in increasing order; otherwise each
 * free list is shuffled with a generator seeded by it (scattered pages). */
int tkv_alloc_create(const tkv_desc *desc, uint64_t shuffle_seed, tkv_alloc **out);
void tkv_alloc_destroy(tkv_alloc *a);
/* Take n free pages of the given width into page_ids_out (host, n entries).
 * On TKV_ERR_POOL_EXHAUSTED nothing is taken. */
int tkv_alloc_pages(tkv_alloc *a, int bits, int32_t n, int32_t *page_ids_out);
/* Return pages to their pools (width follows from the id).  A page that is
 * out of range or already free gives TKV_ERR_PAGE_RANGE and nothing is freed. */
int tkv_free_pages(tkv_alloc *a, const int32_t *page_ids, int32_t n);
int32_t tkv_alloc_free_count(const tkv_alloc *a, int bits);

/* ------------------------------------------------------------------ */
/* Per-sequence page table (host).  A sequence owns two page streams:   */
/* its INT2 tokens fill INT2 pages in arrival order, its INT4 tokens    */
/* INT4 pages.  Listing INT2 pages before INT4 pages is the partition   */
/* that lets decode run width-homogeneous work (Sec. 3.2.3, "Decode",   */
/* phase 1).                                                            */
/* ------------------------------------------------------------------ */
typedef struct tkv_seq tkv_seq;

int tkv_seq_create(tkv_seq **out);
void tkv_seq_destroy(tkv_seq *s);                      /* does not return pages */
int tkv_seq_release(tkv_seq *s, tkv_alloc *a);         /* returns every page, empties the sequence */
int32_t tkv_seq_n_tokens(const tkv_seq *s, int bits);  /* tokens stored at this width */
int32_t tkv_seq_n_pages(const tkv_seq *s, int bits);
/* Copy the page list, INT2 pages first then INT4 pages, into out (host,
 * capacity entries).  Returns the number of pages or TKV_ERR_CAPACITY. */
int32_t tkv_seq_page_ids(const tkv_seq *s, int32_t *out, int32_t capacity);

/* ------------------------------------------------------------------ */
/* T1: triaxial tagger and tag -> bitwidth lookup (host).               */
/* ------------------------------------------------------------------ */
/*
 * A token's tag is a point of temporal x modal x semantic (Sec. 3.1):
 *   semantic  0 inst, 1 user, 2 assistant, 3 reasoning, 4 tool_call, 5 obs, 6 delim
 *   modal     0 text, 1 image
 *   temporal  0 older, 1 turn_m2, 2 turn_m1, 3 current
 * tag code = (temporal * 2 + modal) * 7 + semantic, 56 codes (TKV_N_TAGS).
 * tkv_tag_tokens derives the temporal axis in one scan from the per-token
 * semantic role and modality that the chat template gives (host, u8[n_tokens]
 * each): a turn runs from one user message up to, not including, the next;
 * a user message starts at a `user` token that does not follow a `user`
 * token; tokens before the first user message are turn 0.  tags_out: host
 * u8[n_tokens].  TKV_ERR_INVALID_ARG on a null array or an axis value out of
 * range (nothing is written then).
 * tkv_tags_to_bits looks every tag up in the calibrated map b*: S -> {2, 4}
 * (table, host u8[56]) and yields the per-token bitwidth array that
 * tkv_plan_append and tkv_quantize_append take (Sec. 3.2.3, "Tagging").
 * TKV_ERR_INVALID_ARG on a tag >= 56, TKV_ERR_BAD_BITS on a table entry other
 * than 2 or 4.  tkv_tag_counts adds the tokens of each tag to counts (host
 * i64[56], the N_k of Eq. 3); the caller zeroes it first.
 */
enum { TKV_N_TAGS = 56 };
int tkv_tag_tokens(const uint8_t *semantic, const uint8_t *modal, int32_t n_tokens, uint8_t *tags_out);
int tkv_tags_to_bits(const uint8_t *tags, int32_t n_tokens, const uint8_t *table, uint8_t *bits_out);
int tkv_tag_counts(const uint8_t *tags, int32_t n_tokens, int64_t *counts);

/* ------------------------------------------------------------------ */
/* A1: tag -> bitwidth allocation (host).                               */
/* ------------------------------------------------------------------ */
/*
 * Chooses b_k in {2, 4} for every tag k so that the total distortion
 * sum_k D_k(b_k) is small under the budget sum_k N_k b_k <= B sum_k N_k
 * (Sec. 3.1.3, Eq. 3).  All arrays are host memory.
 *   n_tags   number of tags (the paper's triaxial space has 56)
 *   N        i64[n_tags]  token count of each tag, >= 0
 *   D2, D4   f64[n_tags]  distortion of the tag at 2 / 4 bits, finite
 *   B        target average bitwidth, 2 <= B <= 4
 *   bits_out u8[n_tags]   2 or 4 per tag
 * The budget is T = B * sum N in binary64 with a relative slack of 2^-40 (a
 * decimal B is not a binary64 number); bits in use are counted exactly.
 * tkv_allocate_bits_greedy is Alg. 1: per-bit gain rho_k = (D_k(2) - D_k(4)) /
 * (2 N_k) (Eq. 4; +inf / 0 / -inf by the sign of the gain when N_k = 0), tags
 * visited by rho descending (ties in tag order), a tag is upgraded whenever its
 * 2 N_k extra bits still fit.  tkv_allocate_bits_exhaustive visits all 2^n_tags
 * allocations (n_tags <= 22, as in the paper) and returns the feasible one of
 * least total distortion; ties go to fewer total bits, then to the smaller mask
 * (tag 0 = lowest bit, set = 4 bits).
 * Errors: TKV_ERR_INVALID_ARG (null array, negative count, non-finite distortion,
 * B outside [2, 4], n_tags < 0 or > 22 for the exhaustive search).
 */
int tkv_allocate_bits_greedy(int32_t n_tags, const int64_t *N, const double *D2, const double *D4,
                             double B, uint8_t *bits_out);
int tkv_allocate_bits_exhaustive(int32_t n_tags, const int64_t *N, const double *D2, const double *D4,
                                 double B, uint8_t *bits_out);

/* ------------------------------------------------------------------ */
/* Q1: route newly arrived tokens to slots (host).                      */
/* ------------------------------------------------------------------ */
/*
 * Residual policy of the per-channel INT2 keys (Sec. 3.2.1): of the tokens
 * tagged INT2 in tag_bits (host, u8[n_tokens], one arriving chunk of one
 * sequence) the last (count mod 32) do not fill a block and are stored at
 * INT4.  bits_out (host, u8[n_tokens], may alias tag_bits) receives the
 * per-token widths to hand to tkv_plan_append and tkv_quantize_append.
 * Errors: TKV_ERR_INVALID_ARG, TKV_ERR_BAD_BITS.
 */
int tkv_route_residual(const uint8_t *tag_bits, int32_t n_tokens, uint8_t *bits_out);

/* Upper bound of pages one tkv_plan_append call over n_tokens can touch. */
int32_t tkv_plan_append_max_work(int32_t n_tokens);
/*
 * tag_bits (host, u8[n_tokens]) is the per-token bitwidth array produced by
 * the tagger and the tag -> bitwidth table (Sec. 3.2.3, "Tagging").  Tokens
 * of each width are appended, in order, to the sequence's page stream of that
 * width; new pages come from the matching allocator.  Outputs (host):
 *   slot_ids_out[n_tokens]      page_id * 64 + slot of every token (the
 *                               per-token pointer of the page table);
 *   work_pages_out[max_work]    the distinct pages that receive tokens;
 *   work_src_out[max_work*64]   for each such page and slot, token_base +
 *                               index of the token that goes there, or -1;
 *   *n_work_out                 number of pages listed.
 * token_base lets several sequences' plans address one concatenated K/V
 * tensor.  With TKV_KEYS_PER_CHANNEL the number of INT2 tokens must be a
 * multiple of 32 (TKV_ERR_INVALID_ARG otherwise; see tkv_route_residual).
 * On any error the sequence and the allocator are left unchanged.
 */
int tkv_plan_append(tkv_alloc *a, tkv_seq *s, const uint8_t *tag_bits, int32_t n_tokens,
                    int32_t token_base, int32_t *slot_ids_out, int32_t *work_pages_out,
                    int32_t *work_src_out, int32_t max_work, int32_t *n_work_out);

/* ------------------------------------------------------------------ */
/* Q2-Q5: quantise and pack (device).                                   */
/* ------------------------------------------------------------------ */
/*
 * For every listed page and kv head: asymmetric min/max quantisation of each
 * group of 32 channels of each arriving token (zero = fp16(min), scale =
 * fp16((max-min)/(2^b-1)), code = round-half-even((x-zero)*(1/scale)) clamped),
 * per-token for K and V at both widths, or, with TKV_KEYS_PER_CHANNEL, the
 * keys of INT2 pages per channel over each block of 32 slots (Sec. 3.2.1),
 * packed into the page's planes; bit_map[page] is set to the page's width.
 * Bits of slots whose work_src entry is -1 are left untouched.  With
 * TKV_KEYS_PER_CHANNEL the 32 slots of a block of an INT2 page must all be
 * named or all be -1; a block named in part is skipped (keys and values) and
 * TKV_STATUS_BLOCK_PARTIAL is raised.
 *   pool       device, tkv_pool_bytes(desc) bytes, 256-byte aligned
 *   bit_map    device u8[n_pages_int2 + n_pages_int4]
 *   K, V       device bf16 [n_tokens, n_kv_heads, head_dim], contiguous
 *   tag_bits   device u8[n_tokens]; a token whose width differs from its
 *              page's pool is skipped and TKV_STATUS_TAG_MISMATCH is raised
 *   work_pages device i32[n_work], work_src device i32[n_work*64] as written
 *              by tkv_plan_append; a page may appear at most once per call
 *   status     device i32, may be NULL; kernels OR TKV_STATUS_* bits into it
 * group_size must be 32.  n_work = 0 is a no-op.
 */
int tkv_quantize_append(const tkv_desc *desc, void *pool, uint8_t *bit_map,
                        const void *K, const void *V, const uint8_t *tag_bits,
                        int32_t n_tokens, int32_t group_size,
                        const int32_t *work_pages, const int32_t *work_src, int32_t n_work,
                        int32_t *status, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* P1: prefill gather-dequant (device).                                 */
/* ------------------------------------------------------------------ */
/*
 * Reads the listed pages of a matched prefix from the pool, unpacks every
 * listed slot, dequantises it into FP16 and writes dense K / V rows for an
 * FP16 prefill attention kernel (Sec. 3.2.3, "Prefill").  Each value is the
 * binary16 nearest-even rounding of the exact code * scale + zero.
 *   pool, bit_map  device, as filled by tkv_quantize_append
 *   work_pages     device i32[n_work]: the pages to read, each at most once
 *   work_dst       device i32[n_work*64]: for each page and slot the output
 *                  row (token index) or -1 to skip the slot; the lists that
 *                  tkv_plan_append wrote (work_pages_out, work_src_out) name
 *                  exactly the rows the tokens came from
 *   K_out, V_out   device fp16 [n_tokens, n_kv_heads, head_dim], contiguous,
 *                  16-byte aligned; rows that no slot names are left untouched
 *   status         device i32, may be NULL: TKV_STATUS_PAGE_RANGE (page id
 *                  outside the pool), TKV_STATUS_BITMAP_MISMATCH (page never
 *                  written at its pool's width), TKV_STATUS_DST_RANGE; the
 *                  page or slot concerned is skipped
 * n_work = 0 is a no-op.
 */
int tkv_gather_dequant(const tkv_desc *desc, const void *pool, const uint8_t *bit_map,
                       const int32_t *work_pages, const int32_t *work_dst, int32_t n_work,
                       void *K_out, void *V_out, int32_t n_tokens,
                       int32_t *status, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* D1: cut page lists into work items (host).                           */
/* ------------------------------------------------------------------ */
/*
 * Split-K over a sequence's page list (Sec. 3.2.3, "Decode"): a work item is a
 * contiguous range of one sequence's page list (INT2 pages first); one
 * wavefront per (item, kv head) leaves a partial (m, l, acc) that
 * tkv_decode_reduce merges.  Items are balanced by decode cost (an INT2 page
 * weighs 6, an INT4 page 7): the planner finds the smallest bound on an item's
 * cost for which the batch still splits into at most target_items items and
 * cuts every sequence into equal parts below that bound, so the number of items
 * never exceeds target_items unless there are more non-empty sequences than
 * that (then one item each).  Where the longest such part has two pages (or
 * three, with at most four INT4 pages in five and, per-channel keys, a fifth of
 * target_items to spare; or four, with per-token keys and at most two INT4
 * pages in five) and target_items times the kv heads fit the 3072 wavefronts
 * that a whole MI355X holds at once, every item gets as many pages as that part
 * instead: fewer items, none with more pages than the longest equal part and,
 * at four pages, none of a greater cost than the heaviest.  Under the same
 * condition, where the longest part has one page (two pages) and the pages times
 * the kv heads are more than 2048 (4096) and at most 3072 (6144), an item gets a
 * page more than that.
 * A plan depends only on the page COUNTS of the sequences: it stays valid while
 * tokens are appended to open pages (the kernel reads the token counts from the
 * device arrays and masks by them) and must be made again when a sequence gains
 * a page -- at most every 64 decoded tokens per sequence.  With a stale plan the
 * new page is simply not read.  Layers that share a page table share the plan.
 *   page_indptr   host i32[batch+1], page-list offsets of the sequences
 *   n_tok_int2/4  host i32[batch], valid tokens per width (last page may be partial;
 *                 with TKV_KEYS_PER_CHANNEL n_tok_int2 must be a multiple of 32)
 *   target_items  wanted number of items over the whole batch (>= 1)
 *   items_out     host i32[4*capacity]: {sequence, first page, end page, partial
 *                 slot}, page indices relative to the sequence's list.  Items
 *                 are listed in LAUNCH order (the kernel runs item k as its
 *                 k-th group of workgroups): by falling share of INT2 pages,
 *                 so that the wavefronts that end up on one SIMD mix ranges
 *                 that keep it busy (INT2) with ranges that mostly wait for
 *                 memory (INT4).  The partial of an item is written to slot
 *                 `partial slot` of the workspace; the slots are a permutation
 *                 of 0 .. n_items-1 in sequence order.
 *   seq_item_indptr_out  host i32[batch+1]: sequence b owns the partial slots
 *                 [indptr[b], indptr[b+1]); a sequence without tokens has none
 * Returns the number of items (>= 0) or a negative status.
 */
int32_t tkv_plan_decode_capacity(int32_t batch, int32_t target_items);
int32_t tkv_plan_decode(const tkv_desc *desc, int32_t batch, const int32_t *page_indptr,
                        const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                        int32_t target_items, int32_t *items_out, int32_t capacity,
                        int32_t *seq_item_indptr_out);

/* ------------------------------------------------------------------ */
/* D2-D7: decode attention (device).                                    */
/* ------------------------------------------------------------------ */
/* Bytes of workspace that decode attention over n_items work items needs: the partial (m, l, acc[head_dim]) in
 * fp32 of every (item, query head), which the split kernel writes and the cross-split merge reads (Sec. 3.2.3,
 * "Decode": splits merged by log-sum-exp).  Device memory, 16-byte aligned, owned by the caller; it needs no
 * initialisation and may be shared by calls on the same stream.  0 on a bad descriptor or count; host only. */
size_t tkv_decode_workspace_bytes(const tkv_desc *desc, int32_t n_items, int32_t n_q_heads);
/*
 * Decode attention over the mixed-precision paged cache (Sec. 3.2.3, "Decode"):
 * out[b, h, :] = softmax(sm_scale * q[b, h, :] . K^T) V over the dequantised
 * tokens of sequence b's pages, query head h reading kv head
 * h / (n_q_heads / n_kv_heads); every page runs the dequantisation path of its
 * pool (INT2 or INT4).  A sequence with no tokens gives zeros.
 *   pool, bit_map  device, as filled by tkv_quantize_append
 *   q              device bf16 [batch, n_q_heads, head_dim]
 *   page_indptr    device i32[batch+1]
 *   page_ids       device i32[page_indptr[batch]]: per sequence INT2 pages then INT4 pages
 *   n_tok_int2/4   device i32[batch]
 *   items          device i32[4*n_items], seq_item_indptr device i32[batch+1] (tkv_plan_decode)
 *   out            device fp32 [batch, n_q_heads, head_dim]
 *   workspace      device, >= tkv_decode_workspace_bytes(...), 16-byte aligned
 *   status         device i32, may be NULL
 *   items          every item must name a sequence of the batch and a partial
 *                  slot below n_items, each slot once, the slots of a sequence
 *                  as seq_item_indptr lists them.  An item that names no
 *                  sequence of the batch contributes nothing (an empty partial
 *                  in its slot) and raises TKV_STATUS_BAD_ITEM; so does one
 *                  with a slot out of range, which cannot write anything: the
 *                  sequence that owns the slot it should have named then reads
 *                  what the workspace held before.  The page range of an item
 *                  is clamped to the sequence's pages.
 * The page tables on the device must describe the same sequences as the host
 * arrays the plan was made from (tkv_plan_decode above says when a plan ages).
 * Preconditions on the cache contents: stored scales and zeros finite; V scales
 * up to 255 are used exactly, larger ones are clamped there (the kernel forms
 * softmax weight x V scale in fp16 and keeps it finite); with
 * TKV_KEYS_PER_CHANNEL the scales of the INT2 keys likewise up to 1023 (the
 * kernel forms q x K scale in fp16), and every n_tok_int2 is a multiple of 32.
 * Preconditions on q: finite, and no sum of a head's q over one of the four
 * groups of 32 channels beyond 65504 in magnitude (the kernel keeps these sums
 * in fp16 pieces).  A query head that breaks them gives NaN; NaN and infinities
 * in it leave the other heads alone.  The query heads of a kv head share one
 * power of two: what is far below the largest finite |q| of theirs is rounded to
 * 2^-30 of that (TKV_KEYS_PER_CHANNEL: 2^-24).
 * A clamped scale raises TKV_STATUS_SCALE_SATURATED: the output is then finite
 * but not the attention over the stored values.
 * n_q_heads / n_kv_heads must be 1, 2, 4 or 8.  Two launches on `stream`:
 * the split kernel, then the cross-split reduction.
 */
int tkv_decode_attention(const tkv_desc *desc, const void *pool, const uint8_t *bit_map,
                         const void *q, const int32_t *page_indptr, const int32_t *page_ids,
                         const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                         const int32_t *items, const int32_t *seq_item_indptr, int32_t n_items,
                         int32_t batch, int32_t n_q_heads, float sm_scale, float *out,
                         void *workspace, size_t workspace_bytes, int32_t *status,
                         void *stream /* hipStream_t */);

/*
 * The two launches of tkv_decode_attention as separate calls, same arguments
 * and the same checks: D2-D6, the split kernel, which leaves one partial
 * (m, l, acc) per work item and query head in `workspace`; and D7, the
 * cross-split merge by log-sum-exp (Sec. 3.2.3), which reads the partials
 * and writes `out`.  tkv_decode_attention is exactly one call of each.
 */
int tkv_decode_split(const tkv_desc *desc, const void *pool, const uint8_t *bit_map,
                     const void *q, const int32_t *page_indptr, const int32_t *page_ids,
                     const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                     const int32_t *items, int32_t n_items, int32_t batch, int32_t n_q_heads,
                     float sm_scale, void *workspace, size_t workspace_bytes, int32_t *status,
                     void *stream /* hipStream_t */);
int tkv_decode_reduce(const tkv_desc *desc, const int32_t *seq_item_indptr, int32_t n_items,
                      int32_t batch, int32_t n_q_heads, float *out, const void *workspace,
                      size_t workspace_bytes, void *stream /* hipStream_t */);

/*
 * tkv_decode_attention for callers that cannot allocate device memory or pass
 * a workspace: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, same checks, same two launches and
 * the same results; the partials live in a fixed device array inside the
 * library (TKV_DECODE_STATIC_SCRATCH_BYTES per GPU, held until the process
 * ends) instead of a caller workspace.  The call allocates and frees nothing.
 * TKV_ERR_WORKSPACE_TOO_SMALL when tkv_decode_workspace_bytes(desc, n_items,
 * n_q_heads) exceeds the array (nothing is launched); TKV_ERR_HIP when the
 * array's address cannot be obtained.  The device that owns `stream` must be
 * the current device.  All calls on one GPU share the array: two calls whose
 * kernels may overlap in time (different streams, or replays of captured
 * graphs running concurrently) race on it; calls on one stream are ordered
 * and safe.
 */
#define TKV_DECODE_STATIC_SCRATCH_BYTES (16u << 20)
int tkv_decode_attention_static(const tkv_desc *desc, const void *pool, const uint8_t *bit_map,
                                const void *q, const int32_t *page_indptr, const int32_t *page_ids,
                                const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                                const int32_t *items, const int32_t *seq_item_indptr, int32_t n_items,
                                int32_t batch, int32_t n_q_heads, float sm_scale, float *out,
                                int32_t *status, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* D8: decode attention over shared prefixes (host plan, device).       */
/* ------------------------------------------------------------------ */
/*
 * Groups of sequences whose contexts begin with the same tokens (a system
 * prompt with its tools, a document) list the pages of that prefix once, as a
 * page list of the group; the sequences' own page lists hold what follows.  A
 * sequence may be a member of several groups (a prompt of all, a document of
 * some) or of none.  Attention does not depend on the order of tokens, so
 * several prefixes need none.
 *   n_groups, n_members   groups; entries of member_seqs
 *   tile_rows             query rows of an item, 16, 64 or 128, as tkv_plan_decode_shared chooses them
 *   n_items               prefix work items
 *   page_indptr  device i32[n_groups+1] page-list offsets of the groups
 *   page_ids     device i32: per group INT2 pages, then INT4 pages, of the same pool as the sequences' own
 *   n_tok_int2/4 device i32[n_groups] valid tokens per width
 *   member_indptr device i32[n_groups+1], member_seqs device i32[n_members]: sequences of each group
 *   member_slots device i32[n_members], items device i32[5*n_items]: as written by tkv_plan_decode_shared
 */
typedef struct tkv_prefix {
    int32_t n_groups, n_members, tile_rows, n_items;
    const int32_t *page_indptr;
    const int32_t *page_ids;
    const int32_t *n_tok_int2;
    const int32_t *n_tok_int4;
    const int32_t *member_indptr;
    const int32_t *member_seqs;
    const int32_t *member_slots;
    const int32_t *items;
} tkv_prefix;

/* Upper bound of the items that tkv_plan_decode_shared makes. */
int32_t tkv_plan_shared_capacity(int32_t n_groups, int32_t n_members, int32_t target_cus);
/*
 * Cuts the groups' page lists into parts, and those and the groups' query rows
 * (of one kv head: n_q_heads / n_kv_heads of each member) into work items, and
 * gives every (part, member) a partial slot behind the n_own_items slots of the
 * sequences' own items (tkv_plan_decode).  An item is one workgroup per kv head
 * for tile_rows rows: with 16 its eight wavefronts work on a page each at a
 * time, with 64 and 128 on two pages together.  The number of rows is the one
 * that is expected to take least time, and parts are equal numbers of whole
 * steps, as small as still gives no more workgroups than target_cus compute
 * units, less those that the own items take (or none, where these are few
 * beside the prefixes).  Depends on the page counts and members only, and ages
 * as a decode plan does.
 *   n_tok_int2/4   host i32[n_groups]
 *   member_indptr  host i32[n_groups+1], from 0; member_seqs host i32[member_indptr[n_groups]],
 *                  below batch, each at most once in a group
 *   target_cus     compute units to fill (>= 1)
 *   items_out      host i32[5*capacity]: {group, first page, end page, number of the part in the group, first row}
 *   member_slots_out  host i32[members]: slot of the member's partial of the group's first part, the others follow
 *   seq_slot_indptr_out  host i32[batch+1]: slots of each sequence, from n_own_items on
 *   tile_rows_out  host i32
 * Returns the number of items (>= 0) or a negative status.
 */
int32_t tkv_plan_decode_shared(const tkv_desc *desc, int32_t batch, int32_t n_q_heads, int32_t n_groups,
                               const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                               const int32_t *member_indptr, const int32_t *member_seqs, int32_t target_cus,
                               int32_t n_own_items, int32_t *items_out, int32_t capacity,
                               int32_t *member_slots_out, int32_t *seq_slot_indptr_out, int32_t *tile_rows_out);
/*
 * tkv_decode_attention over each sequence's prefixes and its own tokens
 * together.  Values, and the keys of items of 64 and 128 rows, are dequantised
 * to fp16 as tkv_gather_dequant does (as a prefill over them saw them); other
 * keys are not rounded.  Softmax weights are fp16, sums 32 bits.  The output is
 * bf16, as the projection behind it takes it.  A sequence without tokens gives zeros.
 *   q, page_indptr .. n_items, sm_scale   as for tkv_decode_attention (own tokens; n_items may be 0)
 *   prefix         host struct of device arrays, above; n_items may be 0
 *   slot_indptr    device i32[2*(batch+1)]: seq_item_indptr_out of tkv_plan_decode, then seq_slot_indptr_out
 *   n_slots        seq_slot_indptr_out[batch]
 *   out            device bf16 [batch, n_q_heads, head_dim], 16-byte aligned
 *   workspace      device, >= tkv_decode_workspace_bytes(desc, n_slots, n_q_heads), 16-byte aligned
 *   status         device i32, may be NULL; bits as for tkv_decode_attention.  Members outside the batch, slots outside
 *                  [n_items, n_slots) and items outside the groups raise TKV_STATUS_BAD_ITEM: what they name is not stored,
 *                  and the sequence reads what the workspace held before
 * Preconditions: stored scales and zeros finite, values within fp16, and so 14
 * times the scales of INT4 keys and twice those of INT2 keys; with
 * TKV_KEYS_PER_CHANNEL every n_tok_int2 a multiple of 32.  q may hold any values
 * whose products with sm_scale, and the logits that they give (times log2 e), are
 * finite in 32 bits; a query head of NaN or infinities gives NaN and leaves the
 * others alone.  n_q_heads / n_kv_heads is 1, 2, 4 or 8.  Two launches on `stream`:
 * attention, then the merge.
 */
int tkv_decode_attention_shared(const tkv_desc *desc, const void *pool, const uint8_t *bit_map, const void *q,
                                const int32_t *page_indptr, const int32_t *page_ids,
                                const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                                const int32_t *items, int32_t n_items, const tkv_prefix *prefix,
                                const int32_t *slot_indptr, int32_t n_slots, int32_t batch, int32_t n_q_heads,
                                float sm_scale, void *out, void *workspace, size_t workspace_bytes,
                                int32_t *status, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* Q1 on the GPU: page tables of a batch in device memory.              */
/* ------------------------------------------------------------------ */
/*
 * The page tables, token counts and free lists of n_seqs sequences, all in
 * device memory that the caller owns (4-byte aligned), for loops that the host
 * does not take part in: a captured decode step, drafting and rejecting.  The
 * same page streams as a tkv_seq has: row b of page_ids holds the sequence's
 * INT2 pages, then its INT4 pages, then -1; with page_indptr[b] = b * max_pages
 * (i32[n_seqs+1]) it is what tkv_decode_attention and tkv_decode_split take.
 * Free lists are stacks, the next page to hand out last: free_pages[0 ..
 * n_free[0]) those of the INT2 pool, free_pages[n_pages_int2 .. n_pages_int2 +
 * n_free[1]) those of the INT4 pool; behind them anything.
 * A decode plan (tkv_plan_decode) made for more INT4 pages than a sequence has
 * yet stays valid while it grows into them: what an item names beyond the
 * sequence's pages is not read.  Pages beyond the plan's are not read either, and
 * no status bit says so: the plan is made, by the host, for the pages that the
 * sequences can have when the next one replaces it.  (A sequence of n tokens of
 * a width has at most (n + 63) / 64 pages of it, and the host knows how many
 * tokens it has handed in, if not how many were cut off.)
 */
typedef struct tkv_table {
    int32_t n_seqs;
    int32_t max_pages;      /* entries of a row, at most 2^24; n_seqs * max_pages < 2^31 */
    int32_t *page_ids;      /* i32[n_seqs * max_pages] */
    int32_t *n_tok_int2;    /* i32[n_seqs] */
    int32_t *n_tok_int4;    /* i32[n_seqs] */
    int32_t *free_pages;    /* i32[n_pages_int2 + n_pages_int4] */
    int32_t *n_free;        /* i32[2] */
} tkv_table;

/* No sequence has tokens and all pages are free, handed out in increasing order (one launch). */
int tkv_table_reset(const tkv_desc *desc, const tkv_table *table, void *stream /* hipStream_t */);
/* Upper bound of the pages that n_tokens tokens for n_seqs sequences can touch. */
int32_t tkv_table_max_work(int32_t n_seqs, int32_t n_tokens);
/* Bytes of workspace of tkv_table_append; 0 on a bad count. */
size_t tkv_table_workspace_bytes(int32_t n_seqs, int32_t n_tokens);
/*
 * First cuts every sequence b back to its first keep_int2[b] tokens of the INT2
 * stream and keep_int4[b] of the INT4 stream (0: a request that has ended; a
 * few less: rejected drafts; as many or more than there are: nothing); pages
 * that hold none of them return to the free lists, the first page of the first
 * sequence on top, so that the same tokens appended again get the same pages.
 * Then appends n_new[b] tokens to sequence b: the next ones of tag_bits (the
 * sequences' tokens lie one behind the other), each to the stream of its width,
 * pages from the top of the free lists, sequences in order: what one
 * tkv_plan_append per sequence does.
 *   keep_int2/4   device i32[n_seqs], or NULL: nothing is cut
 *   n_new         device i32[n_seqs], or NULL: nothing arrives
 *   tag_bits      device u8[n_tokens], 2 or 4; may be NULL if n_tokens = 0.  The
 *                 lengths sum to at most n_tokens; tokens behind the last
 *                 sequence (a padded batch) are no tokens
 *   token_indptr  device i32[n_seqs+1] or NULL: first token of each sequence
 *   positions     device i32[n_tokens] or NULL: place of each token in its
 *                 sequence, over both widths; -1 behind the last sequence
 *   slot_ids      device i32[n_tokens] or NULL: page * 64 + slot; -1 behind
 *   work_pages, work_src   device i32[max_work], i32[max_work*64]: as written by
 *                 tkv_plan_append (of each sequence INT2 pages, then INT4 pages);
 *                 entries behind the last are page 0 with no slot named, which
 *                 tkv_quantize_append passes over: it can be called with
 *                 n_work = max_work from code that does not know n_work.
 *                 max_work: see tkv_table_max_work
 *   n_work        device i32: number of pages listed
 *   workspace     device, >= tkv_table_workspace_bytes(...), 16-byte aligned,
 *                 needs no initialisation, may be shared by calls on one stream
 *   status        device i32, may be NULL
 * All or nothing: where lengths are negative or sum to more than n_tokens, a
 * width is neither 2 nor 4, counts of per-channel INT2 keys are no multiples of
 * 32 (arriving or kept) or a count of the table cannot be (tokens below zero or
 * beyond max_pages, free pages below zero or, with those given back, more than
 * the pool has: TKV_STATUS_TABLE_REFUSED), a pool has too few pages
 * (TKV_STATUS_POOL_EXHAUSTED), or max_pages or max_work does not suffice
 * (TKV_STATUS_CAPACITY), the table stays as it is, n_work and token_indptr are
 * 0, no slot is named, and slot_ids and positions are -1.
 * Page ids are not compared with their pools: what a row or a free list holds is
 * handed on as it is, and tkv_quantize_append and attention leave out a page
 * that is none or not of its width, with their own status bits.
 * One launch for up to 1024 sequences, 6144 tokens and max_work of 1024, else up
 * to four.
 */
int tkv_table_append(const tkv_desc *desc, const tkv_table *table, const int32_t *keep_int2, const int32_t *keep_int4,
                     const int32_t *n_new, const uint8_t *tag_bits, int32_t n_tokens,
                     int32_t *token_indptr, int32_t *positions, int32_t *slot_ids,
                     int32_t *work_pages, int32_t *work_src, int32_t max_work, int32_t *n_work,
                     void *workspace, size_t workspace_bytes, int32_t *status, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* R1: norm and rotation of queries and keys (device), its table (host).*/
/* ------------------------------------------------------------------ */
/*
 * What stands between the projections and the cache, which takes keys with
 * their positions encoded (Sec. 3.2.3).  A position has one to four axes
 * (text: one; images and video: time, height, width); each pair of channels
 * turns with one of them.
 *
 * tkv_rope_table (host): one word per pair of channels, table_out[i] = the
 * turns per position of pair i, inv_freq[i] / 2 pi, modulo 1, in units of
 * 2^-64, rounded to a multiple of four units (2^-63 turns), which leaves its
 * lowest two bits for the pair's axis.
 *   rotary_dim  channels 0 .. rotary_dim-1 of a head turn, a multiple of 16,
 *               0 .. 128; the others keep their place
 *   sections    host i32[n_axes], pairs of each axis, summing to rotary_dim/2;
 *               NULL for one axis
 *   interleaved 0: the first sections[0] pairs turn with axis 0, the next
 *               sections[1] with axis 1, ...; 1: pairs are dealt out in turn
 *               (pair i to axis i mod n_axes), and an axis whose section is
 *               used up passes its turn to axis 0
 *   inv_freq    host f64[rotary_dim/2], angle per position of each pair, or
 *               NULL for theta^(-2 i / rotary_dim)
 *   table_out   host u64[rotary_dim/2]
 * Errors: TKV_ERR_BAD_SHAPE (rotary_dim, n_axes not in 1..4, sections that do
 * not fit), TKV_ERR_INVALID_ARG (null table, theta <= 0 or a frequency that is
 * not finite).
 */
typedef struct tkv_rope {
    int32_t rotary_dim;
    int32_t n_axes;
    int32_t adjacent;       /* 0: pair i is channels (i, i + rotary_dim/2); 1: channels (2i, 2i+1) */
    float scale;            /* factor of cosine and sine, 1 unless the frequencies were stretched with one */
    const uint64_t *table;  /* device, u64[rotary_dim/2] as written by tkv_rope_table, 8-byte aligned */
} tkv_rope;
int tkv_rope_table(int32_t rotary_dim, int32_t n_axes, const int32_t *sections, int32_t interleaved,
                   double theta, const double *inv_freq, uint64_t *table_out);
/*
 * For every token t and head h of q and k: the RMS norm over the head's 128
 * channels, x * rsqrt(mean(x^2) + eps) * weight, where a weight is given, then
 * the rotation of its pairs: (a, b) becomes (a cos - b sin, a sin + b cos) *
 * scale with angle positions[axis][t] * frequency.  Values v, if given, are
 * copied.  All in 32 bits (angles: what the table holds to 2^-33 turns at any
 * position), rounded once.
 *   q, k, v      device bf16, 16-byte aligned; token t, head h, channel c at
 *                t * stride + h * 128 + c with the tensor's own stride in
 *                elements (a multiple of 8): parts of a packed projection, or
 *                tensors of their own.  q may be NULL if n_q_heads = 0; k and v
 *                if n_kv_heads = 0; v may be NULL at any time
 *   positions    device i32[n_axes][n_tokens], any value; unused (may be NULL)
 *                if rotary_dim = 0
 *   q_weight,    device bf16[128], 16-byte aligned, or NULL: no norm
 *   k_weight
 *   q_out, k_out, device bf16 [n_tokens, heads, 128], contiguous, 16-byte
 *   v_out        aligned; an output may be its input, if that is contiguous,
 *                and overlaps no other buffer of the call
 * The sum of a row's squares must be finite in 32 bits (a row beyond that gives
 * zeros, one that holds NaN or infinities NaN; other rows are left alone), and
 * with eps = 0 a row whose mean square is below 2^-126, the smallest normal
 * number, gives NaN or infinities.  At most 2^31 - 4096 rows of heads in
 * all.  n_tokens = 0 is a no-op.  One launch on `stream`.
 */
int tkv_norm_rope(const tkv_rope *rope, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                  const void *v, int64_t v_stride, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                  const int32_t *positions, const void *q_weight, const void *k_weight, float eps,
                  void *q_out, void *k_out, void *v_out, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* P2: attention of prompts over a gathered prefix (host plan, device). */
/* ------------------------------------------------------------------ */
/* Types of rows where an entry point takes more than one. */
enum { TKV_BF16 = 0, TKV_FP16 = 1, TKV_FP32 = 2 };
/*
 * Plan of tkv_prefill_attention: which query rows meet which keys in which
 * workgroup.  All host memory.  Row r of a sequence and kv head is query head
 * r mod R of new token r / R, R = n_q_heads / n_kv_heads.  An item is a tile of
 * tile_rows such rows (the same tile of every kv head) and a range of tiles of
 * keys (32 with 32 rows, 64 with 128 and 256), those of the prefix first; where
 * there are too few tiles of rows to fill target_cus compute units, long ranges
 * are cut into equal parts, whose partial results lie in a workspace and are
 * joined.  The number of rows is the one that is expected to take least time.
 * Items come by falling length (of 128 rows, if none is cut, the first target_cus
 * workgroups by rising length).  The plan depends on the lengths alone: layers,
 * and replays of the same requests, share it.
 *   desc             n_kv_heads and geometry; the pools may be empty
 *   seq_indptr       host i32[batch+1], from 0: the sequences' new tokens
 *   prefix_indptr    host i32[batch+1], from 0, or NULL: their prefix rows
 *   target_cus       compute units to fill (>= 1)
 *   items_out        host i32[16*capacity]: {first new token, new tokens, first
 *                    prefix row, prefix rows, first row, first key tile, end,
 *                    partial slot or -1, part, parts; and in the k-th item, of
 *                    the k-th tile that is cut, first new token, new tokens,
 *                    first row, first slot, parts; 0}
 *   tile_rows_out    host i32: 32, 128 or 256
 *   n_slots_out      host i32: partial slots, 0 if no range is cut
 *   n_cut_out        host i32: tiles whose ranges are cut
 * Returns the number of items (>= 0) or a negative status.  A sequence without
 * new tokens has none.  At most 2^30 rows (tokens * R) a sequence, 2^31 - 1 in
 * all, 65535 kv heads (and query heads, if there is more than one token: the
 * token stride), 2^25 - 1 workgroups (items * kv heads) and 2^31 - 1 rows
 * of tiles that are cut (tiles * kv heads * tile_rows); the call takes no more.
 * tkv_plan_prefill_capacity: an upper bound of the items for n_tokens new tokens.
 */
int32_t tkv_plan_prefill_capacity(const tkv_desc *desc, int32_t batch, int32_t n_tokens, int32_t n_q_heads, int32_t target_cus);
int32_t tkv_plan_prefill(const tkv_desc *desc, int32_t batch, int32_t n_q_heads, const int32_t *seq_indptr, const int32_t *prefix_indptr,
                         int32_t target_cus, int32_t *items_out, int32_t capacity, int32_t *tile_rows_out, int32_t *n_slots_out,
                         int32_t *n_cut_out);
typedef struct tkv_prefill {
    int32_t tile_rows, n_items, n_slots, n_cut;   /* as tkv_plan_prefill gives them */
    const int32_t *items;                  /* device, 4-byte aligned */
} tkv_prefill;
/* Bytes of workspace that n_slots partial slots take; 0 on a bad argument or if there are none. */
size_t tkv_prefill_workspace_bytes(const tkv_desc *desc, int32_t n_slots, int32_t tile_rows);
/*
 * Causal attention of packed sequences (Sec. 3.2.3, "Prefill"): for new token i
 * of a sequence and query head h, which reads kv head h / R,
 *   out[i, h] = softmax_j(sm_scale * q[i, h] . k_j) v_j
 * over the sequence's prefix rows (fp16, as tkv_gather_dequant writes them) and
 * its new tokens' rows 0 .. i: a prompt, a chunk of one, or a single token.
 *   q            device bf16 or fp16 (q_type), K, V bf16 or fp16 (kv_type):
 *                bf16 queries go with either, fp16 ones with fp16.  16-byte
 *                aligned; token t, head h, channel c at t * stride + h * 128 +
 *                c with the tensor's own stride in elements (a multiple of 8,
 *                below 2^23): parts of a packed projection, or tensors of their own
 *   K_prefix,    device fp16 [n_prefix, n_kv_heads, 128], contiguous, 16-byte
 *   V_prefix     aligned; may be NULL if n_prefix = 0
 *   prefill      host struct, above; its items are for these lengths
 *   out          device bf16 or fp16 (out_type) [n_tokens, n_q_heads, 128],
 *                contiguous, 16-byte aligned, overlaps no input; rows that no
 *                item covers (behind the last sequence) stay as they were
 *   workspace    device, >= tkv_prefill_workspace_bytes(...), 16-byte aligned,
 *                needs no initialisation; calls that overlap in time need one each
 *   status       device i32, may be NULL: TKV_STATUS_BAD_ITEM
 * Products are exact and summed in 32 bits; weights are rounded to the values'
 * type, their sum is that of the rounded ones; those of fp16 values (all of a
 * prefix) that lie below 2^-23 of the row's largest are rounded to multiples of
 * 2^-33 of it or less; bf16 queries meet fp16 keys as
 * fp16 numbers with a power of two of their row (what lies 2^-24 below the
 * row's largest, or below 2^-144, rounds to the grid of the subnormals).
 * q . k (for bf16 queries over fp16 keys also sm_scale times the row's largest
 * |q|) must be finite in 32 bits, and sm_scale * q . k * log2 e below 2^26 in
 * magnitude, where the rounding of a row's reference still leaves its weights
 * in the range of fp16; a row that goes beyond is NaN or off.  256 times the sum
 * of |v| over the keys that a row sees must be finite in 32 bits.  A row of q that
 * holds NaN or infinities gives NaN and leaves the others alone; what
 * stands in keys and values that a token does not see does not reach it, an
 * infinite or NaN value that it sees makes that channel infinite or NaN.
 * A prefill with other lengths or heads than the call's gives what its items
 * say, or BAD_ITEM.  sm_scale > 0.  n_q_heads must be a multiple of n_kv_heads.
 * One launch on `stream`, a second one if n_cut > 0.
 */
int tkv_prefill_attention(const tkv_desc *desc, int32_t n_q_heads, const void *q, int64_t q_stride, int32_t q_type,
                          const void *K, int64_t k_stride, const void *V, int64_t v_stride, int32_t kv_type, int32_t n_tokens,
                          const void *K_prefix, const void *V_prefix, int32_t n_prefix, const tkv_prefill *prefill, float sm_scale,
                          void *out, int32_t out_type, void *workspace, size_t workspace_bytes, int32_t *status,
                          void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* C1: what calibration replays (host plan, device).                    */
/* ------------------------------------------------------------------ */
/*
 * The tokens at INT2 of every sequence, 32 a block in order of arrival, for
 * per-channel keys: blocks_out host i32[32*capacity], token numbers over the
 * whole of tag_bits (host, u8[seq_indptr[batch]]; other widths are passed over).
 * A sequence whose INT2 tokens are no multiple of 32 is TKV_ERR_INVALID_ARG
 * (tkv_route_residual first).  Returns the number of blocks or a negative status.
 */
int32_t tkv_plan_row_blocks(const uint8_t *tag_bits, const int32_t *seq_indptr, int32_t batch, int32_t *blocks_out, int32_t capacity);
/*
 * Keys and values as the cache would give them back: fp16 rows of what
 * tkv_quantize_append stores and tkv_gather_dequant reads, for the tokens that
 * tag_bits puts at INT2 or INT4; other tokens (width 0) are rounded to fp16.
 * (Calibration replays attention with the tokens of one tag at one width,
 * Sec. 3.1.3.)
 *   desc         n_kv_heads and int2_key_axis; the pools may be empty
 *   K, V         device bf16, 16-byte aligned, with a token stride each (in
 *                elements, a multiple of 8): [n_tokens, n_kv_heads, 128]
 *   tag_bits     device u8[n_tokens]: 0, 2 or 4; a token with another width is
 *                skipped (TKV_STATUS_TAG_MISMATCH)
 *   blocks       device i32[32*n_blocks] (tkv_plan_row_blocks), may be NULL if
 *                n_blocks = 0.  With TKV_KEYS_PER_CHANNEL the keys of INT2
 *                tokens are those of their block, and a key that no block names
 *                stays as it was; with TKV_KEYS_PER_TOKEN n_blocks must be 0.
 *                A block that names a token outside the call or not at INT2 is
 *                skipped (TKV_STATUS_BLOCK_PARTIAL); no token in two blocks
 *   K_out, V_out device fp16 [n_tokens, n_kv_heads, 128], contiguous, 16-byte
 *                aligned, overlapping no input
 *   status       device i32, may be NULL
 * Inputs at width 2 or 4 finite and at most 65504.  One launch.
 */
int tkv_quantize_rows(const tkv_desc *desc, const void *K, int64_t k_stride, const void *V, int64_t v_stride, const uint8_t *tag_bits,
                      int32_t n_tokens, const int32_t *blocks, int32_t n_blocks, void *K_out, void *V_out, int32_t *status,
                      void *stream /* hipStream_t */);
/*
 * out[b, h] = mean over the tokens of sequence b and the 128 channels of
 * (x - y)^2, in 64 bits, added up in the same order every time; 0 for a sequence
 * without tokens: the distortion of a replay (Sec. 3.1.3).
 *   x, y         device [n_tokens, n_heads, 128] of `type` (TKV_BF16, TKV_FP16 or
 *                TKV_FP32), contiguous, 16-byte aligned
 *   seq_indptr   device i32[batch+1], not falling, within [0, n_tokens]; a
 *                sequence of which that does not hold gives NaN, and what the
 *                others then give is not defined
 *   out          device f64 [batch, n_heads]
 *   workspace    device, >= tkv_distortion_workspace_bytes(...), 16-byte aligned,
 *                needs no initialisation; calls that overlap in time need one each
 * NaN and infinities stay in their sequence and head.  One launch, or two.
 */
size_t tkv_distortion_workspace_bytes(int32_t batch, int32_t n_tokens, int32_t n_heads);
int tkv_head_distortion(const void *x, const void *y, int32_t type, const int32_t *seq_indptr, int32_t batch, int32_t n_tokens,
                        int32_t n_heads, double *out, void *workspace, size_t workspace_bytes, void *stream /* hipStream_t */);

/* ------------------------------------------------------------------ */
/* Measurement aid (device).                                            */
/* ------------------------------------------------------------------ */
/*
 * Streams `bytes` (a multiple of 16) of the device buffer `buf` (16-byte
 * aligned) through the GPU with 128-bit non-temporal loads (the kind the
 * kernels use for the records of the cache) and discards them: the
 * read-bandwidth ceiling of the device for a scan such as the decode kernel's
 * pass over the pool.  For benchmarks that report a kernel against what the
 * memory system delivers as well as against the published peak; it computes
 * nothing of the method.  `sink` (device u32, may be NULL) is never written
 * in practice.  One launch on `stream`; TKV_ERR_INVALID_ARG on a null or
 * misaligned buffer.
 */
int tkv_probe_stream_read(const void *buf, size_t bytes, uint32_t *sink, void *stream /* hipStream_t */);
/*
 * Fetches the records that a decode plan reads, in the decode kernel's own
 * decomposition (Sec. 3.2.3, "Decode": one wavefront per (work item, kv head),
 * whole records, the next one requested when the current one has arrived) and
 * discards them: what the memory system delivers to that access pattern, with
 * none of the arithmetic.
 *   walk = 1  addresses come from the items and the device page tables exactly
 *             as in tkv_decode_split (same arguments, same meaning): the
 *             kernel's memory skeleton, start-up chain included;
 *   walk = 0  wavefront w of the n_items * n_kv_heads reads records w, w + W,
 *             ... of the whole pool, addresses computed; the page tables and
 *             items are not read (may be NULL).
 * sink as for tkv_probe_stream_read.  n_items = 0 or an empty pool is a no-op.
 */
int tkv_probe_decode_reads(const tkv_desc *desc, const void *pool, const int32_t *page_indptr,
                           const int32_t *page_ids, const int32_t *n_tok_int2, const int32_t *n_tok_int4,
                           const int32_t *items, int32_t n_items, int32_t batch, int32_t walk,
                           uint32_t *sink, void *stream /* hipStream_t */);
/*
 * Streams read_parts * unit_bytes out of `src` and writes write_parts *
 * unit_bytes into `dst` (device, 16-byte aligned, unit_bytes a multiple of 16)
 * with 128-bit accesses (ordinary loads, non-temporal stores: the fastest
 * combination): the ceiling of the device for a kernel that reads and
 * writes in that byte ratio.  Supported ratios: 4 : 1 (tkv_quantize_append reads
 * 512 B of bf16 per 96..160 B it writes), 1 : 4 (tkv_gather_dequant), 1 : 1.
 * What is written is a fold of what was read.  unit_bytes = 0 is a no-op.
 */
int tkv_probe_stream_mix(const void *src, void *dst, size_t unit_bytes, int32_t read_parts,
                         int32_t write_parts, void *stream /* hipStream_t */);

#ifdef __cplusplus
}
#endif
#endif /* TKV_H */
