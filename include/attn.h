/*
 * attn.h -- C ABI of the gfx950 fused multi-head attention forward.
 *
 * The operation is the attention kernel class that the paper names first
 * among the specialised LLM kernels (Introduction) and evaluates as one of
 * six kernels (Table 2: B, n_head, seq_len, d_head).  The paper gives no
 * formula; the definition is the standard one:
 *
 *     for every batch b, head h, query row i:
 *         J      = {0..S-1}                     causal == 0
 *                = {0..i}                       causal != 0 (diagonal included)
 *         s_j    = scale * sum_d q[i,d] k[j,d]
 *         lse_i  = ln sum_{j in J} exp(s_j)                 (natural log)
 *         O[i,:] = sum_{j in J} exp(s_j - lse_i) v[j,:]
 *
 * One fixed kernel per (D, dtype, causal) with a hand-set instruction
 * schedule -- the paper's framing of a fixed kernel whose schedule is tuned
 * for throughput (Sections 2.4 and 3.5) -- never visible through this ABI.
 */
#ifndef PAPER_2501_08071_ATTN_H
#define PAPER_2501_08071_ATTN_H

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of q, k and v.  o and lse are always fp32. */
typedef enum { ATTN_F16 = 0, ATTN_BF16 = 1 } attn_dtype_t;

typedef enum {
    ATTN_OK = 0,
    ATTN_ERR_NULL = -1,        /* a tensor that the call needs is NULL               */
    ATTN_ERR_SHAPE = -2,       /* B, H, S or D <= 0, or a tensor above 2^40 elements;
                                  on a paged cache: sizes out of the limits below    */
    ATTN_ERR_DTYPE = -3,       /* dtype is not an attn_dtype_t                       */
    ATTN_ERR_SCALE = -4,       /* scale is NaN or infinite                           */
    ATTN_ERR_UNSUPPORTED = -5, /* valid request with no kernel instance (D)          */
    ATTN_ERR_LAUNCH = -6,      /* the HIP runtime refused the launch                 */
    ATTN_ERR_ALIGN = -7,       /* a pointer is not 16-byte aligned (on a paged cache
                                  pointers to int, and lse: 4-byte)                  */
    ATTN_ERR_WORKSPACE = -8    /* attn_paged_fwd: the workspace is missing or small  */
} attn_status_t;

/*
 * Fused attention forward (the attention row of Table 2; definition above).
 *
 *   q, k, v  DEVICE pointers, [B,H,S,D] contiguous with D fastest, elements of
 *            type `dtype` (IEEE binary16 or bfloat16).  Read only.
 *   o        DEVICE pointer, [B,H,S,D] contiguous fp32.  Written.
 *   lse      DEVICE pointer, [B,H,S] fp32, natural-log logsumexp of the scaled,
 *            masked logits; may be NULL (then it is not written).
 *   B,H,S,D  batch, heads, sequence length (queries == keys), head dimension.
 *            Any S >= 1; D must be 32, 64 or 128.
 *   causal   0: every key visible; non-zero: key j visible to query i iff j <= i.
 *            Masked keys enter the second product with weight 0, so q, k and v must be
 *            finite everywhere: a non-finite row j of v spoils, next to the rows of O
 *            that see key j, the earlier rows of the same block of keys (attn_tile_keys of them; at D = 32 of the
 *            same tile of rows; 0 * Inf).
 *   scale    multiplies q.k before the softmax; any finite value.
 *   dtype    attn_dtype_t of q, k, v.
 *   stream   hipStream_t to enqueue on (NULL = the default stream).
 *
 * Ownership: the caller owns every buffer; the library allocates nothing and
 * never synchronises.  Its only state is one flag per device and kernel
 * instance: that the runtime has been told the instance's LDS size (set once,
 * atomically; calls from several host threads are safe).  The call is asynchronous: outputs are valid
 * once `stream` has been synchronised.  o and lse must not alias q, k or v.
 * All pointers must be 16-byte aligned.  Runs repeat bit for bit.  The last bits of a row may differ between
 * problems: which kernel serves one, and in how many parts it adds up a row's keys, depends on B, H and S
 * (attn_kernel_name).
 *
 * Errors: returns an attn_status_t and never throws or aborts.  Every argument
 * is checked before the first HIP call, so bad arguments are reported on a
 * machine without a GPU too.
 */
int attn_fwd(const void *q, const void *k, const void *v, float *o, float *lse,
             int B, int H, int S, int D, int causal, float scale, int dtype, void *stream);

/*
 * The same operation with O written in the type of q, k and v (Table 2 gives the kernel's inputs as
 * fp16 tensors; a layer that feeds the next one in half precision wants O that way), rounded to
 * nearest even from the fp32 result (so its error is that of attn_fwd plus one rounding of O: at most
 * 2^-8 |O| for bfloat16, 2^-11 |O| for binary16).  `o` is [B,H,S,D] contiguous in `dtype`; lse stays fp32.  Every
 * other argument, the ownership and error rules are those of attn_fwd; both share one kernel.
 */
int attn_fwd_o16(const void *q, const void *k, const void *v, void *o, float *lse,
                 int B, int H, int S, int D, int causal, float scale, int dtype, void *stream);

/* 1 if attn_fwd has a kernel instance for this request, else 0 (no HIP call). */
int attn_supported(int S, int D, int dtype, int causal);

/* Static, NUL-terminated description of an attn_status_t (never NULL). */
const char *attn_status_str(int status);

/*
 * Name of the kernel attn_fwd launches for this very problem (the symbol a
 * profiler reports; it depends on B and H because small problems take the
 * instance with fewer query rows, see attn_workgroup_rows), or NULL if
 * unsupported.  A string constant: no HIP call, safe from any thread.
 */
const char *attn_kernel_name(int B, int H, int S, int D, int dtype, int causal);

/*
 * Query rows per tile and keys per inner-loop block of the kernel for problems that fill the chip
 * (0 if unsupported).  For harnesses that pick tile-edge rows to check.
 */
int attn_tile_rows(int D, int dtype, int causal);
int attn_tile_keys(int D, int dtype, int causal);

/*
 * attn_tile_rows ("..., 8>" in the kernel's name), or half of it ("..., 4>") when this very problem has so few tiles of that many
 * rows that half of the chip would be idle, or when they would fill it unevenly.  0 if unsupported.
 */
int attn_launch_rows(int B, int H, int S, int D, int dtype, int causal);

/*
 * Query rows a workgroup of attn_kernel_name's kernel owns for this very problem: attn_launch_rows, but 32 or 64 (32 times the last
 * template argument but one) in "attn_fwd_halves_stream_kernel", whose wavefronts each stream keys of their own.  Every workgroup
 * reads all the keys its rows see.  0 if unsupported.  For harnesses that pick rows at the edges or count what is read.
 */
int attn_workgroup_rows(int B, int H, int S, int D, int dtype, int causal);

/*
 * ---- Attention over a paged key/value cache ------------------------------------------------------
 *
 * The serving form of the operation: a batch of B sequences, each with some new tokens (one in a decode step, a few drafted ones,
 * a piece of a prompt), whose keys and values lie in pages of page_size tokens.  The new tokens of all sequences are rows of one
 * array of T tokens, sequence after sequence.  Every length lies on the device, so a step can be captured in a graph.
 *
 *   k, v         DEVICE pointers, pages [n_pages][Hk][page_size][D], elements of `dtype`.  A page is contiguous; consecutive pages
 *                begin page_stride elements apart (Hk * page_size * D or more, a multiple of 8: k and v may be interleaved).
 *   page_table   DEVICE pointer, [B] rows of `width` page numbers, table_stride elements apart: key j of sequence b lies in page
 *                page_table[b][j / page_size], slot j % page_size.  What entries past a sequence's last key hold does not matter.
 *   cu_q         DEVICE pointer, [B + 1]: the new tokens of sequence b are rows cu_q[b] .. cu_q[b + 1] - 1.  May be none.
 *   kv_len       DEVICE pointer, [B]: keys of the sequence in its pages, the new tokens' among them.
 *   page_size    a power of two.      D: 32, 64 or 128.      Hk: key heads.
 *
 * Limits: B <= 2^20, T <= 2^22, T times the larger of Hq and Hk <= 2^28, B * Hk <= 2^22, width * page_size <= 2^30 keys a sequence,
 * page_stride * n_pages <= 2^40 elements; with T and B not 0, n_pages at least 1.
 *
 * Values on the device cannot be checked by the host.  Whatever they are, nothing outside the buffers is touched: a page number
 * outside 0 .. n_pages - 1 is a page of absent keys, lengths are cut to the table's width, rows to T.
 */
typedef struct {
    void *k, *v;
    long long page_stride;
    int n_pages, page_size, Hk, D, dtype;
    const int *page_table;
    int table_stride, width;
    const int *cu_q, *kv_len;
    int B, T;
} attn_paged_t;

/*
 * Appends the new tokens' keys and values to their pages, and rotates queries and keys by their positions on the way.
 *
 * Token i of the n new ones of sequence b becomes key p = kv_len[b] - n + i (kv_len is the length after this call).  Its angles are
 * row p + pos_offset of cos and sin (clamped to the rows there are; pos_offset: the length of a shared prefix, else 0).  In 32 bits,
 * rounded once: a pair (x, y) becomes (x cos - y sin, y cos + x sin).
 *
 *   q, k, v      DEVICE pointers, T tokens of Hq, Hk and Hk heads of D elements; tokens q_stride, k_stride, v_stride elements
 *                apart (multiples of 8), so that the three may be parts of one projection's rows.  q may be NULL with Hq 0.
 *   q_out        DEVICE pointer, [T][Hq][D] contiguous: the rotated queries.  May be q where q is contiguous.
 *   cos, sin     DEVICE pointers, [n_angles][rot / 2] fp32; NULL with rot 0: nothing is rotated.
 *   rot          how many of a head's D elements are rotated: 0 or a multiple of 16 up to D.
 *   interleaved  0: pairs (j, j + rot / 2); non-zero: pairs (2 j, 2 j + 1).
 *
 * A token whose page does not exist (above), or that no sequence owns, is not stored.  Two tokens never share a slot of a page.
 * Ownership, asynchrony, errors: as attn_fwd.
 */
int attn_kv_append(const attn_paged_t *cache, const void *q, const void *k, const void *v, long long q_stride,
                   long long k_stride, long long v_stride, void *q_out, const float *cos, const float *sin, int rot,
                   int interleaved, int n_angles, int pos_offset, int Hq, void *stream);

/*
 * Attention of the new tokens over the cache.  Query head h reads key head h / (Hq / Hk).  Token i of the n new ones of sequence b
 * sees, in this order, the prefix_len keys of the shared prefix and the first kv_len[b] - n + i + 1 keys of the sequence's own:
 *
 *     s_j = scale * q . k_j,   lse = ln sum_j exp(s_j),   o = sum_j exp(s_j - lse) v_j        (no key: o = 0, lse = -inf)
 *
 *   q            DEVICE pointer, T tokens of Hq heads of D elements, tokens q_stride elements apart (a multiple of 8).
 *   o            DEVICE pointer, [T][Hq][D] contiguous in `dtype`.  Written.  Not q.
 *   lse          DEVICE pointer, [T][Hq] fp32, or NULL.
 *   prefix_table DEVICE pointer, the pages of a prefix that all sequences share, or NULL with prefix_len 0.  Its keys are read once
 *                for all of the batch's rows that fit a tile, not once a sequence.
 *   max_q        the most new tokens any sequence has; rows past it, and rows that no sequence owns, are not written.  It chooses the kernel:
 *                a number that is too large costs speed (a decode step told of T new tokens a sequence may take twice as long).
 *   max_kv       the most keys of its own any sequence has: only a hint of how to share out the work.
 *   workspace    DEVICE pointer of attn_paged_workspace(...) bytes (16-byte aligned) that no other call uses meanwhile; NULL where that is 0.
 *
 * Logits, statistics and sums are fp32.  Two roundings to `dtype`: of the weights exp(s_j - reference) before they meet the values (their sum is taken
 * before it), and of o.  With u = 2^-8 for bfloat16 and 2^-11 for binary16 they move o by up to u sum_j p_j |v_j| + u |o|, p_j the share of
 * key j (binary16 weights below 2^-14 also lose up to 2^-25 each); against 64 bits the error is measured at 1.2 to 1.4 times that of an evaluation
 * in fp32 that is rounded once.
 *
 * Values that only some rows of a sequence's new tokens see must be finite for the others too (a hidden one has weight 0,
 * and 0 * Inf is not 0).  Keys that a row does not see, and slots past kv_len, may hold anything.  Runs repeat bit for bit.  Else as attn_fwd.
 */
int attn_paged_fwd(const attn_paged_t *cache, const void *q, long long q_stride, void *o, float *lse,
                   const int *prefix_table, int prefix_len, int Hq, int max_q, int max_kv, float scale,
                   void *workspace, long long workspace_bytes, void *stream);

/* Bytes of workspace for these sizes (0: none; -1: sizes that attn_paged_fwd refuses).  No HIP call. */
long long attn_paged_workspace(int B, int T, int Hq, int Hk, int D, int max_q, int max_kv, int prefix_len);

#ifdef __cplusplus
}
#endif
#endif
