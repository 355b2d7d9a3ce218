/*
 * dq.h -- C ABI of the D-Quant hot path on MI355X (gfx950).
 *
 * D-Quant (arXiv 2609.19880) stores each token's key or value vector as a
 * fixed-size record: Hadamard rotation, (keys) windowed channel-mean removal,
 * a token-wise min-max affine grid with M levels, a rate-constrained
 * assignment ("drift") that makes the entropy-coded length fit the record,
 * and rANS with a static table derived from standard-normal CDF mass
 * (Sec. 4, Alg. 1).  Decode attention reads the records at fixed stride,
 * rANS-decodes them (Alg. 2) and attends with the affine folded into the
 * contractions (App. A, Eq. fold-key / fold-value).
 *
 * One stream is one (token, KV head): n = head_dim values.  A record of C
 * bytes is laid out as
 *     [scale fp16 LE][offset fp16 LE][rANS state u32 LE][renorm bytes, in the
 *     order the decoder reads them][zero padding]
 * so its rANS budget (Eq. budget) is B = 8 (C - 4) - 32 bits.  The rANS state
 * lives in [2^21, 2^29) and is renormalized one byte at a time.
 *
 * Conventions for every call:
 *  - Device pointers are plain device addresses on the device that was current
 *    when the tables were built; the caller owns every device buffer.
 *  - Work is enqueued on `stream` (a hipStream_t, NULL = the null stream) and
 *    is asynchronous: no call synchronizes, and device-side errors are reported
 *    through the caller's `status` word (see DQ_STATUS_*), readable once the
 *    stream has finished.
 *  - Host-side validation failures return an error code before anything is
 *    enqueued.  No C++ exception crosses this interface.
 *  - bf16 and fp16 values are passed as their 16-bit patterns.
 */
#ifndef DQ_H
#define DQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
#define DQ_OK 0
#define DQ_ERR_INVALID_ARG 1 /* a size, pointer or layout is out of range    */
#define DQ_ERR_INFEASIBLE 2  /* n * min cost exceeds the budget (Tab. 2 "--") */
#define DQ_ERR_HIP 3         /* a HIP runtime call or a launch failed          */
#define DQ_ERR_WORKSPACE 4   /* the workspace is missing or too small          */

/* Bits OR-ed into the caller's device status word. */
#define DQ_STATUS_RANGE 1u    /* encode: non-finite input, or scale/offset/mean overflowed fp16 */
#define DQ_STATUS_OVERFLOW 2u /* encode: a stream could not be fitted into its record (written as
                                 zeros); the coded-length bound makes this unreachable for n <= 1024 */
#define DQ_STATUS_CORRUPT 4u  /* decode: a record did not end in state 2^21 inside its C bytes  */
#define DQ_STATUS_WINDOW 8u   /* residual window: append to a full ring, or commit more than it holds */
#define DQ_STATUS_PAGE 16u    /* paged layout: a block-table entry outside the page pool (skipped)     */

/* Fixed parameters of the format. */
#define DQ_MEAN_WINDOW 128 /* tokens per key-mean window (windows start at token 0) */
#define DQ_MAX_LEVELS 64

/*
 * Coding parameters of one tensor (keys or values).  The per-token bit budget
 * is given as the record size: bits per element = 8 * record_bytes / head_dim
 * (Sec. 4.2 Eq. budget; Sec. 4.4 lets keys and values differ).
 */
typedef struct dq_config {
    int32_t head_dim;       /* n: values per stream, a power of 2 in 64..1024;
                               encode takes n <= 256, decode attention n = 128 */
    int32_t levels;         /* M: quantization levels, 2..64 (Eq. affine_token) */
    int32_t precision_bits; /* p: rANS precision, 8..12 (Eq. rans)              */
    int32_t record_bytes;   /* C: record size in bytes, 9..2n+8                 */
    double alpha;           /* sharpening exponent, >= 1 (Sec. 4.4; paper 1.4)  */
    int32_t prerotated;     /* 0: the library rotates every head's vector with
                               the Hadamard matrix (Sec. 4.2; keys need this,
                               RoPE does not commute with it).  1: the tensor
                               arrives already in the rotated basis, as values
                               do when the rotation is folded into the
                               projection weights offline (Sec. 4.2): no
                               online rotation, see dq_decode_attention.     */
} dq_config;

typedef struct dq_table_info {
    int32_t record_bytes;   /* C                                                 */
    int32_t feasible;       /* 1 if n * min_cost_q16 <= budget_q16               */
    int32_t cheapest;       /* lowest-index symbol of minimum cost               */
    int32_t reserved;
    int64_t budget_q16;     /* B = (8 (C - 4) - 32) * 2^16                       */
    int64_t min_cost_q16;   /* n * min_m R_m                                     */
    double expected_max;    /* a_n = E[max of n standard normals]                */
} dq_table_info;

/* Opaque coding tables: host copy plus a device copy, immutable once built. */
typedef struct dq_tables dq_tables;

/*
 * Builds the entropy model on the host only (no GPU needed):
 * level probabilities from normal CDF mass on the grid [-a_n, a_n] (the
 * order-statistics model of normal samples, Sec. 4.2), sharpened p^alpha
 * (Sec. 4.4), apportioned to integers summing to 2^p (Eq. rans), Q16 costs R_m = round(2^16 (p - log2 f_m))
 * (Alg. 1), the lambda grid 2^(k/512) as fp32, and the feasibility test.
 * Output arrays may be NULL; sizes: freq, cum, cost_q16: levels entries;
 * sym_of_z: 2^p entries; lambda512: 512 entries.
 * Returns DQ_OK, DQ_ERR_INVALID_ARG, or DQ_ERR_INFEASIBLE (info is filled).
 */
int dq_compute_tables(const dq_config* cfg, dq_table_info* info, int32_t* freq,
                      int32_t* cum, int32_t* cost_q16, uint8_t* sym_of_z,
                      float* lambda512);

/*
 * Same tables, copied to the current HIP device.  On DQ_OK *out owns host and
 * device memory until dq_free_tables.  An infeasible configuration returns
 * DQ_ERR_INFEASIBLE with *out = NULL and info filled.
 */
int dq_build_tables(const dq_config* cfg, dq_tables** out, dq_table_info* info);
void dq_free_tables(dq_tables* tables);

/*
 * Encodes new tokens into records (Fig. 1; Alg. 1 and the rANS coder).
 *   kv:      bf16 [batch][tokens][kv_heads][head_dim] at element strides
 *            (stride_b, stride_t, stride_h); channels contiguous.  Token i of
 *            the input becomes cache token t0 + i.
 *   records: u8 [batch][kv_heads][t_cap][C]; writes tokens [t0, t0 + n_new).
 *   mean_q, mean_scale: keys only -- int8 [batch][kv_heads][t_cap/128][head_dim]
 *            and fp16 [batch][kv_heads][t_cap/128]: the per-window INT8
 *            channel mean of the rotated keys, which is removed before
 *            quantization (Sec. 4.2).  Both NULL for values (no mean removal);
 *            with them, t0 and n_new must be multiples of 128.
 *   status:  device u32, may be NULL; DQ_STATUS_RANGE / DQ_STATUS_OVERFLOW.
 * Every stream is rotated with the unnormalized Sylvester Hadamard matrix,
 * unless the tables were built with prerotated = 1 (then the input is coded
 * as it is).  The records are bit-identical to the reference definition of
 * the format.
 * Requires head_dim <= 256, 1 <= kv_heads <= 65535, 0 <= batch <= 65535,
 * t0 >= 0, n_new >= 0, t0 + n_new <= t_cap and non-negative strides; with the
 * mean buffers also t0, n_new and t_cap multiples of 128.  Returns DQ_OK
 * (nothing is launched when batch or n_new is 0), DQ_ERR_INVALID_ARG, or
 * DQ_ERR_HIP if a launch fails.
 */
int dq_encode_kv(const dq_tables* tables, const uint16_t* kv, int64_t stride_b,
                 int64_t stride_t, int64_t stride_h, int32_t batch,
                 int32_t kv_heads, int32_t t0, int32_t n_new, int32_t t_cap,
                 uint8_t* records, int8_t* mean_q, uint16_t* mean_scale,
                 uint32_t* status, void* stream);

/* Workspace bytes dq_decode_attention needs for these sizes. */
size_t dq_decode_workspace_bytes(int32_t batch, int32_t q_heads, int32_t kv_heads,
                                 int32_t t_cap, int32_t head_dim);

/*
 * One decode step of attention over the compressed cache (Sec. 4.5 decoding,
 * App. A): logits softmax_scale * q . k_hat over the first seq_lens[b] tokens,
 * output sum_t a_t v_hat_t, with query head i reading KV head
 * i / (q_heads / kv_heads).  q and out are in the basis the caller gives keys
 * and values in: with online rotation (prerotated = 0) that is the original
 * basis (the query is rotated and the output rotated back inside); with
 * prerotated keys the query must come in the keys' basis, and with
 * prerotated values the output stays in the values' basis (the caller's
 * output projection absorbs the rotation).  The raw tokens of a residual
 * window are taken in the same bases.
 *   q:        bf16 [batch][q_heads][head_dim]
 *   k_records, v_records: u8 [batch][kv_heads][t_cap][C_k or C_v]
 *   k_mean_q, k_mean_scale: as written by dq_encode_kv for the keys
 *   seq_lens: device int32 [batch], each in [0, t_cap]
 *   out:      fp32 [batch][q_heads][head_dim] (a sequence of length 0 gives 0)
 *   workspace: device memory of dq_decode_workspace_bytes(...) bytes
 *   status:   device u32, may be NULL; DQ_STATUS_CORRUPT for malformed records
 * Requires head_dim = 128 for both tables, record lengths C_k and C_v that
 * are multiples of 4 in [12, 64], t_cap a positive multiple of 128,
 * 1 <= batch <= 65535, 1 <= kv_heads <= 65535, q_heads a multiple of kv_heads
 * with q_heads / kv_heads <= 8.  Returns DQ_OK, DQ_ERR_INVALID_ARG (nothing
 * launched), DQ_ERR_WORKSPACE (workspace missing or too small) or DQ_ERR_HIP.
 */
int dq_decode_attention(const dq_tables* k_tables, const dq_tables* v_tables,
                        const uint16_t* q, int32_t batch, int32_t q_heads,
                        int32_t kv_heads, const uint8_t* k_records,
                        const int8_t* k_mean_q, const uint16_t* k_mean_scale,
                        const uint8_t* v_records, const int32_t* seq_lens,
                        int32_t t_cap, float softmax_scale, float* out,
                        void* workspace, size_t workspace_bytes,
                        uint32_t* status, void* stream);

/*
 * dq_decode_attention without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, serving loops and
 * harnesses that forbid hipMalloc).  The split-K workspace lives in a static
 * device array of DQ_NO_ALLOC_SCRATCH_BYTES inside the library, one per
 * device, held until the process ends; its address is looked up on the first
 * call on each device (with that device current).  Arguments, layouts,
 * results and status bits are those of dq_decode_attention, and the same
 * kernels run.  No call allocates or frees memory.
 * Every call on a device shares that device's array, which keeps the last
 * call's contents: calls that overlap on one device (different streams, or
 * different host threads) race and give undefined results; serialize them.
 * The workspace this needs is 256 + 520 batch q_heads (chunks + 4) bytes,
 * chunks being the context split chosen from (batch, kv_heads, t_cap) and the
 * CU count (2 for 16 x 32768 tokens x 8 KV heads on 256 CUs: 1.6 MB).
 * Returns DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE when the sizes need more
 * than the array holds (dq_last_error says how much), or DQ_ERR_HIP.
 */
#define DQ_NO_ALLOC_SCRATCH_BYTES (8u << 20)
int dq_decode_attention_no_alloc(const dq_tables* k_tables, const dq_tables* v_tables,
                                 const uint16_t* q, int32_t batch, int32_t q_heads,
                                 int32_t kv_heads, const uint8_t* k_records,
                                 const int8_t* k_mean_q, const uint16_t* k_mean_scale,
                                 const uint8_t* v_records, const int32_t* seq_lens,
                                 int32_t t_cap, float softmax_scale, float* out,
                                 uint32_t* status, void* stream);

/*
 * The two halves of dq_decode_attention, for callers that merge partial
 * results themselves (e.g. context split over devices) or time them apart.
 * _partial writes one (max, sum, accumulator) triple per (sequence, query
 * head, context chunk) into the workspace (online-softmax state over the
 * chunk); _merge combines the chunks by log-sum-exp, undoes the value
 * rotation and writes `out`.  Arguments mean what they mean above; the chunk
 * size is chosen from (batch, kv_heads, t_cap) and the device's CU count and
 * recorded in the workspace, so both halves must be called with the same
 * sizes and workspace, on the same device and stream.
 */
int dq_decode_attention_partial(const dq_tables* k_tables, const dq_tables* v_tables,
                                const uint16_t* q, int32_t batch, int32_t q_heads,
                                int32_t kv_heads, const uint8_t* k_records,
                                const int8_t* k_mean_q, const uint16_t* k_mean_scale,
                                const uint8_t* v_records, const int32_t* seq_lens,
                                int32_t t_cap, float softmax_scale, void* workspace,
                                size_t workspace_bytes, uint32_t* status, void* stream);
int dq_decode_attention_merge(int32_t batch, int32_t q_heads, int32_t kv_heads,
                              const int32_t* seq_lens, int32_t t_cap, const void* workspace,
                              size_t workspace_bytes, float* out, void* stream);

/*
 * Residual window (Sec. 5.1 keeps the most recent tokens in BF16).  The raw
 * keys and values of a sequence's newest tokens live in a ring:
 *   res_k, res_v: bf16 [batch][kv_heads][r_cap][head_dim], 16-byte aligned,
 *            r_cap <= 256; residual token i of sequence b sits in slot
 *            (seq_lens[b] + i) mod r_cap, in the original basis (no
 *            rotation, no mean removal).
 *   seq_lens: device int32 [batch], the compressed tokens of each sequence;
 *   res_lens: device int32 [batch], its residual tokens (<= r_cap).
 * With r_cap a multiple of 128 and seq_lens[b] a multiple of 128, the oldest
 * 128 residual tokens are the contiguous slots [seq_lens[b] mod r_cap, + 128):
 * encode them with dq_encode_kv at t0 = seq_lens[b] (element strides
 * r_cap * head_dim between heads and head_dim between tokens), then call
 * dq_residual_commit(..., 128).
 *
 * dq_decode_attention_residual writes the residual window's softmax partial
 * into the workspace: call it after dq_decode_attention_partial and before
 * dq_decode_attention_merge, with the same sizes and workspace; the merge then
 * attends over the compressed tokens and the residual tokens together
 * (a sequence with neither gives 0).  head_dim is 128; q_heads / kv_heads <= 8;
 * q, res_k and res_v 16-byte aligned.
 * Returns DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 */
int dq_decode_attention_residual(const uint16_t* q, int32_t batch, int32_t q_heads,
                                 int32_t kv_heads, const uint16_t* res_k,
                                 const uint16_t* res_v, const int32_t* seq_lens,
                                 const int32_t* res_lens, int32_t r_cap, int32_t t_cap,
                                 float softmax_scale, void* workspace,
                                 size_t workspace_bytes, void* stream);

/*
 * The residual window and the merge in one launch (Sec. 5.1, Alg. 2): after
 * dq_decode_attention_partial (or any other _partial call) with the same
 * sizes and workspace, writes `out` as dq_decode_attention_residual followed
 * by dq_decode_attention_merge would (equal up to fp32 rounding order), one
 * kernel instead of two.  The workspace is read, not written, so the
 * residual slots it holds for the two-call form are ignored.  Arguments as
 * for the two calls; q 16-byte aligned (as for dq_decode_attention_residual).
 * Returns DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 */
int dq_decode_attention_merge_residual(const uint16_t* q, int32_t batch, int32_t q_heads,
                                       int32_t kv_heads, const uint16_t* res_k,
                                       const uint16_t* res_v, const int32_t* seq_lens,
                                       const int32_t* res_lens, int32_t r_cap, int32_t t_cap,
                                       float softmax_scale, const void* workspace,
                                       size_t workspace_bytes, float* out, void* stream);

/*
 * Appends one token per sequence to its ring: k_new, v_new bf16
 * [batch][kv_heads][head_dim] go to slot (seq_lens[b] + res_lens[b]) mod
 * r_cap, and res_lens[b] grows by one.  A full ring is left unchanged and
 * sets DQ_STATUS_WINDOW.  Returns DQ_OK, DQ_ERR_INVALID_ARG or DQ_ERR_HIP.
 */
int dq_residual_append(const uint16_t* k_new, const uint16_t* v_new, int32_t batch,
                       int32_t kv_heads, int32_t head_dim, uint16_t* res_k, uint16_t* res_v,
                       const int32_t* seq_lens, int32_t* res_lens, int32_t r_cap,
                       uint32_t* status, void* stream);

/*
 * The oldest n residual tokens of every sequence have been encoded:
 * seq_lens[b] += n, res_lens[b] -= n.  A sequence holding fewer than n is
 * left unchanged and sets DQ_STATUS_WINDOW.
 */
int dq_residual_commit(int32_t* seq_lens, int32_t* res_lens, int32_t batch, int32_t n,
                       uint32_t* status, void* stream);

/*
 * Paged layout, for serving engines that allocate the cache in pages.  The
 * records and key means of every sequence live in fixed-size pages of a pool:
 *   record pools:    u8 [num_pages][kv_heads][page_tokens][C]
 *   mean_q pool:     int8 [num_pages][kv_heads][page_tokens/128][head_dim]
 *   mean_scale pool: fp16 [num_pages][kv_heads][page_tokens/128]
 *   block_table:     device int32 [batch][max_pages]; logical page i of
 *                    sequence b (tokens [i page_tokens, (i+1) page_tokens)) is
 *                    pool page block_table[b * max_pages + i].
 * page_tokens is a power of two in [128, 2^20]; the logical capacity t_cap =
 * max_pages * page_tokens takes the place of t_cap above (workspace size,
 * the merge).  Otherwise the calls mean what their contiguous forms mean.  A
 * block-table entry outside [0, num_pages) sets DQ_STATUS_PAGE: the encoder
 * writes nothing through it, the attention reads page 0 in its place.
 */
int dq_encode_kv_paged(const dq_tables* tables, const uint16_t* kv, int64_t stride_b,
                       int64_t stride_t, int64_t stride_h, int32_t batch, int32_t kv_heads,
                       int32_t t0, int32_t n_new, const int32_t* block_table,
                       int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                       uint8_t* record_pool, int8_t* mean_q_pool, uint16_t* mean_scale_pool,
                       uint32_t* status, void* stream);
int dq_decode_attention_paged_partial(const dq_tables* k_tables, const dq_tables* v_tables,
                                      const uint16_t* q, int32_t batch, int32_t q_heads,
                                      int32_t kv_heads, const uint8_t* k_pool,
                                      const int8_t* mean_q_pool, const uint16_t* mean_scale_pool,
                                      const uint8_t* v_pool, const int32_t* block_table,
                                      int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                                      const int32_t* seq_lens, float softmax_scale,
                                      void* workspace, size_t workspace_bytes, uint32_t* status,
                                      void* stream);

/*
 * Per-token streams (Sec. 4.1, Sec. 4.5 "Decoding", Sec. 5.1): the paper's
 * default grouping, one stream of n = 128 kv_heads values per token spanning
 * every KV head (e.g. 1024 values for 8 heads, with 331 + 4 and 231 + 4 byte
 * records), instead of one stream per (token, KV head).  The stream takes the
 * heads in order, each head rotated on its own and, for keys, minus its own
 * window mean (the means are per head exactly as above); one (s, o) header
 * serves the whole token.  Tables are built with head_dim = n = 128 kv_heads.
 *
 * dq_token_record_stride: bytes of one token's record slot S, C rounded up to
 *   a multiple of 16 (the pad bytes are written as zeros); 0 for an invalid
 *   table.
 * Record buffer: u8 [batch][t_cap / 64][S / 8][64][8], 16-byte aligned: per
 *   64-token tile, the 8-byte chunks of the 64 records with the chunk index
 *   outermost (byte k of token t in tile t / 64 at ((k / 8) 64 + t % 64) 8 +
 *   k % 8), so that the 64 tokens' chunk k / 8 are 512 contiguous bytes.
 * dq_encode_kv_token: as dq_encode_kv with kv_heads in {1, 2, 4, 8} and
 *   head_dim 128; writes the record buffer above.
 * dq_decode_attention_token_partial: one decode step over those records
 *   (rANS-decoded once per token and consumed one KV head at a time), into the
 *   workspace of dq_decode_workspace_bytes; finish with
 *   dq_decode_attention_merge (and optionally add a residual window with
 *   dq_decode_attention_residual before it).  q_heads / kv_heads <= 8;
 *   k_mean_q / k_mean_scale as for dq_decode_attention.  Corrupt records set
 *   DQ_STATUS_CORRUPT.
 * Return DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 */
int32_t dq_token_record_stride(const dq_tables* tables);
int dq_encode_kv_token(const dq_tables* tables, const uint16_t* kv, int64_t stride_b,
                       int64_t stride_t, int64_t stride_h, int32_t batch, int32_t kv_heads,
                       int32_t t0, int32_t n_new, int32_t t_cap, uint8_t* records,
                       int8_t* mean_q, uint16_t* mean_scale, uint32_t* status, void* stream);
int dq_decode_attention_token_partial(const dq_tables* k_tables, const dq_tables* v_tables,
                                      const uint16_t* q, int32_t batch, int32_t q_heads,
                                      int32_t kv_heads, const uint8_t* k_records,
                                      const int8_t* k_mean_q, const uint16_t* k_mean_scale,
                                      const uint8_t* v_records, const int32_t* seq_lens,
                                      int32_t t_cap, float softmax_scale, void* workspace,
                                      size_t workspace_bytes, uint32_t* status, void* stream);

/*
 * Per-token records in pool pages (the paged layout above, Sec. 4.1's fixed
 * stride kept within a page): a pool page holds the records of page_tokens
 * tokens in the tile layout of the record buffer, so the record pool is
 * u8 [num_pages][page_tokens / 64][S / 8][64][8] and token t of sequence b is
 * row t mod page_tokens of pool page block_table[b * max_pages + t /
 * page_tokens].  Key-mean pools, the block table, page_tokens, the logical
 * capacity and DQ_STATUS_PAGE are as for dq_encode_kv_paged and
 * dq_decode_attention_paged_partial; otherwise the calls mean what
 * dq_encode_kv_token and dq_decode_attention_token_partial mean.
 */
int dq_encode_kv_token_paged(const dq_tables* tables, const uint16_t* kv, int64_t stride_b,
                             int64_t stride_t, int64_t stride_h, int32_t batch, int32_t kv_heads,
                             int32_t t0, int32_t n_new, const int32_t* block_table,
                             int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                             uint8_t* record_pool, int8_t* mean_q_pool, uint16_t* mean_scale_pool,
                             uint32_t* status, void* stream);
int dq_decode_attention_token_paged_partial(const dq_tables* k_tables, const dq_tables* v_tables,
                                            const uint16_t* q, int32_t batch, int32_t q_heads,
                                            int32_t kv_heads, const uint8_t* k_pool,
                                            const int8_t* mean_q_pool, const uint16_t* mean_scale_pool,
                                            const uint8_t* v_pool, const int32_t* block_table,
                                            int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                                            const int32_t* seq_lens, float softmax_scale,
                                            void* workspace, size_t workspace_bytes, uint32_t* status,
                                            void* stream);

/*
 * Comparator: fixed-width coding at matched storage (App. B).  The same
 * preprocessing as the D-Quant encoder (rotation, key window means, min-max
 * grid, least-squares refit, fp16 s and o), symbols by nearest-level rounding,
 * b = floor(8 (record_bytes - 4) / head_dim) bits each (M = 2^b levels),
 * packed least-significant bit first after the 4-byte header of a record of
 * the same size.  With 36-byte records and head_dim 128 that is 128 two-bit
 * codes sharing one fp16 scale and one fp16 offset: 2.25 bits per value, the
 * 2-bit example of Sec. 3.
 *
 * dq_fixed_bits: b for (head_dim, record_bytes), 0 if no whole bit fits or
 *   more than 8 would.
 * dq_encode_kv_fixed: as dq_encode_kv without tables; head_dim 64, 128 or 256.
 * dq_decode_attention_fixed_partial: one decode step over 36-byte fixed-width
 *   records (head_dim 128, b = 2), same layouts, workspace and merge as
 *   dq_decode_attention_partial; q_heads / kv_heads <= 4.
 * Return DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 */
int32_t dq_fixed_bits(int32_t head_dim, int32_t record_bytes);
int dq_encode_kv_fixed(int32_t head_dim, int32_t record_bytes, const uint16_t* kv, int64_t stride_b,
                       int64_t stride_t, int64_t stride_h, int32_t batch, int32_t kv_heads, int32_t t0,
                       int32_t n_new, int32_t t_cap, uint8_t* records, int8_t* mean_q,
                       uint16_t* mean_scale, uint32_t* status, void* stream);
int dq_decode_attention_fixed_partial(const uint16_t* q, int32_t batch, int32_t q_heads, int32_t kv_heads,
                                      const uint8_t* k_records, const int8_t* k_mean_q,
                                      const uint16_t* k_mean_scale, const uint8_t* v_records,
                                      const int32_t* seq_lens, int32_t t_cap, float softmax_scale,
                                      void* workspace, size_t workspace_bytes, uint32_t* status,
                                      void* stream);

/*
 * Comparator: the same decode step over an uncompressed BF16 cache.
 *   k, v: bf16 [batch][kv_heads][t_cap][head_dim], 16-byte aligned, original
 *         basis; the first seq_lens[b] tokens of sequence b are attended.
 * Writes split-K partials into the workspace (same size rule as above);
 * finish with dq_decode_attention_merge, with the same sizes and workspace.
 * head_dim is 128; t_cap a positive multiple of 128; q_heads / kv_heads <= 8.
 * Returns DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 */
int dq_bf16_decode_attention_partial(const uint16_t* q, int32_t batch, int32_t q_heads,
                                     int32_t kv_heads, const uint16_t* k, const uint16_t* v,
                                     const int32_t* seq_lens, int32_t t_cap,
                                     float softmax_scale, void* workspace,
                                     size_t workspace_bytes, void* stream);

/*
 * The 8-bit cache: between the records and the raw BF16 window, for layers or
 * requests that want the shortest step at half the bytes of BF16.  A block is
 * DQ_Q8_BLOCK = 32 consecutive tokens of one (sequence, KV head): the codes of
 * its keys and of its values (head_dim 128) and one fp32 scale for each.
 *   format: DQ_Q8_INT8 (codes -127..127, Q = 127) or DQ_Q8_E4M3 (OCP 8-bit
 *           floating point, 4 exponent and 3 mantissa bits, Q = 448)
 *   scale = fl32(max |x| / Q) over the block, code = x / scale rounded to the
 *   type's nearest value (of the exact quotient, ties to even), x^ = scale code.
 * A block whose largest magnitude is below 2^-96 is stored as zeros with scale
 * 0.  Infinities and NaN are stored as zeros and set DQ_STATUS_RANGE.
 *   k_data, v_data:   u8 [batch][kv_heads][t_cap / 32][4096], 16-byte aligned
 *   k_scale, v_scale: fp32 [batch][kv_heads][t_cap / 32]
 * The order of the 4096 codes within a block is the order in which the matrix
 * cores take them; dq_q8_decode_kv reads tokens back.  In pool pages (the paged
 * layout above) the same arrays are [num_pages][kv_heads][page_tokens / 32][..].
 * t_cap is a positive multiple of 128; batch and kv_heads are at most 65535.
 *
 * dq_q8_encode_kv: appends tokens [t0, t0 + n_new) of bf16 keys and values
 *   [batch][tokens][kv_heads][128] at element strides (channels contiguous), in
 *   one launch.  t0 is a multiple of 32; a last block that n_new does not fill
 *   is completed with zeros, so the next append starts at its first token (the
 *   residual window holds the tokens of a block that is not full yet).
 * dq_q8_decode_kv: the values of tokens [t0, t0 + n), t0 a multiple of 32, as
 *   bf16 (scale code, rounded once to fp32 and once to bf16) to
 *   [batch][n][kv_heads][128] at element strides.  Nothing else is written.
 */
#define DQ_Q8_BLOCK 32
#define DQ_Q8_INT8 0
#define DQ_Q8_E4M3 1
int dq_q8_encode_kv(int32_t format, const uint16_t* k, int64_t k_stride_b, int64_t k_stride_t, int64_t k_stride_h,
                    const uint16_t* v, int64_t v_stride_b, int64_t v_stride_t, int64_t v_stride_h, int32_t batch,
                    int32_t kv_heads, int32_t t0, int32_t n_new, int32_t t_cap, uint8_t* k_data, float* k_scale,
                    uint8_t* v_data, float* v_scale, uint32_t* status, void* stream);
int dq_q8_encode_kv_paged(int32_t format, const uint16_t* k, int64_t k_stride_b, int64_t k_stride_t,
                          int64_t k_stride_h, const uint16_t* v, int64_t v_stride_b, int64_t v_stride_t,
                          int64_t v_stride_h, int32_t batch, int32_t kv_heads, int32_t t0, int32_t n_new,
                          const int32_t* block_table, int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                          uint8_t* k_pool, float* k_scale_pool, uint8_t* v_pool, float* v_scale_pool,
                          uint32_t* status, void* stream);
int dq_q8_decode_kv(int32_t format, const uint8_t* k_data, const float* k_scale, const uint8_t* v_data,
                    const float* v_scale, int32_t batch, int32_t kv_heads, int32_t t0, int32_t n, int32_t t_cap,
                    uint16_t* k, int64_t k_stride_b, int64_t k_stride_t, int64_t k_stride_h, uint16_t* v,
                    int64_t v_stride_b, int64_t v_stride_t, int64_t v_stride_h, void* stream);
int dq_q8_decode_kv_paged(int32_t format, const uint8_t* k_pool, const float* k_scale_pool, const uint8_t* v_pool,
                          const float* v_scale_pool, int32_t batch, int32_t kv_heads, int32_t t0, int32_t n,
                          const int32_t* block_table, int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                          uint16_t* k, int64_t k_stride_b, int64_t k_stride_t, int64_t k_stride_h, uint16_t* v,
                          int64_t v_stride_b, int64_t v_stride_t, int64_t v_stride_h, uint32_t* status,
                          void* stream);

/*
 * One decode step of attention over the 8-bit cache: logits softmax_scale *
 * q . k^, output sum a v^, as dq_decode_attention over records.
 *   q:  bf16 [batch][q_heads][128], 16-byte aligned
 *   out: fp32 [batch][q_heads][128], 8-byte aligned
 *   seq_lens: device int32 [batch], tokens in the cache (each in [0, t_cap])
 *   window, sinks: window = 0: every token is visible (sinks has to be 0).
 *       window > 0: token t is visible if it is among the first `sinks` or
 *       among the newest `window` of the sequence; only the blocks that hold
 *       such tokens are read.
 *   extra_lens: device int32 [batch] or NULL: tokens of each sequence that
 *       follow the cached ones (a residual window's); the newest `window`
 *       tokens are counted back from their end.  The residual window itself is
 *       always attended to whole, so with it window should be at least r_cap.
 *   block_lse: fp32 [batch][kv_heads][t_cap / 32][q_heads / kv_heads] or NULL:
 *       receives the base-2 logarithm of each visible block's sum of
 *       exponentials, for dq_q8_add_scores (what its rounding to fp32 leaves is
 *       kept in the workspace).  Other entries are left alone.
 *   workspace: dq_decode_workspace_bytes(...) bytes, 16-byte aligned
 * A sequence with no visible token gives zeros; a query head with an infinity
 * or NaN gives NaN, in its KV head's scores too.  Weighted values are summed in
 * fp32 before they are divided by the sum of the weights, so values larger than
 * 2^127 over the number of visible tokens can give infinities.
 * dq_q8_decode_attention_partial writes split-K partials into the workspace;
 * finish it with dq_decode_attention_merge, with dq_decode_attention_residual
 * and dq_decode_attention_merge, or with dq_decode_attention_merge_residual.
 * dq_q8_decode_attention is the partial, the merge and, where scores is not
 * NULL (block_lse is then required), dq_q8_add_scores in one call.
 * Through a block table the step is the same; an entry outside the pool sets
 * DQ_STATUS_PAGE and page 0 is read in its place.
 * q_heads / kv_heads is at most 8.  Returns DQ_OK, DQ_ERR_INVALID_ARG,
 * DQ_ERR_WORKSPACE or DQ_ERR_HIP.
 *
 * dq_q8_add_scores: scores[b][h][j] (fp32 [batch][kv_heads][t_cap / 32]) grows
 * by the attention weight of block j in the step whose partials (of the cached
 * tokens and, if dq_decode_attention_residual ran, of the raw ones) are in the
 * workspace, summed over its tokens and the query heads of KV head h.  The
 * arguments are those of the step.  The step has to be one of the _partial
 * calls: dq_q8_decode_attention, which may finish without the workspace, adds
 * to the scores by itself.  A score holds the weight of the steps that added to
 * it: none of the attention of a prompt, and none of the steps in which the
 * block's tokens were still raw ones of a residual window.
 * dq_q8_merge_scores: dq_decode_attention_merge and dq_q8_add_scores of such a
 * step in one launch.
 */
int dq_q8_decode_attention_partial(int32_t format, const uint16_t* q, int32_t batch, int32_t q_heads,
                                   int32_t kv_heads, const uint8_t* k_data, const float* k_scale,
                                   const uint8_t* v_data, const float* v_scale, const int32_t* seq_lens,
                                   const int32_t* extra_lens, int32_t t_cap, int32_t window, int32_t sinks,
                                   float softmax_scale, float* block_lse, void* workspace, size_t workspace_bytes,
                                   void* stream);
int dq_q8_decode_attention(int32_t format, const uint16_t* q, int32_t batch, int32_t q_heads, int32_t kv_heads,
                           const uint8_t* k_data, const float* k_scale, const uint8_t* v_data, const float* v_scale,
                           const int32_t* seq_lens, int32_t t_cap, int32_t window, int32_t sinks,
                           float softmax_scale, float* out, float* block_lse, float* scores, void* workspace,
                           size_t workspace_bytes, void* stream);
int dq_q8_decode_attention_paged_partial(int32_t format, const uint16_t* q, int32_t batch, int32_t q_heads,
                                         int32_t kv_heads, const uint8_t* k_pool, const float* k_scale_pool,
                                         const uint8_t* v_pool, const float* v_scale_pool,
                                         const int32_t* block_table, int32_t max_pages, int32_t page_tokens,
                                         int32_t num_pages, const int32_t* seq_lens, const int32_t* extra_lens,
                                         int32_t window, int32_t sinks, float softmax_scale, float* block_lse,
                                         void* workspace, size_t workspace_bytes, uint32_t* status, void* stream);
int dq_q8_decode_attention_paged(int32_t format, const uint16_t* q, int32_t batch, int32_t q_heads,
                                 int32_t kv_heads, const uint8_t* k_pool, const float* k_scale_pool,
                                 const uint8_t* v_pool, const float* v_scale_pool, const int32_t* block_table,
                                 int32_t max_pages, int32_t page_tokens, int32_t num_pages,
                                 const int32_t* seq_lens, int32_t window, int32_t sinks, float softmax_scale,
                                 float* out, float* block_lse, float* scores, void* workspace,
                                 size_t workspace_bytes, uint32_t* status, void* stream);
int dq_q8_add_scores(int32_t batch, int32_t q_heads, int32_t kv_heads, const int32_t* seq_lens,
                     const int32_t* extra_lens, int32_t t_cap, int32_t window, int32_t sinks,
                     const float* block_lse, const void* workspace, size_t workspace_bytes, float* scores,
                     void* stream);
int dq_q8_merge_scores(int32_t batch, int32_t q_heads, int32_t kv_heads, const int32_t* seq_lens,
                       const int32_t* extra_lens, int32_t t_cap, int32_t window, int32_t sinks,
                       const float* block_lse, const void* workspace, size_t workspace_bytes, float* out,
                       float* scores, void* stream);

/*
 * Eviction by accumulated attention weight.  Every (sequence, KV head) that
 * holds more than keep / 32 blocks keeps its first `first` / 32 and its newest
 * `last` / 32 blocks and, of the others, those with the largest scores (of
 * equal ones the lower block, so that before the first step with scores the
 * oldest stay; NaN counts as the smallest): keep / 32 blocks in all, in their
 * order.  Codes, scales and scores move to their new places unchanged; shorter
 * sequences keep everything.
 *   keep, first, last: whole blocks, counted as 32 tokens each; first >= 0,
 *       last >= 32, first + last <= keep <= to_cap.  The newest block counts as
 *       one of the last / 32 however few tokens it holds, so between last - 31
 *       and last of a sequence's newest tokens stay for certain.  last = n + 31,
 *       rounded up to a multiple of 32, keeps the newest n at every length.
 *   kept: int32 [batch][kv_heads][keep / 32]: the old index of each kept block,
 *       -1 behind the last
 *   new_lens: device int32 [batch], may be seq_lens: the new lengths,
 *       seq_lens[b] - 32 (blocks evicted)
 *   to_*: the cache that receives the kept blocks: either the same arrays (in
 *       place; to_cap = t_cap) or others, of to_cap tokens, that do not overlap
 *       them.  Scores behind the kept ones become 0, in place up to the old block
 *       count.
 * In pool pages the eviction is in place, so none of the pages may belong to
 * two sequences; pages behind the new length are free for the caller.  An entry
 * outside the pool sets DQ_STATUS_PAGE and nothing is written through it.
 * Returns DQ_OK, DQ_ERR_INVALID_ARG or DQ_ERR_HIP.
 */
int dq_q8_evict(int32_t batch, int32_t kv_heads, const int32_t* seq_lens, int32_t* new_lens, int32_t t_cap,
                int32_t to_cap, int32_t keep, int32_t first, int32_t last, uint8_t* k_data, float* k_scale,
                uint8_t* v_data, float* v_scale, float* scores, uint8_t* to_k_data, float* to_k_scale,
                uint8_t* to_v_data, float* to_v_scale, float* to_scores, int32_t* kept, void* stream);
int dq_q8_evict_paged(int32_t batch, int32_t kv_heads, const int32_t* seq_lens, int32_t* new_lens, int32_t keep,
                      int32_t first, int32_t last, const int32_t* block_table, int32_t max_pages,
                      int32_t page_tokens, int32_t num_pages, uint8_t* k_pool, float* k_scale_pool,
                      uint8_t* v_pool, float* v_scale_pool, float* scores, int32_t* kept, uint32_t* status,
                      void* stream);

/*
 * Rotary positions.  Pair i of a head's first `rotary_dim` channels, (a, b), at
 * position p becomes
 *   (a cos x - b sin x, a sin x + b cos x) magnitude,   x = p freq[i],
 * where the pairs are (i, i + rotary_dim / 2) (DQ_ROPE_HALF) or (2 i, 2 i + 1)
 * (DQ_ROPE_INTERLEAVED); the channels from rotary_dim on stay as they are.  Keys
 * are rotated before they are appended to a cache, queries before they attend.
 * transposed = 1 changes the sign of x: the transposed map, which gives the
 * gradient of the inputs from that of the outputs and, with magnitude 1, turns
 * rotated vectors back.
 *
 * dq_rope_frequencies: host only.  freq fp64 [rotary_dim / 2] receives the angles
 *   per token, *magnitude the factor of the rotated values.  With
 *   f_i = base^(-2 i / rotary_dim):
 *   DQ_ROPE_NONE    f_i
 *   DQ_ROPE_LINEAR  f_i / factor
 *   DQ_ROPE_NTK     the same with base factor^(rotary_dim / (rotary_dim - 2)) in
 *                   base's place (rotary_dim > 2)
 *   DQ_ROPE_BANDS   w f_i + (1 - w) f_i / factor, w rising evenly from 0 at
 *                   turns_low to 1 at turns_high turns of the pair over
 *                   `original` tokens (turns_low < turns_high)
 *   DQ_ROPE_YARN    the same mixture, w falling evenly over the index i from 1 at
 *                   floor(j(turns_high)) to 0 at ceil(j(turns_low)), j(n) =
 *                   rotary_dim ln(original / (2 pi n)) / (2 ln base) (the ends
 *                   kept within 0 and rotary_dim - 1, and at least 0.001 apart);
 *                   the magnitude is 0.1 ln factor + 1 where factor > 1
 *   The magnitude is 1 otherwise.  base > 0 (YARN: other than 1), factor >= 1,
 *   turns and original > 0 where they count; all finite.
 * dq_rope: rotates the queries and the keys of a chunk in one launch.
 *   freq: device fp64 [rotary_dim / 2]; any frequencies, dq_rope_frequencies'
 *       or the caller's
 *   q, k: bf16 [batch][tokens][heads][head_dim] at element strides, channels
 *       contiguous; either may be absent (NULL, 0 heads).  q_out, k_out: where
 *       the results go, at strides of their own: the same tensor (same address
 *       and strides), or one that overlaps neither input, in which no two
 *       elements share an address.  Queries and keys that start at one address
 *       are not rotated in place.
 *   positions: device int32, position of token t of sequence b at
 *       positions[b pos_stride_b + t pos_stride_t], of any sign; or NULL:
 *       positions are t0 + t, plus starts[b] where starts (device int32 [batch])
 *       is not NULL, as the lengths of a cache are.  With positions, starts is
 *       NULL and t0 is 0.
 * Angles are computed in fp64 and reduced to a part of a turn before they are
 * rounded; results are computed in fp32 and rounded to bf16 once.
 * rotary_dim is even, 2 <= rotary_dim <= head_dim <= 1024; heads at most 65535;
 * batch tokens at most 2^26; strides not negative.  Return DQ_OK (nothing is
 * launched when batch or tokens is 0), DQ_ERR_INVALID_ARG or DQ_ERR_HIP.
 */
#define DQ_ROPE_HALF 0
#define DQ_ROPE_INTERLEAVED 1
#define DQ_ROPE_NONE 0
#define DQ_ROPE_LINEAR 1
#define DQ_ROPE_NTK 2
#define DQ_ROPE_BANDS 3
#define DQ_ROPE_YARN 4
int dq_rope_frequencies(int32_t scaling, int32_t rotary_dim, double base, double factor, double original,
                        double turns_low, double turns_high, double* freq, double* magnitude);
int dq_rope(int32_t layout, int32_t transposed, const double* freq, float magnitude, int32_t rotary_dim,
            int32_t head_dim, int32_t batch, int32_t tokens, const uint16_t* q, int64_t q_stride_b,
            int64_t q_stride_t, int64_t q_stride_h, int32_t q_heads, uint16_t* q_out, int64_t qo_stride_b,
            int64_t qo_stride_t, int64_t qo_stride_h, const uint16_t* k, int64_t k_stride_b, int64_t k_stride_t,
            int64_t k_stride_h, int32_t kv_heads, uint16_t* k_out, int64_t ko_stride_b, int64_t ko_stride_t,
            int64_t ko_stride_h, const int32_t* positions, int64_t pos_stride_b, int64_t pos_stride_t,
            const int32_t* starts, int32_t t0, void* stream);

/*
 * Attention of a chunk of tokens over the 8-bit cache: n_q queries of every
 * sequence at once, logits softmax_scale * q . k^, output sum a v^.
 *   q:   bf16 [batch][n_q][q_heads][128] at element strides, channels contiguous;
 *        query head i reads KV head i / (q_heads / kv_heads)
 *   out: bf16 [batch][n_q][q_heads][128] likewise, no two elements at one address
 *        and none at one of the inputs
 *   q_lens: device int32 [batch] or NULL: the first q_lens[b] of the n_q queries
 *        count (each in [0, n_q]); NULL: all.  Output rows behind them are left
 *        as they are.
 *   seq_lens: device int32 [batch], tokens in the cache (each in [0, t_cap])
 *   causal = 1: the queries are those of the sequence's newest tokens, which the
 *        cache holds already: query i of q_len has position p = seq_len - q_len
 *        + i and sees the tokens t <= p.  window > 0: of those, t < sinks or
 *        t > p - window, as the decode step of that token would; only blocks that
 *        hold such tokens are read.  window = 0: all of them (sinks is 0 then).
 *   causal = 0: every query sees all seq_len tokens, as a decoder's queries do
 *        of an encoder's states that the cache holds (window and sinks are 0).
 *   workspace: dq_chunk_workspace_bytes(...) bytes, 16-byte aligned (NULL where
 *        that is 0); calls that may overlap in time need one each
 * A query that sees no token gives zeros; one with an infinity or NaN that sees
 * some gives NaN.  Scores and sums are held in fp32; the weights are rounded to
 * fp16 for the product with the codes of the values, which are exact, and the
 * output to bf16.  (What is rounded is a weight times its block's scale, relative
 * to a query's largest such product: 11 bits down to 2^-14 of that, fewer below,
 * nothing below 2^-25.)  Value blocks may be of any sizes: one that a query does
 * not see, or that has no weight, takes no bits from others, down to 2^-80 of its
 * scale, and values up to bf16's largest give no infinity.
 * (Scales are finite and not negative, as the encoder writes them; one of values
 * that is NaN or infinite gives NaN to the queries that see its block.)
 * The same call gives the same bits again; where long sequences are cut follows
 * from all lengths of the batch, so a sequence's last bits may go by the others.
 * Through a block table the call is the same; an entry outside the pool sets
 * DQ_STATUS_PAGE and page 0 is read in its place.
 * batch and kv_heads at most 65535, n_q q_heads at most 2^26, batch kv_heads
 * ceil(n_q (q_heads / kv_heads) / 128) at most 2^22.  Returns DQ_OK (nothing is
 * launched when batch or n_q is 0), DQ_ERR_INVALID_ARG, DQ_ERR_WORKSPACE or
 * DQ_ERR_HIP.
 *
 * dq_cross_attention: the same, not causal, over an encoder's states in BF16.
 *   k, v: bf16 [batch][n_kv][kv_heads][128] at element strides (0 where sequences
 *        share states), channels contiguous
 *   kv_lens: device int32 [batch] or NULL: states of each sequence (each in
 *        [0, n_kv]); NULL: n_kv
 *   mask: device u8 [batch][n_kv], rows mask_stride_b apart, or NULL: states with
 *        0 are hidden (their keys and values may hold anything)
 * A query whose sequence has no visible state gives zeros.  Infinities and NaN in
 * a query or a visible state give what the formula gives in fp32, in which the
 * scores are held, but a query whose every score is -infinity gives zeros
 * and sums of values above 2^80 may overflow.
 * Weights are rounded for the product with the values, to two terms of bf16 (16
 * bits) where n_q (or q_lens[b]) (q_heads / kv_heads) is at most 64, to one (8 bits)
 * where it is more.  n_kv is at most 2^30.
 *
 * dq_chunk_workspace_bytes: for both; t_cap is the cache's capacity (max_pages *
 * page_tokens) or n_kv.  It holds the outputs of the pieces that the GPU works on
 * at a time, with or without q_lens: at most 121 MB whatever the sizes are, and as
 * much wherever one sequence may be cut into many.  0 for sizes that the calls
 * refuse, and where nothing can be cut.
 */
size_t dq_chunk_workspace_bytes(int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads, int32_t t_cap);
int dq_q8_chunk_attention(int32_t format, const uint16_t* q, int64_t q_stride_b, int64_t q_stride_t,
                          int64_t q_stride_h, int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads,
                          const uint8_t* k_data, const float* k_scale, const uint8_t* v_data, const float* v_scale,
                          const int32_t* q_lens, const int32_t* seq_lens, int32_t t_cap, int32_t causal,
                          int32_t window, int32_t sinks, float softmax_scale, uint16_t* out, int64_t o_stride_b,
                          int64_t o_stride_t, int64_t o_stride_h, void* workspace, size_t workspace_bytes,
                          void* stream);
int dq_q8_chunk_attention_paged(int32_t format, const uint16_t* q, int64_t q_stride_b, int64_t q_stride_t,
                                int64_t q_stride_h, int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads,
                                const uint8_t* k_pool, const float* k_scale_pool, const uint8_t* v_pool,
                                const float* v_scale_pool, const int32_t* block_table, int32_t max_pages,
                                int32_t page_tokens, int32_t num_pages, const int32_t* q_lens,
                                const int32_t* seq_lens, int32_t causal, int32_t window, int32_t sinks,
                                float softmax_scale, uint16_t* out, int64_t o_stride_b, int64_t o_stride_t,
                                int64_t o_stride_h, void* workspace, size_t workspace_bytes, uint32_t* status,
                                void* stream);
int dq_cross_attention(const uint16_t* q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, int32_t batch,
                       int32_t n_q, int32_t q_heads, int32_t kv_heads, const uint16_t* k, int64_t k_stride_b,
                       int64_t k_stride_t, int64_t k_stride_h, const uint16_t* v, int64_t v_stride_b,
                       int64_t v_stride_t, int64_t v_stride_h, int32_t n_kv, const int32_t* q_lens,
                       const int32_t* kv_lens, const uint8_t* mask, int64_t mask_stride_b, float softmax_scale,
                       uint16_t* out, int64_t o_stride_b, int64_t o_stride_t, int64_t o_stride_h, void* workspace,
                       size_t workspace_bytes, void* stream);

/*
 * rANS-decodes records back to symbols (Alg. 2), for parity checks.
 *   records: u8 [n_streams][C]; sym: u8 [n_streams][head_dim];
 *   header:  u16 [n_streams][2] = (scale, offset) fp16 bits; may be NULL;
 *   status:  DQ_STATUS_CORRUPT if a record is malformed; may be NULL.
 */
int dq_decode_symbols(const dq_tables* tables, const uint8_t* records,
                      int64_t n_streams, uint8_t* sym, uint16_t* header,
                      uint32_t* status, void* stream);

/* Static description of a return code. */
const char* dq_strerror(int code);

/* The HIP call that last failed in this thread with DQ_ERR_HIP, and its HIP
 * error name and text ("" if none).  Valid until the next failing call. */
const char* dq_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DQ_H */
