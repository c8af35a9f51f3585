/*
 * ppmm.h - C ABI of the clear track: products of plaintext weights and clear activations, the public K/V cache and
 * attention over it, all held in 4 bits.  Part of the same library as pcmm.h, with its status codes and conventions.
 *
 * A mixed prompt (Section 4.1) has a public prefix and an encrypted suffix.  The public tokens run in the clear through the
 * layers whose weights the encrypted ones are multiplied with (Section 5.1), and leave a public K/V cache, which the encrypted
 * track reads as the plaintext operand of PC-attention (Section 4.2).  Codes and scales are the caller's: nothing here makes
 * them of the integers of a pcmm_plan, or integers of them.  The converted weights of the encrypted track fill
 * most of the memory (Section 5.3), so here a weight, a key or a value takes 4 bits and its share of a group's scale.
 *
 * Conventions.  "device" pointers are HIP device memory on the device that is named.  Matrices are row-major with the row
 * stride given in elements; elements are aligned to their size, nothing more is asked for.  Calls are asynchronous on the
 * given stream (NULL = default stream), allocate nothing and keep nothing between calls, so any number of runs of one plan
 * or one cache may overlap as long as no call writes what another one reads or writes; all of them can be captured into a
 * graph.  Sums are held in 32-bit floating point; results are rounded once, to nearest even.  One factor has fewer bits: what
 * attention weighs a value with, its scale times the exponential of its score, is rounded to 16 bits or more.  No function throws or
 * aborts.
 */
#ifndef PPMM_H
#define PPMM_H

#include "pcmm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PPMM_BF16 = 0,
    PPMM_FP16 = 1,
    PPMM_INT16 = 2 /* fixed point, of ppkv_read only */
} ppmm_type;

typedef struct ppmv_plan ppmv_plan; /* opaque; owns one packed weight matrix */

/*
 * Pack one weight matrix in 4 bits.
 *
 *     w[m][k] = scales[m][k / group] * (c[m][k] - 8) + offsets[m][k / group] ,    c in 0..15
 *
 *   out           receives the plan (set to NULL on failure)
 *   M, K          W is M x K: M output channels, 1 <= M <= 2^24, K input channels, 1 <= K <= 2^22, any number of both
 *   group         input channels that share a scale: 32, 64 or 128; the last group may be shorter
 *   type          type of scales, offsets, activations and results: PPMM_BF16 or PPMM_FP16
 *   codes_dev     device, [M][(K+1)/2] bytes: c of even k in the low half of a byte, of odd k in the high half
 *   scales_dev    device, [M][ceil(K/group)]
 *   offsets_dev   device, as scales_dev, or NULL: no offsets
 *   device        HIP device ordinal the plan lives on
 *   stream        stream of the packing kernels; the call synchronises it before it returns
 *
 * The three arrays are read during this call only.  PCMM_EINVAL for null pointers, sizes out of range and any other
 * group or type; PCMM_EUNSUPPORTED for more than 2^36 packed codes.
 */
pcmm_status ppmv_plan_create(ppmv_plan **out, int64_t M, int64_t K, int32_t group, ppmm_type type, const uint8_t *codes_dev,
                             const void *scales_dev, const void *offsets_dev, int32_t device, void *stream);

/* Device bytes the plan owns: the codes and scales, with M filled up to 16 and K to 128.  0 for NULL. */
size_t ppmv_plan_workspace_bytes(const ppmv_plan *plan);

/*
 * Y = X W^T for T tokens: y[t][m] = sum_k x[t][k] w[m][k].
 *
 *   T        tokens, 0 <= T <= 2^24; 0 does nothing
 *   x_dev    device, T rows of K elements, row stride ldx >= 0 (0: all tokens are the same row)
 *   y_dev    device, T rows of M elements, row stride ldy >= M; must not overlap x_dev
 *
 * A result does not depend on the other tokens' values, but its last bits may depend on how many there are.  An x that is
 * not finite makes every result of its token NaN or infinite, and so may a sum of 31 |x| over a group that 32-bit floating
 * point does not hold.  PCMM_EINVAL for null pointers, negative T, strides that
 * are too small, y_dev == x_dev; PCMM_EUNSUPPORTED for larger T or more than 2^22 tiles of 16 x 64 results.
 */
pcmm_status ppmv_run(const ppmv_plan *plan, int64_t T, const void *x_dev, int64_t ldx, void *y_dev, int64_t ldy, void *stream);

/*
 * The gated feed-forward products: h[t][m] = silu(x Wg^T)[t][m] * (x Wu^T)[t][m], silu(a) = a / (1 + exp(-a)).  Neither
 * projection is rounded or stored.  The two plans agree in M, K, group, type and device (PCMM_EINVAL otherwise), and
 * both have offsets or neither has; they may be the same plan.  Everything else as for ppmv_run.
 */
pcmm_status ppmv_gated_run(const ppmv_plan *gate, const ppmv_plan *up, int64_t T, const void *x_dev, int64_t ldx, void *h_dev,
                           int64_t ldh, void *stream);

/* Frees everything a plan owns.  NULL is ignored.  No run of the plan may still be in flight. */
void ppmv_plan_destroy(ppmv_plan *plan);

/*
 * The public K/V cache: pages of page_size tokens, each with the keys and values of kv_heads heads of head_dim channels
 * in 4 bits.  32 channels of one token's key (or value) share a scale s and an offset b, both bf16:
 *
 *     s = bf16((max - min) / 15) ,  b = bf16(min - 16 s) ,  code = clamp(rint((x - b) / s) - 16, 0, 15) ,
 *     value = s (16 + code) + b ,
 *
 * computed in 64-bit floating point, s and b through 32 bits, ties to even; a scale below 2^-126 counts as 0 and then
 * every code is 0.  32 channels that hold a NaN or an infinity, or whose b does not fit, read as NaN.  The layout inside the
 * pool is the library's own; ppkv_read gives the values.
 */
typedef struct {
    void *pool;        /* device, ppkv_pool_bytes bytes, aligned to 16 bytes; need not be cleared */
    int64_t pages;     /* 1 .. 2^31 - 1 */
    int32_t page_size; /* tokens, a multiple of 16 up to 65536 */
    int32_t kv_heads;  /* 1 .. 1024 */
    int32_t head_dim;  /* 64 or 128 */
} ppkv_cache;

/* Bytes of a pool (1.25 head_dim for a token's key and value of one head).  0 for sizes out of range or 2^47 bytes and more. */
size_t ppkv_pool_bytes(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim);

/*
 * The new tokens of a batch of sequences.  Row n of a packed array belongs to sequence b if starts[b] <= n < starts[b+1],
 * and is that sequence's token number lens[b] - (starts[b+1] - n): lens counts the cached tokens with the new ones.  Token
 * i of sequence b lies in page table[b][i / page_size].  The arrays are on the device and are not checked by the host.
 * Whatever they hold, nothing outside the pool and the arrays' given sizes is read or written:
 *   - rows that belong to no sequence (before the first, behind the last one) are left as they were;
 *   - a token with a negative number, a number beyond the table's width or a page outside 0..pages-1 is not written, reads
 *     as zeros and is not attended to.
 */
typedef struct {
    const int32_t *starts; /* device, [batch + 1], ascending */
    const int32_t *lens;   /* device, [batch] */
    const int32_t *table;  /* device, [batch][table_width] page numbers */
    int32_t batch;         /* 1 .. 65535 */
    int32_t table_width;   /* pages a sequence may have, >= 1; table_width * page_size < 2^31 */
} ppkv_batch;

/*
 * Quantise the keys and values of new tokens into the cache.
 *
 *   k_dev, v_dev           device, [tokens][kv_heads][head_dim] with the given strides (in elements, >= 0) of tokens and heads
 *   type                   PPMM_BF16 or PPMM_FP16
 *   tokens                 rows of k_dev and v_dev, 0 <= tokens < 2^31
 *
 * No two tokens of one call may have the same place in the cache.  PCMM_EINVAL for null pointers, sizes and strides out of range;
 * PCMM_EUNSUPPORTED, here and in ppkv_read, for tokens kv_heads head_dim above 2^34 - 1024.
 */
pcmm_status ppkv_append(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, const void *k_dev,
                        int64_t k_token_stride, int64_t k_head_stride, const void *v_dev, int64_t v_token_stride,
                        int64_t v_head_stride, int32_t device, void *stream);

/*
 * The values of the same tokens: the inverse of ppkv_append.  k_dev or v_dev may be NULL: not wanted.  The strides must
 * keep the rows apart.  A value is rounded to 32 bits first.  PPMM_INT16 writes rint(value 2^frac_bits), ties to even, held to
 * [-32768, 32639] and 0 for NaN:
 * the 16-bit plaintext operand of pcmm_plan_create.  With the strides of [kv_heads][tokens][head_dim] every head's keys
 * are such an operand.  0 <= frac_bits <= 30, and 0 for the other types.
 */
pcmm_status ppkv_read(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, int32_t frac_bits,
                      void *k_dev, int64_t k_token_stride, int64_t k_head_stride, void *v_dev, int64_t v_token_stride,
                      int64_t v_head_stride, int32_t device, void *stream);

/*
 * Attention of the new tokens over the cache:
 *
 *     out[n][h] = sum_i softmax_i( scale <q[n][h], key_i> ) value_i ,    key and value of head h / (heads / kv_heads) ,
 *
 * over the tokens i of the row's sequence, i < lens[b], and, if causal, i not behind the row's own token.  A row that
 * attends to nothing is zero.  A token behind a causal row does not reach it, whatever it holds; of the tokens that a row
 * attends to, a NaN key makes the whole row NaN, and values that read as NaN make those 32 channels of it NaN.  So may scores
 * that 32-bit floating point does not hold, and values 2^8 times whose magnitudes it does not hold the sum of.
 *
 *   q_dev, out_dev   device, [tokens][heads][head_dim] with strides; the rows of out_dev must be apart; out_dev != q_dev
 *   heads            a multiple of kv_heads, heads / kv_heads <= 65536; max_q heads / kv_heads below 2^31 - 64
 *   max_q            no sequence has more new tokens; rows beyond are left as they were
 *   max_len          expected largest lens[b], for the division of the work only (0: table_width * page_size)
 *   scratch          device, ppkv_attention_scratch_bytes(same sizes) bytes, at most 2^27, aligned to 16 bytes, for this call alone
 *                    until it has finished; need not be cleared; may be NULL where that is 0
 *
 * PCMM_EINVAL for null pointers, sizes and strides out of range and too little scratch; PCMM_EUNSUPPORTED for 2^24 work-groups and
 * more: batch kv_heads times a sequence's max_q heads / kv_heads rows by sixteens (at least one).
 *
 * The last bits of a result may depend on the sizes of the call, not on what else is in the batch.  The work of every sequence is divided
 * by max_q and max_len alike: a prompt and single tokens are better given in two calls.
 */
size_t ppkv_attention_scratch_bytes(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, int32_t heads,
                                    int32_t max_q, int64_t max_len, int32_t device);
pcmm_status ppkv_attention(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, int32_t heads,
                           const void *q_dev, int64_t q_token_stride, int64_t q_head_stride, void *out_dev,
                           int64_t out_token_stride, int64_t out_head_stride, float scale, int32_t causal, int32_t max_q,
                           int64_t max_len, void *scratch, size_t scratch_bytes, int32_t device, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PPMM_H */
