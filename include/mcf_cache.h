/*
 * mcf -- what the softmax chain needs around it where keys and values are kept between calls (the key and
 * value matrices B and D of mcf.h, held for many sequences in pages, in 8 bits), on AMD MI355X (gfx950):
 *
 *   mcf_norm_rotate            RMS norm of queries and keys for each head and the position rotation, in one pass
 *   mcf_norm_rotate_backward   its gradients
 *   mcf_cache_append           new keys (normed and rotated on the way) and values into the cache, with a scale
 *                              for each page and head; the queries of the same tokens go through the same launch
 *   mcf_cache_attention        softmax(scale Q K^T) V over the cache: single tokens, a few, pieces of prompts
 *
 * C ABI, as mcf.h: every call returns an mcf_status (mcf.h) and launches asynchronously on the caller's stream;
 * structs are HOST memory, every pointer in them is a DEVICE pointer owned by the caller; nothing is allocated and
 * nothing synchronises.  What a call cannot see from the host (positions, tables, lengths) the kernels check
 * themselves, as written at each: no value there makes them read or write outside of the buffers named here.
 */
#ifndef MCF_CACHE_H
#define MCF_CACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* A tensor [batch, tokens, heads, size]: element strides of the first three dimensions, the last one packed.  Strides
 * are multiples of 8 elements and the pointer 16-byte aligned (MCF_EALIGN). */
typedef struct mcf_rows {
    void *data;
    int64_t stride[3]; /* batch, token, head */
} mcf_rows;

/*
 * For every row x (one head of one token) of q and of k, with its weight w and its position p:
 *     r = 1 / sqrt(mean(x^2) + eps)       y = R(p) (x r w)
 * R(p) turns the pairs (y_a, y_b) of the first `rotary` elements by the angle whose cosine and sine stand in row p
 * of the tables: (a, b) = (j, j + rotary/2), or (2j, 2j + 1) with interleaved != 0; the other elements stay.  A weight
 * of NULL leaves out the norm of that tensor, tables of NULL (rotary = 0) the rotation.
 *   dtype          MCF_F16 or MCF_BF16, of q, k, the weights (weight_f32 = 0) and the results; all arithmetic is fp32,
 *                  rounded once.  weight_f32 = 1: the weights are fp32
 *   size           a multiple of 16 up to 512; rotary a multiple of 16, at most size
 *   cos, sin       fp32 [table_rows, rotary / 2], packed
 *   positions      NULL: a token's index in its batch row; else [tokens] (position_batch = 0) or [batch, tokens]
 *                  (position_batch = tokens), of 4 or 8 bytes (position_bytes).  A position outside of the tables
 *                  gives NaN in the rotated elements
 *   k.data NULL    (k_heads 0) only q
 * Results may be written in place (q_out = q), else they overlap no operand (the caller's to see to).
 * Backward: dq, dk are the gradients of the results, q, k what the forward call took; q_out, k_out receive the gradients
 * of q and k (they may be dq and dk), dq_weight, dk_weight (fp32 [size], NULL without a weight) those of the weights: sums
 * over all tokens and heads in fp32, in an order that the shapes fix.
 */
typedef struct mcf_norm_rotate_call {
    int32_t dtype, weight_f32, interleaved, position_bytes;
    int64_t batch, tokens, q_heads, k_heads, size, rotary, table_rows, position_batch;
    double eps;
    const float *cos, *sin;
    const void *positions, *q_weight, *k_weight;
    mcf_rows q, k, q_out, k_out;
    mcf_rows dq, dk;                 /* backward only */
    float *dq_weight, *dk_weight;    /* backward only */
} mcf_norm_rotate_call;
int mcf_norm_rotate(const mcf_norm_rotate_call *call, void *hip_stream);
/* Bytes of device memory that the backward call wants (16-byte aligned, in use until its work is done); host only. */
int mcf_norm_rotate_backward_workspace(const mcf_norm_rotate_call *call, int64_t *bytes);
int mcf_norm_rotate_backward(const mcf_norm_rotate_call *call, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * The cache: keys and values as e4m3 (no infinities, NaN = 0x7f), [pages, heads, page_size, size], the last two
 * dimensions packed, element strides of the first two multiples of 16 and that of the pages below 2^32 (pointers 16-byte aligned), and an fp32 scale for
 * each page and head, [pages, heads] with a stride of its own and packed heads, not negative: the value held is e4m3 * scale, NaN where the
 * scale is not finite.
 * page_size: 16, 32, 64 or 128; size: 64, 80, 96, 128, 192 or 256.
 */
typedef struct mcf_kv_cache {
    int64_t pages, heads, page_size, size;
    void *k, *v;
    float *k_scale, *v_scale;
    int64_t k_stride[2], v_stride[2]; /* page, head */
    int64_t k_scale_stride, v_scale_stride;
} mcf_kv_cache;

/*
 * The sequences of a call: rows starts[b] .. starts[b + 1] - 1 of the call's token tensors belong to sequence b (starts
 * NULL: one row each, row b); rows outside of every sequence are not written, and what they hold has no effect.  Starts ascend: with others, rows that
 * several sequences claim get the result of any of them, and rows may be left out.  lengths[b] counts the tokens of the
 * sequence, those rows the last of them: row i of n is token lengths[b] - n + i.  Token t is held in place
 * t % page_size of page table[b][t / page_size] (`table_width` columns; stride in elements).  A token whose page number
 * is outside of the cache, or that is beyond the table, is not there: nothing is written for it and nobody sees it.
 * starts, lengths and table are int32.
 */
typedef struct mcf_sequences {
    int64_t batch, tokens;  /* sequences; rows of the token tensors */
    int64_t table_width, table_stride;
    const int32_t *starts, *lengths, *table;
} mcf_sequences;

/*
 * k and v [tokens, heads, size] (mcf_rows with the batch stride unused) go into the cache.  Keys get mcf_norm_rotate's norm
 * (k_weight) and rotation (tables) first, with the token's place in its sequence as the position, in 64 bits, rounded
 * to fp32 and then to e4m3.  The scale of a page and head is the least power of two, 2^-100 at least, that brings its largest
 * finite value to 448 at most; where a page holds earlier tokens of the sequence, its scale only grows, and they are
 * rounded again when it does.  (Scales are powers of two because e4m3 then loses nothing by them but what falls below
 * its smallest exponent.)  Values that are not finite are held as NaN.  A page that is written belongs to one sequence.
 * q (NULL: none) [tokens, q_heads, size] -> q_out gets its norm and rotation in the same launch; it may be in place.
 */
typedef struct mcf_append_call {
    int32_t dtype, weight_f32, interleaved, reserved;
    int64_t q_heads, rotary, table_rows;
    double eps;
    const float *cos, *sin;
    const void *q_weight, *k_weight;
    mcf_rows q, q_out, k, v;
    mcf_kv_cache cache;
    mcf_sequences seq;
} mcf_append_call;
int mcf_cache_append(const mcf_append_call *call, void *hip_stream);

/*
 * out[t, h] = sum_j softmax_j(scale q[t, h] . k_j) v_j over the tokens j of the row's sequence that it sees: all of them, or
 * with causal != 0 those up to itself; query head h reads head h / (q_heads / heads) of the cache.  A row that sees no token is
 * written as zeros, whatever its query holds; where it sees any, a query that is not finite gives NaN.  q and out are MCF_F16 or MCF_BF16; scores, weights and sums are fp32, the weights are rounded once to
 * the type of q.  (fp16: scales of V below 2^-60 count as 2^-60, which no fp16 result can tell, above 2^126 as 2^126.)  What a row does not see has no effect on it, NaN included.
 * The tokens of a sequence are split over blocks where rows are few; the parts stand in the workspace and are joined in a
 * fixed order.  mcf_cache_attention_workspace: its bytes (host only); with less (NULL and 0) nothing is split.
 */
typedef struct mcf_attention_call {
    int32_t dtype, causal;
    int64_t q_heads;
    float scale;
    int32_t reserved;
    mcf_rows q, out;
    mcf_kv_cache cache;
    mcf_sequences seq;
} mcf_attention_call;
int mcf_cache_attention_workspace(const mcf_attention_call *call, int64_t *bytes);
int mcf_cache_attention(const mcf_attention_call *call, void *workspace, int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MCF_CACHE_H */
