/*
 * lc_serve.h -- what a program that answers with a restored checkpoint needs next to lc.h: weights held in 4 bits with
 * group scales and their products with activations, and a paged cache of keys and values in 8 or 4 bits, written, read
 * back and attended to.  Hand-written HIP kernels for MI355X (gfx950) behind the same C ABI as lc.h.
 *
 * As in lc.h: every pointer is a DEVICE pointer unless a parameter says "host"; `stream` is a hipStream_t passed as
 * void* (NULL = the null stream).  Every call here enqueues on `stream` and returns at once with an lc_status; it
 * allocates nothing, waits for nothing and keeps nothing, so all of them may be captured into a graph.  Arguments are
 * checked on the host before anything is enqueued; a refused call (LC_ERR_BADARG) leaves every buffer as it was.
 * dtype: LC_F32, LC_BF16 or LC_F16 (LC_F64 is refused).  Arrays need the alignment of their element unless said
 * otherwise.  Outputs must not overlap inputs.
 */
#ifndef LC_SERVE_H
#define LC_SERVE_H

#include "lc.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A matrix w[n][k] in 4 bits.  Groups of `group` elements along k (the last one of a row may be shorter) share a scale:
 *     s = bf16(max |w| * fl32(1/7)),  q = rint(w * fl32(1/s)) limited to [-7, 7],  stored as the nibble q + 8,
 * both roundings to nearest even; the value that is meant is q * s.  A group whose scale would be below the smallest normal
 * number (2^-126) gets scale 0 and zeros; one that holds an infinity or NaN gets a NaN scale, so that all of it reads
 * back as NaN.  A nibble of 0 (q = -8) is never written but is read as what it stands for.
 * Element j of a row is the low (j even) or high (j odd) half of its byte j/2.
 */
typedef struct lc_w4 {
    void* codes;            /* 16-byte aligned; row i begins at codes + i * codes_pitch */
    void* scales;           /* bf16; row i begins at element i * scales_pitch */
    uint64_t n, k;          /* at most 2^31 - 1 each */
    uint64_t codes_pitch;   /* bytes: a multiple of 16, at least lc_w4_row_bytes(k) */
    uint64_t scales_pitch;  /* elements: at least ceil(k / group) */
    int group;              /* 32, 64 or 128 */
} lc_w4;

/* Bytes of a row of k codes: ceil(k / 2) rounded up to 16 (0 if k is 0 or above 2^31 - 1).  Host only. */
size_t lc_w4_row_bytes(uint64_t k);

/*
 * w [n][k] of type dtype, row i at element i * ldw (ldw >= k), into w4's codes and scales.  Of every row lc_w4_row_bytes(k) bytes
 * are written, nibbles behind the row's end as zeros (8).
 */
int lc_w4_quantize(const void* w, uint64_t ldw, int dtype, const lc_w4* w4, void* stream);

/* The values that w4 stands for, each fl32(q * s) rounded once to dtype, into w [n][k] (row i at element i * ldw). */
int lc_w4_dequantize(const lc_w4* w4, void* w, uint64_t ldw, int dtype, void* stream);

/*
 * y[i][j] = sum over l of x[i][l] * (q * s)[j][l], plus bias[j] if bias is not NULL: x [m][k] (row i at element i * ldx), bias [n],
 * y [m][n] (row i at element i * ldy), all of type dtype.  Sums are held in 32 bits, codes enter them exactly, each
 * group's sum is multiplied by its scale once, and y is rounded once.  (fp32 x is split into three bf16 parts that add up to it
 * exactly.  For bf16 and fp16 x a group's sum passes through 136 or 72 times the sum of its |x|, whose roundings leave up to some 2e-5 or 1e-5 of
 * the result where x has a mean and groups are of 128, and a tenth of that where it has none; the result's own rounding is 1.6e-3 or 2e-4.)
 * An infinity or NaN in x gives what the formula gives: a result that is not finite is added up again by itself, as far as its first NaN, so that a
 * row with an infinity takes some 0.15 ms more at a width of 4096.  m may be 0 and is at most 2^19; k = 0 gives the bias.
 */
int lc_w4_matmul(const void* x, uint64_t ldx, uint64_t m, const lc_w4* w4, const void* bias, void* y, uint64_t ldy,
                 int dtype, void* stream);

/*
 * A paged cache of keys and values.  A slot is page * page_tokens + token.  Codes lie as [page][head][token][dim],
 * dim elements in dim * bits / 8 bytes; scales as [page][head][token], one fp32 for the dim elements of a key or value:
 *     s = max |v| * fl32(1/most),  q = rint(v * fl32(1/s)) limited to [-most, most],  the value meant is q * s,
 * with most = 127 and q a two's complement byte (bits = 8), or most = 7 and q + 8 a nibble, the even element in the
 * low half (bits = 4).  Scales below 2^-126 and vectors that are not finite as for lc_w4.
 */
typedef struct lc_kv_cache {
    void *k, *v;                /* codes, 16-byte aligned */
    float *k_scale, *v_scale;   /* 16-byte aligned */
    uint64_t pages;             /* pages * page_tokens at most 2^31 */
    int page_tokens;            /* a power of two, 8 to 1024 */
    int heads;                  /* at most 1024 */
    int dim;                    /* a multiple of 32, at most 256 */
    int bits;                   /* 8 or 4 */
} lc_kv_cache;

/*
 * Quantises the keys and values of `tokens` tokens into the cache: k and v are [tokens][heads][dim] of type dtype, token i at
 * element i * ld_token, head h at h * ld_head behind that (both may be any multiple of 1 that keeps vectors apart).
 * slots: int64 [tokens], the slot of each token; a slot outside [0, pages * page_tokens) is passed over.  If a slot
 * occurs twice, what it holds afterwards is not defined: its codes and scales may come from either of the tokens.
 */
int lc_kv_write(const lc_kv_cache* cache, const void* k, const void* v, uint64_t ld_token, uint64_t ld_head, const int64_t* slots,
                uint64_t tokens, int dtype, void* stream);

/* Reads back the tokens at `slots` (int64 [tokens]) into k and v (laid out as for lc_kv_write), each value fl32(q * s)
 * rounded once to dtype; a slot outside the cache reads as zeros. */
int lc_kv_read(const lc_kv_cache* cache, const int64_t* slots, uint64_t tokens, void* k, void* v, uint64_t ld_token, uint64_t ld_head,
               int dtype, void* stream);

/*
 * Attention of nq drafted tokens a sequence over its cached tokens, the drafted ones already written among them:
 *   q, out  [batch][nq][heads][dim] of type dtype, contiguous, 16-byte aligned; heads a multiple of cache->heads, at most 4096, and head h
 *           reads the cache's head h / (heads / cache->heads)
 *   table   int32 [batch][ld_table]: the pages of a sequence, in order; lens int32 [batch]: its cached tokens, of which
 *           the newest nq are the drafted ones (fewer than nq: the drafted tokens that would lie before the first do not exist).
 *           A length is held to what the table has room for (table_pages pages, at most 2^30 tokens); a page outside the cache counts as not seen.
 *   mask    NULL, or uint64 [batch][nq]: drafted token i sees drafted token j iff bit j of mask[i] is set (a tree's ancestors and
 *           itself).  NULL: j <= i.  Everything before the drafted tokens is seen by all of them.  nq is at most 64; nq = 1 is
 *           the step of one token.
 *   out     softmax over the seen tokens of (scale * q . k), times v; zeros where a token sees nothing, NaN where it sees anything with
 *           an infinity or NaN in q.  Scores, maxima and sums are held in 32 bits; probabilities, times the values' scales, enter the product with the values
 *           rounded to nearest with 16 bits or more (fp32: 24), 2^-16 of each at most.  A head's sum of |q|, and |v| summed over the tokens
 *           seen, have to stay below 2^120.  Keys and values that are not seen do not matter, whatever they hold.
 *   ws      scratch, 256-byte aligned, lc_kv_workspace_bytes; its content need not be anything.  Calls that may run at the same
 *           time (on different streams) need areas of their own.
 */
size_t lc_kv_workspace_bytes(uint64_t batch, int nq, int heads, int kv_heads, int dim);
int lc_kv_attend(const lc_kv_cache* cache, const void* q, uint64_t batch, int nq, int heads, const int32_t* table, uint64_t ld_table,
                 uint64_t table_pages, const int32_t* lens, const uint64_t* mask, float scale, void* out, int dtype, void* ws,
                 size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LC_SERVE_H */
