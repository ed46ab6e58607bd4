/*
 * lc_serve.h -- what a program that answers with a restored checkpoint needs next to lc.h: weights held in 4 bits with
 * group scales or in 8 with one a row, and their products with activations; a paged cache of keys and values in 8 or 4 bits,
 * its pages given out and taken back, written, read back and attended to; and drafted tokens judged.  Hand-written HIP kernels for MI355X (gfx950) behind the same C ABI as lc.h.
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
 * A matrix q[n][k] in 8 bits, one scale a row: weights (a row is an output channel) or activations (a row is a token).
 *     s = max |w| * fl32(1/127),  q = rint(fl32(w * fl32(1/s))) limited to [-127, 127], a two's complement byte;  the value meant is q * s.
 * Scales below 2^-126 and rows that are not finite as for lc_w4.  A byte of -128 is never written but is read as what it stands for.
 */
typedef struct lc_i8 {
    void* codes;            /* int8, 16-byte aligned; row i begins at codes + i * pitch */
    float* scales;          /* [n] */
    uint64_t n, k;          /* n at most 2^31 - 1, k at most LC_I8_MAX_K */
    uint64_t pitch;         /* bytes: a multiple of 16, at least k */
} lc_i8;
#define LC_I8_MAX_K 131072  /* so that a sum of k products of codes, of which one side is never -128, fits 32 bits */

/* w [n][k] of type dtype, row i at element i * ldw (ldw >= k), into w8's codes and scales.  Bytes behind a row's end are written as zeros up to the
 * next multiple of 16. */
int lc_i8_quantize(const void* w, uint64_t ldw, int dtype, const lc_i8* w8, void* stream);

/* The values that w8 stands for, each fl32(q * s) rounded once to dtype, into w [n][k] (row i at element i * ldw). */
int lc_i8_dequantize(const lc_i8* w8, void* w, uint64_t ldw, int dtype, void* stream);

/*
 * y[i][j] = (sum over l of qx[i][l] * qw[j][l]) * sx[i] * sw[j], plus bias[j] if bias is not NULL: x8 [m][k] with m at most 2^19, w8 [n][k], bias [n] and
 * y [m][n] (row i at element i * ldy) of type dtype.  The sum of codes is exact, rounded once to 32 bits, multiplied by x's scale and then by w's in 32 bits (the sum times
 * x's scale has to stay below 2^128), and y is rounded once more.  Bytes of a row of x8 behind k
 * have to be zeros up to the next multiple of 16, as lc_i8_quantize leaves them; those of w8 may be anything.
 */
int lc_i8_matmul(const lc_i8* x8, const lc_i8* w8, const void* bias, void* y, uint64_t ldy, int dtype, void* stream);

/*
 * The same for x [m][k] of type dtype, row i at element i * ldx: its rows are put into 8 bits first, as by lc_i8_quantize, with the same results.  ws: scratch,
 * 256-byte aligned, lc_i8_workspace_bytes(m, k); its content need not be anything.  Calls that may run at the same time need areas of their own.
 */
size_t lc_i8_workspace_bytes(uint64_t m, uint64_t k);
int lc_i8_linear(const void* x, uint64_t ldx, uint64_t m, const lc_i8* w8, const void* bias, void* y, uint64_t ldy, int dtype, void* ws, size_t ws_bytes,
                 void* stream);

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

/*
 * The same attention for the new tokens of several prompts, or pieces of them, of any number each:
 *   q, out  [tokens][heads][dim] of type dtype, token i at element i * ld (a multiple of 8; of 4 for LC_F32), 16-byte aligned; tokens at most 2^24, heads as above,
 *           tokens * heads at most 2^30
 *   starts  int32 [batch + 1], none below the one before it, in [0, tokens]: sequence b's new tokens are starts[b] .. starts[b + 1] - 1, in order.  Rows of out that
 *           belong to no sequence are left as they were.
 *   table, lens, scale: as above; the newest cached tokens of a sequence are the new ones, and each sees what is cached up to itself.  A new token
 *           that would lie before the first cached one gets zeros.
 * Keys and values that a token does not see do not matter, whatever they hold (in bf16 and fp16 as long as no scale of a later token's value, among the 64 that begin at a multiple of 64, is
 * above 2^90 times the largest that it sees).
 * Roundings: probabilities times the values' scales are rounded once, in bf16 and fp16 to 11 bits, or to 2^-31 of the largest scale that the token sees times its largest probability, if that is
 * more; in fp32 to 24.  Sums, maxima and scores are held in 32 bits, with the ranges of lc_kv_attend.
 * ws: scratch, 256-byte aligned, lc_kv_prompt_workspace_bytes of these very sizes: fewer tokens may need more (rows enough to fill the chip are not split).  An area for calls of
 * several sizes has lc_kv_prompt_workspace_most, which is enough for every call of up to that many tokens and sequences.
 */
size_t lc_kv_prompt_workspace_bytes(uint64_t tokens, uint64_t batch, int heads, int kv_heads, int dim);
size_t lc_kv_prompt_workspace_most(uint64_t tokens, uint64_t batch, int heads, int kv_heads, int dim);
int lc_kv_attend_prompt(const lc_kv_cache* cache, const void* q, uint64_t ld_q, uint64_t tokens, int heads, const int32_t* starts, uint64_t batch,
                        const int32_t* table, uint64_t ld_table, uint64_t table_pages, const int32_t* lens, float scale, void* out, uint64_t ld_out, int dtype,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * The pages of sequences that share a cache.  table and lens are those that attention takes; free_pages is a stack of the pages that nobody has, with
 * *free_count of them (both on the device), the next one to be given out last.  No page is on the stack twice, and none has two owners: a page that two rows of the
 * table name would go back twice.
 */
typedef struct lc_kv_pages {
    int32_t* table;         /* [batch][ld_table]; entries behind a sequence's pages may hold anything */
    int32_t* lens;          /* [batch] cached tokens, a negative number counts as 0 */
    int32_t* free_pages;    /* [free_room] */
    int32_t* free_count;    /* [1], held to [0, free_room] */
    uint64_t batch;         /* at most 65535 */
    uint64_t ld_table, table_pages;     /* table_pages * page_tokens at most 2^30 */
    uint64_t free_room;     /* at most 2^31 - 1 */
    int page_tokens;        /* a power of two, 8 to 1024 */
} lc_kv_pages;

/*
 * Room for add[b] (int32 [batch]; not above 0: none) more tokens of every sequence: the pages that it needs are taken off the stack, in order of the sequences and of
 * the tokens, and written into the table.  A sequence that has no room in its row of the table, for which the stack does not suffice, or whose tokens would pass
 * `room`, gets nothing, and neither do those behind it.  Then
 *   new_lens [batch], new_count [1]   the lengths with the tokens that found room, and what is left on the stack; may be lens and free_count themselves
 *   starts   int32 [batch + 1]        where each sequence's new tokens begin among all that found room
 *   slots    int64 [room]             of each new token its slot (page * page_tokens + token), -1 behind the last one
 *   places   int32 [room]             its place in the sequence, or -1;  owners int32 [room]: the sequence, or -1.  Either may be NULL.
 * The stack itself is read only.  One call at a time on the same pages.
 */
int lc_kv_extend(const lc_kv_pages* pages, const int32_t* add, uint64_t room, int32_t* new_lens, int32_t* new_count, int32_t* starts, int64_t* slots,
                 int32_t* places, int32_t* owners, void* stream);

/*
 * Of every sequence the first keep[b] tokens stay (int32 [batch]; at most its length, a negative number counts as 0), and the pages behind them go back on the stack, the
 * last one first: what an extension took, taken back, leaves the stack as it was.  The table is read only.  Pages for which the stack has no room are lost.
 * new_lens and new_count as for lc_kv_extend.
 */
int lc_kv_trim(const lc_kv_pages* pages, const int32_t* keep, int32_t* new_lens, int32_t* new_count, void* stream);

/*
 * Drafted tokens judged against the model's probabilities, with given random numbers, so that what is written has the model's distribution:
 *   target  [batch][nodes][vocab] of type dtype: the model's probabilities behind each node; row (b, i) at element b * ld_batch + i * ld_row (rows may share memory).  nodes 1 to 64, vocab 1 to 2^24.
 *           Values that are negative or not finite count as zero.
 *   tokens  int32 [batch][nodes].  Node 0 is the token that is known (its number is not looked at); a number outside the vocabulary has probability zero.
 *   draft   the probabilities that the tokens of nodes 1, 2 ... were drawn from, [batch][nodes - 1][vocab] with pitches of its own, or NULL: the tokens are
 *           guesses that nothing was drawn for
 *   parent  int32 [batch][nodes], only without draft: the node below which each was drafted, smaller than itself; NULL: the one before.
 *   count   NULL, or int32 [batch]: how many of the nodes exist (held to 1 .. nodes)
 *   uniform fp32 [batch][nodes], in [0, 1)
 * The path begins with node 0.  Below its end nodes are tried in order.  With draft, i is taken if uniform[i] * q(token i) < p(token i), with p behind the path's end and
 * q that i was drawn from; else the path ends, and what is left is max(p - q, 0).  Without, i is taken if uniform[i] * rest < p(token i), where rest is 1 less the
 * probabilities of what was refused here before, and those tokens are left out of p (the same token refused again has probability zero).  A node without
 * nodes below it leaves p.  Then
 *   path    int32 [batch][nodes]: the nodes of the path, -1 behind them;  length int32 [batch]: how many
 *   next    int32 [batch]: the first token at which the running sum of what is left exceeds uniform[0] times all of it; where nothing is left, of p; where that is zero
 *           everywhere, -1
 * Sums are held in 64 bits.  ws: scratch, 256-byte aligned, lc_draft_workspace_bytes(batch); its content need not be anything.  Calls that may run
 * at the same time need areas of their own.
 */
size_t lc_draft_workspace_bytes(uint64_t batch);
int lc_draft_verify(const void* target, uint64_t ld_batch, uint64_t ld_row, uint64_t batch, int nodes, uint64_t vocab, const int32_t* tokens, const void* draft,
                    uint64_t ld_draft_batch, uint64_t ld_draft_row, const int32_t* parent, const int32_t* count, const float* uniform, int dtype,
                    int32_t* path, int32_t* length, int32_t* next, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LC_SERVE_H */
