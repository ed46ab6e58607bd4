/*
 * lc_serve.h -- what a program that answers with a restored checkpoint needs next to lc.h: weights held in 4 bits with
 * group scales and their products with activations.  Hand-written HIP kernels for MI355X (gfx950) behind the same C ABI as lc.h.
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
 * exactly.)  An infinity or NaN in x gives what the formula gives.  m may be 0; k = 0 gives the bias.
 */
int lc_w4_matmul(const void* x, uint64_t ldx, uint64_t m, const lc_w4* w4, const void* bias, void* y, uint64_t ldy,
                 int dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LC_SERVE_H */
