/*
 * fewbit_residual.h -- C ABI of the operators between the products of a
 * transformer block, and of the product in 8-bit integers, for AMD MI355X
 * (gfx950); same library as fewbit.h (libfewbit.so) and the conventions of
 * fewbit_block.h: plain C types, device pointers and a hipStream_t as void*,
 * every buffer the caller's, argument checks on the host before anything is
 * launched, no synchronisation, no device memory of the library's own, no
 * exception across the interface, every call may be captured into a graph,
 * FEWBIT_* status codes and storage types.
 *
 *   dropout        from a counter: the backward forms the mask again
 *   rnorm          dropout of a branch, its addition to the residual stream and
 *                  the RMS norm of the sum; keeps the sum alone, which the next
 *                  addition reads anyway.  For serving, the norm's result in 8
 *                  bits with a scale per token
 *   rows8          any rows in 8 bits with a scale per row
 *   mm8            the product of such rows with weights in 8 bits
 *
 * Pointers are 16-byte aligned, but for rnorm's and rows8's `scale`, dw and a
 * seed's place, which need no more than their type.
 */
#ifndef FEWBIT_RESIDUAL_H
#define FEWBIT_RESIDUAL_H

#include <stdint.h>

#include "fewbit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ */
/* Dropout                                                             */
/* ------------------------------------------------------------------ */
/*
 * With t = p * 65536 rounded to the nearest whole number (p is taken in steps
 * of 2^-16), element e of a tensor of n is kept where u_e >= t and then
 * multiplied by 65536 / (65536 - t), else it becomes 0 whatever it was; the
 * gradient is the same function of the incoming one.  u_e has 16 bits: of the
 * generator Philox 4x32 with 7 rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw,
 * "Parallel random numbers: as easy as 1, 2, 3", 2011) with key (low, high
 * word of the seed) and counter (low, high word of e / 8, site, 0), word
 * e % 8 / 2 of the result, its low half for even e.
 *
 * The seed is `seed`, or what is at *seed_at on the device when the kernels
 * run: a graph that is replayed draws anew where its program has changed that.
 * `site` tells apart places of a program that share a seed.
 */
typedef struct fewbit_drop {
    double p;                     /* 0 .. 1                                    */
    int64_t seed;
    const int64_t* seed_at;       /* device, or NULL                           */
    uint32_t site;
    uint32_t reserved;            /* must be 0                                 */
} fewbit_drop;

/* y may be x; both are 16-byte aligned.  n is at most 2^37 - 8192
 * (a launch has fewer than 2^32 threads). */
int fewbit_dropout(const fewbit_drop* d, int32_t dtype, int64_t n, const void* x, void* y,
                   void* stream);

/* ------------------------------------------------------------------ */
/* Residual addition with RMS norm; rows in 8 bits                      */
/* ------------------------------------------------------------------ */
/*
 * For every row of `width` elements,
 *   h = residual + dropout(x) rounded to the storage type,
 *   y = h r w,  r = 1 / sqrt(mean(h^2) + eps),  of h as it was rounded.
 * Dropout counts the elements of x as if it were dense.  residual may be NULL:
 * h = dropout(x), and where p takes nothing away either h is x and is not
 * written.
 *
 * In 8 bits: with a = h w and m = max |a| over the row,
 *   code = 127 a / m to the nearest whole number, halves to the even one,
 *   scale = r m / 127,  so that code * scale stands for y;
 * for rows8 a = x and r = 1.  Codes are exact: of 16-bit storage no rounding
 * lies between h and w and their code, as long as h w is not below fp32's
 * normal range (of fp32 those of 64-bit products).  A row of zeros has codes
 * and scale 0; a row that holds a NaN or an infinity (in h w) has codes 0 and
 * scale NaN.
 *
 * Backward, from dh and dy, the gradients of h and y (dh may be NULL: 0):
 *   g = dy w,  dresidual = dh + r (g - h r^2 mean(g h)),
 *   dx = dropout of dresidual before it is rounded,  dw = sum over rows of dy h r.
 *
 * Squares are formed in fp32: magnitudes past 2^63 make r 0, those below 2^-63
 * count only as far as eps lets them.  With eps = 0 a row of zeros has no r: y
 * and the gradients are NaN, as the formulas make them (codes and scale are 0).
 *
 * x, residual, dh and dy have `width` contiguous elements per row and strides
 * {outer, row} in elements; rows start at multiples of 16 bytes.  h, y, dx and
 * dresidual are dense, as are codes; scale has one float per row.  Everything
 * is computed in fp32 and rounded once; dw is summed in an order that depends
 * on the sizes alone.  outer * rows stays below 2^31, and a launch has fewer than
 * 2^32 threads: 64 a row of up to 2048 elements, 256 up to 8192, 1024 beyond.
 */
#define FEWBIT_RNORM_MOST 32768   /* elements of a row                         */

typedef struct fewbit_rnorm {
    int32_t dtype;                /* storage type of all but scale (and dw)    */
    int32_t width;                /* a multiple of 8, 8 .. FEWBIT_RNORM_MOST   */
    int64_t outer, rows;
    int64_t x_stride[2], residual_stride[2];
    int64_t dh_stride[2], dy_stride[2];
    float eps;                    /* >= 0, finite                              */
    int32_t dw_dtype;             /* storage type of dw: FEWBIT_F32 or dtype   */
    fewbit_drop drop;             /* p = 0: none                               */
} fewbit_rnorm;

int fewbit_rnorm_fwd(const fewbit_rnorm* a, const void* x, const void* residual, const void* w,
                     void* h, void* y, void* stream);

/* No dropout here: drop.p has to be 0. */
int fewbit_rnorm_int8(const fewbit_rnorm* a, const void* x, const void* residual, const void* w,
                      void* h, int8_t* codes, float* scale, void* stream);

/* Of a, dtype, width, outer, rows and x_stride are used. */
int fewbit_rows8(const fewbit_rnorm* a, const void* x, int8_t* codes, float* scale, void* stream);

/* Bytes of workspace that the backward needs; negative: a status. */
int64_t fewbit_rnorm_workspace(const fewbit_rnorm* a);

/* dresidual may be NULL: it is not written then.  Where p takes nothing away
 * dx is it, and dresidual has to be NULL. */
int fewbit_rnorm_bwd(const fewbit_rnorm* a, const void* dh, const void* dy, const void* h,
                     const void* w, void* dx, void* dresidual, void* dw, void* workspace,
                     int64_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ */
/* Product in 8-bit integers                                           */
/* ------------------------------------------------------------------ */
/*
 *   y[m][n] = act(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n])
 * The sum is exact (32-bit integers: width up to 131056); the rest is formed in
 * fp32, the sum times x_scale first, and rounded once: x_scale from 2^-126 to
 * 2^96, where such a product neither vanishes nor overflows, w_scale any.
 * act: FEWBIT_MM8_LINEAR, or FEWBIT_GELU or FEWBIT_SILU of fewbit.h.
 *
 * x and w have `width` contiguous codes per row and rows that start at
 * multiples of 16 bytes, at most FEWBIT_MM8_STRIDE apart; the scales are dense, bias (may
 * be NULL) has the type of y, and y is dense.  Codes may be -128.  rows and out stay
 * below 2^31, and what a launch takes below 2^32 threads (512 for 256 x 256 results
 * where there are many).
 */
#define FEWBIT_MM8_LINEAR (-1)
#define FEWBIT_MM8_STRIDE 8388608  /* 2^23 */

typedef struct fewbit_mm8 {
    int32_t dtype;                /* of y and bias                             */
    int32_t act;
    int64_t rows, out;
    int32_t width;                /* a multiple of 16, 16 .. 131056            */
    int32_t reserved;             /* must be 0                                 */
    int64_t x_stride, w_stride;
} fewbit_mm8;

/* Bytes of workspace that the product needs; negative: a status. */
int64_t fewbit_mm8_workspace(const fewbit_mm8* a);

int fewbit_mm8_fwd(const fewbit_mm8* a, const int8_t* x, const float* x_scale, const int8_t* w,
                   const float* w_scale, const void* bias, void* y, void* workspace,
                   int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FEWBIT_RESIDUAL_H */
