/*
 * fewbit_block.h -- C ABI of the operators around the activation in a
 * transformer block, for AMD MI355X (gfx950); same library as fewbit.h
 * (libfewbit.so) and the same conventions: plain C types, device pointers and
 * a hipStream_t as void*, every buffer the caller's, argument checks on the
 * host before anything is launched, no synchronisation, no device memory of
 * the library's own, no exception across the interface, every call may be
 * captured into a graph, FEWBIT_* status codes and storage types.
 *
 * Three operators, each keeping little for its backward pass:
 *   attention      keeps its output and one number per row; the backward
 *                  recomputes the probabilities
 *   qk_norm_rope   keeps its inputs alone; the backward recomputes the norms
 *   adamw          moments in 8 bits per element (or in 32)
 */
#ifndef FEWBIT_BLOCK_H
#define FEWBIT_BLOCK_H

#include <stdint.h>

#include "fewbit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ */
/* Attention                                                           */
/* ------------------------------------------------------------------ */
/*
 * For query row i and key row j of one sequence and one query head,
 *   s_ij = scale * <q_i, k_j>,  p_ij = exp(s_ij - lse_i) where the mask lets
 *   (i, j) through and 0 elsewhere,  lse_i = log sum_j exp(s_ij),
 *   out_i = sum_j p_ij v_j.
 * A row whose mask leaves nothing has out = 0 and lse = -inf, and gives no
 * gradient.  Query heads share key heads in runs: query head h reads key head
 * h / (heads_q / heads_kv).
 *
 * Sequences.  Fixed: `batch` sequences of rows_q queries and rows_k keys, of
 * which the first k_len[b] are there (k_len, clamped to 0..rows_k; NULL: all
 * of them); rows past them are never read.  Packed (cu_q and cu_k not NULL):
 * tensors of rows_q and rows_k rows hold `batch` sequences one after another;
 * sequence b has the rows cu[b] .. cu[b+1]-1 (the first starts at row 0
 * whatever cu[0] is; bounds are clamped to the tensor and to the one before).
 * Rows past cu[batch] belong to none: they see nothing and nothing sees them.
 *
 * Mask.  With nq queries and nk keys in a sequence, query i stands at key
 * i + nk - nq.  causal: j <= i + nk - nq.  window w > 0 (with causal only):
 * also j > i + nk - nq - w.
 *
 * Layouts.  q, k, v and dout have head_dim elements in a row and strides
 * {sequence, row, head} in elements (packed: the first is not used), each a
 * multiple of 8 and not negative; pointers are 16-byte aligned.  out, dq, dk
 * and dv are dense: [batch,] rows, heads, head_dim.  lse is dense: [batch,]
 * heads_q, rows_q.  A launch has fewer than 2^32 threads: sizes that take more
 * are refused (the backward takes 512 for 128 or 256 keys of a key head).
 *
 * Values of k and v that no row of a sequence sees but that lie inside it
 * have to be finite, and so does dout: masked products are 0 times them.
 *
 * Sums, softmax statistics and gradients are accumulated in fp32.  What the
 * matrix instructions take is rounded to 16 bits once: p and its gradient ds =
 * p (<dout_i, v_j> - <dout_i, out_i>) to the storage type before the products
 * with v and dout, and with k and q.  For dk the p in ds has the 11 bits of
 * fp16, whatever the type, and is 0 below 2^-39.  In fp16 ds is multiplied by
 * a power of two of each row's (dq) or key's (dk) own first, so that small
 * gradients keep their bits and large ones do not pass its range.  <dout_i,
 * out_i> is of out as it was rounded, but for rows that see few keys.  Results
 * do not depend on the order in which anything runs.
 */
typedef struct fewbit_attn {
    int32_t dtype;                /* FEWBIT_F16 / FEWBIT_BF16                  */
    int32_t heads_q, heads_kv;    /* heads_q a multiple of heads_kv            */
    int32_t head_dim;             /* a multiple of 8, 8 .. 128                 */
    int32_t causal;               /* 0 / 1                                     */
    int32_t window;               /* 0: none                                   */
    float scale;                  /* > 0, finite                               */
    int32_t reserved;             /* must be 0                                 */
    int64_t batch;                /* sequences                                 */
    int64_t rows_q, rows_k;       /* per sequence; packed: of all together     */
    const int32_t* cu_q;          /* device, batch + 1 entries, or NULL        */
    const int32_t* cu_k;          /* device, batch + 1 entries, or NULL        */
    const int32_t* k_len;         /* device, batch entries, or NULL            */
    int64_t q_stride[3], k_stride[3], v_stride[3], dout_stride[3];
} fewbit_attn;

/* Bytes of workspace that the forward (backward = 0) or the backward needs;
 * negative: a status. */
int64_t fewbit_attn_workspace(const fewbit_attn* a, int32_t backward);

int fewbit_attn_fwd(const fewbit_attn* a, const void* q, const void* k, const void* v, void* out,
                    float* lse, void* workspace, int64_t workspace_bytes, void* stream);

/* The gradients of q, k and v from out and lse of the forward and out's
 * gradient. */
int fewbit_attn_bwd(const fewbit_attn* a, const void* dout, const void* q, const void* k,
                    const void* v, const void* out, const float* lse, void* dq, void* dk, void* dv,
                    void* workspace, int64_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ */
/* RMS norm of query and key heads with their rotary position           */
/* ------------------------------------------------------------------ */
/*
 * For every token and head, x a row of head_dim elements and w the weight of
 * its kind (queries or keys):
 *   u = x / sqrt(mean(x^2) + eps) * w
 * and the first `rot` elements of u turned by the token's angles: pair t of
 * rot / 2 is (t, t + rot/2), or (2t, 2t+1) if interleaved, and becomes
 *   (a cos - b sin, b cos + a sin),  cos and sin from row `position` of
 * tables with table_rows rows of rot / 2 floats.  The other elements of u are
 * left as they are.  A token whose position is not in the tables gets NaN in
 * its rotated elements (and in its gradient).
 *
 * q and k have head_dim contiguous elements per row and strides {batch, token,
 * head} in elements; rows start at multiples of 16 bytes.  positions (may be
 * NULL: the token's place in its sequence) has 8-byte integers and strides
 * {batch, token}.  Outputs and gradients are dense [batch, tokens, heads,
 * head_dim]; the gradients of the weights are fp32.
 *
 * Everything is computed in fp32 and rounded once.  The weights' gradients
 * are summed in an order that depends on the sizes alone.  batch * tokens *
 * (heads + 1) stays below 2^31, and the forward takes fewer than 2^32 threads: 4,
 * 8 or 16 (head_dim up to 64, 128, 256) for two heads of a token.
 */
typedef struct fewbit_qk {
    int32_t dtype;                /* storage type of q, k and their weights    */
    int32_t heads_q, heads_k;     /* either may be 0                           */
    int32_t head_dim;             /* a multiple of 16, 16 .. 256               */
    int32_t rot;                  /* a multiple of 16, 0 .. head_dim           */
    int32_t interleaved;          /* 0 / 1                                     */
    float eps;                    /* >= 0, finite                              */
    int32_t reserved;             /* must be 0                                 */
    int64_t batch, tokens;
    int64_t table_rows;
    int64_t q_stride[3], k_stride[3];
    int64_t dq_stride[3], dk_stride[3];       /* of the incoming gradients     */
    int64_t position_stride[2];
} fewbit_qk;

int fewbit_qk_fwd(const fewbit_qk* a, const void* q, const void* k, const void* q_weight,
                  const void* k_weight, const float* cos, const float* sin,
                  const int64_t* positions, void* q_out, void* k_out, void* stream);

/* Bytes of workspace that the backward needs; negative: a status.  The gradient
 * of a weight without heads or tokens is 0; that of one without heads may be
 * NULL. */
int64_t fewbit_qk_workspace(const fewbit_qk* a);

int fewbit_qk_bwd(const fewbit_qk* a, const void* dq_out, const void* dk_out, const void* q,
                  const void* k, const void* q_weight, const void* k_weight, const float* cos,
                  const float* sin, const int64_t* positions, void* dq, void* dk,
                  float* dq_weight, float* dk_weight, void* workspace, int64_t workspace_bytes,
                  void* stream);

/* ------------------------------------------------------------------ */
/* AdamW over many tensors                                             */
/* ------------------------------------------------------------------ */
/*
 * For every element of every tensor, in fp32,
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   w = w (1 - lr weight_decay)
 *       - lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps);
 * w is the master copy where there is one, else the parameter; the parameter
 * receives w rounded to its type.
 *
 * Moments lie in two flat buffers: tensor i's start at element 256 B_i, B_i
 * the number of 256-element blocks of the tensors before it (a tensor's last
 * block may be partly used).  The master copy lies alike.
 *   state_bits 32: fp32.
 *   state_bits 8:  8-bit floating point (1 sign, 4 exponent, 3 mantissa bits,
 *     largest 448, no infinity) times one power of two per block and moment,
 *     the least that takes the block's largest finite magnitude to at most
 *     448 (and at least 2^-125).  A value between two codes becomes the upper
 *     one with the probability of its distance from the lower one, so that
 *     the running means, which move by less than a code's step at a time, are
 *     kept in the mean.  A second moment that is not 0 never becomes 0 (an
 *     update divides by its root).  NaN and infinities become NaN.
 *   The probabilities' numbers follow from `seed` and the element's place e
 *   in the buffer alone: x = e * 0x9E3779B1 + seed * 0x6A09E667 + 0x3C6EF372,
 *   x = (x ^ x >> 15) * 0xBB67AE85, x ^= x >> 13, all modulo 2^32; the first
 *   moment's is the high half of x, the second's the low half, over 2^16.
 */
#define FEWBIT_ADAMW_BLOCK 256    /* elements that share a scale; tensors start at whole blocks */

typedef struct fewbit_adamw_tensor {
    void* param;                  /* n elements, contiguous                    */
    const void* grad;             /* n elements in the same order; NULL: the
                                     tensor and its moments stay as they are   */
    int64_t n;                    /* >= 0                                      */
} fewbit_adamw_tensor;

typedef struct fewbit_adamw {
    int32_t param_dtype;          /* FEWBIT_F32 / F16 / BF16                   */
    int32_t grad_dtype;           /* the parameters' or FEWBIT_F32             */
    int32_t state_bits;           /* 8 or 32                                   */
    int32_t reserved;             /* must be 0                                 */
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;                 /* >= 1                                      */
    int64_t seed;                 /* its low 32 bits are used                  */
} fewbit_adamw;

/* m, v: fp32 or 8-bit codes; m_scale, v_scale: one float per block with
 * 8-bit moments, else not used; master: fp32 or NULL.  `tensors` is a host
 * array, read before the call returns.  Takes one launch per 256 tensors (and
 * per 3.4e10 elements); if one fails the earlier ones are done. */
int fewbit_adamw_step(const fewbit_adamw* a, const fewbit_adamw_tensor* tensors, int32_t count,
                      void* m, void* v, float* m_scale, float* v_scale, float* master,
                      void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FEWBIT_BLOCK_H */
