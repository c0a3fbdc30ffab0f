/*
 * lsgd_layers.h - the ends of the step's buffers in a language model, exported
 * by liblsgd.so: what a worker computes from the parameters that the step
 * copies out, and what it writes into the gradient buffers that the step reads,
 * for the two kinds of parameters that make up nearly all of such a model.
 *
 *   token table     lsgd_embed_lookup reads rows of a copy, lsgd_embed_grad
 *                   writes the table's gradient: one worker's (an input of
 *                   lsgd_step), or the mean over many (what lsgd_sgd_step takes).
 *   linear layers   lsgd_copy_out8 writes copies of the parameters in 8 bits,
 *                   lsgd_quant8 brings activations into 8 bits, lsgd_matmul8
 *                   multiplies the two, lsgd_weight_grad8 computes the gradient
 *                   of the parameters from the 8-bit activations, which are all
 *                   that the forward pass has to keep.
 *
 * 8-bit tensors. A matrix of `rows` by `cols` is held as
 *   codes   rows x pitch bytes, pitch = lsgd_pitch8(cols) = cols rounded up to a
 *           multiple of 128; each byte a number of 1 sign, 4 exponent and 3
 *           mantissa bits (e4m3, largest 448, no infinity, NaN = 0x7f or
 *           0xff); columns from `cols` on hold 0.
 *   scales  ceil(rows/block) x lsgd_scale_pitch8(cols) bytes (ceil(cols/128)
 *           rounded up to a multiple of 4); byte x stands for 2^(x-127); one for
 *           each `block` rows by 128 columns, block 1 (activations) or 128
 *           (parameters); bytes behind the last block of columns hold 127.
 * An element is code * scale. The scale of a block whose largest finite
 * magnitude is A > 0 is 2^e with the smallest e in [-126, 127] for which
 * A / 2^e <= 448, and 1 for A = 0; elements are divided by it exactly and
 * rounded to the nearest code, ties to the even one; NaN and infinities become
 * NaN. (A power of two costs a floating format no relative precision, is
 * divided by and multiplied with exactly, and makes a transposed copy hold the
 * same numbers.) Scales made elsewhere may be bytes 1 to 254.
 *
 * The conventions of lsgd.h hold (memory, streams, validation, aliasing,
 * errors; every matrix is contiguous, row-major): buffers are 16-byte aligned,
 * arrays of tokens aligned to their elements. Results do not depend on
 * scheduling: the same call on the same data gives the same bits.
 */
#ifndef LSGD_LAYERS_H
#define LSGD_LAYERS_H

#include "../lsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lsgd_index_type {
    LSGD_I32 = 0, /* int32_t */
    LSGD_I64 = 1  /* int64_t */
} lsgd_index_type;

/*
 * Rows of a token table, scaled:
 *   out[i][j] = scale * table[tokens[i]][j],  0 where tokens[i] is outside [0, rows)
 * (binary32 product, rounded once to odt, nearest-even).
 * table  rows x dim elements of dtype tdt (a copy of the parameters, or the
 *        parameters); tokens  n_tokens indices; out  n_tokens x dim of odt.
 * n_tokens == 0 or dim == 0 is a no-op. Errors: LSGD_ERR_DTYPE, LSGD_ERR_SIZE (a
 * negative size, rows, dim or n_tokens above 2^31 - 1), LSGD_ERR_NULL,
 * LSGD_ERR_ALIGN, LSGD_ERR_ALIAS, LSGD_ERR_HIP.
 */
LSGD_API lsgd_status lsgd_embed_lookup(const void* table, lsgd_dtype tdt, int64_t rows,
                                       int64_t dim, const void* tokens, lsgd_index_type it,
                                       int64_t n_tokens, float scale, void* out, lsgd_dtype odt,
                                       void* stream);

/*
 * The gradient of lsgd_embed_lookup's table, summed over n_workers workers:
 *   out[v][j] = scale * sum of grads[w][i][j] over all w, i with tokens[w][i] == v
 *               (+ out[v][j] if accumulate is nonzero)
 * Every row of out is written (rows that no token names become 0); with
 * accumulate only those that a token names. Tokens outside [0, rows) are
 * skipped, and so are their gradients, whatever they hold.
 * One worker with the scale of its lookup gives that worker's gradient buffer;
 * all workers of equal groups with that scale / n_workers give the mean
 * gradient of Alg. 2, the grad_mean of lsgd_sgd_step, without a buffer of the
 * table's size for each worker.
 * grads   [n_workers] device pointers, each n_tokens x dim of dtype gdt.
 * tokens  [n_workers] device pointers, each n_tokens indices.
 * out     rows x dim of dtype odt.
 * Sums are binary32, in an order that the tokens alone decide (by worker, then
 * position, in pieces), times scale, rounded once to odt.
 * workspace: device memory of at least lsgd_embed_grad_workspace_size bytes,
 * 256-byte aligned; its contents are not needed between calls, and calls that
 * share one must be ordered on one stream.
 * 1 <= n_workers <= LSGD_MAX_WORKERS; n_workers * n_tokens at most 2^28, rows below
 * 2^31, dim at most 2^24. lsgd_embed_grad_workspace_size may give 0 bytes (few
 * tokens), and workspace may then be NULL.
 * Errors as lsgd_embed_lookup.
 */
LSGD_API lsgd_status lsgd_embed_grad_workspace_size(int32_t n_workers, int64_t n_tokens, int64_t rows,
                                                    int64_t dim, size_t* bytes);

LSGD_API lsgd_status lsgd_embed_grad(const void* const* grads, lsgd_dtype gdt,
                                     const void* const* tokens, lsgd_index_type it,
                                     int32_t n_workers, int64_t n_tokens, int64_t rows, int64_t dim,
                                     float scale, void* out, lsgd_dtype odt, int32_t accumulate,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* Bytes from one row of codes to the next, and of scales. */
LSGD_API int64_t lsgd_pitch8(int64_t cols);
LSGD_API int64_t lsgd_scale_pitch8(int64_t cols);

/*
 * Activations in 8 bits, block 1: codes and scales (see above) of x, rows x cols
 * of dtype xdt. rows == 0 or cols == 0 is a no-op. Errors as lsgd_embed_lookup.
 */
LSGD_API lsgd_status lsgd_quant8(const void* x, lsgd_dtype xdt, int64_t rows, int64_t cols,
                                 void* codes, void* scales, void* stream);

/*
 * lsgd_copy_out in 8 bits, block 128: every one of the n_replicas copies
 * receives the codes and scales of params (rows x cols, binary32), and every
 * one of the n_transposed copies those of its transpose (cols x rows: codes of
 * pitch lsgd_pitch8(rows)), which the gradient of a layer's input needs. The
 * arrays are host arrays of device pointers (NULL for a count of 0). Counts in
 * [0, LSGD_MAX_REPLICAS]; rows at most 65535 * 128. No-op where rows or cols is 0,
 * or both counts are.
 * Errors as lsgd_embed_lookup.
 */
LSGD_API lsgd_status lsgd_copy_out8(const float* params, int64_t rows, int64_t cols,
                                    void* const* codes, void* const* scales, int32_t n_replicas,
                                    void* const* codes_t, void* const* scales_t,
                                    int32_t n_transposed, void* stream);

/*
 * The product of two 8-bit matrices over their columns:
 *   out[i][j] = sum over c < k of a[i][c] * b[j][c]
 * a: m x k, b: n x k (codes and scales as above, a_block and b_block 1 or 128,
 * else LSGD_ERR_UNSUPPORTED; k at most 2^23); out: m x n of dtype odt. With activations a and
 * parameters b: a layer's output; with an output gradient a and transposed
 * parameters b: the gradient of its input.
 * Products are exact, sums binary32, rounded once to odt (matrix instructions on
 * bfloat16, which holds every element between 2^-126 and 2^128 exactly;
 * smaller ones may count as 0).
 * k == 0 gives 0. No-op where m or n is 0. Errors as lsgd_embed_lookup.
 */
LSGD_API lsgd_status lsgd_matmul8(const void* a, const void* a_scales, int32_t a_block, int64_t m,
                                  const void* b, const void* b_scales, int32_t b_block, int64_t n,
                                  int64_t k, void* out, lsgd_dtype odt, void* stream);

/*
 * The gradient of a linear layer's parameters from its activations in 8 bits:
 *   out[j][c] = sum over i < m of grad[i][j] * x[i][c]  (+ out[j][c] if accumulate)
 * grad: m x n, bfloat16 (the gradient of the layer's output); x: m x k in 8
 * bits, block 1; out: n x k of dtype odt, a worker's gradient buffer; n and k at
 * most 2^24. Products
 * are exact (elements of x between 2^-126 and 2^128), sums binary32, rounded
 * once to odt. m == 0 gives 0 (with accumulate: a no-op); no-op where n or k is 0.
 * workspace as for lsgd_embed_grad; lsgd_weight_grad8_workspace_size may give 0
 * bytes, and workspace may then be NULL. Errors as lsgd_embed_lookup.
 */
LSGD_API lsgd_status lsgd_weight_grad8_workspace_size(int64_t m, int64_t n, int64_t k,
                                                      size_t* bytes);

LSGD_API lsgd_status lsgd_weight_grad8(const void* grad, const void* x, const void* x_scales,
                                       int64_t m, int64_t n, int64_t k, void* out, lsgd_dtype odt,
                                       int32_t accumulate, void* workspace, size_t workspace_bytes,
                                       void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LSGD_LAYERS_H */
