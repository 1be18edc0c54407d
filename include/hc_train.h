/*
 * hc_train.h -- C ABI of the training-side operators around the compressed
 * aggregation of hc.h, in the same library (libhc.so, gfx950): what makes the
 * row-sparse gradients that compress best, and what takes a recovered sum to
 * the weights.
 *
 *   hc_embed                 embedding lookup with scaling
 *   hc_embed_grad            its gradient, dense: the token ids are sorted and
 *                            the gradients of equal ids summed in a fixed order
 *   hc_embed_grad_rows       the same for the touched rows alone
 *   hc_embed_grad_bytes      workspace of both
 *   hc_orthogonalise         Newton-Schulz orthogonalisation of matrices, as
 *                            the Muon optimiser does with an update
 *   hc_orthogonalise_bytes   its workspace
 *
 * The conventions are those of hc.h: device pointers unless marked "host",
 * memory owned by the caller, calls asynchronous on `stream`, errors returned
 * as hc_status before anything is enqueued, messages by hc_last_error().
 * Workspaces are 256-byte aligned, their contents on entry ignored; a
 * workspace belongs to one call at a time.  Data need the alignment of their
 * element type (16-byte aligned rows are fastest).  Outputs may not overlap
 * inputs or the workspace.
 */
#ifndef HC_TRAIN_H
#define HC_TRAIN_H

#include "hc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types; the first two are hc_vtype's. */
typedef enum { HC_T_I32 = 0, HC_T_F32 = 1, HC_T_BF16 = 2, HC_T_F16 = 3 } hc_type;

/* A table of `vocab` rows of `dim` elements and `count` token ids. */
typedef struct {
    uint64_t vocab;     /* rows of the table, 1 .. 2^31 - 1                       */
    uint64_t count;     /* token ids, 0 .. 2^31 - 1 (gradients: 2^30)             */
    uint64_t dim;       /* elements of a row, 1 .. 2^22                           */
    uint64_t table_ld;  /* elements between rows of the table, of its gradient or
                           of the rows' values, >= dim                            */
    uint64_t x_ld;      /* elements between rows of the lookups or of their
                           gradient, >= dim                                       */
    int64_t padding;    /* an id whose row gets no gradient; negative: none       */
    uint32_t id_bits;   /* 32 or 64: token ids are int32 or int64                 */
    uint32_t reserved;  /* must be 0                                              */
    float scale;        /* factor of the lookup and of its gradient, finite       */
    float fixed;        /* int32 gradients: units per 1.0 of the fixed point,
                           finite and > 0 (not read otherwise)                    */
} hc_embed_params;

/* out[i] = scale * table[ids[i]] for i < count, in 32 bits and rounded once to
 * `type` (HC_T_F32, HC_T_BF16 or HC_T_F16: the table's and out's).  An id
 * outside [0, vocab) reads nothing and gives a row of zeros.  `padding` is not
 * looked at. */
hc_status hc_embed(const hc_embed_params *p, hc_type type, const void *table, const void *ids,
                   void *out, hipStream_t stream);

/* Workspace bytes (HOST pointer) of the two gradient calls, for any types; they
 * do for fewer ids of the same vocab and dim too. */
hc_status hc_embed_grad_bytes(const hc_embed_params *p, size_t *bytes);

/* dtable[v] = scale * sum of dout[i] over the i with ids[i] = v, for all v <
 * vocab; ids outside [0, vocab) and the padding id add nothing.  dout: x_type
 * (HC_T_F32, HC_T_BF16, HC_T_F16); dtable: g_type.
 *   HC_T_F32, HC_T_BF16, HC_T_F16  products and sums in fp32, summed in an
 *       order that depends on the ids alone (two calls agree bit for bit) and
 *       rounded once.
 *   HC_T_I32  the fixed point that the int32 encodes take: every contribution
 *       scale * dout * fixed (two fp32 products) is rounded to the nearest
 *       whole number, ties to even, saturating at +-(2^31 - 1) (NaN: 0), and
 *       their 64-bit sum saturates the same way.  Exact, so free of any order.
 * accumulate = 0 writes every row (zeros where no id points); otherwise the
 * sums are added to what dtable holds (a tied head's gradient, an earlier
 * micro-batch's) and untouched rows are left alone. */
hc_status hc_embed_grad(const hc_embed_params *p, hc_type x_type, const void *dout,
                        const void *ids, hc_type g_type, void *dtable, int accumulate, void *ws,
                        size_t ws_bytes, hipStream_t stream);

/* The touched rows alone: rows[u] (uint32, ascending) are the distinct valid
 * ids and values[u * table_ld ..] their sums as above, for u < cap; entries
 * past cap are not written (cap = 0: rows and values may be NULL).  *touched
 * (uint32, DEVICE) is how many there are, at most min(count, vocab).  Row r's
 * elements are parameters r * dim .. of a flat gradient: with its index expanded
 * this is hc_encode_coo's input. */
hc_status hc_embed_grad_rows(const hc_embed_params *p, hc_type x_type, const void *dout,
                             const void *ids, hc_type g_type, uint32_t *rows, void *values,
                             uint64_t cap, uint32_t *touched, void *ws, size_t ws_bytes,
                             hipStream_t stream);

/* `batch` matrices of m x n, rows contiguous.  Matrix b's row i starts at
 * x + b * x_stride + i * x_ld elements. */
typedef struct {
    uint64_t m, n;        /* 1 .. 65536 each                                      */
    uint64_t batch;       /* 0 .. 65535                                           */
    uint64_t x_ld, x_stride;      /* elements; x_ld >= n                          */
    uint64_t out_ld, out_stride;  /* the same of the output, whose matrices lie one
                                     after the other, or all their rows i before
                                     any row i + 1                                */
    uint32_t type;        /* hc_type of x and out: HC_T_F32 or HC_T_BF16          */
    uint32_t steps;       /* Newton-Schulz steps, 0 .. 32                         */
    const float *coeffs;  /* HOST: a, b, c of each step (3 * steps values), or
                             NULL: 3.4445, -4.7750, 2.0315 in every step          */
    float eps;            /* added to the norm, 2^-100 or more                    */
    float scale;          /* factor of the output, finite                         */
} hc_orthogonalise_params;

/* out = scale * X_steps with X_0 = x / (|x|_F + eps) and
 *   X_{t+1} = a X_t + (b A + c A^2) X_t,  A = X_t X_t^T
 * (or from the right with X_t^T X_t where m > n: the same matrix).  Singular
 * values s of X_t become a s + b s^3 + c s^5; the default coefficients (Muon's,
 * Jordan et al. 2024) bring those above a few thousandths to about 1 in five
 * steps.  Works on the matrix cores with sums in 32 bits.  HC_T_F32, and
 * HC_T_BF16 whose shorter side is at most 256: operands of two times 11 bits, X
 * in fp32 between the steps: in the 2-norm five steps are 1e-6 to 9e-6 from the
 * exact result, before a bf16 result is rounded.  HC_T_BF16 otherwise: operands
 * of 11 bits, X as an operand and an 11-bit rest (22 bits, none below 2^-38): with
 * the result's rounding (1.7e-3) five steps are 1.8e-3 to 2.7e-3 off, twelve up to
 * 7e-3; matrices all of whose elements are below about 1e-10 eps lose more, and
 * below 1e-12 eps give zeros.  HC_T_F32 has no such limit.  The coefficients must
 * keep the bound on the singular values (1, mapped through every step) within
 * 2^-10 .. 2^10 and b A + c A^2 within 2^10 (HC_EUNSUPPORTED).  NaN or infinity
 * in a matrix makes that matrix's output NaN; other matrices are unaffected. */
hc_status hc_orthogonalise_bytes(const hc_orthogonalise_params *p, size_t *bytes);
hc_status hc_orthogonalise(const hc_orthogonalise_params *p, const void *x, void *out, void *ws,
                           size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
