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
 *   hc_dropout               dropout, or its gradient, with a residual; the mask
 *                            is made from a seed and a place, and not stored
 *   hc_linear                matrix product with bias, activation, dropout and
 *                            residual
 *   hc_linear_bytes          its workspace
 *   hc_linear_grad           its gradient: of the input, the weight and the bias
 *   hc_linear_grad_bytes     its workspace
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

/* Dropout's masks.  Element (r, c) of a call is dropped where 16 bits, uniform
 * and independent, are below T = round(65536 p); what is kept is scaled by
 * 65536 / (65536 - T).  So p is rounded to a multiple of 2^-16, and below 2^-17
 * nothing is dropped.  The bits depend on seed, draw, r and c alone, not on the
 * shape, the type or the operator: a backward pass gives the same seed and draw
 * and gets the forward pass's mask.  They are those of Philox4x32-10 (Salmon et
 * al. 2011) with key = seed (low word first) and counter = (c div 8, r, draw mod
 * 2^32, draw div 2^32): element c takes half c mod 2 (0: the low one) of word
 * (c mod 8) div 2.  `counter` (DEVICE, or NULL) is a number that is added to
 * draw when the kernels run: a captured graph whose counter goes on between the
 * replays draws a new mask in each. */
typedef struct {
    uint64_t rows;         /* 0 .. 2^31 - 1                                       */
    uint64_t cols;         /* 1 .. 2^31 - 1; at most 2^35 elements in all         */
    uint64_t x_ld, residual_ld, out_ld; /* elements between rows, >= cols          */
    uint64_t seed, draw;   /* a program's seed, and which of its draws this is    */
    float p;               /* probability of a drop, 0 .. 1                       */
    uint32_t reserved;     /* must be 0                                           */
} hc_dropout_params;

/* out = residual + mask * x (residual NULL: mask * x), in 32 bits and rounded
 * once to `type` (HC_T_F32, HC_T_BF16, HC_T_F16: all three buffers').  A dropped
 * element adds nothing, whatever x holds there.  On an output gradient this is
 * the gradient: the residual's is the output's itself.  out may be x or residual
 * (at the same address and stride). */
hc_status hc_dropout(const hc_dropout_params *p, hc_type type, const void *x, const void *residual,
                     void *out, const uint64_t *counter, hipStream_t stream);

/* Activations: max(z, 0), z Phi(z), z s(z), tanh z, s(z) with s the logistic
 * function and Phi the normal distribution's. */
typedef enum {
    HC_ACT_NONE = 0, HC_ACT_RELU = 1, HC_ACT_GELU = 2, HC_ACT_SILU = 3, HC_ACT_TANH = 4,
    HC_ACT_SIGMOID = 5
} hc_act;

/* A layer of n outputs and k inputs on m rows: x [m, k], w [n, k], all else
 * [m, n], rows contiguous.  m n, m k and n k are at most 2^34. */
typedef struct {
    uint64_t m;            /* 0 .. 2^27                                           */
    uint64_t n, k;         /* 1 .. 2^24                                           */
    uint64_t x_ld, w_ld;   /* elements between rows, here and below: at least the
                              columns, at most 2^31                               */
    uint64_t y_ld;         /* of y; of dy in the gradient                         */
    uint64_t z_ld, residual_ld;
    uint64_t dx_ld, dw_ld; /* gradient                                            */
    uint64_t seed, draw;   /* as in hc_dropout; the place is y's                  */
    float p;
    uint32_t act;          /* hc_act                                              */
    float fixed;           /* gradient, int32: units per 1.0 of the fixed point,
                              finite and > 0 (not read otherwise)                 */
    uint32_t reserved;     /* must be 0                                           */
} hc_linear_params;

/* z = x w^T + bias (NULL: none), y = residual (NULL: none) + mask * act(z), with
 * products and sums in fp32 (z is not rounded before act).  All of `type`
 * (HC_T_F32, HC_T_BF16, HC_T_F16).  z (NULL: not wanted) is what the gradient of
 * an activation asks for.  Sums are taken in an order that depends on the shape, the
 * type, the strides and, in 16-bit types, on whether x and w begin at multiples of 16
 * bytes, and on nothing else: two calls agree bit for bit.  (A 16-bit x or w that does
 * not, though its stride is a multiple of 8, is multiplied by a slower way: 170 to 400
 * TFLOP/s.)  Large fp32 products run as three
 * of fp16 parts with fp32 sums: an element of x or w keeps 22 bits if it is no
 * smaller than 2^-29 of the largest in its row, fewer below, none below 2^-51 of it;
 * small ones are fp32 products.  An infinity may come out as NaN.  y may be residual
 * (same address and stride).
 * The workspace does for fewer rows of the same n, k and strides too. */
hc_status hc_linear_bytes(const hc_linear_params *p, hc_type type, size_t *bytes);
hc_status hc_linear(const hc_linear_params *p, hc_type type, const void *x, const void *w,
                    const void *bias, const void *residual, void *y, void *z,
                    const uint64_t *counter, void *ws, size_t ws_bytes, hipStream_t stream);

/* dz = act'(z) * mask * dy, then dx = dz w, dw = dz^T x and db = the sum of dz's
 * rows; each may be NULL (not wanted), and x, w, z where nothing wanted reads
 * them (w: dx; x: dw; z: an activation).  The residual's gradient is dy itself.
 * A dropped element's dz is 0, whatever dy and z hold there.
 * dy, x, w, z and dx: `type`.  z holds what hc_linear wrote there (for HC_ACT_RELU
 * y itself does where there is neither dropout nor residual).
 *   dw and db: g_type, fp32 sums rounded once, or HC_T_I32: a sum times `fixed`,
 * rounded to the nearest whole number, ties to even, saturating at +-(2^31 - 1)
 * (NaN: 0).  accumulate != 0 adds them to what dw and db hold (int32 saturating).
 *   16-bit types: dx, and a 16-bit dw, take dz rounded to `type`; a dw of
 * HC_T_F32 or HC_T_I32 takes it in three bf16 parts (24 bits) or two fp16 ones
 * (22 bits), three or two times the products.  An fp16 dz is held in units of 2^e, the
 * smallest power of two, 1 or more, that dropout's scale times the largest slope (1.13
 * for GELU and SiLU, 1 otherwise) does not exceed: it does not overflow, and below its
 * normal range it is up to 2^(e - 25) off, in two parts 2^(e - 36).  Without activation
 * and dropout dz is dy.  db takes dz unrounded.
 *   m = 0 gives zeros.  Order, fp32 parts (there by the rows of dz and the columns
 * of w, the columns of dz and of x) and infinities as in hc_linear; dx goes by w's
 * stride and address, dw by x's and by g_type, db by neither, all by whether dz is dy,
 * and none by what else is wanted. */
hc_status hc_linear_grad_bytes(const hc_linear_params *p, hc_type type, size_t *bytes);
hc_status hc_linear_grad(const hc_linear_params *p, hc_type type, const void *dy, const void *x,
                         const void *w, const void *z, void *dx, hc_type g_type, void *dw,
                         void *db, int accumulate, const uint64_t *counter, void *ws,
                         size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
