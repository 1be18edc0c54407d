// hc_train_internal.h -- host-side launchers of the training-side kernels
// (internal to libhc; the public surface is include/hc_train.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/hc_train.h"

namespace hc {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// ---- embedding -------------------------------------------------------------------

hipError_t launch_embed(const hc_embed_params& p, hc_type type, const void* table, const void* ids,
                        void* out, hipStream_t s);

size_t embed_grad_bytes(const hc_embed_params& p);

// Dense: dst is the table's gradient.  By rows: dst is the values, and
// rows/cap/touched are as in hc_embed_grad_rows.
struct EmbedGradOut {
    void* dst;
    hc_type type;
    bool accumulate, by_rows;
    uint32_t* rows;
    uint64_t cap;
    uint32_t* touched;
};
hipError_t launch_embed_grad(const hc_embed_params& p, hc_type x_type, const void* dout,
                             const void* ids, const EmbedGradOut& out, void* ws, hipStream_t s);

// ---- orthogonalisation -----------------------------------------------------------

// Powers of two by which a step's operands are held in fp16 (x, A = X X^T and
// b A + c A^2), and the step's coefficients.
struct OrthoStep {
    float a, b, c;
    int ex, ea, eb;
    int ex_next;  // of the X that the step makes
};
constexpr int kOrthoMaxSteps = 32;

size_t orthogonalise_bytes(const hc_orthogonalise_params& p);
hipError_t launch_orthogonalise(const hc_orthogonalise_params& p, const OrthoStep* steps,
                                const void* x, void* out, void* ws, hipStream_t s);

}  // namespace hc
