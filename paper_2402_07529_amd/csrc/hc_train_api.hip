// hc_train_api.hip -- the C ABI of include/hc_train.h: argument validation,
// workspace sizing and launches.  Host code only.
#include <math.h>

#include "hc_internal.h"
#include "hc_train_internal.h"

namespace hc {

namespace {

size_t type_bytes(uint32_t t) { return t == HC_T_I32 || t == HC_T_F32 ? 4 : 2; }
bool float_type(uint32_t t) { return t == HC_T_F32 || t == HC_T_BF16 || t == HC_T_F16; }

hc_status check_embed(const hc_embed_params* p, uint64_t max_count) {
    if (p == nullptr) return fail(HC_EINVAL, "params is NULL");
    if (p->vocab < 1 || p->vocab > 0x7fffffffull) return fail(HC_EINVAL, "vocab must be in [1, 2^31 - 1]");
    if (p->count > max_count)
        return fail(HC_EINVAL, "count must be at most 2^31 - 1 (gradients: 2^30)");
    if (p->dim < 1 || p->dim > (1ull << 22)) return fail(HC_EINVAL, "dim must be in [1, 2^22]");
    if (p->table_ld < p->dim || p->x_ld < p->dim)
        return fail(HC_EINVAL, "row strides must be at least dim");
    if (p->table_ld > (1ull << 31) || p->x_ld > (1ull << 31))
        return fail(HC_EINVAL, "row strides must be at most 2^31 elements");
    if (p->id_bits != 32 && p->id_bits != 64) return fail(HC_EINVAL, "id_bits must be 32 or 64");
    if (p->reserved != 0) return fail(HC_EINVAL, "reserved must be 0");
    if (!isfinite(p->scale)) return fail(HC_EINVAL, "scale must be finite");
    return HC_OK;
}

hc_status check_embed_grad(const hc_embed_params* p, uint32_t x_type, const void* dout,
                           const void* ids, uint32_t g_type, bool has_dst, const void* dst,
                           const void* ws, size_t ws_bytes) {
    const hc_status s = check_embed(p, 1ull << 30);
    if (s != HC_OK) return s;
    if (!float_type(x_type)) return fail(HC_EINVAL, "unknown x_type");
    if (!float_type(g_type) && g_type != HC_T_I32) return fail(HC_EINVAL, "unknown g_type");
    if (g_type == HC_T_I32 && (!isfinite(p->fixed) || !(p->fixed > 0.0f)))
        return fail(HC_EINVAL, "fixed must be finite and > 0");
    if ((has_dst && !dst) || !ws || (p->count != 0 && (!dout || !ids)))
        return fail(HC_EINVAL, "buffers must be non-NULL");
    if (!aligned(dout, type_bytes(x_type)) || !aligned(ids, p->id_bits / 8) ||
        !aligned(dst, type_bytes(g_type)))
        return fail(HC_EINVAL, "buffers must be aligned to their elements");
    if (!aligned(ws, 256)) return fail(HC_EINVAL, "ws must be 256-byte aligned");
    if (ws_bytes < embed_grad_bytes(*p))
        return fail(HC_EWORKSPACE, "workspace smaller than hc_embed_grad_bytes reports");
    return HC_OK;
}

// Bounds on the singular values and on b A + c A^2 through the steps give the
// powers of two of the fp16 operands.  A factor of two is left for rounding.
const float kMuon[3] = {3.4445f, -4.7750f, 2.0315f};
constexpr double kBound = 1024.0;

int half_shift(double bound) {
    // largest e with bound * 2^e <= 2^15, half of what fp16 holds
    int e = 0;
    frexp(bound, &e);  // bound in [2^(e-1), 2^e)
    return 15 - e;
}

// max over s in [0, top] of |f(s)|, f odd or even with the given extrema
double max_abs_poly(double a, double b, double c, double top) {
    // |a s + b s^3 + c s^5| on [0, top]
    double best = fabs(((c * top * top + b) * top * top + a) * top);
    const double A = 5 * c, B = 3 * b;  // derivative a + B z + A z^2, z = s^2
    double z[2] = {-1, -1};
    if (A != 0) {
        const double d = B * B - 4 * A * a;
        if (d >= 0) {
            z[0] = (-B + sqrt(d)) / (2 * A);
            z[1] = (-B - sqrt(d)) / (2 * A);
        }
    } else if (B != 0) {
        z[0] = -a / B;
    }
    for (double v : z)
        if (v > 0 && v < top * top)
            best = fmax(best, fabs(((c * v + b) * v + a) * sqrt(v)));
    return best;
}

hc_status ortho_steps(const hc_orthogonalise_params* p, OrthoStep* out) {
    double s = 1.0 + 1e-6;
    for (uint32_t t = 0; t < p->steps; t++) {
        const float* q = p->coeffs ? p->coeffs + 3 * t : kMuon;
        if (!isfinite(q[0]) || !isfinite(q[1]) || !isfinite(q[2]))
            return fail(HC_EINVAL, "coefficients must be finite");
        const double a = q[0], b = q[1], c = q[2], z = s * s;
        double poly = fabs(b * z + c * z * z);  // |b z + c z^2| on [0, s^2]
        if (c != 0) {
            const double v = -b / (2 * c);
            if (v > 0 && v < z) poly = fmax(poly, fabs(b * v + c * v * v));
        }
        const double next = max_abs_poly(a, b, c, s);
        if (!(poly <= kBound) || !(next <= kBound) || !(next >= 1.0 / kBound))
            return fail(HC_EUNSUPPORTED,
                        "coefficients take the singular values out of 2^-10 .. 2^10");
        out[t].a = q[0];
        out[t].b = q[1];
        out[t].c = q[2];
        out[t].ex = half_shift(s);
        out[t].ea = half_shift(z);
        out[t].eb = half_shift(fmax(poly, 1.0 / kBound));
        // rounding of the operands can carry a singular value a little further
        s = next * (1.0 + 1e-2);
        out[t].ex_next = half_shift(s);
    }
    return HC_OK;
}

hc_status check_ortho(const hc_orthogonalise_params* p, OrthoStep* steps) {
    if (p == nullptr) return fail(HC_EINVAL, "params is NULL");
    if (p->m < 1 || p->n < 1 || p->m > 65536 || p->n > 65536)
        return fail(HC_EINVAL, "m and n must be in [1, 65536]");
    if (p->batch > 65535) return fail(HC_EINVAL, "batch must be at most 65535");
    if (p->x_ld < p->n || p->out_ld < p->n)
        return fail(HC_EINVAL, "row strides must be at least n");
    if (p->x_ld > (1ull << 40) || p->out_ld > (1ull << 40) || p->x_stride > (1ull << 46) ||
        p->out_stride > (1ull << 46))
        return fail(HC_EINVAL, "row strides must be at most 2^40 elements, matrix strides 2^46");
    // one matrix after the other, or all matrices' row i before any row i + 1
    if (p->batch > 1 && p->out_stride < (p->m - 1) * p->out_ld + p->n &&
        (p->out_stride < p->n || (p->m > 1 && p->out_ld < (p->batch - 1) * p->out_stride + p->n)))
        return fail(HC_EINVAL, "the output's matrices overlap");
    if (p->type != HC_T_F32 && p->type != HC_T_BF16)
        return fail(HC_EINVAL, "type must be HC_T_F32 or HC_T_BF16");
    if (p->steps > (uint32_t)kOrthoMaxSteps) return fail(HC_EINVAL, "steps must be at most 32");
    if (!isfinite(p->scale)) return fail(HC_EINVAL, "scale must be finite");
    if (!isfinite(p->eps) || !(p->eps >= 0x1p-100f))
        return fail(HC_EINVAL, "eps must be finite and at least 2^-100");
    return ortho_steps(p, steps);
}

}  // namespace

}  // namespace hc

using namespace hc;

extern "C" {

hc_status hc_embed(const hc_embed_params* p, hc_type type, const void* table, const void* ids,
                   void* out, hipStream_t stream) {
    clear_error();
    const hc_status s = check_embed(p, 0x7fffffffull);
    if (s != HC_OK) return s;
    if (!float_type(type)) return fail(HC_EINVAL, "unknown type");
    if (p->count == 0) return HC_OK;
    if (!table || !ids || !out) return fail(HC_EINVAL, "buffers must be non-NULL");
    if (!aligned(table, type_bytes(type)) || !aligned(out, type_bytes(type)) ||
        !aligned(ids, p->id_bits / 8))
        return fail(HC_EINVAL, "buffers must be aligned to their elements");
    const hipError_t e = launch_embed(*p, type, table, ids, out, stream);
    return e == hipSuccess ? HC_OK : fail_hip(e, "hc_embed");
}

hc_status hc_embed_grad_bytes(const hc_embed_params* p, size_t* bytes) {
    clear_error();
    const hc_status s = check_embed(p, 1ull << 30);
    if (s != HC_OK) return s;
    if (!bytes) return fail(HC_EINVAL, "bytes is NULL");
    *bytes = embed_grad_bytes(*p);
    return HC_OK;
}

hc_status hc_embed_grad(const hc_embed_params* p, hc_type x_type, const void* dout,
                        const void* ids, hc_type g_type, void* dtable, int accumulate, void* ws,
                        size_t ws_bytes, hipStream_t stream) {
    clear_error();
    const hc_status s = check_embed_grad(p, x_type, dout, ids, g_type, true, dtable, ws, ws_bytes);
    if (s != HC_OK) return s;
    EmbedGradOut o = {};
    o.dst = dtable;
    o.type = g_type;
    o.accumulate = accumulate != 0;
    const hipError_t e = launch_embed_grad(*p, x_type, dout, ids, o, ws, stream);
    return e == hipSuccess ? HC_OK : fail_hip(e, "hc_embed_grad");
}

hc_status hc_embed_grad_rows(const hc_embed_params* p, hc_type x_type, const void* dout,
                             const void* ids, hc_type g_type, uint32_t* rows, void* values,
                             uint64_t cap, uint32_t* touched, void* ws, size_t ws_bytes,
                             hipStream_t stream) {
    clear_error();
    const hc_status s = check_embed_grad(p, x_type, dout, ids, g_type, cap != 0, values, ws, ws_bytes);
    if (s != HC_OK) return s;
    if ((cap != 0 && !rows) || !touched)
        return fail(HC_EINVAL, "rows and touched must be non-NULL");
    if (!aligned(rows, 4) || !aligned(touched, 4))
        return fail(HC_EINVAL, "buffers must be aligned to their elements");
    EmbedGradOut o = {};
    o.dst = values;
    o.type = g_type;
    o.by_rows = true;
    o.rows = rows;
    o.cap = cap;
    o.touched = touched;
    const hipError_t e = launch_embed_grad(*p, x_type, dout, ids, o, ws, stream);
    return e == hipSuccess ? HC_OK : fail_hip(e, "hc_embed_grad_rows");
}

hc_status hc_orthogonalise_bytes(const hc_orthogonalise_params* p, size_t* bytes) {
    clear_error();
    OrthoStep steps[kOrthoMaxSteps];
    const hc_status s = check_ortho(p, steps);
    if (s != HC_OK) return s;
    if (!bytes) return fail(HC_EINVAL, "bytes is NULL");
    *bytes = orthogonalise_bytes(*p);
    return HC_OK;
}

hc_status hc_orthogonalise(const hc_orthogonalise_params* p, const void* x, void* out, void* ws,
                           size_t ws_bytes, hipStream_t stream) {
    clear_error();
    OrthoStep steps[kOrthoMaxSteps];
    const hc_status s = check_ortho(p, steps);
    if (s != HC_OK) return s;
    if (p->batch == 0) return HC_OK;
    if (!x || !out || !ws) return fail(HC_EINVAL, "buffers must be non-NULL");
    if (!aligned(x, type_bytes(p->type)) || !aligned(out, type_bytes(p->type)))
        return fail(HC_EINVAL, "buffers must be aligned to their elements");
    if (!aligned(ws, 256)) return fail(HC_EINVAL, "ws must be 256-byte aligned");
    if (ws_bytes < orthogonalise_bytes(*p))
        return fail(HC_EWORKSPACE, "workspace smaller than hc_orthogonalise_bytes reports");
    const hipError_t e = launch_orthogonalise(*p, steps, x, out, ws, stream);
    return e == hipSuccess ? HC_OK : fail_hip(e, "hc_orthogonalise");
}

}  // extern "C"
