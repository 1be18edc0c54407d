// hc_linear.hip -- the linear layer and its gradient (include/hc_train.h).
//
//   forward   D = y,  D[i][j] = sum over l of x[i][l] w[j][l]
//   dx        D = dx, D[i][j] = sum over l of dz[i][l] w[l][j]
//   dw        D = dw, D[i][j] = sum over l of dz[l][i] x[l][j]
#include "hc_layer.h"

namespace hc {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));

enum Kind { FORWARD, DX, DW };

// What a forward product's sums become.
struct Forward {
    const void *bias, *residual;
    void *y, *z;
    uint64_t residual_ld, y_ld, z_ld;
    uint32_t act;
    Dropout drop;
};

template <typename T>
__device__ __forceinline__ void finish_forward(const Forward& f, const Masks& masks, uint64_t row,
                                               uint32_t col, uint32_t count, float (&v)[8]) {
    if (f.bias) {
        float b[8];
        load8(static_cast<const T*>(f.bias) + col, count, b);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += b[e];
    }
    if (f.z) store8(static_cast<T*>(f.z) + row * f.z_ld + col, count, v);
    if (f.act != HC_ACT_NONE)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = activate<T>(f.act, v[e]);
    if (masks.limit) drop8(masks, (uint32_t)row, col / 8, v);
    if (f.residual) {
        float r[8];
        load8(static_cast<const T*>(f.residual) + row * f.residual_ld + col, count, r);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += r[e];
    }
    store8(static_cast<T*>(f.y) + row * f.y_ld + col, count, v);
}

struct Product {
    const void *p, *q;       // operands
    const void* p_rest;      // DW: dz = p + p_rest, or null
    uint64_t p_ld, q_ld;
    uint64_t rows, inner;    // of D; length of l
    uint32_t cols, tiles_j;
    uint64_t tiles;
    uint32_t pieces;         // each tile's l is cut into
    float* part;             // their sums, [piece][rows][part_ld]
    uint32_t part_ld;
    Forward forward;
    Gradient gradient;
};

template <Kind KIND, typename T>
__device__ __forceinline__ void finish8(const Product& g, const Masks& masks, uint64_t row, uint32_t col,
                                        float (&v)[8]) {
    const uint32_t count = g.cols - col;
    if constexpr (KIND == FORWARD) finish_forward<T>(g.forward, masks, row, col, count, v);
    else if constexpr (KIND == DX) store8(static_cast<T*>(g.gradient.out) + row * g.gradient.ld + col, count, v);
    else store_gradient(g.gradient, row, col, count, v);
}

// ---- products of any shape, stride and alignment -----------------------------------

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f4 product16(h8 a, h8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 product16(b8 a, b8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 product16(f8 a, f8 b, f4 c) {
#pragma unroll
    for (int e = 0; e < 8; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// Steps of 32 along l.  Rows of a tile in LDS are padded by 16 bytes, so that a
// fragment's 16 rows start at different banks.
constexpr uint32_t kDirect = 64, kStep = 32;

template <typename T> constexpr uint32_t kDirectLd = kStep + 16 / sizeof(T);

// A lane's 8 elements of a 64 x 32 tile of an operand: along l where its rows lie
// along l, along its rows' index where they are strided.
template <bool STRIDED> struct DirectPlace {
    uint32_t row, l;
    __device__ __forceinline__ DirectPlace() {
        if (STRIDED) {
            l = threadIdx.x / 8;
            row = threadIdx.x % 8 * 8;
        } else {
            row = threadIdx.x / 4;
            l = threadIdx.x % 4 * 8;
        }
    }
};

template <bool STRIDED, typename T>
__device__ __forceinline__ void direct_load(const T* p, uint64_t ld, uint64_t rows, uint64_t row0,
                                            uint64_t l, uint64_t inner, T (&v)[8]) {
    const DirectPlace<STRIDED> at;
    const uint64_t row = row0 + at.row;
    l += at.l;
    const T* src = STRIDED ? p + l * ld + row : p + row * ld + l;
    const bool in = row < rows && l < inner;
    const uint64_t left = in ? (STRIDED ? rows - row : inner - l) : 0;
    if (left >= 8) {
        const typename Eight<T>::V t = *reinterpret_cast<const typename Eight<T>::V*>(src);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (uint64_t)e < left ? src[e] : (T)0.0f;
    }
}

template <bool STRIDED, typename T>
__device__ __forceinline__ void direct_store(T* s, const T (&v)[8]) {
    const DirectPlace<STRIDED> at;
    if constexpr (STRIDED) {
#pragma unroll
        for (int e = 0; e < 8; e++) s[(at.row + e) * kDirectLd<T> + at.l] = v[e];
    } else {
        typedef T V __attribute__((ext_vector_type(8), aligned(16)));
        V t;
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = v[e];
        *reinterpret_cast<V*>(s + at.row * kDirectLd<T> + at.l) = t;
    }
}

// A 64 x 64 tile, or a piece of one, a workgroup of four waves, each 32 x 32 of
// it.  Loads go through registers, which takes any stride, alignment and length,
// zeros where a matrix ends.
template <Kind KIND, typename T>
__global__ __launch_bounds__(256) void direct_kernel(Product g) {
    constexpr bool PS = KIND == DW, QS = KIND != FORWARD;
    typedef T V __attribute__((ext_vector_type(8), aligned(16)));
    __shared__ __align__(16) T s_p[kDirect * kDirectLd<T>], s_q[kDirect * kDirectLd<T>];
    __shared__ __align__(16) float s_out[kDirect * (kDirect + 4)];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t wi = wave / 2 * 32, wj = wave % 2 * 32;
    const uint64_t piece = blockIdx.x / g.tiles, tile = blockIdx.x - piece * g.tiles;
    const uint64_t ti = tile / g.tiles_j, row0 = ti * kDirect;
    const uint32_t col0 = (uint32_t)(tile - ti * g.tiles_j) * kDirect;
    const uint64_t lines = (g.inner + kStep - 1) / kStep, all = g.p_rest ? 2 * lines : lines;
    const uint64_t first = piece * all / g.pieces, end = (piece + 1) * all / g.pieces;
    const T* q = static_cast<const T*>(g.q);
    f4 acc[2][2] = {};
    T rp[8], rq[8];
    auto load = [&](uint64_t s) {
        const bool rest = s >= lines;
        const uint64_t l = (rest ? s - lines : s) * kStep;
        direct_load<PS>(static_cast<const T*>(rest ? g.p_rest : g.p), g.p_ld, g.rows, row0, l, g.inner, rp);
        direct_load<QS>(q, g.q_ld, (uint64_t)g.cols, col0, l, g.inner, rq);
    };
    if (first < end) load(first);
    for (uint64_t s = first; s < end; s++) {
        __syncthreads();
        direct_store<PS>(s_p, rp);
        direct_store<QS>(s_q, rq);
        __syncthreads();
        if (s + 1 < end) load(s + 1);
        V fp[2], fq[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const uint32_t at = (16 * u + (lane & 15)) * kDirectLd<T> + (lane >> 4) * 8;
            fp[u] = *reinterpret_cast<const V*>(s_p + wi * kDirectLd<T> + at);
            fq[u] = *reinterpret_cast<const V*>(s_q + wj * kDirectLd<T> + at);
        }
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int v = 0; v < 2; v++) acc[u][v] = product16(fq[v], fp[u], acc[u][v]);
    }
    constexpr uint32_t LD = kDirect + 4;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
        for (int v = 0; v < 2; v++)
            *reinterpret_cast<f4*>(s_out + (wi + 16 * u + (lane & 15)) * LD + wj + 16 * v + (lane >> 4) * 4) =
                acc[u][v];
    __syncthreads();
    Masks masks = {};
    if constexpr (KIND == FORWARD) masks = masks_of(g.forward.drop);
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t at = threadIdx.x + 256 * k, ii = at / 8, jj = at % 8 * 8;
        const uint64_t row = row0 + ii;
        const uint32_t col = col0 + jj;
        if (row >= g.rows || col >= g.cols) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = s_out[ii * LD + jj + e];
        if (g.pieces > 1)
            store8(g.part + (piece * g.rows + row) * g.part_ld + col, 8, v);
        else
            finish8<KIND, T>(g, masks, row, col, v);
    }
}

// The sums of the tiles' pieces, in order, a lane eight columns of a row.
template <Kind KIND, typename T>
__global__ __launch_bounds__(256) void join_kernel(Product g) {
    const uint32_t groups = g.part_ld / 8;
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = at / groups;
    if (row >= g.rows) return;
    const uint32_t col = (uint32_t)(at - row * groups) * 8;
    const f8* part = reinterpret_cast<const f8*>(g.part + row * g.part_ld + col);
    const uint64_t step = g.rows * g.part_ld / 8;
    f8 sum = {};
    for (uint32_t c = 0; c < g.pieces; c++) sum += part[c * step];
    Masks masks = {};
    if constexpr (KIND == FORWARD) masks = masks_of(g.forward.drop);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = sum[e];
    finish8<KIND, T>(g, masks, row, col, v);
}

// ---- dz and the bias's gradient ----------------------------------------------------

struct DzArgs {
    const void *dy, *z;
    uint64_t dy_ld, z_ld, m;
    uint32_t n, groups;
    uint32_t act;
    uint32_t per;      // rows of a workgroup
    uint32_t width;    // lanes for a row, a power of two up to 64
    Dropout drop;
    void *dz, *rest;   // [m][dz_ld], or null
    uint64_t dz_ld;
    float* part;       // the workgroups' sums, [blocks][n], or null
};

// dz = act'(z) mask dy, and each workgroup's sums of its rows.
template <typename T> __global__ __launch_bounds__(256) void dz_kernel(DzArgs a) {
    __shared__ float s_sum[256 * 8];
    const Masks masks = masks_of(a.drop);
    const uint32_t group = blockIdx.x * a.width + threadIdx.x % a.width, sub = threadIdx.x / a.width;
    const uint32_t step = 256 / a.width, col = group * 8;
    const uint64_t end = min((uint64_t)(blockIdx.y + 1) * a.per, a.m);
    float sum[8] = {};
    if (group < a.groups) {
        const uint32_t count = a.n - col;
        for (uint64_t row = (uint64_t)blockIdx.y * a.per + sub; row < end; row += step) {
            float v[8];
            load8(static_cast<const T*>(a.dy) + row * a.dy_ld + col, count, v);
            if (masks.limit) drop8(masks, (uint32_t)row, group, v);
            if (a.act != HC_ACT_NONE) {
                float z[8];
                load8(static_cast<const T*>(a.z) + row * a.z_ld + col, count, z);
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = backward<T>(a.act, z[e], v[e]);
            }
            if (a.dz) store8(static_cast<T*>(a.dz) + row * a.dz_ld + col, count, v);
            if (a.rest) {
                float r[8];
#pragma unroll
                for (int e = 0; e < 8; e++) r[e] = v[e] - (float)(T)v[e];
                store8(static_cast<T*>(a.rest) + row * a.dz_ld + col, count, r);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) sum[e] += (uint32_t)e < count ? v[e] : 0.0f;
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int e = 0; e < 8; e++) s_sum[threadIdx.x * 8 + e] = sum[e];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.width * 8; c += 256) {
        float t = 0.0f;
        for (uint32_t r = 0; r < step; r++) t += s_sum[r * a.width * 8 + c];
        const uint32_t at = blockIdx.x * a.width * 8 + c;
        if (at < a.n) a.part[(uint64_t)blockIdx.y * a.n + at] = t;
    }
}

// db: the workgroups' sums, 64 columns a workgroup, in 16 shares that are added
// in order.
__global__ __launch_bounds__(1024) void bias_kernel(const float* __restrict__ part, uint32_t blocks, uint32_t n,
                                                    Gradient g) {
    __shared__ float s_sum[16][64];
    const uint32_t lane = threadIdx.x & 63, share = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float t = 0.0f;
    if (col < n)
        for (uint32_t b = blocks * share / 16; b < blocks * (share + 1) / 16; b++) t += part[(uint64_t)b * n + col];
    s_sum[share][lane] = t;
    __syncthreads();
    if (threadIdx.x < 64 && col < n) {
        t = 0.0f;
        for (int k = 0; k < 16; k++) t += s_sum[k][lane];
        float v[8] = {t};
        store_gradient(g, 0, col, 1, v);
    }
}

// ---- layout and launches ------------------------------------------------------------

constexpr uint64_t kSlots = 1024;        // workgroups that a product is cut for
constexpr uint64_t kMostPieces = 64;
constexpr uint64_t kBiasBlocks = 256;    // most workgroups along the rows of dz

uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to; }

struct DirectPlan {
    uint64_t tiles;
    uint32_t tiles_j, pieces;
    size_t part_bytes;
};

DirectPlan direct_plan(uint64_t rows, uint64_t cols, uint64_t lines) {
    DirectPlan d = {};
    d.tiles_j = (uint32_t)up(cols, kDirect);
    d.tiles = up(rows, kDirect) * d.tiles_j;
    uint64_t pieces = d.tiles ? kSlots / d.tiles : 1;
    pieces = pieces > lines / 4 ? lines / 4 : pieces;
    pieces = pieces > kMostPieces ? kMostPieces : pieces < 1 ? 1 : pieces;
    d.pieces = (uint32_t)pieces;
    d.part_bytes = pieces > 1 ? pieces * rows * up(cols, 8) * 32 : 0;
    return d;
}

template <Kind KIND, typename T> hipError_t direct(Product g, float* part, hipStream_t s) {
    const uint64_t lines = up(g.inner, kStep) * (g.p_rest ? 2 : 1);
    const DirectPlan d = direct_plan(g.rows, g.cols, lines);
    g.tiles = d.tiles;
    g.tiles_j = d.tiles_j;
    g.pieces = d.pieces;
    g.part = part;
    g.part_ld = (uint32_t)up(g.cols, 8) * 8;
    hipLaunchKernelGGL((direct_kernel<KIND, T>), dim3((uint32_t)(d.tiles * d.pieces)), dim3(256), 0, s, g);
    if (d.pieces > 1)
        hipLaunchKernelGGL((join_kernel<KIND, T>), dim3((uint32_t)up(g.rows * (g.part_ld / 8), 256)),
                           dim3(256), 0, s, g);
    return hipGetLastError();
}

template <Kind KIND> hipError_t product(const Product& g, hc_type type, float* part, hipStream_t s) {
    if (type == HC_T_F32) return direct<KIND, float>(g, part, s);
    if (type == HC_T_BF16) return direct<KIND, __bf16>(g, part, s);
    return direct<KIND, _Float16>(g, part, s);
}

// Most bytes of partial sums for up to this many rows of D (fewer rows may be cut
// into more pieces).
size_t most_part_bytes(uint64_t rows, uint64_t cols) {
    const uint64_t whole = up(rows, kDirect) * up(cols, kDirect);  // tiles
    const uint64_t most = whole < 1 ? 0 : whole * kMostPieces < kSlots ? whole * kMostPieces : kSlots;
    return most * kDirect * kDirect * 4 + 256;
}

struct GradLayout {
    size_t dz, rest, bias, part, bytes;
    uint64_t dz_ld, per, blocks;
    uint32_t width;
};

GradLayout grad_layout(const hc_linear_params& p, hc_type type) {
    GradLayout L = {};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    const size_t size = type == HC_T_F32 ? 4 : 2;
    L.dz_ld = up(p.n, 8) * 8;
    const uint64_t groups = L.dz_ld / 8;
    L.width = 1;
    while (L.width < 64 && L.width < groups) L.width *= 2;
    const uint64_t step = 256 / L.width;
    L.per = up(up(p.m, kBiasBlocks), step) * step;
    L.blocks = p.m ? up(p.m, L.per) : 0;
    L.dz = take(p.m * L.dz_ld * size);
    L.rest = take(type == HC_T_F32 ? 0 : p.m * L.dz_ld * size);
    L.bias = take(kBiasBlocks * p.n * 4);
    const size_t a = most_part_bytes(p.m, p.k), b = most_part_bytes(p.n, p.k);
    L.part = take(a > b ? a : b);
    L.bytes = at;
    return L;
}

}  // namespace

size_t linear_bytes(const hc_linear_params& p, hc_type) { return most_part_bytes(p.m, p.n); }

hipError_t launch_linear(const hc_linear_params& p, const Dropout& d, hc_type type, const void* x,
                         const void* w, const void* bias, const void* residual, void* y, void* z,
                         void* ws, hipStream_t s) {
    Product g = {};
    g.p = x;
    g.q = w;
    g.p_ld = p.x_ld;
    g.q_ld = p.w_ld;
    g.rows = p.m;
    g.cols = (uint32_t)p.n;
    g.inner = p.k;
    g.forward = {bias, residual, y, z, p.residual_ld, p.y_ld, p.z_ld, p.act, d};
    return product<FORWARD>(g, type, static_cast<float*>(ws), s);
}

size_t linear_grad_bytes(const hc_linear_params& p, hc_type type) { return grad_layout(p, type).bytes; }

hipError_t launch_linear_grad(const hc_linear_params& p, const Dropout& d, hc_type type,
                              const LinearGrad& q, void* ws_, hipStream_t s) {
    const GradLayout L = grad_layout(p, type);
    char* ws = static_cast<char*>(ws_);
    const bool plain = p.act == HC_ACT_NONE && d.limit == 0;
    const bool rest = !plain && q.dw && type != HC_T_F32 && (q.g_type == HC_T_F32 || q.g_type == HC_T_I32);
    const bool dz = !plain && (q.dx || q.dw);
    const Gradient gradient = {nullptr, 0, (uint32_t)q.g_type, q.accumulate ? 1u : 0u, p.fixed};
    if ((dz || q.db) && p.m) {
        DzArgs a = {};
        a.dy = q.dy;
        a.z = q.z;
        a.dy_ld = p.y_ld;
        a.z_ld = p.z_ld;
        a.m = p.m;
        a.n = (uint32_t)p.n;
        a.groups = (uint32_t)(L.dz_ld / 8);
        a.act = p.act;
        a.per = (uint32_t)L.per;
        a.width = L.width;
        a.drop = d;
        a.dz = dz ? ws + L.dz : nullptr;
        a.rest = rest ? ws + L.rest : nullptr;
        a.dz_ld = L.dz_ld;
        a.part = q.db ? reinterpret_cast<float*>(ws + L.bias) : nullptr;
        const dim3 grid((uint32_t)up(a.groups, L.width), (uint32_t)L.blocks);
        if (type == HC_T_F32) hipLaunchKernelGGL(dz_kernel<float>, grid, dim3(256), 0, s, a);
        else if (type == HC_T_BF16) hipLaunchKernelGGL(dz_kernel<__bf16>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(dz_kernel<_Float16>, grid, dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (q.db) {
        Gradient b = gradient;
        b.out = q.db;
        hipLaunchKernelGGL(bias_kernel, dim3((uint32_t)up(p.n, 64)), dim3(1024), 0, s,
                           reinterpret_cast<const float*>(ws + L.bias), (uint32_t)L.blocks, (uint32_t)p.n, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    Product g = {};
    g.p = dz ? ws + L.dz : q.dy;
    g.p_ld = dz ? L.dz_ld : p.y_ld;
    float* part = reinterpret_cast<float*>(ws + L.part);
    if (q.dx && p.m) {
        Product h = g;
        h.q = q.w;
        h.q_ld = p.w_ld;
        h.rows = p.m;
        h.cols = (uint32_t)p.k;
        h.inner = p.n;
        h.gradient.out = q.dx;
        h.gradient.ld = p.dx_ld;
        const hipError_t e = product<DX>(h, type, part, s);
        if (e != hipSuccess) return e;
    }
    if (q.dw) {
        Product h = g;
        if (rest) h.p_rest = ws + L.rest;
        h.q = q.x;
        h.q_ld = p.x_ld;
        h.rows = p.n;
        h.cols = (uint32_t)p.k;
        h.inner = p.m;
        h.gradient = gradient;
        h.gradient.out = q.dw;
        h.gradient.ld = p.dw_ld;
        return product<DW>(h, type, part, s);
    }
    return hipSuccess;
}

}  // namespace hc
