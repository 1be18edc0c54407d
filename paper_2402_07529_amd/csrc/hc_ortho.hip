// hc_ortho.hip -- Newton-Schulz orthogonalisation (include/hc_train.h).
//
// X_0 = x / (|x|_F + eps), held with its shorter side (r) as rows and its longer
// side (k) as columns; then per step A = X X^T, B = b A + c A^2 and
// X <- a X + B X.  The three products run on the matrix cores.
//
// Precision.  The operands of the products are fp16 times a power of two that
// the bound on the singular values allows (so nothing overflows and what
// matters stays normal), sums are fp32, and X itself is kept in fp32 beside its
// operands: a X is added in fp32, so that rounding an operand only reaches X
// through B, which is small where X's singular values are.  For bf16 matrices
// one fp16 plane: on random and on low-rank matrices with sides of 256 or more
// the result is 3e-4 to 2.0e-3 from the exact one, about the 1.7e-3 of rounding
// it to bf16 (bf16 operands: 2e-3 to 1.4e-2; fp16 operands without the fp32 X: up
// to 2e-2).  For fp32 matrices an operand is the sum of two fp16 planes and a
// product three matrix products (high x high, high x low, low x high): 22 bits,
// 5e-8 to 3e-7 from the exact result, as fp32 arithmetic.
#include "hc_device.h"
#include "hc_internal.h"
#include "hc_train_internal.h"

namespace hc {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// ---- operand planes --------------------------------------------------------------

// An operand matrix of `cols` columns (a multiple of 64) is stored by rows.
// One plane: fp16 values in order.  Two planes: every 32 values are 32 high
// parts followed by their 32 low parts, so a row of 64 stored values is one
// 128-byte line in either form.
template <int PLANES> __device__ __forceinline__ size_t operand_at(size_t row, uint32_t cols, uint32_t col) {
    if constexpr (PLANES == 1) return row * cols + col;
    return row * (2 * (size_t)cols) + (col >> 5) * 64 + (col & 31);
}

template <int PLANES> __device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    if constexpr (PLANES == 2) lo = (_Float16)(v - (float)hi);
}

// ---- norm and operands of X_0 ----------------------------------------------------

constexpr int kPrepBlock = 256;
constexpr uint32_t kNormParts = 256;

template <typename T>
__global__ __launch_bounds__(kPrepBlock) void norm_kernel(const T* __restrict__ x, uint64_t rows,
                                                          uint64_t cols, uint64_t ld,
                                                          uint64_t stride,
                                                          double* __restrict__ partial) {
    __shared__ double s_sum[kPrepBlock / 64];
    const T* m = x + (uint64_t)blockIdx.y * stride;
    double acc = 0.0;
    if (rows == 1) {
        for (uint64_t i = (uint64_t)blockIdx.x * kPrepBlock + threadIdx.x; i < cols;
             i += (uint64_t)gridDim.x * kPrepBlock) {
            const double v = (double)(float)m[i];
            acc += v * v;
        }
    } else {
        for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
            for (uint64_t i = threadIdx.x; i < cols; i += kPrepBlock) {
                const double v = (double)(float)m[r * ld + i];
                acc += v * v;
            }
    }
    for (int d = 32; d > 0; d >>= 1) acc += __shfl_xor(acc, d);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = acc;
    lds_barrier();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < kPrepBlock / 64; w++) t += s_sum[w];
        partial[(uint64_t)blockIdx.y * kNormParts + blockIdx.x] = t;
    }
}

// 1 / (norm + eps), or NaN where the norm is not finite.  Every lane calls it.
__device__ __forceinline__ float inverse_norm(const double* partial, uint32_t parts, float eps) {
    double t = 0.0;
    for (uint32_t i = lane_id(); i < parts; i += 64) t += partial[i];
    for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
    const double n = sqrt(t);
    return n < __builtin_inf() ? (float)(1.0 / (n + (double)eps)) : __builtin_nanf("");
}

struct PrepArgs {
    uint64_t m, n, ld, stride;
    uint32_t r, k;    // padded shorter and longer side
    bool tall;        // m > n: X is the transpose of x
    uint32_t parts;
    float eps;
    int shift;
    const double* partial;
    float* master;
    _Float16 *x, *xt;
};

// A 64 x 64 tile of x, scaled by the inverse norm: the fp32 X, its operand and
// its transpose's.  Tiles cover the padded sides; the padding is zero.
template <typename T, int PLANES>
__global__ __launch_bounds__(kPrepBlock) void prepare_kernel(PrepArgs a, const T* __restrict__ x) {
    __shared__ float s_tile[64][65];
    const uint32_t b = blockIdx.z;
    const float f = inverse_norm(a.partial + (uint64_t)b * kNormParts, a.parts, a.eps);
    const float scale = __builtin_ldexpf(1.0f, a.shift);
    const T* m = x + (uint64_t)b * a.stride;
    const uint32_t row0 = blockIdx.y * 64, col0 = blockIdx.x * 64;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t base = (size_t)b * a.r * a.k;
    // x's own orientation: X's where it is wide, X^T's where it is tall
    const uint32_t cols = a.tall ? a.r : a.k, rows = a.tall ? a.k : a.r;
    _Float16* straight = (a.tall ? a.xt : a.x) + base * PLANES;
    _Float16* turned = (a.tall ? a.x : a.xt) + base * PLANES;
    for (uint32_t j = wave; j < 64; j += 4) {
        const uint32_t r = row0 + j, c = col0 + lane;
        const float v = r < a.m && c < a.n ? (float)m[(uint64_t)r * a.ld + c] * f : 0.0f;
        s_tile[j][lane] = v;
        const size_t at = operand_at<PLANES>(r, cols, c);
        _Float16 hi, lo = 0;
        split<PLANES>(v * scale, hi, lo);
        straight[at] = hi;
        if (PLANES == 2) straight[at + 32] = lo;
        if (!a.tall) a.master[base + (size_t)r * cols + c] = v;
    }
    lds_barrier();
    for (uint32_t j = wave; j < 64; j += 4) {
        const uint32_t r = col0 + j, c = row0 + lane;
        const float v = s_tile[lane][j];
        const size_t at = operand_at<PLANES>(r, rows, c);
        _Float16 hi, lo = 0;
        split<PLANES>(v * scale, hi, lo);
        turned[at] = hi;
        if (PLANES == 2) turned[at + 32] = lo;
        if (a.tall) a.master[base + (size_t)r * rows + c] = v;
    }
}

// No steps: the normalised matrix itself.
template <typename T>
__global__ __launch_bounds__(kPrepBlock) void normalise_kernel(hc_orthogonalise_params p,
                                                               const T* __restrict__ x,
                                                               T* __restrict__ out,
                                                               const double* __restrict__ partial,
                                                               uint32_t parts) {
    const float f = inverse_norm(partial + (uint64_t)blockIdx.y * kNormParts, parts, p.eps);
    const T* m = x + (uint64_t)blockIdx.y * p.x_stride;
    T* o = out + (uint64_t)blockIdx.y * p.out_stride;
    for (uint64_t r = blockIdx.x; r < p.m; r += gridDim.x)
        for (uint64_t i = threadIdx.x; i < p.n; i += kPrepBlock)
            o[r * p.out_ld + i] = (T)((float)m[r * p.x_ld + i] * f * p.scale);
}

// ---- products --------------------------------------------------------------------

// C[i][j] = sum over l of P[i][l] Q[j][l]: both operands by rows along l.
//   GRAM    P = Q = X            A = C                        symmetric
//   SQUARE  P = Q = A            B = b A + c C                symmetric
//   APPLY   P = B, Q = X^T       X <- a X + C
// Of a symmetric result the tiles on and below the diagonal are computed and
// the others mirrored.
enum Kind { GRAM, SQUARE, APPLY };

struct Product {
    const _Float16 *p, *q;
    uint32_t inner;                  // length of l, a multiple of 64
    uint32_t tiles_i, tiles_j;       // of a result that is not symmetric
    size_t p_stride, q_stride;       // between matrices of the batch (stored values)
    float factor;                    // takes the sum to the result's unit
    float factor2;                   // SQUARE: takes the operand A to it; APPLY: a
    float next;                      // APPLY: power of two of the next operands
    // results
    _Float16 *d;                     // A or B, [r][r], or X, [r][k]
    _Float16 *dt;                    // APPLY: X^T, [k][r]
    uint32_t r, k;                   // padded
    float* master;                   // APPLY: X in fp32
    // APPLY, last step: the output instead
    void* out;
    uint64_t m, n, out_ld, out_stride;
    float out_scale;
    bool tall;
};

constexpr int kBM = 128, kBN = 128, kGemmBlock = 256;
constexpr int kLine = 64;  // stored values of a tile's row: 128 bytes

// 16-byte chunk `c` of row `row` of a tile in LDS, stored at c ^ (row mod 8): a
// wave's reads of one chunk of 16 rows then touch all banks evenly.
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c) {
    return row * kLine + ((c ^ (row & 7u)) << 3);
}

// Result (i, j) of a wave's 64 x 64: its 4-value group is turned by i, so that a
// column is spread over the banks.
__device__ __forceinline__ uint32_t staged(uint32_t i, uint32_t j) {
    return i * 64 + ((((j >> 2) ^ i) & 15u) << 2) + (j & 3u);
}

template <typename T> __device__ __forceinline__ T to_out(float v) { return (T)v; }

template <Kind KIND, int PLANES, typename TO>
__global__ __launch_bounds__(kGemmBlock) void product_kernel(Product g) {
    // main loop: two operand tiles; afterwards each wave's 64 x 64 results
    __shared__ __align__(16) char s_mem[kGemmBlock / 64 * 64 * 64 * 4];
    _Float16* sp = reinterpret_cast<_Float16*>(s_mem);
    _Float16* sq = sp + kBM * kLine;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    const uint32_t batch = blockIdx.y;
    uint32_t ti, tj;
    if constexpr (KIND == APPLY) {
        ti = blockIdx.x % g.tiles_i;
        tj = blockIdx.x / g.tiles_i;
    } else {
        // row ti of the lower triangle begins at ti (ti + 1) / 2
        ti = (uint32_t)((sqrtf(8.0f * (float)blockIdx.x + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > blockIdx.x) ti--;
        while ((ti + 1) * (ti + 2) / 2 <= blockIdx.x) ti++;
        tj = blockIdx.x - ti * (ti + 1) / 2;
    }
    const uint32_t i0 = ti * kBM, j0 = tj * kBN;
    const size_t line = (size_t)g.inner * PLANES;  // stored values of an operand's row
    const _Float16* P = g.p + batch * g.p_stride + (size_t)i0 * line;
    const _Float16* Q = g.q + batch * g.q_stride + (size_t)j0 * line;

    f4 acc[4][4] = {};
    const uint32_t row = threadIdx.x >> 3, chunk = threadIdx.x & 7;  // 32 rows a round
    const uint32_t lines = (uint32_t)(line / kLine);
    h8 rp[4], rq[4];
    auto fetch = [&](uint32_t l) {
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const size_t at = (size_t)(row + 32 * u) * line + (size_t)l * kLine + chunk * 8;
            rp[u] = *reinterpret_cast<const h8*>(P + at);
            rq[u] = *reinterpret_cast<const h8*>(Q + at);
        }
    };
    fetch(0);
    for (uint32_t l = 0; l < lines; l++) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; u++) {
            *reinterpret_cast<h8*>(sp + swizzled(row + 32 * u, chunk)) = rp[u];
            *reinterpret_cast<h8*>(sq + swizzled(row + 32 * u, chunk)) = rq[u];
        }
        __syncthreads();
        if (l + 1 < lines) fetch(l + 1);
        // fragments: lane holds row lane % 16, 8 values from chunk 4 h + lane / 16
        h8 fp[2][4], fq[2][4];
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const uint32_t c = 4 * h + (lane >> 4);
                fp[h][u] = *reinterpret_cast<const h8*>(sp + swizzled(wi + 16 * u + (lane & 15), c));
                fq[h][u] = *reinterpret_cast<const h8*>(sq + swizzled(wj + 16 * u + (lane & 15), c));
            }
        // the first operand gives the result's 4 consecutive values of a lane:
        // Q first, so that they lie along j
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int v = 0; v < 4; v++) {
                acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[0][v], fp[0][u], acc[u][v], 0, 0, 0);
                if constexpr (PLANES == 1) {
                    acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[1][v], fp[1][u], acc[u][v], 0, 0, 0);
                } else {
                    acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[1][v], fp[0][u], acc[u][v], 0, 0, 0);
                    acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[0][v], fp[1][u], acc[u][v], 0, 0, 0);
                }
            }
    }
    __syncthreads();

    // result (i, j .. j + 3) of fragment (u, v): i = lane % 16, j = 4 (lane / 16)
    float* stage = reinterpret_cast<float*>(s_mem) + wave * 64 * 64;  // [i][j], see staged()
    const uint32_t fi = lane & 15, fj = (lane >> 4) * 4;
    const uint32_t width = KIND == APPLY ? g.k : g.r;
    const size_t dbase = (size_t)batch * g.r * width;
    const bool last = KIND == APPLY && g.out != nullptr;
    float factor = g.factor, factor2 = g.factor2;
#pragma unroll
    for (int u = 0; u < 4; u++)
#pragma unroll
        for (int v = 0; v < 4; v++) {
            const uint32_t i = i0 + wi + 16 * u + fi, j = j0 + wj + 16 * v + fj;
            f4 w = acc[u][v] * factor;
            if constexpr (KIND == SQUARE) {
                const _Float16* A = g.p + batch * g.p_stride + operand_at<PLANES>(i, g.r, j);
                const h4 hi = *reinterpret_cast<const h4*>(A);
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] += (float)hi[e] * factor2;
                if constexpr (PLANES == 2) {
                    const h4 lo = *reinterpret_cast<const h4*>(A + 32);
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] += (float)lo[e] * factor2;
                }
            }
            if constexpr (KIND == APPLY) {
                f4* mm = reinterpret_cast<f4*>(g.master + dbase + (size_t)i * width + j);
                w += *mm * factor2;
                if (!last) *mm = w;
                w *= last ? g.out_scale : g.next;
            }
            if (last) {
                if (!g.tall && i < g.m) {
                    TO* o = static_cast<TO*>(g.out) + batch * g.out_stride + (uint64_t)i * g.out_ld + j;
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (j + e < g.n) o[e] = to_out<TO>(w[e]);
                }
            } else {
                h4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    _Float16 a, b = 0;
                    split<PLANES>(w[e], a, b);
                    hi[e] = a;
                    lo[e] = b;
                }
                _Float16* D = g.d + dbase * PLANES + operand_at<PLANES>(i, width, j);
                *reinterpret_cast<h4*>(D) = hi;
                if constexpr (PLANES == 2) *reinterpret_cast<h4*>(D + 32) = lo;
            }
            *reinterpret_cast<f4*>(stage + staged(16 * u + fi, 16 * v + fj)) = w;
        }
    __syncthreads();
    // the transpose, a row of 64 i's at a time
    if (KIND != APPLY && ti == tj) return;
    if (last) {
        if (!g.tall) return;
        for (uint32_t jj = 0; jj < 64; jj++) {
            const uint32_t j = j0 + wj + jj, i = i0 + wi + lane;
            if (j < g.m && i < g.n)
                static_cast<TO*>(g.out)[batch * g.out_stride + (uint64_t)j * g.out_ld + i] =
                    to_out<TO>(stage[staged(lane, jj)]);
        }
        return;
    }
    _Float16* DT = (KIND == APPLY ? g.dt : g.d) + dbase * PLANES;
    for (uint32_t jj = 0; jj < 64; jj++) {
        _Float16 hi, lo = 0;
        split<PLANES>(stage[staged(lane, jj)], hi, lo);
        const size_t at = operand_at<PLANES>(j0 + wj + jj, g.r, i0 + wi + lane);
        DT[at] = hi;
        if (PLANES == 2) DT[at + 32] = lo;
    }
}

// ---- layout and launches ---------------------------------------------------------

// bf16 matrices with a side of at most this take two planes too: the rounding
// of few entries does not average out (a 64-bit model of one plane's roundings:
// up to 9.6e-3 off at a side of 4, 3e-3 at 16 to 64, 2.0e-3 at 256), and small
// sides are bound by launches, not by products.
constexpr uint64_t kTwoPlaneSide = 256;

struct OrthoLayout {
    uint32_t r, k;  // padded
    int planes;
    size_t partial, master, x, xt[2], a, b, bytes;
};

OrthoLayout ortho_layout(const hc_orthogonalise_params& p) {
    OrthoLayout L;
    const uint64_t r = p.m < p.n ? p.m : p.n, k = p.m < p.n ? p.n : p.m;
    L.r = (uint32_t)((r + kBM - 1) / kBM * kBM);
    L.k = (uint32_t)((k + kBN - 1) / kBN * kBN);
    L.planes = p.type == HC_T_F32 || r <= kTwoPlaneSide ? 2 : 1;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    const size_t xs = p.batch * L.r * L.k, as = p.batch * L.r * L.r;
    L.partial = take(p.batch * kNormParts * sizeof(double));
    const bool any = p.steps > 0;
    L.master = take(any ? xs * 4 : 0);
    L.x = take(any ? xs * 2 * L.planes : 0);
    L.xt[0] = take(any ? xs * 2 * L.planes : 0);
    L.xt[1] = take(any ? xs * 2 * L.planes : 0);
    L.a = take(any ? as * 2 * L.planes : 0);
    L.b = take(any ? as * 2 * L.planes : 0);
    L.bytes = at;
    return L;
}

template <typename T, int PLANES>
hipError_t orthogonalise_typed(const hc_orthogonalise_params& p, const OrthoStep* steps,
                               const void* x, void* out, char* ws, hipStream_t s) {
    const OrthoLayout L = ortho_layout(p);
    const uint32_t batch = (uint32_t)p.batch;
    double* partial = reinterpret_cast<double*>(ws + L.partial);
    const bool flat = p.x_ld == p.n;
    const uint64_t rows = flat ? 1 : p.m, cols = flat ? p.m * p.n : p.n;
    uint64_t parts = flat ? (cols + kPrepBlock * 16 - 1) / (kPrepBlock * 16) : p.m;
    if (parts > kNormParts) parts = kNormParts;
    hipLaunchKernelGGL(norm_kernel<T>, dim3((uint32_t)parts, batch), dim3(kPrepBlock), 0, s,
                       static_cast<const T*>(x), rows, cols, p.x_ld, p.x_stride, partial);
    if (p.steps == 0) {
        hipLaunchKernelGGL(normalise_kernel<T>, dim3((uint32_t)(p.m < 1024 ? p.m : 1024), batch),
                           dim3(kPrepBlock), 0, s, p, static_cast<const T*>(x), static_cast<T*>(out),
                           partial, (uint32_t)parts);
        return hipGetLastError();
    }
    _Float16* X = reinterpret_cast<_Float16*>(ws + L.x);
    _Float16* XT[2] = {reinterpret_cast<_Float16*>(ws + L.xt[0]),
                       reinterpret_cast<_Float16*>(ws + L.xt[1])};
    _Float16* A = reinterpret_cast<_Float16*>(ws + L.a);
    _Float16* B = reinterpret_cast<_Float16*>(ws + L.b);
    PrepArgs q = {};
    q.m = p.m;
    q.n = p.n;
    q.ld = p.x_ld;
    q.stride = p.x_stride;
    q.r = L.r;
    q.k = L.k;
    q.tall = p.m > p.n;
    q.parts = (uint32_t)parts;
    q.eps = p.eps;
    q.shift = steps[0].ex;
    q.partial = partial;
    q.master = reinterpret_cast<float*>(ws + L.master);
    q.x = X;
    q.xt = XT[0];
    const dim3 tiles = q.tall ? dim3(L.r / 64, L.k / 64, batch) : dim3(L.k / 64, L.r / 64, batch);
    hipLaunchKernelGGL((prepare_kernel<T, PLANES>), tiles, dim3(kPrepBlock), 0, s, q,
                       static_cast<const T*>(x));
    const uint32_t tr = L.r / kBM, tk = L.k / kBN;
    for (uint32_t t = 0; t < p.steps; t++) {
        const OrthoStep& st = steps[t];
        Product g = {};
        g.r = L.r;
        g.k = L.k;
        g.p = g.q = X;
        g.inner = L.k;
        g.p_stride = g.q_stride = (size_t)L.r * L.k * PLANES;
        g.factor = ldexpf(1.0f, st.ea - 2 * st.ex);
        g.d = A;
        hipLaunchKernelGGL((product_kernel<GRAM, PLANES, T>), dim3(tr * (tr + 1) / 2, batch),
                           dim3(kGemmBlock), 0, s, g);
        g.p = g.q = A;
        g.inner = L.r;
        g.p_stride = g.q_stride = (size_t)L.r * L.r * PLANES;
        g.factor = ldexpf(st.c, st.eb - 2 * st.ea);
        g.factor2 = ldexpf(st.b, st.eb - st.ea);
        g.d = B;
        hipLaunchKernelGGL((product_kernel<SQUARE, PLANES, T>), dim3(tr * (tr + 1) / 2, batch),
                           dim3(kGemmBlock), 0, s, g);
        g.p = B;
        g.q = XT[t & 1];
        g.tiles_i = tr;
        g.tiles_j = tk;
        g.q_stride = (size_t)L.r * L.k * PLANES;
        g.factor = ldexpf(1.0f, -st.eb - st.ex);
        g.factor2 = st.a;
        g.next = ldexpf(1.0f, st.ex_next);
        g.d = X;
        g.dt = XT[(t + 1) & 1];
        g.master = q.master;
        if (t + 1 == p.steps) {
            g.out = out;
            g.m = p.m;
            g.n = p.n;
            g.out_ld = p.out_ld;
            g.out_stride = p.out_stride;
            g.out_scale = p.scale;
            g.tall = q.tall;
        }
        hipLaunchKernelGGL((product_kernel<APPLY, PLANES, T>), dim3(tr * tk, batch),
                           dim3(kGemmBlock), 0, s, g);
    }
    return hipGetLastError();
}

}  // namespace

size_t orthogonalise_bytes(const hc_orthogonalise_params& p) { return ortho_layout(p).bytes; }

hipError_t launch_orthogonalise(const hc_orthogonalise_params& p, const OrthoStep* steps,
                                const void* x, void* out, void* ws, hipStream_t s) {
    if (p.type == HC_T_F32)
        return orthogonalise_typed<float, 2>(p, steps, x, out, static_cast<char*>(ws), s);
    if (ortho_layout(p).planes == 2)
        return orthogonalise_typed<__bf16, 2>(p, steps, x, out, static_cast<char*>(ws), s);
    return orthogonalise_typed<__bf16, 1>(p, steps, x, out, static_cast<char*>(ws), s);
}

}  // namespace hc
