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
constexpr uint32_t kNormParts = 1024;

// 16 bytes at the alignment of their elements
template <typename T> struct Wide16 {
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Sum of squares in 64 bits, a workgroup a part: 16-byte loads, four in flight a
// lane.  rows == 1: the matrix lies in one piece.
template <typename T>
__global__ __launch_bounds__(kPrepBlock) void norm_kernel(const T* __restrict__ x, uint64_t rows,
                                                          uint64_t cols, uint64_t ld,
                                                          uint64_t stride,
                                                          double* __restrict__ partial) {
    typedef typename Wide16<T>::V V;
    constexpr int VEC = 16 / sizeof(T);
    __shared__ double s_sum[kPrepBlock / 64];
    const T* m = x + (uint64_t)blockIdx.y * stride;
    double acc = 0.0;
    auto span = [&](const T* p, uint64_t count, uint64_t first, uint64_t step) {
        const uint64_t vectors = count / VEC;
        auto add = [&](V v) {
#pragma unroll
            for (int e = 0; e < VEC; e++) acc += (double)(float)v[e] * (double)(float)v[e];
        };
        uint64_t i = first;
        for (; i + 3 * step < vectors; i += 4 * step) {
            V v[4];
#pragma unroll
            for (int u = 0; u < 4; u++) v[u] = *reinterpret_cast<const V*>(p + (i + u * step) * VEC);
#pragma unroll
            for (int u = 0; u < 4; u++) add(v[u]);
        }
        for (; i < vectors; i += step) add(*reinterpret_cast<const V*>(p + i * VEC));
        if (first < count - vectors * VEC) {
            const double v = (double)(float)p[vectors * VEC + first];
            acc += v * v;
        }
    };
    if (rows == 1) {
        span(m, cols, (uint64_t)blockIdx.x * kPrepBlock + threadIdx.x, (uint64_t)gridDim.x * kPrepBlock);
    } else {
        // a wave a row
        const uint32_t wave = blockIdx.x * (kPrepBlock / 64) + (threadIdx.x >> 6);
        for (uint64_t r = wave; r < rows; r += (uint64_t)gridDim.x * (kPrepBlock / 64))
            span(m + r * ld, cols, threadIdx.x & 63, 64);
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
    uint32_t rows, cols;  // padded m and n
    uint32_t parts;
    float eps;
    int shift;
    const double* partial;
    float* inverse;                // 1 / (norm + eps) of each matrix
    _Float16 *straight, *turned;   // operands in x's orientation and transposed
};

// A 64 x 64 tile of x, scaled by the inverse norm, as operands in both
// orientations.  Tiles cover the padded sides; the padding is zero.
template <typename T, int PLANES>
__global__ __launch_bounds__(kPrepBlock) void prepare_kernel(PrepArgs a, const T* __restrict__ x) {
    __shared__ float s_tile[64][65];
    const uint32_t b = blockIdx.z;
    const float f = inverse_norm(a.partial + (uint64_t)b * kNormParts, a.parts, a.eps);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.inverse[b] = f;
    const float scale = __builtin_ldexpf(1.0f, a.shift);
    const T* m = x + (uint64_t)b * a.stride;
    const uint32_t row0 = blockIdx.y * 64, col0 = blockIdx.x * 64;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t base = (size_t)b * a.rows * a.cols * PLANES;
    for (uint32_t j = wave; j < 64; j += 4) {
        const uint32_t r = row0 + j, c = col0 + lane;
        const float v = r < a.m && c < a.n ? (float)m[(uint64_t)r * a.ld + c] * f * scale : 0.0f;
        s_tile[j][lane] = v;
        _Float16* d = a.straight + base + operand_at<PLANES>(r, a.cols, c);
        _Float16 hi, lo = 0;
        split<PLANES>(v, hi, lo);
        d[0] = hi;
        if (PLANES == 2) d[32] = lo;
    }
    lds_barrier();
    for (uint32_t j = wave; j < 64; j += 4) {
        const uint32_t r = col0 + j, c = row0 + lane;
        _Float16* d = a.turned + base + operand_at<PLANES>(r, a.rows, c);
        _Float16 hi, lo = 0;
        split<PLANES>(s_tile[lane][j], hi, lo);
        d[0] = hi;
        if (PLANES == 2) d[32] = lo;
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

// D[i][j] = sum over l of P[i][l] Q[j][l]: both operands by rows along l.
//   GRAM    P = Q = X            D = A                        symmetric
//   SQUARE  P = Q = A            D = B = b A + c (sum)        symmetric
//   APPLY   P = B, Q = X^T       D = X <- a X + (sum), or, where x is tall,
//           P = X^T, Q = B       D = X^T <- a X^T + (sum): x's own orientation
// Of a symmetric result the tiles on and below the diagonal are computed and
// the others mirrored.
enum Kind { GRAM, SQUARE, APPLY };

struct Product {
    const _Float16 *p, *q;
    uint32_t inner;                  // length of l, a multiple of 64
    uint32_t tiles_i, tiles_j;       // tiles_j: of a result that is not symmetric
    size_t p_stride, q_stride;       // between matrices of the batch (stored values)
    float factor;                    // takes the sum to the result's unit
    float factor2;                   // SQUARE: takes the operand A to it; APPLY: a
    float next;                      // APPLY: power of two of the next operands
    // results: rows x cols (padded), as operands, and transposed
    _Float16 *d, *dt;
    uint32_t rows, cols;
    // APPLY: X in fp32; in the first step x itself is read, times the inverse norm
    float* master;
    const void* x;
    const float* inverse;
    uint64_t m, n, x_ld, x_stride;
    // APPLY, last step: the output instead of the operands
    void* out;
    uint64_t out_ld, out_stride;
    float out_scale;
};

constexpr int kLine = 64;  // stored values of a tile's row in LDS: 128 bytes

// A workgroup's tile: BM x BN, a wave's part WM x WN.
template <int BM_, int BN_, int WM_, int WN_> struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kWaves = (BM / WM) * (BN / WN);
    static constexpr int kThreads = kWaves * 64;
    static constexpr int kStageBytes = (BM + BN) * kLine * 2;
    // a wave's results pass through LDS in blocks of EM x EN
    static constexpr int EM = WM < 64 ? WM : 64, EN = WN < 64 ? WN : 64;
    static constexpr int kLdsBytes =
        2 * kStageBytes > kWaves * EM * EN * 4 ? 2 * kStageBytes : kWaves * EM * EN * 4;
};

// Result (i, j) of a block in LDS, [i][EN]: its 4-value group is turned by i so
// that rows written and columns read are spread over the banks.
template <int EN> __device__ __forceinline__ uint32_t staged(uint32_t i, uint32_t j) {
    return i * EN + ((((j >> 2) ^ i ^ (i >> 3)) & (EN / 4 - 1)) << 2) + (j & 3u);
}

// 16-byte chunk c of row `row` of an operand tile in LDS lies at c ^ (row mod
// 8): the reads of one chunk of 16 rows then touch all banks evenly.
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c) {
    return row * kLine + ((c ^ (row & 7u)) << 3);
}

typedef __attribute__((address_space(3))) void lds_void;

// Fragments and products of one 128-byte step l.  A lane holds row lane % 16 of a
// fragment, 8 values from chunk 4 h + lane / 16.  The first operand of the
// instruction gives a lane's 4 consecutive results: Q, so that they lie along j.
template <int PLANES, typename S, typename F>
__device__ __forceinline__ void main_loop(f4 (&acc)[S::WM / 16][S::WN / 16], const F& fetch,
                                          const char* s_mem, uint32_t lines, uint32_t wi,
                                          uint32_t wj, uint32_t lane) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    for (uint32_t l = 0; l < lines; l++) {
        // this wave's loads have landed, then everybody's; and everybody is done
        // reading the other buffer
        __syncthreads();
        if (l + 1 < lines) fetch(l + 1, (l + 1) & 1);
        const _Float16* sp = reinterpret_cast<const _Float16*>(s_mem + (l & 1) * S::kStageBytes);
        const _Float16* sq = sp + S::BM * kLine;
        h8 fp[2][FM], fq[2][FN];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t c = 4 * h + (lane >> 4);
#pragma unroll
            for (int u = 0; u < FM; u++)
                fp[h][u] = *reinterpret_cast<const h8*>(sp + swizzled(wi + 16 * u + (lane & 15), c));
#pragma unroll
            for (int v = 0; v < FN; v++)
                fq[h][v] = *reinterpret_cast<const h8*>(sq + swizzled(wj + 16 * v + (lane & 15), c));
            if constexpr (PLANES == 1) {
#pragma unroll
                for (int u = 0; u < FM; u++)
#pragma unroll
                    for (int v = 0; v < FN; v++)
                        acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[h][v], fp[h][u], acc[u][v], 0, 0, 0);
            }
        }
        if constexpr (PLANES == 2) {  // high x high, low x high, high x low
#pragma unroll
            for (int t = 0; t < 3; t++)
#pragma unroll
                for (int u = 0; u < FM; u++)
#pragma unroll
                    for (int v = 0; v < FN; v++)
                        acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[t == 1][v], fp[t == 2][u], acc[u][v], 0, 0, 0);
        }
    }
}

// A barrier that keeps every instruction on its side.
__device__ __forceinline__ void phase_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Eight waves, two on each SIMD: a step is two halves, a half one phase of LDS
// reads and one phase of products, with a barrier after every phase.  The second
// four waves run one phase behind, so that on every SIMD one wave multiplies
// while the other reads.  Buffers: the first four waves read step l in phases 4 l
// and 4 l + 2, the second in 4 l + 1 and 4 l + 3, so from phase 4 l + 4 on the
// buffer is free and takes step l + 2, which each wave asks for in its first
// phase of step l + 1 and waits for before the barrier that ends phase 4 l + 7.
template <int PLANES, typename S, typename F>
__device__ __forceinline__ void main_loop_paired(f4 (&acc)[S::WM / 16][S::WN / 16], const F& fetch,
                                                 const char* s_mem, uint32_t lines, uint32_t wi,
                                                 uint32_t wj, uint32_t lane, uint32_t wave) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    const bool second = wave >= 4;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    phase_barrier();
    if (second) phase_barrier();
    for (uint32_t l = 0; l < lines; l++) {
        const _Float16* sp = reinterpret_cast<const _Float16*>(s_mem + (l & 1) * S::kStageBytes);
        const _Float16* sq = sp + S::BM * kLine;
        h8 fp[2][FM], fq[2][FN];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            // one plane: a half is 32 of the 64 values of l.  Two planes: a half is
            // half of the rows, with all of Q read in the first
#pragma unroll
            for (int c2 = 0; c2 < 2; c2++) {
                if (PLANES == 1 && c2 != h) continue;
                const uint32_t c = 4 * c2 + (lane >> 4);
#pragma unroll
                for (int v = 0; v < FN; v++)
                    if (PLANES == 1 || h == 0)
                        fq[c2][v] = *reinterpret_cast<const h8*>(sq + swizzled(wj + 16 * v + (lane & 15), c));
#pragma unroll
                for (int u = 0; u < FM; u++)
                    if (PLANES == 1 || u / (FM / 2) == h)
                        fp[c2][u] = *reinterpret_cast<const h8*>(sp + swizzled(wi + 16 * u + (lane & 15), c));
            }
            if (h == 0 && l + 1 < lines) fetch(l + 1, (l + 1) & 1);
            if (second && h == 1) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
            __builtin_amdgcn_s_waitcnt(0xc07f);                        // lgkmcnt(0)
            phase_barrier();
            __builtin_amdgcn_s_setprio(1);
            if constexpr (PLANES == 1) {
#pragma unroll
                for (int u = 0; u < FM; u++)
#pragma unroll
                    for (int v = 0; v < FN; v++)
                        acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[h][v], fp[h][u], acc[u][v], 0, 0, 0);
            } else {
#pragma unroll
                for (int t = 0; t < 3; t++)
#pragma unroll
                    for (int u = h * FM / 2; u < (h + 1) * FM / 2; u++)
#pragma unroll
                        for (int v = 0; v < FN; v++)
                            acc[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[t == 1][v], fp[t == 2][u], acc[u][v], 0, 0, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            if (!second && h == 1) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
            phase_barrier();
        }
    }
    if (!second) phase_barrier();
}

template <Kind KIND, int PLANES, typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Product g) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    extern __shared__ __align__(16) char s_mem[];
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t wi = wave / (S::BN / S::WN) * S::WM, wj = wave % (S::BN / S::WN) * S::WN;
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
    const uint32_t i0 = ti * S::BM, j0 = tj * S::BN;
    const size_t line = (size_t)g.inner * PLANES;  // stored values of an operand's row
    const _Float16* P = g.p + batch * g.p_stride + (size_t)i0 * line;
    const _Float16* Q = g.q + batch * g.q_stride + (size_t)j0 * line;
    const uint32_t lines = (uint32_t)(line / kLine);

    // Tiles go from memory to LDS directly, 8 rows of 128 bytes an instruction:
    // lane l writes 16 bytes at 16 l, so it reads the chunk that belongs there.
    const __amdgpu_buffer_rsrc_t rp = buffer_rsrc(P, (uint32_t)(S::BM * line * 2));
    const __amdgpu_buffer_rsrc_t rq = buffer_rsrc(Q, (uint32_t)(S::BN * line * 2));
    const uint32_t voff = (uint32_t)((lane >> 3) * line * 2) + (((lane & 7u) ^ (lane >> 3)) << 4);
    auto fetch = [&](uint32_t l, uint32_t buf) {
        char* base = s_mem + buf * S::kStageBytes;
        constexpr int GP = S::BM / 8 / S::kWaves, GQ = S::BN / 8 / S::kWaves;
#pragma unroll
        for (int u = 0; u < GP; u++) {
            const uint32_t rows8 = wave * GP + u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rp, (lds_void*)(base + rows8 * 1024), 16, voff,
                (uint32_t)(rows8 * 8 * line * 2) + l * 128, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < GQ; u++) {
            const uint32_t rows8 = wave * GQ + u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rq, (lds_void*)(base + S::BM * kLine * 2 + rows8 * 1024), 16, voff,
                (uint32_t)(rows8 * 8 * line * 2) + l * 128, 0, 0);
        }
    };

    f4 acc[FM][FN] = {};
    fetch(0, 0);
    if constexpr (S::kWaves == 8)
        main_loop_paired<PLANES, S>(acc, fetch, s_mem, lines, wi, wj, lane, wave);
    else
        main_loop<PLANES, S>(acc, fetch, s_mem, lines, wi, wj, lane);
    __syncthreads();

    // Results: fragment (u, v) holds i = lane % 16, j = 4 (lane / 16) .. + 3.
    constexpr int EM = S::EM, EN = S::EN;
    float* stage = reinterpret_cast<float*>(s_mem) + wave * EM * EN;
    const uint32_t fi = lane & 15, fj = (lane >> 4) * 4;
    const size_t base = (size_t)batch * g.rows * g.cols;
    const bool last = KIND == APPLY && g.out != nullptr;
    const bool first = KIND == APPLY && g.x != nullptr;
    const float inverse = first ? g.inverse[batch] * g.factor2 : 0.0f;
#pragma unroll
    for (int eu = 0; eu < S::WM / EM; eu++)
#pragma unroll
        for (int ev = 0; ev < S::WN / EN; ev++) {
            const uint32_t ib = i0 + wi + eu * EM, jb = j0 + wj + ev * EN;
#pragma unroll
            for (int u = 0; u < EM / 16; u++)
#pragma unroll
                for (int v = 0; v < EN / 16; v++) {
                    const uint32_t i = ib + 16 * u + fi, j = jb + 16 * v + fj;
                    f4 w = acc[eu * (EM / 16) + u][ev * (EN / 16) + v] * g.factor;
                    if constexpr (KIND == SQUARE) {
                        const _Float16* A = g.p + batch * g.p_stride + operand_at<PLANES>(i, g.inner, j);
                        const h4 hi = *reinterpret_cast<const h4*>(A);
#pragma unroll
                        for (int e = 0; e < 4; e++) w[e] += (float)hi[e] * g.factor2;
                        if constexpr (PLANES == 2) {
                            const h4 lo = *reinterpret_cast<const h4*>(A + 32);
#pragma unroll
                            for (int e = 0; e < 4; e++) w[e] += (float)lo[e] * g.factor2;
                        }
                    }
                    if constexpr (KIND == APPLY) {
                        f4* mm = reinterpret_cast<f4*>(g.master + base + (size_t)i * g.cols + j);
                        if (first) {
                            const T* xr = static_cast<const T*>(g.x) + batch * g.x_stride + i * g.x_ld + j;
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                if (i < g.m && j + e < g.n) w[e] += (float)xr[e] * inverse;
                        } else {
                            w += *mm * g.factor2;
                        }
                        if (!last) *mm = w;
                        w *= last ? g.out_scale : g.next;
                    }
                    if (last) {
                        T* o = static_cast<T*>(g.out) + batch * g.out_stride + i * g.out_ld + j;
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (i < g.m && j + e < g.n) o[e] = (T)w[e];
                    } else {
                        h4 hi, lo;
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            _Float16 a, b = 0;
                            split<PLANES>(w[e], a, b);
                            hi[e] = a;
                            lo[e] = b;
                        }
                        _Float16* D = g.d + base * PLANES + operand_at<PLANES>(i, g.cols, j);
                        *reinterpret_cast<h4*>(D) = hi;
                        if constexpr (PLANES == 2) *reinterpret_cast<h4*>(D + 32) = lo;
                        *reinterpret_cast<f4*>(stage + staged<EN>(16 * u + fi, 16 * v + fj)) = w;
                    }
                }
            if (last || (KIND != APPLY && ti == tj)) continue;
            // the transpose: 8 consecutive i of one j a lane (only this wave's results)
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_wave_barrier();
            constexpr int kPer = EM / 8;  // lanes for one j
#pragma unroll
            for (int q = 0; q < EN * kPer / 64; q++) {
                const uint32_t jj = q * (64 / kPer) + lane / kPer, ii = lane % kPer * 8;
                h8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    _Float16 a, b = 0;
                    split<PLANES>(stage[staged<EN>(ii + e, jj)], a, b);
                    hi[e] = a;
                    lo[e] = b;
                }
                _Float16* D = g.dt + base * PLANES + operand_at<PLANES>(jb + jj, g.rows, ib + ii);
                *reinterpret_cast<h8*>(D) = hi;
                if constexpr (PLANES == 2) *reinterpret_cast<h8*>(D + 32) = lo;
            }
            __builtin_amdgcn_wave_barrier();
        }
}

// ---- layout and launches ---------------------------------------------------------

typedef Shape<256, 256, 128, 64> Large;
typedef Shape<128, 128, 64, 64> Medium;
typedef Shape<64, 64, 32, 32> Small;

// bf16 matrices with a side of at most this take two planes too: the rounding
// of few entries does not average out (a 64-bit model of one plane's roundings:
// up to 9.6e-3 off at a side of 4, 3e-3 at 16 to 64, 2.0e-3 at 256), and small
// sides are bound by launches, not by products.
constexpr uint64_t kTwoPlaneSide = 256;

struct OrthoLayout {
    uint32_t rows, cols, r;  // padded m, n and their smaller
    int planes;
    bool tall;
    int tile;
    size_t partial, inverse, master, x, xt[2], a, b, bytes;
};

int tile_for(const hc_orthogonalise_params& p) {
    const uint64_t r = p.m < p.n ? p.m : p.n;
    return r > 1536 ? 256 : r > 64 ? 128 : 64;
}

OrthoLayout ortho_layout(const hc_orthogonalise_params& p) {
    OrthoLayout L;
    const uint64_t r = p.m < p.n ? p.m : p.n;
    L.tile = tile_for(p);
    const uint64_t t = L.tile;
    L.rows = (uint32_t)((p.m + t - 1) / t * t);
    L.cols = (uint32_t)((p.n + t - 1) / t * t);
    L.tall = p.m > p.n;
    L.r = L.tall ? L.cols : L.rows;
    L.planes = p.type == HC_T_F32 || r <= kTwoPlaneSide ? 2 : 1;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    const bool any = p.steps > 0;
    const size_t xs = any ? p.batch * L.rows * L.cols : 0, as = any ? p.batch * L.r * L.r : 0;
    L.partial = take(p.batch * kNormParts * sizeof(double));
    L.inverse = take(p.batch * 4);
    L.master = take(xs * 4);
    L.x = take(xs * 2 * L.planes);
    L.xt[0] = take(xs * 2 * L.planes);
    L.xt[1] = take(xs * 2 * L.planes);
    L.a = take(as * 2 * L.planes);
    L.b = take(as * 2 * L.planes);
    L.bytes = at;
    return L;
}

template <Kind KIND, int PLANES, typename T, typename S>
hipError_t product_shape(Product g, uint32_t batch, hipStream_t s) {
    const auto kernel = &product_kernel<KIND, PLANES, T, S>;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), S::kLdsBytes);
    if (e != hipSuccess) return e;
    g.tiles_i = g.rows / S::BM;
    g.tiles_j = g.cols / S::BN;
    const uint32_t tiles = KIND == APPLY ? g.tiles_i * g.tiles_j : g.tiles_i * (g.tiles_i + 1) / 2;
    hipLaunchKernelGGL(kernel, dim3(tiles, batch), dim3(S::kThreads), S::kLdsBytes, s, g);
    return hipGetLastError();
}

template <Kind KIND, int PLANES, typename T>
hipError_t product(const Product& g, int tile, uint32_t batch, hipStream_t s) {
    if (tile == 256) return product_shape<KIND, PLANES, T, Large>(g, batch, s);
    if (tile == 128) return product_shape<KIND, PLANES, T, Medium>(g, batch, s);
    return product_shape<KIND, PLANES, T, Small>(g, batch, s);
}

template <typename T, int PLANES>
hipError_t orthogonalise_typed(const hc_orthogonalise_params& p, const OrthoStep* steps,
                               const void* x, void* out, char* ws, hipStream_t s) {
    const OrthoLayout L = ortho_layout(p);
    const uint32_t batch = (uint32_t)p.batch;
    double* partial = reinterpret_cast<double*>(ws + L.partial);
    const bool flat = p.x_ld == p.n;
    const uint64_t rows = flat ? 1 : p.m, cols = flat ? p.m * p.n : p.n;
    uint64_t parts = flat ? (cols + kPrepBlock * 16 - 1) / (kPrepBlock * 16) : (p.m + 3) / 4;
    if (parts > kNormParts) parts = kNormParts;
    hipLaunchKernelGGL(norm_kernel<T>, dim3((uint32_t)parts, batch), dim3(kPrepBlock), 0, s,
                       static_cast<const T*>(x), rows, cols, p.x_ld, p.x_stride, partial);
    if (p.steps == 0) {
        hipLaunchKernelGGL(normalise_kernel<T>, dim3((uint32_t)(p.m < 1024 ? p.m : 1024), batch),
                           dim3(kPrepBlock), 0, s, p, static_cast<const T*>(x), static_cast<T*>(out),
                           partial, (uint32_t)parts);
        return hipGetLastError();
    }
    _Float16* X = reinterpret_cast<_Float16*>(ws + L.x);  // by the shorter side's rows
    _Float16* XT[2] = {reinterpret_cast<_Float16*>(ws + L.xt[0]),
                       reinterpret_cast<_Float16*>(ws + L.xt[1])};
    _Float16* A = reinterpret_cast<_Float16*>(ws + L.a);
    _Float16* B = reinterpret_cast<_Float16*>(ws + L.b);
    float* inverse = reinterpret_cast<float*>(ws + L.inverse);
    PrepArgs q = {};
    q.m = p.m;
    q.n = p.n;
    q.ld = p.x_ld;
    q.stride = p.x_stride;
    q.rows = L.rows;
    q.cols = L.cols;
    q.parts = (uint32_t)parts;
    q.eps = p.eps;
    q.shift = steps[0].ex;
    q.partial = partial;
    q.inverse = inverse;
    q.straight = L.tall ? XT[0] : X;
    q.turned = L.tall ? X : XT[0];
    hipLaunchKernelGGL((prepare_kernel<T, PLANES>), dim3(L.cols / 64, L.rows / 64, batch),
                       dim3(kPrepBlock), 0, s, q, static_cast<const T*>(x));
    hipError_t e = hipGetLastError();
    const size_t x_size = (size_t)L.rows * L.cols * PLANES, a_size = (size_t)L.r * L.r * PLANES;
    for (uint32_t t = 0; t < p.steps && e == hipSuccess; t++) {
        const OrthoStep& st = steps[t];
        Product g = {};
        g.p = g.q = X;
        g.p_stride = g.q_stride = x_size;
        g.inner = L.tall ? L.rows : L.cols;
        g.factor = ldexpf(1.0f, st.ea - 2 * st.ex);
        g.rows = g.cols = L.r;
        g.d = g.dt = A;
        e = product<GRAM, PLANES, T>(g, L.tile, batch, s);
        if (e != hipSuccess) return e;
        g.p = g.q = A;
        g.p_stride = g.q_stride = a_size;
        g.inner = L.r;
        g.factor = ldexpf(st.c, st.eb - 2 * st.ea);
        g.factor2 = ldexpf(st.b, st.eb - st.ea);
        g.d = g.dt = B;
        e = product<SQUARE, PLANES, T>(g, L.tile, batch, s);
        if (e != hipSuccess) return e;
        g.p = L.tall ? XT[t & 1] : B;
        g.q = L.tall ? B : XT[t & 1];
        g.p_stride = L.tall ? x_size : a_size;
        g.q_stride = L.tall ? a_size : x_size;
        g.factor = ldexpf(1.0f, -st.eb - st.ex);
        g.factor2 = st.a;
        g.next = ldexpf(1.0f, st.ex_next);
        g.rows = L.rows;
        g.cols = L.cols;
        g.d = L.tall ? XT[(t + 1) & 1] : X;
        g.dt = L.tall ? X : XT[(t + 1) & 1];
        g.master = reinterpret_cast<float*>(ws + L.master);
        g.m = p.m;
        g.n = p.n;
        if (t == 0) {
            g.x = x;
            g.inverse = inverse;
            g.x_ld = p.x_ld;
            g.x_stride = p.x_stride;
        }
        if (t + 1 == p.steps) {
            g.out = out;
            g.out_ld = p.out_ld;
            g.out_stride = p.out_stride;
            g.out_scale = p.scale;
        }
        e = product<APPLY, PLANES, T>(g, L.tile, batch, s);
    }
    return e;
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
