// hc_ortho.hip -- Newton-Schulz orthogonalisation (include/hc_train.h).
//
// X_0 = x / (|x|_F + eps), held with its shorter side (r) as rows and its longer
// side (k) as columns; then per step A = X X^T, B = b A + c A^2 and
// X <- a X + B X.  The three products run on the matrix cores.
//
// Precision.  The operands of the products are fp16 times a power of two that
// the bound on the singular values allows (so nothing overflows and what
// matters stays normal), sums are fp32, and X itself is kept with 22 bits or
// more beside its operands: a X is added in fp32, so that rounding an operand
// only reaches X through B, which is small where X's singular values are.  For
// bf16 matrices one fp16 plane, X being its operand plus an fp16 rest: five steps
// leave the result 1.8e-3 (low rank over noise) to 2.7e-3 (400 x 5000, random)
// from the exact one, of which rounding it to bf16 is 1.7e-3, what fp32 products
// leave; nine steps up to 4.9e-3, twelve 6.9e-3 (library products in bf16, five
// steps: 1.7e-2 and more; fp16 operands without the rest: up to 2e-2).  That
// form holds X to 2^-38, so where all of x is below about 1e-10 eps the result
// loses bits, and below 1e-12 eps it is zero.  For fp32 matrices an operand is
// the sum of two fp16 planes and a product three matrix products (high x high,
// high x low, low x high), X is fp32: five steps 1e-6 to 9e-6 from the exact
// result, 0.35 to 1.15 times what fp32 products of the matrix library leave.
//
// What bounds it.  Large matrices: the matrix cores, of which the main loop of a
// 256-tile gets 1.31 PFLOP/s (4096 x 25088, the apply without its results; a
// library product of 8192^3 1.37), and then X's way to memory and back in the
// apply (10 or 16 bytes a value), hardly overlapped as all CUs end their tiles
// together: 780 us where the products alone take 629.  Half of the Gram product
// and of the square are computed and mirrored.  Small ones: the chain of
// launches, three a step (thin ones one or two) of 6 to 8 us each.
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

// Value (i, j) of a block in LDS, [i][EN]: its 4-value group is turned by i so
// that rows written and columns read are spread over the banks.
template <int EN> __device__ __forceinline__ uint32_t staged(uint32_t i, uint32_t j) {
    return i * EN + ((((j >> 2) ^ i ^ (i >> 3)) & (EN / 4 - 1)) << 2) + (j & 3u);
}

// ---- norm and operands of X_0 ----------------------------------------------------

constexpr int kPrepBlock = 256, kNormBlock = 1024;
constexpr uint32_t kNormParts = 256;  // every wave of the next launch sums them

// 16 bytes at the alignment of their elements
template <typename T> struct Wide16 {
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Sum of squares in 64 bits, a workgroup a part: 16-byte loads, four in flight a
// lane.  rows == 1: the matrix lies in one piece.  4096 x 25088 bf16: 52 us, 4.0
// TB/s.
template <typename T>
__global__ __launch_bounds__(kNormBlock) void norm_kernel(const T* __restrict__ x, uint64_t rows,
                                                          uint64_t cols, uint64_t ld,
                                                          uint64_t stride,
                                                          double* __restrict__ partial) {
    typedef typename Wide16<T>::V V;
    constexpr int VEC = 16 / sizeof(T);
    __shared__ double s_sum[kNormBlock / 64];
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
        span(m, cols, (uint64_t)blockIdx.x * kNormBlock + threadIdx.x, (uint64_t)gridDim.x * kNormBlock);
    } else {
        // a wave a row
        const uint32_t wave = blockIdx.x * (kNormBlock / 64) + (threadIdx.x >> 6);
        for (uint64_t r = wave; r < rows; r += (uint64_t)gridDim.x * (kNormBlock / 64))
            span(m + r * ld, cols, threadIdx.x & 63, 64);
    }
    for (int d = 32; d > 0; d >>= 1) acc += __shfl_xor(acc, d);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = acc;
    lds_barrier();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < kNormBlock / 64; w++) t += s_sum[w];
        partial[(uint64_t)blockIdx.y * kNormParts + blockIdx.x] = t;
    }
}

// 1 / (norm + eps), or NaN where the norm is not finite, as two factors: the norm
// of finite fp32 values reaches 2^144, whose inverse no fp32 holds.  From 2^64 on
// `pre` is 2^-64 (what it takes below the normal range is nothing beside the norm).
struct Inverse {
    float pre, rest;
    __device__ __forceinline__ float of(float v) const { return v * pre * rest; }
};

// Every lane calls it.
__device__ __forceinline__ Inverse inverse_norm(const double* partial, uint32_t parts, float eps) {
    double t = 0.0;
    for (uint32_t i = lane_id(); i < parts; i += 64) t += partial[i];
    for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
    const double n = sqrt(t);
    const float pre = n >= 0x1p64 ? 0x1p-64f : 1.0f;
    return {pre, n < __builtin_inf() ? (float)(1.0 / ((n + (double)eps) * pre)) : __builtin_nanf("")};
}

struct PrepArgs {
    uint64_t m, n, ld, stride;
    uint32_t rows, cols;  // padded m and n
    uint32_t parts;
    float eps;
    int shift;
    const double* partial;
    Inverse* inverse;              // 1 / (norm + eps) of each matrix
    _Float16 *straight, *turned;   // operands in x's orientation and transposed
};

// A 64 x 64 tile of x, scaled by the inverse norm, as operands in both
// orientations.  Tiles cover the padded sides; the padding is zero.  4096 x 25088
// bf16: 107 us, 5.8 TB/s (275 with 2-byte stores and four times the parts).
template <typename T, int PLANES>
__global__ __launch_bounds__(kPrepBlock) void prepare_kernel(PrepArgs a, const T* __restrict__ x) {
    __shared__ __align__(16) float s_tile[64 * 64];
    const uint32_t b = blockIdx.z;
    const Inverse f = inverse_norm(a.partial + (uint64_t)b * kNormParts, a.parts, a.eps);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.inverse[b] = f;
    const float scale = __builtin_ldexpf(1.0f, a.shift);
    const T* m = x + (uint64_t)b * a.stride;
    const uint32_t row0 = blockIdx.y * 64, col0 = blockIdx.x * 64;
    const size_t base = (size_t)b * a.rows * a.cols * PLANES;
    // 8 values of a row a lane, then 8 of a column: 16-byte stores
    typedef T T8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    float v[2][8];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t q = threadIdx.x + kPrepBlock * k;
        const uint32_t r = row0 + q / 8, c = col0 + q % 8 * 8;
        const T* p = m + (uint64_t)r * a.ld + c;
        if (r < a.m && c + 7 < a.n) {
            const T8 t = *reinterpret_cast<const T8*>(p);
#pragma unroll
            for (int e = 0; e < 8; e++) v[k][e] = (float)t[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) v[k][e] = r < a.m && c + e < a.n ? (float)p[e] : 0.0f;
        }
    }
    auto store = [](_Float16* d, const float (&w)[8]) {
        h8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            _Float16 x, y = 0;
            split<PLANES>(w[e], x, y);
            hi[e] = x;
            lo[e] = y;
        }
        *reinterpret_cast<h8*>(d) = hi;
        if constexpr (PLANES == 2) *reinterpret_cast<h8*>(d + 32) = lo;
    };
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t q = threadIdx.x + kPrepBlock * k, ii = q / 8, jj = q % 8 * 8;
        const bool in = row0 + ii < a.m;
#pragma unroll
        for (int e = 0; e < 8; e++)  // the padding stays zero whatever f is
            v[k][e] = in && col0 + jj + e < a.n ? f.of(v[k][e]) * scale : 0.0f;
#pragma unroll
        for (int h = 0; h < 2; h++)
            *reinterpret_cast<f4*>(s_tile + staged<64>(ii, jj + 4 * h)) =
                f4{v[k][4 * h], v[k][4 * h + 1], v[k][4 * h + 2], v[k][4 * h + 3]};
        store(a.straight + base + operand_at<PLANES>(row0 + ii, a.cols, col0 + jj), v[k]);
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t q = threadIdx.x + kPrepBlock * k, jj = q / 8, ii = q % 8 * 8;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; e++) w[e] = s_tile[staged<64>(ii + e, jj)];
        store(a.turned + base + operand_at<PLANES>(col0 + jj, a.rows, row0 + ii), w);
    }
}

// No steps: the normalised matrix itself.
template <typename T>
__global__ __launch_bounds__(kPrepBlock) void normalise_kernel(hc_orthogonalise_params p,
                                                               const T* __restrict__ x,
                                                               T* __restrict__ out,
                                                               const double* __restrict__ partial,
                                                               uint32_t parts) {
    const Inverse f = inverse_norm(partial + (uint64_t)blockIdx.y * kNormParts, parts, p.eps);
    const T* m = x + (uint64_t)blockIdx.y * p.x_stride;
    T* o = out + (uint64_t)blockIdx.y * p.out_stride;
    for (uint64_t r = blockIdx.x; r < p.m; r += gridDim.x)
        for (uint64_t i = threadIdx.x; i < p.n; i += kPrepBlock)
            o[r * p.out_ld + i] = (T)(f.of((float)m[r * p.x_ld + i]) * p.scale);
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
// APPLY's step: the first reads x itself, the last writes the output.
enum Step { MIDDLE = 0, FIRST = 1, LAST = 2 };

// Few tiles: each is cut along l into pieces, one or two a workgroup, whose sums
// a launch of its own adds up.  The first `tiles` of them in `first` pieces, the
// others in `second`.  first == 1: those fill the CUs whole, in a launch before
// (528 tiles of 4096 x 4096 on 512 places, bf16: 104 us as whole tiles, 88).
struct Cuts {
    uint32_t tiles, first, others, second;
    __host__ __device__ uint32_t whole() const { return first == 1 ? tiles : 0; }
    __host__ __device__ uint32_t first_pieces() const { return first == 1 ? 0 : tiles * first; }
    __host__ __device__ uint32_t pieces() const { return first_pieces() + others * second; }
    __host__ __device__ uint32_t groups() const { return max(first_pieces(), others * second); }
};

struct Product {
    const _Float16 *p, *q;
    uint32_t inner;                  // length of l, a multiple of 64
    uint32_t tiles_i, tiles_j;       // tiles_j: of a result that is not symmetric
    uint32_t tiles;                  // of one matrix that this launch makes
    uint32_t first;                  // APPLY: first of them along the longer side
    uint32_t batch;
    Cuts cuts;
    float* part;                     // sums of the tiles' pieces
    size_t p_stride, q_stride;       // between matrices of the batch (stored values)
    float factor;                    // takes the sum to the result's unit
    float factor2;                   // SQUARE: takes the operand A to it; APPLY: a
    float next;                      // APPLY: power of two of the next operands
    // results: rows x cols (padded), as operands, and transposed
    _Float16 *d, *dt;
    uint32_t rows, cols;
    // APPLY: X between the steps: fp32 (two planes), or its operand `prev` and the
    // fp16 rest `master` in the same unit (one); in the first step x itself is
    // read, times the inverse norm
    void* master;
    const _Float16* prev;
    const void* x;
    const Inverse* inverse;
    uint64_t m, n, x_ld, x_stride;
    // APPLY, last step: the output instead of the operands
    void* out;
    uint64_t out_ld, out_stride;
    float out_scale;
};

constexpr int kLine = 64;  // stored values of a tile's row in LDS: 128 bytes

// A workgroup's tile: BM x BN, a wave's part WM x WN.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_> struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kStages = STAGES_;
    static constexpr int kWaves = (BM / WM) * (BN / WN);
    static constexpr int kThreads = kWaves * 64;
    static constexpr int kStageBytes = (BM + BN) * kLine * 2;
    // a wave's results pass through LDS in blocks of EM x EN
    static constexpr int EM = WM < 64 ? WM : 64, EN = WN < 64 ? WN : 64;
    static constexpr int kLdsBytes =
        kStages * kStageBytes > kWaves * EM * EN * 4 ? kStages * kStageBytes : kWaves * EM * EN * 4;
};

// 16-byte chunk c of row `row` of an operand tile in LDS lies at c ^ (row mod
// 8): the reads of one chunk of 16 rows then touch all banks evenly.
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c) {
    return row * kLine + ((c ^ (row & 7u)) << 3);
}

typedef __attribute__((address_space(3))) void lds_void;

// A barrier that keeps every instruction on its side.
__device__ __forceinline__ void phase_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ f4 product16(h8 a, h8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Fragments and products of one 128-byte step l.  A lane holds row lane % 16 of a
// fragment, 8 values from chunk 4 h + lane / 16.  The first operand of the
// instruction gives a lane's 4 consecutive results: Q, so that they lie along j.
template <int PLANES, typename S, typename F>
__device__ __forceinline__ void main_loop(f4 (&acc)[S::WM / 16][S::WN / 16], const F& fetch,
                                          const char* s_mem, uint32_t lines, uint32_t wi,
                                          uint32_t wj, uint32_t lane) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    constexpr uint32_t N = S::kStages;
    constexpr uint32_t kLoads = (S::BM + S::BN) / 8 / S::kWaves;  // of a wave and step
#pragma unroll
    for (uint32_t l = 1; l + 1 < N; l++)
        if (l < lines) fetch(l, l);
    uint32_t buf = 0;
    for (uint32_t l = 0; l < lines; l++) {
        // this wave's loads of step l have landed (those of later steps may be on
        // their way), then everybody's; and everybody is done with step l - 1
        if (l + N - 2 < lines)
            __builtin_amdgcn_s_waitcnt(0x0f70 | ((N - 2) * kLoads & 15) |
                                       ((N - 2) * kLoads >> 4) << 14);
        else
            __builtin_amdgcn_s_waitcnt(0x0f70);
        phase_barrier();
        if (l + N - 1 < lines) fetch(l + N - 1, buf == 0 ? N - 1 : buf - 1);
        const _Float16* sp = reinterpret_cast<const _Float16*>(s_mem + buf * S::kStageBytes);
        buf = buf + 1 == N ? 0 : buf + 1;
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
                        acc[u][v] = product16(fq[h][v], fp[h][u], acc[u][v]);
            }
        }
        if constexpr (PLANES == 2) {  // high x high, low x high, high x low
#pragma unroll
            for (int t = 0; t < 3; t++)
#pragma unroll
                for (int u = 0; u < FM; u++)
#pragma unroll
                    for (int v = 0; v < FN; v++)
                        acc[u][v] = product16(fq[t == 1][v], fp[t == 2][u], acc[u][v]);
        }
    }
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
                        acc[u][v] = product16(fq[h][v], fp[h][u], acc[u][v]);
            } else {
#pragma unroll
                for (int t = 0; t < 3; t++)
#pragma unroll
                    for (int u = h * FM / 2; u < (h + 1) * FM / 2; u++)
#pragma unroll
                        for (int v = 0; v < FN; v++)
                            acc[u][v] = product16(fq[t == 1][v], fp[t == 2][u], acc[u][v]);
            }
            __builtin_amdgcn_s_setprio(0);
            if (!second && h == 1) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
            phase_barrier();
        }
    }
    if (!second) phase_barrier();
}

// A tile's matrix and place.
struct Tile {
    uint32_t batch, ti, tj;
};

template <Kind KIND> __device__ __forceinline__ Tile tile_at(const Product& g, uint32_t t) {
    Tile o;
    o.batch = t / g.tiles;
    t -= o.batch * g.tiles;
    if constexpr (KIND == APPLY) {
        // blocks of 8 tiles along the shorter side (B's) by 4 along the longer:
        // the 32 tiles that an XCD works on then read 12 panels, not 18
        const bool wide = g.tiles_i <= g.tiles_j;
        const uint32_t across = wide ? g.tiles_i : g.tiles_j, along = g.tiles / across;
        const uint32_t stripe = t / (4 * across);
        t -= stripe * 4 * across;
        const uint32_t w = min(4u, along - 4 * stripe), block = t / (8 * w);
        t -= block * 8 * w;
        const uint32_t h = min(8u, across - 8 * block);
        const uint32_t r = 8 * block + t % h, k = g.first + 4 * stripe + t / h;
        o.ti = wide ? r : k;
        o.tj = wide ? k : r;
    } else {
        // the lower triangle in squares of 4 x 4 tiles, so that tiles near each
        // other in the order share rows of both operands; row I of squares begins
        // at 8 I^2 + 2 I
        uint32_t I = (uint32_t)(sqrtf((float)t * 0.125f));
        while (I > 0 && 8 * I * I + 2 * I > t) I--;
        while (8 * (I + 1) * (I + 1) + 2 * (I + 1) <= t) I++;
        uint32_t q = t - (8 * I * I + 2 * I);
        const uint32_t h = min(4u, g.tiles_i - 4 * I);  // rows of this row of squares
        if (q < I * 4 * h) {
            const uint32_t J = q / (4 * h);
            q -= J * 4 * h;
            o.ti = 4 * I + q % h;
            o.tj = 4 * J + q / h;
        } else {
            q -= I * 4 * h;
            const uint32_t r = q < 1 ? 0 : q < 3 ? 1 : q < 6 ? 2 : 3;
            o.ti = 4 * I + r;
            o.tj = 4 * I + q - r * (r + 1) / 2;
        }
    }
    return o;
}

// Workgroups go to the 8 XCDs in turn; each XCD takes a contiguous share of the
// tiles, so that what neighbouring tiles read is shared in its L2.
__device__ __forceinline__ uint32_t by_xcd(uint32_t block, uint32_t blocks) {
    const uint32_t xcd = block & 7u, k = block >> 3, per = blocks >> 3, more = blocks & 7u;
    return xcd * per + min(xcd, more) + k;
}

// Steps [l0, l1) of a tile, added to acc.
template <int PLANES, typename S>
__device__ __forceinline__ void accumulate(const Product& g, const Tile& tile, uint32_t l0,
                                           uint32_t l1, char* s_mem,
                                           f4 (&acc)[S::WM / 16][S::WN / 16]) {
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t wi = wave / (S::BN / S::WN) * S::WM, wj = wave % (S::BN / S::WN) * S::WN;
    const size_t line = (size_t)g.inner * PLANES;  // stored values of an operand's row
    const _Float16* P = g.p + tile.batch * g.p_stride + (size_t)tile.ti * S::BM * line;
    const _Float16* Q = g.q + tile.batch * g.q_stride + (size_t)tile.tj * S::BN * line;
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
                (uint32_t)(rows8 * 8 * line * 2) + (l0 + l) * 128, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < GQ; u++) {
            const uint32_t rows8 = wave * GQ + u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rq, (lds_void*)(base + S::BM * kLine * 2 + rows8 * 1024), 16, voff,
                (uint32_t)(rows8 * 8 * line * 2) + (l0 + l) * 128, 0, 0);
        }
    };
    fetch(0, 0);
    if constexpr (S::kWaves == 8)
        main_loop_paired<PLANES, S>(acc, fetch, s_mem, l1 - l0, wi, wj, lane, wave);
    else
        main_loop<PLANES, S>(acc, fetch, s_mem, l1 - l0, wi, wj, lane);
    __syncthreads();
}

// What a tile's sums become, and where they go.
template <Kind KIND, int STEP, int PLANES, typename T, typename S> struct Results {
    const Product& g;
    size_t base;      // of the matrix
    uint32_t batch;
    bool turn;        // the transpose is stored too
    float addend_pre, addend_factor;
    static constexpr bool first = KIND == APPLY && (STEP & FIRST), last = KIND == APPLY && (STEP & LAST);

    __device__ __forceinline__ Results(const Product& g_, const Tile& t)
        : g(g_), base((size_t)t.batch * g_.rows * g_.cols), batch(t.batch),
          turn(KIND == APPLY ? !last : t.ti != t.tj),
          addend_pre(first ? g_.inverse[t.batch].pre : 1.0f),
          addend_factor(first ? g_.inverse[t.batch].rest * g_.factor2 : g_.factor2) {}

    // X between two steps passes the caches by in the tiles of large matrices,
    // which they cannot hold: 2 % of 4096 x 25088 (of twelve 768 x 768, in smaller
    // tiles, it would cost 2 %).
    template <typename V> __device__ __forceinline__ static V load_x(const V* p) {
        if constexpr (S::BM == 256) return __builtin_nontemporal_load(p);
        return *p;
    }
    template <typename V> __device__ __forceinline__ static void store_x(V* p, V v) {
        if constexpr (S::BM == 256) __builtin_nontemporal_store(v, p);
        else *p = v;
    }

    // What is added to the sums of (i, j .. j + 7): A, or X, or x in the first step.
    __device__ __forceinline__ void addend(uint32_t i, uint32_t j, f4 (&w)[2]) const {
        if constexpr (KIND == SQUARE) {
            const _Float16* A = g.p + batch * g.p_stride + operand_at<PLANES>(i, g.inner, j);
            const h8 hi = *reinterpret_cast<const h8*>(A);
#pragma unroll
            for (int e = 0; e < 8; e++) w[e >> 2][e & 3] = (float)hi[e];
            if constexpr (PLANES == 2) {
                const h8 lo = *reinterpret_cast<const h8*>(A + 32);
#pragma unroll
                for (int e = 0; e < 8; e++) w[e >> 2][e & 3] += (float)lo[e];
            }
        }
        if constexpr (first) {
            typedef T T8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
            const T* xr = static_cast<const T*>(g.x) + batch * g.x_stride + i * g.x_ld + j;
            if (i < g.m && j + 7 < g.n) {
                const T8 v = *reinterpret_cast<const T8*>(xr);
#pragma unroll
                for (int e = 0; e < 8; e++) w[e >> 2][e & 3] = (float)v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    w[e >> 2][e & 3] = i < g.m && j + e < g.n ? (float)xr[e] : 0.0f;
            }
        } else if constexpr (KIND == APPLY) {
            const size_t at = base + (size_t)i * g.cols + j;
            if constexpr (PLANES == 2) {
                const f4* mm = reinterpret_cast<const f4*>(static_cast<const float*>(g.master) + at);
                w[0] = load_x(mm);
                w[1] = load_x(mm + 1);
            } else {
                const h8 hi = load_x(reinterpret_cast<const h8*>(g.prev + at));
                const h8 lo = load_x(reinterpret_cast<const h8*>(static_cast<const _Float16*>(g.master) + at));
#pragma unroll
                for (int e = 0; e < 8; e++) w[e >> 2][e & 3] = (float)hi[e] + (float)lo[e];
            }
        }
    }

    // A block's sums in LDS become its results, 8 consecutive j of one i a lane, so
    // that rows of 128 bytes are read and stored; what the transpose needs goes
    // back to LDS.  N rounds of lanes `at`, at + step, ...: all addends are asked
    // for before the first store, so that the loads do not wait for each other.
    template <int N>
    __device__ __forceinline__ void straight(float* stage, uint32_t ib, uint32_t jb, uint32_t at,
                                             uint32_t step) const {
        constexpr int kPer = S::EN / 8;  // lanes for one i
        f4 add[N][2];
        if constexpr (KIND != GRAM)
#pragma unroll
            for (int k = 0; k < N; k++) {
                const uint32_t q = at + k * step;
                addend(ib + q / kPer, jb + q % kPer * 8, add[k]);
            }
#pragma unroll
        for (int k = 0; k < N; k++) {
            const uint32_t q = at + k * step;
            const uint32_t ii = q / kPer, jj = q % kPer * 8, i = ib + ii, j = jb + jj;
            f4 w[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                f4* at_stage = reinterpret_cast<f4*>(stage + staged<S::EN>(ii, jj + 4 * h));
                w[h] = *at_stage * g.factor;
                if constexpr (first) add[k][h] *= addend_pre;
                if constexpr (KIND != GRAM) w[h] += add[k][h] * addend_factor;
                if (turn) *at_stage = w[h];
            }
            if constexpr (last) {
                typedef T T8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
                T* o = static_cast<T*>(g.out) + batch * g.out_stride + i * g.out_ld + j;
                if (i < g.m && j + 7 < g.n) {
                    T8 v;
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = (T)(w[e >> 2][e & 3] * g.out_scale);
                    *reinterpret_cast<T8*>(o) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (i < g.m && j + e < g.n) o[e] = (T)(w[e >> 2][e & 3] * g.out_scale);
                }
            } else {
                const size_t mat = base + (size_t)i * g.cols + j;
                if constexpr (KIND == APPLY && PLANES == 2) {
                    f4* mm = reinterpret_cast<f4*>(static_cast<float*>(g.master) + mat);
                    store_x(mm, w[0]);
                    store_x(mm + 1, w[1]);
                }
                h8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    _Float16 x, y;
                    split<2>(w[e >> 2][e & 3] * (KIND == APPLY ? g.next : 1.0f), x, y);
                    hi[e] = x;
                    lo[e] = y;
                }
                _Float16* D = g.d + base * PLANES + operand_at<PLANES>(i, g.cols, j);
                *reinterpret_cast<h8*>(D) = hi;
                if constexpr (PLANES == 2)
                    *reinterpret_cast<h8*>(D + 32) = lo;
                else if constexpr (KIND == APPLY)
                    store_x(reinterpret_cast<h8*>(static_cast<_Float16*>(g.master) + mat), lo);
            }
        }
    }

    // The transpose of a block in LDS: 8 consecutive i of one j a lane.  Lanes
    // `at`, at + step, ... of the EM EN / 8.
    __device__ __forceinline__ void turned(const float* stage, uint32_t ib, uint32_t jb, uint32_t at,
                                           uint32_t step) const {
        constexpr int kPer = S::EM / 8;  // lanes for one j
        for (uint32_t q = at; q < S::EN * kPer; q += step) {
            const uint32_t jj = q / kPer, ii = q % kPer * 8;
            h8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                _Float16 x, y = 0;
                split<PLANES>(stage[staged<S::EN>(ii + e, jj)] * (KIND == APPLY ? g.next : 1.0f), x, y);
                hi[e] = x;
                lo[e] = y;
            }
            _Float16* D = g.dt + base * PLANES + operand_at<PLANES>(jb + jj, g.rows, ib + ii);
            *reinterpret_cast<h8*>(D) = hi;
            if constexpr (PLANES == 2) *reinterpret_cast<h8*>(D + 32) = lo;
        }
    }
};

// A workgroup's sums of a whole tile become its results, a wave its own part:
// fragment (u, v) of a lane holds i = lane % 16, j = 4 (lane / 16) .. + 3.
template <Kind KIND, int STEP, int PLANES, typename T, typename S>
__device__ __forceinline__ void finish(const Product& g, const Tile& tile, char* s_mem,
                                       f4 (&acc)[S::WM / 16][S::WN / 16]) {
    constexpr int EM = S::EM, EN = S::EN;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t i0 = tile.ti * S::BM + wave / (S::BN / S::WN) * S::WM;
    const uint32_t j0 = tile.tj * S::BN + wave % (S::BN / S::WN) * S::WN;
    const uint32_t fi = lane & 15, fj = (lane >> 4) * 4;
    float* stage = reinterpret_cast<float*>(s_mem) + wave * EM * EN;
    const Results<KIND, STEP, PLANES, T, S> out(g, tile);
#pragma unroll
    for (int eu = 0; eu < S::WM / EM; eu++)
#pragma unroll
        for (int ev = 0; ev < S::WN / EN; ev++) {
            const uint32_t ib = i0 + eu * EM, jb = j0 + ev * EN;
#pragma unroll
            for (int u = 0; u < EM / 16; u++)
#pragma unroll
                for (int v = 0; v < EN / 16; v++)
                    *reinterpret_cast<f4*>(stage + staged<EN>(16 * u + fi, 16 * v + fj)) =
                        acc[eu * (EM / 16) + u][ev * (EN / 16) + v];
            // only this wave's results are read
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_wave_barrier();
            out.template straight<EM * EN / 512>(stage, ib, jb, lane, 64);
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_wave_barrier();
            if (out.turn) out.turned(stage, ib, jb, lane, 64);
            __builtin_amdgcn_wave_barrier();
        }
}

// One tile a workgroup.
template <Kind KIND, int STEP, int PLANES, typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Product g) {
    extern __shared__ __align__(16) char s_mem[];
    const Tile tile = tile_at<KIND>(g, by_xcd(blockIdx.x, gridDim.x));
    f4 acc[S::WM / 16][S::WN / 16] = {};
    accumulate<PLANES, S>(g, tile, 0, g.inner * PLANES / kLine, s_mem, acc);
    finish<KIND, STEP, PLANES, T, S>(g, tile, s_mem, acc);
}

// Pieces of the tiles.  Neighbouring workgroups of an XCD take the same piece of
// neighbouring tiles, and begin together, so that its L2 serves most of what they
// read: 4096 x 25088 (bf16, 136 tiles on 256 CUs) 368 us, 412 with equal shares of
// all steps in a row, which run at no common phase; 1500 x 6000 (fp32) 52, 64.
template <Kind KIND, int PLANES, typename S>
__global__ __launch_bounds__(S::kThreads) void pieces_kernel(Product g) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    extern __shared__ __align__(16) char s_mem[];
    const uint32_t lines = g.inner * PLANES / kLine, w = by_xcd(blockIdx.x, gridDim.x);
    for (uint32_t k = 0; k < 2; k++) {
        const uint32_t tiles = k == 0 ? g.cuts.tiles : g.cuts.others;
        const uint32_t cuts = k == 0 ? g.cuts.first : g.cuts.second;
        if (w >= (k == 0 ? g.cuts.first_pieces() : tiles * cuts)) continue;
        const uint32_t piece = w / tiles, t = (k == 0 ? 0 : g.cuts.tiles) + w - piece * tiles;
        f4 acc[FM][FN] = {};
        accumulate<PLANES, S>(g, tile_at<KIND>(g, t), piece * lines / cuts,
                              (piece + 1) * lines / cuts, s_mem, acc);
        f4* part = reinterpret_cast<f4*>(g.part) +
                   (size_t)((k == 0 ? 0 : g.cuts.first_pieces()) + w) * (S::BM * S::BN / 4);
#pragma unroll
        for (int u = 0; u < FM; u++)
#pragma unroll
            for (int v = 0; v < FN; v++) part[(u * FN + v) * S::kThreads + threadIdx.x] = acc[u][v];
    }
}

// The sums of the tiles' pieces, in order.  A workgroup takes an EM x EN block of
// a wave's part, a wave of it 16 rows.
template <Kind KIND, int PLANES, typename T, typename S>
__global__ __launch_bounds__(S::EM * 4) void join_kernel(Product g) {
    constexpr int FN = S::WN / 16, EM = S::EM, EN = S::EN;
    constexpr uint32_t kBlocks = S::kWaves * (S::WM / EM) * (S::WN / EN);  // of a tile
    __shared__ __align__(16) float s_stage[EM * EN];
    const uint32_t tile_block = blockIdx.x / kBlocks, block = blockIdx.x - tile_block * kBlocks;
    const uint32_t t = g.cuts.whole() + tile_block;
    const uint32_t wave = block % S::kWaves, sub = block / S::kWaves;
    const uint32_t eu = sub / (S::WN / EN), ev = sub % (S::WN / EN);
    const bool second = t >= g.cuts.tiles;
    const uint32_t cuts = second ? g.cuts.second : g.cuts.first;
    const uint32_t step = second ? g.cuts.others : g.cuts.tiles;  // from piece to piece
    const size_t piece0 = second ? g.cuts.first_pieces() + (t - g.cuts.tiles) : t;
    const uint32_t lane = threadIdx.x & 63, u = threadIdx.x >> 6;
    const f4* part = reinterpret_cast<const f4*>(g.part) +
                     ((eu * (EM / 16) + u) * FN + ev * (EN / 16)) * S::kThreads + wave * 64 + lane;
    constexpr int kAhead = 4;  // pieces asked for at once: one at a time 16 us for 18, 4 us more a piece
    f4 acc[EN / 16] = {};
    for (uint32_t c = 0; c < cuts; c += kAhead) {
        f4 v[kAhead][EN / 16];
#pragma unroll
        for (int q = 0; q < kAhead; q++)
#pragma unroll
            for (int k = 0; k < EN / 16; k++)
                if (c + q < cuts)
                    v[q][k] = part[(piece0 + (size_t)(c + q) * step) * (S::BM * S::BN / 4) +
                                   k * S::kThreads];
#pragma unroll
        for (int q = 0; q < kAhead; q++)
#pragma unroll
            for (int k = 0; k < EN / 16; k++)
                if (c + q < cuts) acc[k] += v[q][k];
    }
    const Tile tile = tile_at<KIND>(g, t);
    const Results<KIND, MIDDLE, PLANES, T, S> out(g, tile);
    const uint32_t ib = tile.ti * S::BM + wave / (S::BN / S::WN) * S::WM + eu * EM;
    const uint32_t jb = tile.tj * S::BN + wave % (S::BN / S::WN) * S::WN + ev * EN;
    const uint32_t fi = 16 * u + (lane & 15), fj = (lane >> 4) * 4;
#pragma unroll
    for (int v = 0; v < EN / 16; v++)
        *reinterpret_cast<f4*>(s_stage + staged<EN>(fi, 16 * v + fj)) = acc[v];
    lds_barrier();
    out.template straight<EN / 32>(s_stage, ib, jb, threadIdx.x, EM * 4);
    lds_barrier();
    if (out.turn) out.turned(s_stage, ib, jb, threadIdx.x, EM * 4);
}

// ---- thin matrices ---------------------------------------------------------------

// A shorter side of at most 128: a step is one launch.  A workgroup owns columns
// of X (along the longer side), 64 at a time.  It sums all workgroups' parts of
// A = X X^T from the launch before, in order, squares A in LDS, multiplies its
// columns by B, and leaves its part of the next A.  What bounds it is the chain
// of latencies of a launch, so nothing but X and the parts of A goes to memory:
// 64 x 576 7.7 us a step, in three products 20.
//
// A wave multiplies 16 of the 64 columns: a lane holds column lane % 16, rows
// 16 u + 4 (lane / 16) .. + 3, which is what its product with B gives again, and
// what the next takes as its second operand if B's columns are read in the same
// order: chunk c of a line of 32 holds 4 c .. 4 c + 3 and 16 + 4 c .. + 3.  Two
// planes always.
struct Thin {
    uint64_t m, n, x_ld, x_stride, out_ld, out_stride;
    bool tall;
    uint32_t slabs, per, parts;    // 64-column slabs, of a workgroup, workgroups
    uint32_t parts_in;             // parts of A to sum (1: summed by a launch between)
    const void* x;
    void* out;                     // last step
    float* master;                 // X in fp32, in the lanes' order
    const float* part_in;          // parts of A, [batch][parts_in][R][R]
    float* part_out;
    const double* norm;            // first launch
    uint32_t norm_parts;
    float eps, out_scale;
    float a, sb, sc;               // step: a; factors of A and of its square in B
    float x_unit, factor;          // unit of X's operands, factor of the sums of B X
    float gram_x, gram;            // unit of the next X's operands, factor of their A
};

// Where 4 consecutive columns from l (a multiple of 4) of a row lie in a line.
template <int R> __device__ __forceinline__ uint32_t thin_at(uint32_t row, uint32_t l, bool low) {
    const uint32_t q = l & 31u;
    return (l >> 5) * (R * kLine) + swizzled(row, ((q & 15u) >> 2) + (low ? 4u : 0u)) + (q >> 4) * 4;
}

__device__ __forceinline__ void split4(f4 w, h4& hi, h4& lo) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        _Float16 x, y;
        split<2>(w[e], x, y);
        hi[e] = x;
        lo[e] = y;
    }
}

// (high + low) x (high + low).  The low x low product, which the other kernels
// leave out, costs nothing here and takes 50 x 3000 from 1.8e-6 to 1.5e-6.
__device__ __forceinline__ f4 mfma4(h8 ah, h8 al, h8 bh, h8 bl, f4 c) {
    c = product16(ah, bh, c);
    c = product16(al, bh, c);
    c = product16(ah, bl, c);
    return product16(al, bl, c);
}

template <typename T, int R, bool FIRST>
__global__ __launch_bounds__(256) void thin_kernel(Thin g) {
    constexpr int RT = R / 16, RS = R / 32;   // row tiles, lines of 32
    constexpr int GT = RT / 4;                // row tiles of a wave in A and B
    extern __shared__ __align__(16) char s_mem[];
    _Float16* s_b = reinterpret_cast<_Float16*>(s_mem);  // A, then B: [RS][R][64]
    _Float16* s_x = s_b + (FIRST ? 0 : RS * R * kLine);  // 64 columns of X: [2][R][64]
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t li = lane & 15, lg = lane >> 4;
    const uint32_t batch = blockIdx.y;
    Inverse f = {};
    if constexpr (FIRST) {
        f = inverse_norm(g.norm + (uint64_t)batch * kNormParts, g.norm_parts, g.eps);
    } else {
        // A: the parts' sum
        const f4* in = reinterpret_cast<const f4*>(g.part_in) + (size_t)batch * g.parts_in * (R * R / 4);
        constexpr int N = R * R / 4 / 256;
        f4 sum[N] = {};
#pragma unroll 2
        for (uint32_t w = 0; w < g.parts_in; w++)
#pragma unroll
            for (int k = 0; k < N; k++) sum[k] += in[(size_t)w * (R * R / 4) + k * 256 + threadIdx.x];
#pragma unroll
        for (int k = 0; k < N; k++) {
            const uint32_t at = (k * 256 + threadIdx.x) * 4, i = at / R, j = at % R;
            h4 hi, lo;
            split4(sum[k], hi, lo);
            *reinterpret_cast<h4*>(s_b + thin_at<R>(i, j, false)) = hi;
            *reinterpret_cast<h4*>(s_b + thin_at<R>(i, j, true)) = lo;
        }
        lds_barrier();
        // B = sb A + sc A A, rows 16 (GT wave + u) of it
        f4 acc[GT][RT] = {};
#pragma unroll
        for (int s = 0; s < RS; s++) {
            const _Float16* line = s_b + s * (R * kLine);
            h8 ph[GT], pl[GT];
#pragma unroll
            for (int u = 0; u < GT; u++) {
                const uint32_t row = 16 * (GT * wave + u) + li;
                ph[u] = *reinterpret_cast<const h8*>(line + swizzled(row, lg));
                pl[u] = *reinterpret_cast<const h8*>(line + swizzled(row, lg + 4));
            }
#pragma unroll
            for (int v = 0; v < RT; v++) {
                const h8 qh = *reinterpret_cast<const h8*>(line + swizzled(16 * v + li, lg));
                const h8 ql = *reinterpret_cast<const h8*>(line + swizzled(16 * v + li, lg + 4));
#pragma unroll
                for (int u = 0; u < GT; u++) acc[u][v] = mfma4(qh, ql, ph[u], pl[u], acc[u][v]);
            }
        }
#pragma unroll
        for (int u = 0; u < GT; u++)
#pragma unroll
            for (int v = 0; v < RT; v++) {
                const uint32_t i = 16 * (GT * wave + u) + li, j = 16 * v + 4 * lg;
                const h4 hi = *reinterpret_cast<const h4*>(s_b + thin_at<R>(i, j, false));
                const h4 lo = *reinterpret_cast<const h4*>(s_b + thin_at<R>(i, j, true));
#pragma unroll
                for (int e = 0; e < 4; e++)
                    acc[u][v][e] = acc[u][v][e] * g.sc + ((float)hi[e] + (float)lo[e]) * g.sb;
            }
        lds_barrier();
#pragma unroll
        for (int u = 0; u < GT; u++)
#pragma unroll
            for (int v = 0; v < RT; v++) {
                const uint32_t i = 16 * (GT * wave + u) + li, j = 16 * v + 4 * lg;
                h4 hi, lo;
                split4(acc[u][v], hi, lo);
                *reinterpret_cast<h4*>(s_b + thin_at<R>(i, j, false)) = hi;
                *reinterpret_cast<h4*>(s_b + thin_at<R>(i, j, true)) = lo;
            }
        lds_barrier();
    }
    f4 gram[GT][RT] = {};
    const bool last = !FIRST && g.out != nullptr;
    const uint32_t slab0 = blockIdx.x * g.per, slab1 = min(slab0 + g.per, g.slabs);
    for (uint32_t slab = slab0; slab < slab1; slab++) {
        const uint32_t col = slab * 64 + wave * 16 + li;  // along the longer side
        f4* master = reinterpret_cast<f4*>(g.master) +
                     (((size_t)batch * g.slabs + slab) * 4 + wave) * (RT * 64) + lane;
        f4 mine[RT];
        if constexpr (FIRST) {
            const T* x = static_cast<const T*>(g.x) + batch * g.x_stride;
#pragma unroll
            for (int u = 0; u < RT; u++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t row = 16 * u + 4 * lg + e;
                    const uint64_t i = g.tall ? col : row, j = g.tall ? row : col;
                    mine[u][e] = i < g.m && j < g.n ? f.of((float)x[i * g.x_ld + j]) : 0.0f;
                }
        } else {
#pragma unroll
            for (int u = 0; u < RT; u++) mine[u] = master[u * 64];
            h8 xh[RS], xl[RS];
#pragma unroll
            for (int s = 0; s < RS; s++)
#pragma unroll
                for (int q = 0; q < 2; q++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        _Float16 hi, lo;
                        split<2>(mine[2 * s + q][e] * g.x_unit, hi, lo);
                        xh[s][4 * q + e] = hi;
                        xl[s][4 * q + e] = lo;
                    }
#pragma unroll
            for (int u = 0; u < RT; u++) {
                f4 sum = {};
#pragma unroll
                for (int s = 0; s < RS; s++) {
                    const _Float16* line = s_b + s * (R * kLine);
                    const h8 bh = *reinterpret_cast<const h8*>(line + swizzled(16 * u + li, lg));
                    const h8 bl = *reinterpret_cast<const h8*>(line + swizzled(16 * u + li, lg + 4));
                    sum = mfma4(bh, bl, xh[s], xl[s], sum);
                }
                mine[u] = mine[u] * g.a + sum * g.factor;
            }
        }
        if (last) {
            T* out = static_cast<T*>(g.out) + batch * g.out_stride;
#pragma unroll
            for (int u = 0; u < RT; u++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t row = 16 * u + 4 * lg + e;
                    const uint64_t i = g.tall ? col : row, j = g.tall ? row : col;
                    if (i < g.m && j < g.n) out[i * g.out_ld + j] = (T)(mine[u][e] * g.out_scale);
                }
            continue;
        }
#pragma unroll
        for (int u = 0; u < RT; u++) master[u * 64] = mine[u];
        // the columns' part of the next A
        _Float16* sx = s_x + (wave >> 1) * (R * kLine);
        const uint32_t c = (wave & 1) * 16 + li;  // of 32 in a line
        lds_barrier();                            // the last slab's are read
#pragma unroll
        for (int u = 0; u < RT; u++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint32_t row = 16 * u + 4 * lg + e;
                _Float16 hi, lo;
                split<2>(mine[u][e] * g.gram_x, hi, lo);
                sx[swizzled(row, c >> 3) + (c & 7u)] = hi;
                sx[swizzled(row, (c >> 3) + 4) + (c & 7u)] = lo;
            }
        lds_barrier();
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const _Float16* line = s_x + s * (R * kLine);
            h8 ph[GT], pl[GT];
#pragma unroll
            for (int u = 0; u < GT; u++) {
                const uint32_t row = 16 * (GT * wave + u) + li;
                ph[u] = *reinterpret_cast<const h8*>(line + swizzled(row, lg));
                pl[u] = *reinterpret_cast<const h8*>(line + swizzled(row, lg + 4));
            }
#pragma unroll
            for (int v = 0; v < RT; v++) {
                const h8 qh = *reinterpret_cast<const h8*>(line + swizzled(16 * v + li, lg));
                const h8 ql = *reinterpret_cast<const h8*>(line + swizzled(16 * v + li, lg + 4));
#pragma unroll
                for (int u = 0; u < GT; u++) gram[u][v] = mfma4(qh, ql, ph[u], pl[u], gram[u][v]);
            }
        }
    }
    if (last) return;
    f4* out = reinterpret_cast<f4*>(g.part_out) + ((size_t)batch * g.parts + blockIdx.x) * (R * R / 4);
#pragma unroll
    for (int u = 0; u < GT; u++)
#pragma unroll
        for (int v = 0; v < RT; v++)
            out[((16 * (GT * wave + u) + li) * R + 16 * v + 4 * lg) / 4] = gram[u][v] * g.gram;
}

// Many parts of A, summed by a launch of its own: a wave takes 64 groups of 4
// values and a quarter of the parts, in order, and the quarters are added in order.
template <int R>
__global__ __launch_bounds__(256) void thin_sum_kernel(const float* __restrict__ part_in, uint32_t parts,
                                                       float* __restrict__ a) {
    constexpr uint32_t N = R * R / 4;
    __shared__ f4 s_sum[4][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t at = blockIdx.x * 64 + lane;
    const f4* in = reinterpret_cast<const f4*>(part_in) + (size_t)blockIdx.y * parts * N + at;
    const uint32_t per = (parts + 3) / 4, end = min((wave + 1) * per, parts);
    f4 sum = {};
    for (uint32_t w = wave * per; w < end; w += 8) {
        f4 v[8];
#pragma unroll
        for (int q = 0; q < 8; q++)
            if (w + q < end) v[q] = in[(size_t)(w + q) * N];
#pragma unroll
        for (int q = 0; q < 8; q++)
            if (w + q < end) sum += v[q];
    }
    s_sum[wave][lane] = sum;
    lds_barrier();
    if (wave == 0)
        reinterpret_cast<f4*>(a)[(size_t)blockIdx.y * N + at] =
            ((s_sum[0][lane] + s_sum[1][lane]) + s_sum[2][lane]) + s_sum[3][lane];
}

// ---- layout and launches ---------------------------------------------------------

typedef Shape<256, 256, 128, 64, 2> Large;
typedef Shape<128, 128, 64, 64, 2> Medium;
typedef Shape<64, 64, 32, 32, 3> Small;

// bf16 matrices with a side of at most this take two planes too: the rounding
// of few entries does not average out (a 64-bit model of one plane's roundings:
// up to 9.6e-3 off at a side of 4, 3e-3 at 16 to 64, 2.0e-3 at 256), and small
// sides are bound by launches, not by products.
constexpr uint64_t kTwoPlaneSide = 256;

// How a product runs: the tile, and how it is cut (cuts.tiles = 0: not).  APPLY:
// `cut` values of the longer side in tiles of `tile`, the rest in tiles of `rest`.
struct Way {
    int tile;
    Cuts cuts;
    uint32_t cut;
    int rest;
};

// Estimated time of a product in us, from measured ones: a step of 128 bytes
// takes a workgroup `alone` on its CU, or `shared` by as many as fit; a tile's
// first loads and its results take `ends`.  (One plane: a 4096 x 25088 Gram
// product in 256-tiles, 136 of them, 574 us, its square 98; two planes, 6000 x
// 1500: Gram 329, 159 and 94 us in tiles of 256, 128 and 64, square 101, 44 and
// 30, apply 116, 113 and 133.)
struct TileCost {
    int tile, resident;
    double alone, shared, ends;  // one plane
    double alone2, shared2;      // two
};
constexpr TileCost kTileCosts[3] = {
    {256, 1, 1.50, 1.50, 8.0, 2.20, 2.20},
    {128, 2, 0.50, 0.86, 8.0, 0.70, 0.98},
    {64, 4, 0.35, 0.70, 6.0, 0.45, 0.92},
};
// Pieces of tiles: a piece's first loads and the tile of sums that it writes take
// `ends`; the sums go to memory and back in a launch of its own.
struct PieceCost {
    uint32_t least;  // steps of a piece
    double ends;
};
constexpr PieceCost kPieceCosts[3] = {{4, 8.0}, {4, 5.0}, {4, 4.0}};
constexpr double kJoin = 7.0, kJoinPart = 0.2;  // and for each of a tile's parts

constexpr double kLaunch = 4.0, kBytesPerUs = 5e6;

double plain_cost(const TileCost& c, uint64_t tiles, uint32_t lines, int planes, int cus) {
    const double alone = planes == 1 ? c.alone : c.alone2, shared = planes == 1 ? c.shared : c.shared2;
    const uint64_t slots = (uint64_t)cus * c.resident, full = tiles / slots, rest = tiles % slots;
    double t = (double)full * (lines * shared + c.ends);
    if (rest) {
        const double filled = c.resident == 1 || rest <= (uint64_t)cus
                                  ? 0.0
                                  : (double)(rest - cus) / (double)(slots - cus);
        t += lines * (alone + filled * (shared - alone)) + c.ends;
    }
    return t;
}

// Products that are cut into pieces.  Those of 256-tiles in two planes, and of
// 64-tiles in a square in one, are never the least estimate (not once in 900,000
// random sides and batches) and not built.
constexpr bool has_pieces(Kind kind, int planes, int tile) {
    return kind == APPLY ? false : planes == 2 ? tile < 256 : kind == GRAM || tile > 64;
}

// With a workgroup on every CU (full = 0) or as many as fit: every tile in as
// many pieces as there is room for; one more of as many tiles as that leaves room
// for, the others in the pieces that fill it; or whole rounds of whole tiles, the
// others in pieces.
void try_pieces(int k, int full, uint64_t n, uint32_t lines, int planes, int cus, double* best,
                Way* way) {
    const TileCost& T = kTileCosts[k];
    const PieceCost& c = kPieceCosts[k];
    if (full && T.resident == 1) return;
    const uint64_t slots = (uint64_t)cus * (full ? T.resident : 1), most = lines / c.least;
    const uint64_t round = (uint64_t)cus * T.resident;
    if (n == 0 || most < 2) return;
    const double step = planes == 1 ? (full ? T.shared : T.alone) : (full ? T.shared2 : T.alone2);
    const double size = 4.0 * T.tile * T.tile;
    auto pieces = [&](uint64_t tiles, uint64_t cuts) {
        return tiles == 0 ? 0.0
                          : (lines + cuts - 1) / cuts * step + c.ends +
                                ((cuts + 1) * tiles) * size / kBytesPerUs + kJoinPart * cuts;
    };
    auto consider = [&](double t, uint64_t tiles, uint64_t first, uint64_t second) {
        if (t >= *best) return;
        *best = t;
        *way = Way{T.tile, {(uint32_t)tiles, (uint32_t)first, (uint32_t)(n - tiles), (uint32_t)second}, 0, 0};
    };
    if (n < slots) {
        for (int more = 0; more < 2; more++) {
            const uint64_t first = slots / n + more < most ? slots / n + more : most;
            if (first < 2) continue;
            const uint64_t take = slots / first < n ? slots / first : n, others = n - take;
            const uint64_t second = others == 0 ? 0 : slots / others < most ? slots / others : most;
            consider(pieces(take, first) + pieces(others, second) + kJoin, take, first, second);
        }
    }
    const uint64_t whole = n / round * round, others = n - whole;
    if (whole && others && slots / others >= 2) {
        const uint64_t second = slots / others < most ? slots / others : most;
        consider(plain_cost(T, whole, lines, planes, cus) + kLaunch + pieces(others, second) + kJoin,
                 whole, 1, second);
    }
}

double best_way(Kind kind, uint64_t tiles256, uint64_t tiles128, uint64_t tiles64, uint32_t lines,
                int planes, int cus, Way* way) {
    const uint64_t tiles[3] = {tiles256, tiles128, tiles64};
    double best = 1e30;
    for (int k = 0; k < 3; k++) {
        if (tiles[k] == 0) continue;  // the sides are no multiples of this tile
        const double t = plain_cost(kTileCosts[k], tiles[k], lines, planes, cus);
        if (t < best) {
            best = t;
            *way = Way{kTileCosts[k].tile, {}, 0, 0};
        }
    }
    for (int k = 0; k < 3; k++) {
        if (!has_pieces(kind, planes, kTileCosts[k].tile)) continue;
        for (int full = 0; full < 2; full++) try_pieces(k, full, tiles[k], lines, planes, cus, &best, way);
    }
    return best;
}

// CUs of the gfx950; a product is split over no more.
constexpr int kMaxCus = 256;

// APPLY, whose results are r x k: tiles of one size, or as many as fill whole
// rounds of the CUs and smaller ones for the rest of the longer side.
double best_apply(uint64_t batch, uint64_t r, uint64_t k, uint64_t pad, uint32_t lines, int planes,
                  int cus, Way* way) {
    double best = 1e30;
    for (int c = 0; c < 3; c++) {
        const TileCost& T = kTileCosts[c];
        const uint64_t tile = T.tile;
        if (tile > pad) continue;
        const uint64_t across = batch * (r / tile), along = k / tile;
        const double whole = plain_cost(T, across * along, lines, planes, cus);
        if (whole < best) {
            best = whole;
            *way = Way{T.tile, {}, (uint32_t)k, 0};
        }
        const uint64_t slots = (uint64_t)cus * T.resident;
        const uint64_t part = across * along / slots * slots / across;  // whole rounds
        if (part == 0 || part == along) continue;
        for (int d = c + 1; d < 3; d++) {
            const uint64_t small = kTileCosts[d].tile;
            const double t = plain_cost(T, across * part, lines, planes, cus) + kLaunch +
                             plain_cost(kTileCosts[d], batch * (r / small) * ((k - part * tile) / small),
                                        lines, planes, cus);
            if (t < best) {
                best = t;
                *way = Way{T.tile, {}, (uint32_t)(part * tile), kTileCosts[d].tile};
            }
        }
    }
    return best;
}

constexpr uint64_t kThinSide = 128;
constexpr uint32_t kFewParts64 = 16, kFewParts128 = 4;

struct OrthoLayout {
    uint32_t rows, cols, r;  // padded m, n and their smaller
    int planes;
    bool tall, thin;
    Way way[3];  // by Kind
    uint32_t slabs, per, parts;  // thin
    bool sum_parts;
    size_t partial, inverse, master, x, xt[2], a, b, part, bytes;
};

// Pads the sides to multiples of 64, 128 or 256 and picks every product's way,
// for the least estimated time of a step.
void plan_products(const hc_orthogonalise_params& p, int cus, OrthoLayout* L) {
    double best = 1e30;
    for (uint64_t pad = 64; pad <= 256; pad *= 2) {
        const uint64_t rows = (p.m + pad - 1) / pad * pad, cols = (p.n + pad - 1) / pad * pad;
        const uint64_t r = L->tall ? cols : rows, k = L->tall ? rows : cols;
        uint64_t half[3] = {};  // tiles of 256, 128, 64
        for (int s = 0; s < 3; s++) {
            const uint64_t t = 256 >> s;
            if (t > pad) continue;
            half[s] = p.batch * (r / t) * (r / t + 1) / 2;
        }
        Way way[3] = {};
        const double t =
            best_way(GRAM, half[0], half[1], half[2], (uint32_t)(k * L->planes / kLine), L->planes, cus,
                     &way[GRAM]) +
            best_way(SQUARE, half[0], half[1], half[2], (uint32_t)(r * L->planes / kLine), L->planes, cus,
                     &way[SQUARE]) +
            best_apply(p.batch, r, k, pad, (uint32_t)(r * L->planes / kLine), L->planes, cus, &way[APPLY]) +
            // what an apply reads and writes, 10 or 16 bytes a value with its
            // padding, is hardly overlapped with its products
            (double)(p.batch * rows * cols * (L->planes == 1 ? 10 : 16)) / kBytesPerUs;
        if (t < best) {
            best = t;
            L->rows = (uint32_t)rows;
            L->cols = (uint32_t)cols;
            for (int s = 0; s < 3; s++) L->way[s] = way[s];
        }
    }
}

OrthoLayout ortho_layout(const hc_orthogonalise_params& p) {
    OrthoLayout L = {};
    if (p.batch == 0) return L;  // no matrices: nothing to plan, no workspace
    const uint64_t r = p.m < p.n ? p.m : p.n;
    L.tall = p.m > p.n;
    L.thin = r <= kThinSide;
    L.planes = p.type == HC_T_F32 || r <= kTwoPlaneSide ? 2 : 1;
    if (L.thin) {
        // a workgroup a slab, up to two workgroups a CU; few parts of A (16 KiB
        // each with 64 rows, 64 KiB with 128) are read by every workgroup, more are
        // summed between the steps (120 x 4000: 16 parts read by all 195 us)
        L.r = r <= 64 ? 64 : 128;
        L.slabs = (uint32_t)(((L.tall ? p.m : p.n) + 63) / 64);
        const uint64_t most = 2 * kMaxCus, groups = (uint64_t)L.slabs * p.batch;
        const uint32_t few = r <= 64 ? kFewParts64 : kFewParts128;
        L.per = (uint32_t)(groups > most ? (groups + most - 1) / most : 1);
        L.parts = (L.slabs + L.per - 1) / L.per;
        L.sum_parts = L.parts > few;
    } else {
        plan_products(p, kMaxCus, &L);
        L.r = L.tall ? L.cols : L.rows;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    const bool any = p.steps > 0;
    L.partial = take(p.batch * kNormParts * sizeof(double));
    if (L.thin) {
        const size_t part = any ? p.batch * L.parts * L.r * L.r * 4 : 0;
        L.master = take(any ? p.batch * L.slabs * 64 * L.r * 4 : 0);
        L.xt[0] = take(part);  // the parts of A, of this step and the next
        L.xt[1] = take(part);
        L.a = take(any && L.sum_parts ? p.batch * L.r * L.r * 4 : 0);
        L.bytes = at;
        return L;
    }
    const size_t xs = any ? p.batch * L.rows * L.cols : 0, as = any ? p.batch * L.r * L.r : 0;
    L.inverse = take(p.batch * sizeof(Inverse));
    L.master = take(xs * 2 * L.planes);
    L.x = take(xs * 2 * L.planes);
    L.xt[0] = take(xs * 2 * L.planes);
    L.xt[1] = take(xs * 2 * L.planes);
    L.a = take(as * 2 * L.planes);
    L.b = take(as * 2 * L.planes);
    size_t part = 0;
    for (const Way& w : L.way) {
        const size_t bytes = (size_t)w.cuts.pieces() * w.tile * w.tile * 4;
        part = bytes > part ? bytes : part;
    }
    L.part = take(any ? part : 0);
    L.bytes = at;
    return L;
}

template <typename S, typename K>
hipError_t launch_tiles(K kernel, const Product& g, uint32_t groups, hipStream_t s) {
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), S::kLdsBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(S::kThreads), S::kLdsBytes, s, g);
    return hipGetLastError();
}

// [k0, k1) of the longer side (APPLY), or all of it.
template <Kind KIND, int PLANES, typename T, typename S>
hipError_t product_shape(Product g, uint32_t batch, const Cuts& cuts, uint32_t k0, uint32_t k1,
                         hipStream_t s) {
    g.tiles_i = g.rows / S::BM;
    g.tiles_j = g.cols / S::BN;
    if (KIND == APPLY) {
        g.first = k0 / S::BM;
        g.tiles = (g.tiles_i < g.tiles_j ? g.tiles_i : g.tiles_j) * ((k1 - k0) / S::BM);
    } else {
        g.tiles = g.tiles_i * (g.tiles_i + 1) / 2;
    }
    g.batch = batch;
    g.cuts = cuts;
    if constexpr (has_pieces(KIND, PLANES, S::BM)) {
        if (cuts.tiles) {
            hipError_t e = hipSuccess;
            if (cuts.whole())
                e = launch_tiles<S>(&product_kernel<KIND, MIDDLE, PLANES, T, S>, g, cuts.whole(), s);
            if (e == hipSuccess)
                e = launch_tiles<S>(&pieces_kernel<KIND, PLANES, S>, g, cuts.groups(), s);
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL((join_kernel<KIND, PLANES, T, S>),
                               dim3((g.tiles * batch - cuts.whole()) * (S::BM / S::EM) * (S::BN / S::EN)),
                               dim3(S::EM * 4), 0, s, g);
            return hipGetLastError();
        }
    }
    const uint32_t groups = g.tiles * batch;
    if constexpr (KIND == APPLY) {
        switch ((g.x ? FIRST : 0) | (g.out ? LAST : 0)) {
            case FIRST:
                return launch_tiles<S>(&product_kernel<KIND, FIRST, PLANES, T, S>, g, groups, s);
            case LAST:
                return launch_tiles<S>(&product_kernel<KIND, LAST, PLANES, T, S>, g, groups, s);
            case FIRST | LAST:
                return launch_tiles<S>(&product_kernel<KIND, FIRST | LAST, PLANES, T, S>, g, groups, s);
        }
    }
    return launch_tiles<S>(&product_kernel<KIND, MIDDLE, PLANES, T, S>, g, groups, s);
}

template <Kind KIND, int PLANES, typename T>
hipError_t product_tiles(const Product& g, int tile, uint32_t batch, const Cuts& cuts, uint32_t k0,
                         uint32_t k1, hipStream_t s) {
    if (tile == 256) return product_shape<KIND, PLANES, T, Large>(g, batch, cuts, k0, k1, s);
    if (tile == 128) return product_shape<KIND, PLANES, T, Medium>(g, batch, cuts, k0, k1, s);
    return product_shape<KIND, PLANES, T, Small>(g, batch, cuts, k0, k1, s);
}

template <Kind KIND, int PLANES, typename T>
hipError_t product(const Product& g, const OrthoLayout& L, uint32_t batch, hipStream_t s) {
    const Way w = L.way[KIND];
    const hipError_t e = product_tiles<KIND, PLANES, T>(g, w.tile, batch, w.cuts, 0, w.cut, s);
    if (e != hipSuccess || w.rest == 0) return e;
    return product_tiles<KIND, PLANES, T>(g, w.rest, batch, {}, w.cut, g.rows > g.cols ? g.rows : g.cols, s);
}

template <typename T, int R>
hipError_t thin_typed(const hc_orthogonalise_params& p, const OrthoLayout& L, const OrthoStep* steps,
                      const void* x, void* out, uint32_t norm_parts, char* ws, hipStream_t s) {
    constexpr int kFirstLds = 2 * R * kLine * 2, kStepLds = kFirstLds + R * R * 4;
    hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&thin_kernel<T, R, false>), kStepLds);
    if (e != hipSuccess) return e;
    float* parts[2] = {reinterpret_cast<float*>(ws + L.xt[0]), reinterpret_cast<float*>(ws + L.xt[1])};
    Thin g = {};
    g.m = p.m;
    g.n = p.n;
    g.x_ld = p.x_ld;
    g.x_stride = p.x_stride;
    g.out_ld = p.out_ld;
    g.out_stride = p.out_stride;
    g.tall = L.tall;
    g.slabs = L.slabs;
    g.per = L.per;
    g.parts = L.parts;
    g.x = x;
    g.master = reinterpret_cast<float*>(ws + L.master);
    g.norm = reinterpret_cast<const double*>(ws + L.partial);
    g.norm_parts = norm_parts;
    g.eps = p.eps;
    g.out_scale = p.scale;
    const dim3 grid(L.parts, (uint32_t)p.batch);
    auto next = [&](const OrthoStep& st) {  // units of step st's X and A
        g.gram_x = ldexpf(1.0f, st.ex);
        g.gram = ldexpf(1.0f, st.ea - 2 * st.ex);
    };
    g.part_out = parts[0];
    next(steps[0]);
    hipLaunchKernelGGL((thin_kernel<T, R, true>), grid, dim3(256), kFirstLds, s, g);
    float* a = reinterpret_cast<float*>(ws + L.a);
    for (uint32_t t = 0; t < p.steps; t++) {
        const OrthoStep& st = steps[t];
        g.part_in = parts[t & 1];
        g.parts_in = L.parts;
        if (L.sum_parts) {
            hipLaunchKernelGGL(thin_sum_kernel<R>, dim3(R * R / 256, (uint32_t)p.batch), dim3(256), 0, s,
                               g.part_in, L.parts, a);
            g.part_in = a;
            g.parts_in = 1;
        }
        g.part_out = parts[(t + 1) & 1];
        g.a = st.a;
        g.sb = ldexpf(st.b, st.eb - st.ea);
        g.sc = ldexpf(st.c, st.eb - 2 * st.ea);
        g.x_unit = ldexpf(1.0f, st.ex);
        g.factor = ldexpf(1.0f, -st.eb - st.ex);
        if (t + 1 < p.steps) next(steps[t + 1]);
        else g.out = out;
        hipLaunchKernelGGL((thin_kernel<T, R, false>), grid, dim3(256), kStepLds, s, g);
    }
    return hipGetLastError();
}

template <typename T, int PLANES>
hipError_t orthogonalise_typed(const hc_orthogonalise_params& p, const OrthoStep* steps,
                               const void* x, void* out, char* ws, hipStream_t s) {
    const OrthoLayout L = ortho_layout(p);
    const uint32_t batch = (uint32_t)p.batch;
    double* partial = reinterpret_cast<double*>(ws + L.partial);
    const bool flat = p.x_ld == p.n;
    const uint64_t rows = flat ? 1 : p.m, cols = flat ? p.m * p.n : p.n;
    uint64_t parts = flat ? (cols + kNormBlock * 16 - 1) / (kNormBlock * 16) : (p.m + 15) / 16;
    if (parts > kNormParts) parts = kNormParts;
    hipLaunchKernelGGL(norm_kernel<T>, dim3((uint32_t)parts, batch), dim3(kNormBlock), 0, s,
                       static_cast<const T*>(x), rows, cols, p.x_ld, p.x_stride, partial);
    if (p.steps == 0) {
        hipLaunchKernelGGL(normalise_kernel<T>, dim3((uint32_t)(p.m < 1024 ? p.m : 1024), batch),
                           dim3(kPrepBlock), 0, s, p, static_cast<const T*>(x), static_cast<T*>(out),
                           partial, (uint32_t)parts);
        return hipGetLastError();
    }
    if constexpr (PLANES == 2)
        if (L.thin)
            return L.r == 64 ? thin_typed<T, 64>(p, L, steps, x, out, (uint32_t)parts, ws, s)
                             : thin_typed<T, 128>(p, L, steps, x, out, (uint32_t)parts, ws, s);
    _Float16* X = reinterpret_cast<_Float16*>(ws + L.x);  // by the shorter side's rows
    _Float16* XT[2] = {reinterpret_cast<_Float16*>(ws + L.xt[0]),
                       reinterpret_cast<_Float16*>(ws + L.xt[1])};
    _Float16* A = reinterpret_cast<_Float16*>(ws + L.a);
    _Float16* B = reinterpret_cast<_Float16*>(ws + L.b);
    Inverse* inverse = reinterpret_cast<Inverse*>(ws + L.inverse);
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
        g.part = reinterpret_cast<float*>(ws + L.part);
        g.p = g.q = X;
        g.p_stride = g.q_stride = x_size;
        g.inner = L.tall ? L.rows : L.cols;
        g.factor = ldexpf(1.0f, st.ea - 2 * st.ex);
        g.rows = g.cols = L.r;
        g.d = g.dt = A;
        e = product<GRAM, PLANES, T>(g, L, batch, s);
        if (e != hipSuccess) return e;
        g.p = g.q = A;
        g.p_stride = g.q_stride = a_size;
        g.inner = L.r;
        g.factor = ldexpf(st.c, st.eb - 2 * st.ea);
        g.factor2 = ldexpf(st.b, st.eb - st.ea);
        g.d = g.dt = B;
        e = product<SQUARE, PLANES, T>(g, L, batch, s);
        if (e != hipSuccess) return e;
        g.p = L.tall ? XT[t & 1] : B;
        g.q = L.tall ? B : XT[t & 1];
        g.p_stride = L.tall ? x_size : a_size;
        g.q_stride = L.tall ? a_size : x_size;
        g.factor = ldexpf(1.0f, -st.eb - st.ex);
        // a X, from its unit
        g.factor2 = t > 0 && PLANES == 1 ? ldexpf(st.a, -st.ex) : st.a;
        g.next = ldexpf(1.0f, st.ex_next);
        g.rows = L.rows;
        g.cols = L.cols;
        g.d = L.tall ? XT[(t + 1) & 1] : X;
        g.dt = L.tall ? X : XT[(t + 1) & 1];
        g.master = ws + L.master;
        g.prev = L.tall ? XT[t & 1] : X;
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
        e = product<APPLY, PLANES, T>(g, L, batch, s);
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
