// hc_linear.hip -- the linear layer and its gradient (include/hc_train.h).
//
//   forward   D = y,  D[i][j] = sum over l of x[i][l] w[j][l]
//   dx        D = dx, D[i][j] = sum over l of dz[i][l] w[l][j]
//   dw        D = dw, D[i][j] = sum over l of dz[l][i] x[l][j]
//
// Bias, activation, dropout and residual are applied to the sums before they leave
// the registers; dz = act'(z) mask dy is made in a pass of its own, which leaves the
// column sums (db) too, since both products read it.
//
// Precision.  Products of 16-bit types are exact and summed in fp32; dz is rounded to
// the type for dx and for a 16-bit dw, whose results are rounded to it too (bf16: 2.3e-3
// off in all, 1.7e-3 by the result alone; each further part of dz is another product),
// and taken in two or three parts for a wider one.  fp32: large products as three of
// fp16 parts (22 bits), others by fp32 matrix instructions.  Sums are taken in an order
// that shape, type, strides and the 16-byte alignment of 16-bit operands fix; partial
// sums of a tile's pieces are joined in order.
//
// Three ways.  Tiles of 256, 128 or 64 fed from memory to LDS directly, which need
// rows that are read 16 bytes at a time (others are copied where that pays); small
// tiles whose eight waves share l, for products that are a chain of latencies; and
// 64-tiles through registers, which take anything.  Host estimates pick one for each
// product by itself.
//
// What bounds it (MI355X, a library product of 8192^3 reaches 1.29 to 1.37 PFLOP/s).
// Large products the matrix cores: 4096 x 4096 x 25088 in bf16 takes 666 us without
// epilogue (1.26 PFLOP/s), its dx and dw 683 and 695.  With l of a few hundred the tiles'
// way through L2: 32768 x 768 x 768 (bf16) 57 us in 128-tiles, 40 of them products
// (600 MB from L2) and 17 results, hardly overlapped; 256-tiles read half of that but
// are one round and a half of the CUs.
#include "hc_internal.h"
#include "hc_layer.h"
#include "hc_tiles.h"

namespace hc {

namespace {

typedef float f8 __attribute__((ext_vector_type(8)));

enum Kind { FORWARD, DX, DW };

constexpr uint32_t kCus = 256;  // of the gfx950

// What a forward product's sums become.
struct Forward {
    const void *bias, *residual;
    void *y, *z;
    uint64_t residual_ld, y_ld, z_ld;
    uint32_t act;
    uint32_t stream;  // results pass the caches by
    Dropout drop;
};

template <typename T>
__device__ __forceinline__ void put8(const Forward& f, T* p, uint32_t count, const float (&v)[8]) {
    if (f.stream) store8_past(p, count, v);
    else store8(p, count, v);
}

template <typename T>
__device__ __forceinline__ void finish_forward(const Forward& f, const Masks& masks, uint64_t row, uint64_t rows,
                                               uint32_t col, uint32_t count, const float (&bias)[8],
                                               const T (&residual)[8], float (&v)[8]) {
    if (row >= rows || count == 0) return;
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] += bias[e];
    if (f.z) put8(f, static_cast<T*>(f.z) + row * f.z_ld + col, count, v);
    activate8<T>(f.act, v);
    if (masks.limit) drop8(masks, (uint32_t)row, col / 8, v);
    if (f.residual)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += (float)residual[e];
    put8(f, static_cast<T*>(f.y) + row * f.y_ld + col, count, v);
}

// An operand may be a sum of planes, and a product the sum of some products of
// planes: pass s takes plane p_planes >> 4 s of P and q_planes >> 4 s of Q.  The
// small ones come first; the sums of the first `small` are multiplied by `factor`.
struct Passes {
    uint32_t count, p_planes, q_planes, small;
    float factor;
};
constexpr Passes kOnePass = {1, 0, 0, 0, 1.0f};
// dz in three bf16 parts that follow each other; in an fp16 part and 2^11 times the
// rest, which as it is would lose bits below fp16's normal range
constexpr float kRestUnit = 0x1p11f;
constexpr Passes kRestBf16 = {3, 0x012, 0x000, 0, 1.0f};
constexpr Passes kRestF16 = {2, 0x01, 0x00, 1, 1.0f / kRestUnit};
// fp32 in an fp16 part and 2^11 times the rest, 22 bits: high x rest, rest x high,
// high x high.  The product of the rests is below 2^-22 of the whole.
constexpr Passes kTwoPlanes = {3, 0x010, 0x001, 2, 1.0f / kRestUnit};

struct Product {
    const void *p, *q;       // operands
    uint64_t p_ld, q_ld;
    uint64_t p_cols, q_cols;    // stored elements of a row: its columns, or with zeros behind
    uint64_t p_plane, q_plane;  // elements between planes
    const float *p_most, *q_most;  // planes of fp32: the largest element of each row
    Passes passes;
    uint64_t rows, inner;    // of D; length of l
    uint32_t cols;
    uint32_t tiles_i, tiles_j, stripe;
    uint32_t whole, cut;     // tiles that a workgroup makes whole, and that are cut
    uint32_t pieces;         // along l into this many pieces
    float* part;             // the pieces' sums
    uint32_t part_ld;
    Forward forward;
    Gradient gradient;
};

// Sums of a product with dz, back from the units that an fp16 dz is held in.
template <typename T> __device__ __forceinline__ void from_units(const Gradient& g, float (&v)[8]) {
    if constexpr (std::is_same<T, _Float16>::value)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] *= g.unit;
}

template <Kind KIND, typename T>
__device__ __forceinline__ void finish8(const Product& g, const Masks& masks, uint64_t row, uint32_t col,
                                        float (&v)[8]) {
    const uint32_t count = g.cols - col;
    if constexpr (KIND == FORWARD) {
        const Forward& f = g.forward;
        float bias[8] = {};
        T residual[8];
        if (f.bias) load8(static_cast<const T*>(f.bias) + col, count, bias);
        if (f.residual) load8_raw(static_cast<const T*>(f.residual) + row * f.residual_ld + col, count, residual);
        finish_forward<T>(f, masks, row, g.rows, col, count, bias, residual, v);
    } else {
        from_units<T>(g.gradient, v);
        if constexpr (KIND == DX) store8(static_cast<T*>(g.gradient.out) + row * g.gradient.ld + col, count, v);
        else store_gradient(g.gradient, row, col, count, v);
    }
}

// ---- products of any shape, stride and alignment -----------------------------------

using hc::product16;
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
// zeros where a matrix ends.  fp32: 75 TFLOP/s of the matrix instructions' 157, and
// 65536 x 64 x 128 in 17 us, whose memory takes 8 to 10.
template <Kind KIND, typename T>
__global__ __launch_bounds__(256) void direct_kernel(Product g) {
    constexpr bool PS = KIND == DW, QS = KIND != FORWARD;
    typedef T V __attribute__((ext_vector_type(8), aligned(16)));
    __shared__ __align__(16) T s_p[kDirect * kDirectLd<T>], s_q[kDirect * kDirectLd<T>];
    __shared__ __align__(16) float s_out[kDirect * (kDirect + 4)];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t wi = wave / 2 * 32, wj = wave % 2 * 32;
    const uint32_t piece = blockIdx.x / g.cut, tile = blockIdx.x - piece * g.cut;
    const uint64_t ti = tile / g.tiles_j, row0 = ti * kDirect;
    const uint32_t col0 = (uint32_t)(tile - ti * g.tiles_j) * kDirect;
    const uint64_t lines = (g.inner + kStep - 1) / kStep, all = g.passes.count * lines;
    const uint64_t first = piece * all / g.pieces, end = (piece + 1) * all / g.pieces;
    const T* q = static_cast<const T*>(g.q);
    f4 acc[2][2] = {};
    T rp[8], rq[8];  // of the next step: more would cost workgroups of a CU (65536 x 64 x 128 fp32: 17 us, 20 with four)
    for (uint64_t s = first; s < end;) {
        const uint32_t pass = (uint32_t)(s / lines);
        const uint64_t stop = min(end, (pass + 1) * lines);
        const T* p = static_cast<const T*>(g.p) + (g.passes.p_planes >> 4 * pass & 15u) * g.p_plane;  // Q has one
        auto load = [&](uint64_t l) {
            direct_load<PS>(p, g.p_ld, g.rows, row0, l, g.inner, rp);
            direct_load<QS>(q, g.q_ld, (uint64_t)g.cols, col0, l, g.inner, rq);
        };
        load((s - pass * lines) * kStep);
        for (; s < stop; s++) {
            __syncthreads();
            direct_store<PS>(s_p, rp);
            direct_store<QS>(s_q, rq);
            __syncthreads();
            if (s + 1 < stop) load((s + 1 - pass * lines) * kStep);
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
        if (pass + 1 == g.passes.small)
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int v = 0; v < 2; v++) acc[u][v] *= g.passes.factor;
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
            store8(g.part + ((uint64_t)piece * g.rows + row) * g.part_ld + col, 8, v);
        else
            finish8<KIND, T>(g, masks, row, col, v);
    }
}

// The sums of the tiles' pieces, in order, a lane eight columns of a row.
template <Kind KIND, typename T>
__global__ __launch_bounds__(256) void direct_join_kernel(Product g) {
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

// ---- small products --------------------------------------------------------------

// A tile of 16 x 16 a workgroup, whose eight waves share l: what bounds a small
// product is a chain of latencies, so a wave asks for the fragments of four steps at
// once, from memory to registers, and the waves' sums are added up in LDS in order.
// 16 tokens through 768 x 768 (bf16): one launch of 5.4 us, in 64-tiles 8; 16 x 4096 x
// 4096 in fp32 15, directly 27.
constexpr uint32_t kSplitTile = 16, kSplitWaves = 8, kSplitAhead = 4;

// 8 values of l of an operand's row, zeros behind its ends.
template <bool ACROSS, typename T>
__device__ __forceinline__ void split_load(const T* p, uint64_t ld, uint64_t row, uint64_t rows, uint32_t l,
                                           uint32_t inner, T (&v)[8]) {
    const uint32_t left = row < rows && l < inner ? inner - l : 0;
    if constexpr (ACROSS) {
        const T* at = p + (uint64_t)l * ld + row;
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < left ? at[e * ld] : (T)0.0f;
    } else {
        load8_raw(p + row * ld + l, left, v);
    }
}

template <Kind KIND, typename T>
__device__ __forceinline__ void split_tile(const Product& g, uint32_t tile, float (&s_sum)[kSplitWaves][16][20]) {
    constexpr bool PA = KIND == DW, QA = KIND != FORWARD;
    typedef T V __attribute__((ext_vector_type(8)));
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t ti = tile / g.tiles_j, tj = tile - ti * g.tiles_j;
    const uint64_t row0 = (uint64_t)ti * kSplitTile;
    const uint32_t col0 = tj * kSplitTile, inner = (uint32_t)g.inner;
    const uint32_t lines = (inner + kStep - 1) / kStep;
    // the lanes that store results ask for what is added to them first
    const uint32_t i = threadIdx.x / 2 % 16, j = threadIdx.x % 2 * 8, col = col0 + j;
    const bool finishes = threadIdx.x < 32 && row0 + i < g.rows && col < g.cols;
    float bias[8] = {};
    T residual[8];
    if constexpr (KIND == FORWARD)
        if (finishes) {
            const Forward& f = g.forward;
            if (f.bias) load8(static_cast<const T*>(f.bias) + col, g.cols - col, bias);
            if (f.residual)
                load8_raw(static_cast<const T*>(f.residual) + (row0 + i) * f.residual_ld + col, g.cols - col, residual);
        }
    f4 acc = {};
    for (uint32_t pass = 0; pass < g.passes.count; pass++) {
        const T* p = static_cast<const T*>(g.p) + (g.passes.p_planes >> 4 * pass & 15u) * g.p_plane;
        for (uint32_t s = wave; s < lines; s += kSplitWaves * kSplitAhead) {
            T rp[kSplitAhead][8], rq[kSplitAhead][8];
#pragma unroll
            for (uint32_t k = 0; k < kSplitAhead; k++) {
                const uint32_t l = (s + k * kSplitWaves) * kStep + (lane >> 4) * 8;
                split_load<PA>(p, g.p_ld, row0 + (lane & 15), g.rows, l, inner, rp[k]);
                split_load<QA>(static_cast<const T*>(g.q), g.q_ld, col0 + (lane & 15), g.cols, l, inner, rq[k]);
            }
#pragma unroll
            for (uint32_t k = 0; k < kSplitAhead; k++) {
                V a, b;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    a[e] = rp[k][e];
                    b[e] = rq[k][e];
                }
                acc = product16(b, a, acc);
            }
        }
        if (pass + 1 == g.passes.small) acc *= g.passes.factor;
    }
    *reinterpret_cast<f4*>(&s_sum[wave][lane & 15][(lane >> 4) * 4]) = acc;
    __syncthreads();
    if (!finishes) return;
    float v[8] = {};
    for (uint32_t w = 0; w < kSplitWaves; w++)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += s_sum[w][i][j + e];
    if constexpr (KIND == FORWARD)
        finish_forward<T>(g.forward, masks_of(g.forward.drop), row0 + i, g.rows, col, g.cols - col, bias, residual, v);
    else
        finish8<KIND, T>(g, Masks{}, row0 + i, col, v);
}

template <typename T> __global__ __launch_bounds__(512) void split_forward_kernel(Product g) {
    __shared__ __align__(16) float s_sum[kSplitWaves][16][20];
    split_tile<FORWARD, T>(g, blockIdx.x, s_sum);
}

// The gradients of a small layer in one launch: tiles of dx, then of dw, then 64
// columns of db a workgroup, whose waves take an eighth of the rows each.
struct SplitGrad {
    Product dx, dw;
    uint32_t dx_tiles, dw_tiles;
    const void* dy;   // db: or null
    uint64_t dy_ld, m;
    uint32_t n;
    Gradient db;
};

template <typename T> __global__ __launch_bounds__(512) void split_grad_kernel(SplitGrad g) {
    __shared__ __align__(16) float s_sum[kSplitWaves][16][20];
    if (blockIdx.x < g.dx_tiles) {
        split_tile<DX, T>(g.dx, blockIdx.x, s_sum);
    } else if (blockIdx.x < g.dx_tiles + g.dw_tiles) {
        split_tile<DW, T>(g.dw, blockIdx.x - g.dx_tiles, s_sum);
    } else {
        float* sums = &s_sum[0][0][0];
        const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint32_t col = (blockIdx.x - g.dx_tiles - g.dw_tiles) * 64 + lane;
        const T* dy = static_cast<const T*>(g.dy);
        float t = 0.0f;
        if (col < g.n)
#pragma unroll 8
            for (uint64_t row = g.m * wave / kSplitWaves; row < g.m * (wave + 1) / kSplitWaves; row++)
                t += (float)dy[row * g.dy_ld + col];
        sums[wave * 64 + lane] = t;
        __syncthreads();
        if (wave == 0 && col < g.n) {
            float v[8] = {};
            for (uint32_t w = 0; w < kSplitWaves; w++) v[0] += sums[w * 64 + lane];
            store_gradient(g.db, 0, col, 1, v);
        }
    }
}

// ---- products in tiles fed from memory to LDS directly -------------------------------

// Where a wave's loads of one operand's tile go.  ROWS: of the tile.  Along rows
// a load is 8 rows of 128 bytes, across them 512 / ROWS lines of 2 ROWS bytes;
// lane i writes 16 bytes at 16 i of 1024, so it reads the chunk that belongs
// there.  Bounds are the buffer's, which begins at each step anew: rows and lines
// behind the last read as zero, and so do chunks past the end of l in its rows, whose
// lanes get an offset behind any buffer.  Columns behind the last give what follows
// them in memory, for results that are not stored; of the last line they read as zero.  A stored row is a multiple of 8 elements, so that no
// chunk ends in the middle of a buffer.
constexpr uint32_t kNowhere = 0x80000000u;

__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, char* to, uint32_t at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)to, 16, at, 0, 0, 0);
}

template <bool ACROSS, int ROWS, int WAVES> struct Loads {
    static constexpr int N = ROWS / 8 / WAVES;  // of a wave and step
    static constexpr uint32_t kChunks = ACROSS ? ROWS / 8 : 8, kLines = 64 / kChunks;
    static constexpr uint32_t kBlock = ACROSS ? Across<ROWS>::kBlock : 1024;
    uint32_t at[N];
    uint32_t chunk;      // along rows: the first of the lane's 8 values of l
    uint32_t ld2;        // bytes from line to line
    uint32_t bytes;      // along rows: the tile's buffer; across: of its last line
    const char* first;   // of the tile in plane 0
    const char* base;    // of this step
    uint64_t plane_bytes;

    __device__ __forceinline__ void init(uint64_t ld, uint64_t plane, uint32_t wave, uint32_t lane) {
        ld2 = (uint32_t)(2 * ld);
#pragma unroll
        for (int u = 0; u < N; u++) {
            const uint32_t line = (wave * N + u) * kLines + lane / kChunks;
            const uint32_t c = (lane % kChunks) ^ (ACROSS ? Across<ROWS>::turn(line) : line & 7u);
            at[u] = line * ld2 + c * 16;
            if (!ACROSS) chunk = c * 8;
        }
        plane_bytes = 2 * plane;
    }
    // lines: stored rows of the operand, of `cols` elements; row0: of the tile
    __device__ __forceinline__ void tile(const void* p, uint64_t cols, uint64_t lines, uint64_t row0) {
        first = static_cast<const char*>(p) + row0 * (ACROSS ? 2 : ld2);
        if (ACROSS) bytes = 2 * (uint32_t)min((uint64_t)ROWS, cols - row0);
        else bytes = ((uint32_t)min((uint64_t)ROWS, lines - row0) - 1) * ld2 + 2 * (uint32_t)min((uint64_t)64, cols);
    }
    __device__ __forceinline__ void seek(uint32_t plane, uint32_t l) {
        base = first + plane * plane_bytes + (uint64_t)l * (ACROSS ? ld2 : 2) * 64;
    }
    // left: values of l from this step on
    __device__ __forceinline__ void fetch(char* tile, uint32_t wave, uint32_t left) {
        char* to = tile + wave * (N * kBlock);
        if constexpr (ACROSS) {
            const __amdgpu_buffer_rsrc_t r = buffer_rsrc(base, (min(left, 64u) - 1) * ld2 + bytes);
#pragma unroll
            for (int u = 0; u < N; u++) load_to_lds(r, to + u * kBlock, at[u]);
            base += (uint64_t)ld2 * 64;
        } else {
            const __amdgpu_buffer_rsrc_t r = buffer_rsrc(base, bytes);
            if (left >= 64) {
#pragma unroll
                for (int u = 0; u < N; u++) load_to_lds(r, to + u * kBlock, at[u]);
            } else {
#pragma unroll
                for (int u = 0; u < N; u++)
                    load_to_lds(r, to + u * kBlock, chunk < left ? at[u] : kNowhere);
            }
            base += 128;
        }
    }
};

template <Kind KIND> constexpr bool kPAcross = KIND == DW;
template <Kind KIND> constexpr bool kQAcross = KIND != FORWARD;
template <Kind KIND, typename V, typename S> struct Reads {
    typedef AlongRows<V> Along;
    typedef typename std::conditional<kPAcross<KIND>, AcrossRows<V, S::BM>, Along>::type P;
    typedef typename std::conditional<kQAcross<KIND>, AcrossRows<V, S::BN>, Along>::type Q;
    typedef Stage<S, P, Q> InLds;
    static constexpr uint32_t kLdsBytes = S::kStages * InLds::kBytes;
};

// Tile t: blocks of 8 tiles along i by `stripe` along j, so that the tiles that an
// XCD works on share rows of both operands in its L2.
__device__ __forceinline__ void tile_at(const Product& g, uint32_t t, uint32_t& ti, uint32_t& tj) {
    const uint32_t stripe = t / (g.stripe * g.tiles_i);
    t -= stripe * g.stripe * g.tiles_i;
    const uint32_t w = min(g.stripe, g.tiles_j - g.stripe * stripe), block = t / (8 * w);
    t -= block * 8 * w;
    const uint32_t h = min(8u, g.tiles_i - 8 * block);
    ti = 8 * block + t % h;
    tj = g.stripe * stripe + t / h;
}

// A workgroup's next work: steps [s0, s1) of all passes' steps of a tile, the whole
// of it or a piece.
struct Work {
    uint32_t ti, tj, s0, s1, piece;
    bool whole;
};

// Work i of the launch; workgroup b takes b, b + gridDim.x, ...  Whole tiles come
// first, the tiles of each round so that an XCD has neighbouring ones; then the
// pieces, neighbouring workgroups the same piece of neighbouring tiles.
__device__ __forceinline__ Work work_at(const Product& g, uint32_t i, uint32_t steps) {
    Work w = {0, 0, 0, steps, 0, i < g.whole};
    uint32_t t;
    if (w.whole) {
        const uint32_t round = i / gridDim.x * gridDim.x;
        t = round + by_xcd(i - round, min(gridDim.x, g.whole - round));
    } else {
        w.piece = by_xcd(i - g.whole, g.cut * g.pieces);
        const uint32_t k = w.piece / g.cut;
        t = g.whole + w.piece - k * g.cut;
        w.s0 = (uint32_t)((uint64_t)k * steps / g.pieces);
        w.s1 = (uint32_t)((uint64_t)(k + 1) * steps / g.pieces);
    }
    tile_at(g, t, w.ti, w.tj);
    return w;
}

// Brings the steps of a tile to LDS, one after the other: a pass after the other, or,
// where no factor comes between them (dz in three parts), all passes of a step of l,
// so that x comes from memory once (32768 x 768 x 768: 235 MB read, 340 otherwise).
template <Kind KIND, typename V, typename S> struct Feed {
    static constexpr bool PA = kPAcross<KIND>, QA = kQAcross<KIND>;
    typedef typename Reads<KIND, V, S>::InLds InLds;
    Loads<PA, S::BM, S::kWaves> lp;
    Loads<QA, S::BN, S::kWaves> lq;
    char* s_mem;
    uint32_t inner, wave, lines, pass, l, p_planes, q_planes, mixed;

    __device__ __forceinline__ Feed(const Product& g, char* s_mem_, uint32_t wave_, uint32_t lane)
        : s_mem(s_mem_), inner((uint32_t)g.inner), wave(wave_), lines((uint32_t)((g.inner + 63) / 64)),
          p_planes(g.passes.p_planes), q_planes(g.passes.q_planes),
          mixed(KIND == DW && g.passes.small == 0 && g.passes.count > 1 ? g.passes.count : 0) {
        lp.init(g.p_ld, g.p_plane, wave, lane);
        lq.init(g.q_ld, g.q_plane, wave, lane);
    }
    __device__ __forceinline__ void seek() {
        lp.seek(p_planes >> 4 * pass & 15u, l);
        lq.seek(q_planes >> 4 * pass & 15u, l);
    }
    // the first step is on its way then
    __device__ __forceinline__ void begin(const Product& g, const Work& w) {
        lp.tile(g.p, g.p_cols, PA ? g.inner : g.rows, (uint64_t)w.ti * S::BM);
        lq.tile(g.q, g.q_cols, QA ? g.inner : g.cols, (uint64_t)w.tj * S::BN);
        if (KIND == DW && mixed) {
            l = w.s0 / mixed;
            pass = w.s0 - l * mixed;
        } else {
            pass = w.s0 / lines;
            l = w.s0 - pass * lines;
        }
        seek();
        fetch(0);
    }
    __device__ __forceinline__ void fetch(uint32_t buf) {
        char* base = s_mem + buf * InLds::kBytes;
        const uint32_t left = inner - l * 64;
        lp.fetch(base, wave, left);
        lq.fetch(base + InLds::kQ, wave, left);
        if (KIND == DW && mixed) {
            if (++pass == mixed) {
                pass = 0;
                l++;
            }
            seek();
        } else if (++l == lines) {
            l = 0;
            pass++;
            seek();
        }
    }
};

template <Kind KIND> __device__ __forceinline__ Masks masks_for(const Product& g) {
    Masks masks = {};
    if constexpr (KIND == FORWARD) masks = masks_of(g.forward.drop);
    return masks;
}

// Two neighbouring fragments of a lane, 4 columns of a row each, become 8
// neighbouring columns: odd groups of 16 lanes of the first change places with even
// ones of the second.  Lane group q then has columns 16 (q mod 2) + 8 (q div 2) .. + 7
// of the 32, so that four lanes store 64 bytes of a 16-bit row.
__device__ __forceinline__ uint32_t paired_col(uint32_t lane) { return (lane & 16u) + (lane >> 5) * 8; }
__device__ __forceinline__ void pair_up(const f4& a, const f4& b, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float x = a[e], y = b[e];
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
        const uint32_t first = r[0], second = r[1];
        v[e] = __uint_as_float(first);
        v[4 + e] = __uint_as_float(second);
    }
}

// f(0), f(STEP), ... below END, unrolled however long they are: an index into the sums
// that is not a constant would put them all in memory.
template <int END, int STEP, int I = 0, typename F> __device__ __forceinline__ void unrolled(const F& f) {
    if constexpr (I < END) {
        f(std::integral_constant<int, I>{});
        unrolled<END, STEP, I + STEP>(f);
    }
}

// The power of two that an fp32 row's planes are scaled by: its largest element is
// brought to 2^14 .. 2^15.
__device__ __forceinline__ int scale_of(float most) {
    return most == 0.0f ? 0 : 15 - __builtin_amdgcn_frexp_expf(most);
}

// Columns col .. col + 7 of FM rows 16 apart become results.  What is read for some
// rows is asked for before the first of them is stored: a load behind a store would
// wait for it.
template <Kind KIND, typename T, int FIRST, int FM, int FN>
__device__ __forceinline__ void finish_rows(const Product& g, const Masks& masks, uint64_t row0, uint32_t col,
                                            const f4 (&acc)[FM][FN]) {
    constexpr int N = FM <= 4 ? FM : sizeof(T) == 4 ? 2 : 4;  // rows at a time
    // every lane takes part in the exchange, also those behind the last column
    const uint32_t count = col < g.cols ? g.cols - col : 0;
    // fp32: back from the rows' scales
    float most[8];
    if constexpr (sizeof(T) == 4) load8(g.q_most + col, count, most);
    auto unscale = [&](uint64_t row, float (&v)[8]) __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 4) {
            const int down = row < g.rows ? -scale_of(g.p_most[row]) : 0;
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = __builtin_ldexpf(v[e], down - scale_of(most[e]));
        }
    };
    if constexpr (KIND == FORWARD) {
        const Forward& f = g.forward;
        float bias[8] = {};
        if (f.bias) load8(static_cast<const T*>(f.bias) + col, count, bias);
        unrolled<FM, N>([&](auto u0) __attribute__((always_inline)) {
            T residual[N][8];
            if (f.residual)
#pragma unroll
                for (int u = 0; u < N; u++)
                    load8_raw(static_cast<const T*>(f.residual) + (row0 + 16 * (u0 + u)) * f.residual_ld + col,
                              row0 + 16 * (u0 + u) < g.rows ? count : 0, residual[u]);
            unrolled<N, 1>([&](auto u) __attribute__((always_inline)) {
                float v[8];
                pair_up(acc[u0 + u][FIRST], acc[u0 + u][FIRST + 1], v);
                unscale(row0 + 16 * (u0 + u), v);
                finish_forward<T>(f, masks, row0 + 16 * (u0 + u), g.rows, col, count, bias, residual[u], v);
            });
        });
    } else {
        unrolled<FM, 1>([&](auto u) __attribute__((always_inline)) {
            float v[8];
            pair_up(acc[u][FIRST], acc[u][FIRST + 1], v);
            const uint64_t row = row0 + 16 * u;
            unscale(row, v);
            if (row >= g.rows || count == 0) return;
            from_units<T>(g.gradient, v);
            if constexpr (KIND == DX) store8(static_cast<T*>(g.gradient.out) + row * g.gradient.ld + col, count, v);
            else store_gradient(g.gradient, row, col, count, v);
        });
    }
}

// Workgroups of a CU by what LDS holds, as waves of a SIMD.
template <typename S> constexpr int kWavesOfSimd = S::BM == 64 ? 3 : 2;

// The kernel's arguments, to be loaded again: held over a main loop they would take
// more scalar registers than there are.
__device__ __forceinline__ const Product& again() {
    typedef const __attribute__((address_space(4))) Product ConstantProduct;
    ConstantProduct* p = (ConstantProduct*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Product*)p;
}

// A workgroup takes one tile, or piece of one, after the other.  The first step of
// the next is on its way while results are stored.
template <Kind KIND, typename T, typename V, typename S>
__global__ __launch_bounds__(S::kThreads, kWavesOfSimd<S>) void tiled_kernel(Product g) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    typedef Reads<KIND, V, S> R;
    extern __shared__ __align__(16) char s_mem[];
    const uint32_t steps = g.passes.count * (uint32_t)((g.inner + 63) / 64);
    const uint32_t all = g.whole + g.cut * g.pieces;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t wi = wave / (S::BN / S::WN) * S::WM, wj = wave % (S::BN / S::WN) * S::WN;
    constexpr bool kScaled = KIND == DW || sizeof(T) == 4;
    const float factor = g.passes.factor;
    const uint32_t small = kScaled ? g.passes.small * ((uint32_t)(g.inner + 63) / 64) : 0;  // steps
    Feed<KIND, V, S> feed(g, s_mem, wave, lane);
    uint32_t i = blockIdx.x;
    Work w = work_at(g, i, steps);
    feed.begin(g, w);
    for (;;) {
        float zero = 0.0f;
        asm volatile("" : "+v"(zero));  // or a register for each zero is held throughout
        f4 acc[FM][FN];
#pragma unroll
        for (int u = 0; u < FM; u++)
#pragma unroll
            for (int v = 0; v < FN; v++) acc[u][v] = f4{zero, zero, zero, zero};
        auto run = [&](uint32_t n) {
            auto fetch = [&](uint32_t, uint32_t buf) { feed.fetch(buf); };
            if constexpr (S::kWaves == 8)
                main_loop_paired<1, S, V, typename R::P, typename R::Q>(acc, fetch, s_mem, n, wi, wj, lane, wave);
            else
                main_loop<1, S, V, typename R::P, typename R::Q>(acc, fetch, s_mem, n, wi, wj, lane);
            __syncthreads();
        };
        uint32_t s0 = w.s0;
        if (kScaled && s0 < small) {
            const uint32_t stop = min(w.s1, small);
            run(stop - s0);
#pragma unroll
            for (int u = 0; u < FM; u++)
#pragma unroll
                for (int v = 0; v < FN; v++) acc[u][v] *= factor;
            s0 = stop;
            if (s0 < w.s1) feed.fetch(0);
        }
        if (s0 < w.s1) run(w.s1 - s0);
        const Product& e = again();
        i += gridDim.x;
        Work next = {};
        if (i < all) {
            next = work_at(e, i, steps);
            feed.begin(e, next);
        }
        if (w.whole) {
            const Masks masks = masks_for<KIND>(e);
            const uint64_t row0 = (uint64_t)w.ti * S::BM + wi + (lane & 15);
            const uint32_t col0 = w.tj * S::BN + wj + paired_col(lane);
            unrolled<FN, 2>([&](auto v) __attribute__((always_inline)) {
                finish_rows<KIND, T, v>(e, masks, row0, col0 + 16 * v, acc);
            });
        } else {
            f4* part = reinterpret_cast<f4*>(e.part) + (size_t)w.piece * (S::BM * S::BN / 4);
#pragma unroll
            for (int u = 0; u < FM; u++)
#pragma unroll
                for (int v = 0; v < FN; v++) part[(u * FN + v) * S::kThreads + threadIdx.x] = acc[u][v];
        }
        if (i >= all) return;
        w = next;
    }
}

// The sums of the cut tiles' pieces, in order.  A wave takes two neighbouring
// fragments of a wave's part of a tile.
template <Kind KIND, typename T, typename S> __global__ __launch_bounds__(256) void join_kernel(Product g) {
    constexpr uint32_t FM = S::WM / 16, FN = S::WN / 16, kPairs = S::kWaves * FM * FN / 2;  // of a tile
    const uint32_t at = blockIdx.x * 4 + (threadIdx.x >> 6), c = at / kPairs, pair = at - c * kPairs;
    const uint32_t wave = pair / (FM * FN / 2), u = pair / (FN / 2) % FM, v = pair % (FN / 2) * 2;
    const uint32_t lane = threadIdx.x & 63;
    const f4* part = reinterpret_cast<const f4*>(g.part) + (size_t)c * (S::BM * S::BN / 4) +
                     (u * FN + v) * S::kThreads + wave * 64 + lane;
    const size_t step = (size_t)g.cut * (S::BM * S::BN / 4);
    constexpr uint32_t kAhead = 8;  // pieces asked for at once
    f4 acc[1][2] = {};
    for (uint32_t q0 = 0; q0 < g.pieces; q0 += kAhead) {
        f4 a[kAhead], b[kAhead];
#pragma unroll
        for (uint32_t q = 0; q < kAhead; q++)
            if (q0 + q < g.pieces) {
                a[q] = part[(q0 + q) * step];
                b[q] = part[(q0 + q) * step + S::kThreads];
            }
#pragma unroll
        for (uint32_t q = 0; q < kAhead; q++)
            if (q0 + q < g.pieces) {
                acc[0][0] += a[q];
                acc[0][1] += b[q];
            }
    }
    uint32_t ti, tj;
    tile_at(g, g.whole + c, ti, tj);
    const uint64_t row = (uint64_t)ti * S::BM + wave / (S::BN / S::WN) * S::WM + 16 * u + (lane & 15);
    const uint32_t col = tj * S::BN + wave % (S::BN / S::WN) * S::WN + 16 * v + paired_col(lane);
    finish_rows<KIND, T, 0>(g, masks_for<KIND>(g), row, col, acc);
}

// ---- operands as the tiles take them --------------------------------------------------

struct PackArgs {
    const void* in;
    void* out;
    uint64_t rows, in_ld, out_ld, plane;
    uint32_t cols;
};

// A 16-bit matrix of any stride and alignment as rows of a multiple of 64 values
// with zeros behind them.
template <typename T> __global__ __launch_bounds__(256) void pack_kernel(PackArgs a) {
    const uint32_t groups = (uint32_t)(a.out_ld / 8);
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = at / groups;
    if (row >= a.rows) return;
    const uint32_t col = (uint32_t)(at - row * groups) * 8;
    float v[8];
    load8(static_cast<const T*>(a.in) + row * a.in_ld + (col < a.cols ? col : 0), col < a.cols ? a.cols - col : 0, v);
    store8(static_cast<T*>(a.out) + row * a.out_ld + col, 8, v);
}

// fp32 matrices go in two fp16 planes, scaled by a power of two for each row of the
// product's operand, which leaves the sums by 2^-(both) at the end.  That way 22 bits
// of every element down to 2^-29 of its row's largest are kept, and nothing is lost
// above 2^-51 of it; three products of fp16 then take half the time of six of bf16
// planes, which would need no scale (33278 x 1500 x 700: 427 us).  The largest is
// taken over finite elements; infinity leaves no rest, NaN is NaN in both.
__device__ __forceinline__ void split2(float v, int scale, _Float16& high, _Float16& rest) {
    const float s = __builtin_ldexpf(v, scale);
    high = (_Float16)s;
    const float r = s - (float)high;
    rest = (_Float16)(r - r == 0.0f || s != s ? r * kRestUnit : 0.0f);
}

__device__ __forceinline__ void store_two(void* out, uint64_t plane, uint64_t at, const float (&v)[8],
                                          const int (&scale)[8]) {
    h8 high, rest;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        _Float16 a, b;
        split2(v[e], scale[e], a, b);
        high[e] = a;
        rest[e] = b;
    }
    *reinterpret_cast<h8*>(static_cast<_Float16*>(out) + at) = high;
    *reinterpret_cast<h8*>(static_cast<_Float16*>(out) + plane + at) = rest;
}

// |v| where v is finite, else 0.
__device__ __forceinline__ float finite_size(float v) {
    const float a = fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}

// A workgroup a stored row, which is a row of the operand: its largest element, then
// its planes.  cols_out: the same matrix again by its columns' scales (dz is P along
// its rows for dx and across them for dw).
struct SplitRowsArgs {
    PackArgs pack;
    float* most;             // of each row
    void* cols_out;          // or null
    const float* cols_most;
};

__global__ __launch_bounds__(256) void split_rows_kernel(SplitRowsArgs a) {
    __shared__ float s_most[4];
    const uint32_t groups = (uint32_t)(a.pack.out_ld / 8), cols = a.pack.cols;
    for (uint64_t row = blockIdx.x; row < a.pack.rows; row += gridDim.x) {
        const float* in = static_cast<const float*>(a.pack.in) + row * a.pack.in_ld;
        float v[8], most = 0.0f;
        auto load = [&](uint32_t g) {
            load8(in + (g * 8 < cols ? g * 8 : 0), g * 8 < cols ? cols - g * 8 : 0, v);
        };
        for (uint32_t g = threadIdx.x; g < groups; g += 256) {
            load(g);
#pragma unroll
            for (int e = 0; e < 8; e++) most = fmaxf(most, finite_size(v[e]));
        }
        for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
        __syncthreads();  // the row before is done with
        if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
        __syncthreads();
        most = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
        if (threadIdx.x == 0) a.most[row] = most;
        const int mine = scale_of(most), all[8] = {mine, mine, mine, mine, mine, mine, mine, mine};
        for (uint32_t g = threadIdx.x; g < groups; g += 256) {
            if (groups > 256) load(g);  // otherwise it is still there
            const uint64_t at = row * a.pack.out_ld + g * 8;
            store_two(a.pack.out, a.pack.plane, at, v, all);
            if (!a.cols_out) continue;
            float by[8];
            int scale[8];
            load8(a.cols_most + g * 8, 8, by);
#pragma unroll
            for (int e = 0; e < 8; e++) scale[e] = scale_of(by[e]);
            store_two(a.cols_out, a.pack.plane, at, v, scale);
        }
    }
}

// The largest element of each column, into zeros.  Sizes are compared as the whole
// numbers that their bits are, so that no order of the atomics matters.
__device__ __forceinline__ void columns_most(float* s_most, uint32_t width, uint32_t step, const float (&most)[8],
                                             uint32_t first, uint32_t cols, float* out) {
#pragma unroll
    for (int e = 0; e < 8; e++) s_most[threadIdx.x * 8 + e] = most[e];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < width * 8; c += 256) {
        float t = 0.0f;
        for (uint32_t r = 0; r < step; r++) t = fmaxf(t, s_most[r * width * 8 + c]);
        if (first + c < cols) atomicMax(reinterpret_cast<uint32_t*>(out) + first + c, __float_as_uint(t));
    }
}

__global__ __launch_bounds__(256) void most_kernel(PackArgs a, uint64_t per, float* __restrict__ out) {
    __shared__ float s_most[256 * 8];
    const uint32_t col = (blockIdx.x * 64 + (threadIdx.x & 63)) * 8;
    const uint64_t end = min((uint64_t)(blockIdx.y + 1) * per, a.rows);
    float most[8] = {};
    if (col < a.cols)
        for (uint64_t row = (uint64_t)blockIdx.y * per + (threadIdx.x >> 6); row < end; row += 4) {
            float v[8];
            load8(static_cast<const float*>(a.in) + row * a.in_ld + col, a.cols - col, v);
#pragma unroll
            for (int e = 0; e < 8; e++) most[e] = fmaxf(most[e], finite_size(v[e]));
        }
    columns_most(s_most, 64, 4, most, blockIdx.x * 512, a.cols, out);
}

// A matrix whose columns are the operand's rows, by their scales.
__global__ __launch_bounds__(256) void split_columns_kernel(PackArgs a, const float* __restrict__ most) {
    const uint32_t groups = (uint32_t)(a.out_ld / 8);
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x, row = at / groups;
    if (row >= a.rows) return;
    const uint32_t col = (uint32_t)(at - row * groups) * 8;
    float v[8], by[8];
    int scale[8];
    load8(static_cast<const float*>(a.in) + row * a.in_ld + (col < a.cols ? col : 0), col < a.cols ? a.cols - col : 0, v);
    load8(most + col, 8, by);
#pragma unroll
    for (int e = 0; e < 8; e++) scale[e] = scale_of(by[e]);
    store_two(a.out, a.plane, row * a.out_ld + col, v, scale);
}

// An fp16 dz, up to 65504 times dropout's scale and the largest slope, is held in units of
// the power of two that takes both in, so that it does not overflow: that costs nothing
// in its normal range, and what is lost below it, 2^-25 units, is less than twice what dy,
// off by 2^-25 itself, brings along.  The sums are multiplied by the unit.
float dz_unit(uint32_t act, const Dropout& d) {
    const float slope = act == HC_ACT_GELU || act == HC_ACT_SILU ? 1.13f : 1.0f;
    float unit = 1.0f;
    while (unit < d.scale * slope) unit *= 2.0f;
    return unit;
}

// v = the sum of three bf16 values, exactly where v is no smaller than 2^-110.
// Infinity leaves nothing, NaN is NaN in all.
__device__ __forceinline__ void split3(float v, __bf16 (&w)[3]) {
    w[0] = (__bf16)v;
    const float first = (float)w[0], r = fabsf(first) == __builtin_inff() && v == v ? 0.0f : v - first;
    w[1] = (__bf16)r;
    w[2] = (__bf16)(r - (float)w[1]);
}

// ---- dz and the bias's gradient ----------------------------------------------------

struct DzArgs {
    const void *dy, *z;
    uint64_t dy_ld, z_ld, m;
    uint32_t n, groups;
    uint32_t act;
    uint32_t per;      // rows of a workgroup
    uint32_t width;    // lanes for a row, up to 64
    Dropout drop;
    PackArgs dz;       // where it goes (out: or null), zeros behind its columns
    uint32_t planes;   // 1: in its own type; 2: and 2^11 times the rest; 3: bf16 parts
    float per_unit;    // fp16: dz is multiplied by it, 1 / its unit
    float* most;       // fp32: the largest of each column, or null
    float* part;       // the workgroups' sums, [blocks][n], or null
    Gradient db;       // one workgroup along the rows: the sums themselves
};

// dz = act'(z) mask dy, and each workgroup's sums of its rows.  Memory bounds it: 32768
// x 768 in bf16 through GELU and dropout into three parts, 250 MB, 53 us (115 with 512
// workgroups of columns in powers of two, and a first part that was checked for
// overflow).
template <typename T> __global__ __launch_bounds__(256) void dz_kernel(DzArgs a) {
    __shared__ float s_sum[256 * 8];
    const Masks masks = masks_of(a.drop);
    const uint32_t lane = threadIdx.x % a.width, sub = threadIdx.x / a.width, step = 256 / a.width;
    const uint32_t group = blockIdx.x * a.width + lane, col = group * 8;
    const uint64_t end = min((uint64_t)(blockIdx.y + 1) * a.per, a.m);
    float sum[8] = {}, most[8] = {};
    if (group < a.groups && sub < step) {
        const uint32_t count = col < a.n ? a.n - col : 0;
        for (uint64_t row = (uint64_t)blockIdx.y * a.per + sub; row < end; row += step) {
            float v[8];
            load8(static_cast<const T*>(a.dy) + row * a.dy_ld + col, count, v);
            MaskBits bits = {};
            if (masks.limit) {
                bits = mask_bits(masks, (uint32_t)row, group);
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] *= masks.scale;
            }
            if (a.act != HC_ACT_NONE) {
                float z[8];
                load8(static_cast<const T*>(a.z) + row * a.z_ld + col, count, z);
                backward8<T>(a.act, z, v);
            }
            // after the slope, which may be NaN: a dropped element is 0 whatever z was
            if (masks.limit)
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = bits.kept(e, masks.limit) ? v[e] : 0.0f;
            if (count < 8)
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < count ? v[e] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) sum[e] += v[e];
            if (sizeof(T) == 4 && a.most)
#pragma unroll
                for (int e = 0; e < 8; e++) most[e] = fmaxf(most[e], finite_size(v[e]));
            if (!a.dz.out) continue;
            const uint64_t at = row * a.dz.out_ld + col;
            if (a.planes == 3) {
                b8 w[3];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    __bf16 s[3];
                    split3(v[e], s);
#pragma unroll
                    for (int k = 0; k < 3; k++) w[k][e] = s[k];
                }
#pragma unroll
                for (int k = 0; k < 3; k++)
                    *reinterpret_cast<b8*>(static_cast<__bf16*>(a.dz.out) + k * a.dz.plane + at) = w[k];
            } else {
                if constexpr (std::is_same<T, _Float16>::value)
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] *= a.per_unit;
                store8(static_cast<T*>(a.dz.out) + at, 8, v);
                if (a.planes == 2) {
                    // infinity and NaN leave nothing
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float r = v[e] - (float)(T)v[e];
                        v[e] = r - r == 0.0f ? r * kRestUnit : 0.0f;
                    }
                    store8(static_cast<T*>(a.dz.out) + a.dz.plane + at, 8, v);
                }
            }
        }
    }
    if (sizeof(T) == 4 && a.most) {
        columns_most(s_sum, a.width, step, most, blockIdx.x * a.width * 8, a.n, a.most);
        __syncthreads();
    }
    if (!a.part) return;
#pragma unroll
    for (int e = 0; e < 8; e++) s_sum[threadIdx.x * 8 + e] = sum[e];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.width * 8; c += 256) {
        float t = 0.0f;
        for (uint32_t r = 0; r < step; r++) t += s_sum[r * a.width * 8 + c];
        const uint32_t at = blockIdx.x * a.width * 8 + c;
        if (at >= a.n) continue;
        if (gridDim.y > 1) {
            a.part[(uint64_t)blockIdx.y * a.n + at] = t;
        } else {
            float v[8] = {t};
            store_gradient(a.db, 0, at, 1, v);
        }
    }
}

// db: the workgroups' sums, 16 columns a workgroup, in 64 shares that are added in
// order.
__global__ __launch_bounds__(1024) void bias_kernel(const float* __restrict__ part, uint32_t blocks, uint32_t n,
                                                    Gradient g) {
    __shared__ float s_sum[64][17];
    const uint32_t lane = threadIdx.x & 15, share = threadIdx.x >> 4, col = blockIdx.x * 16 + lane;
    float t = 0.0f;
    if (col < n)
#pragma unroll 8
        for (uint32_t b = blocks * share / 64; b < blocks * (share + 1) / 64; b++) t += part[(uint64_t)b * n + col];
    s_sum[share][lane] = t;
    __syncthreads();
    if (threadIdx.x < 16 && col < n) {
        t = 0.0f;
        for (int k = 0; k < 64; k++) t += s_sum[k][lane];
        float v[8] = {t};
        store_gradient(g, 0, col, 1, v);
    }
}

// ---- layout and launches ------------------------------------------------------------

constexpr uint64_t kDzGroups = 2048;     // workgroups of dz
// db of a dz that is dy, up to these rows and elements, is summed in the launch of small products, or
// alone in such a one: 512 x 512 (fp32) 3.8 us, 2048 x 64 6.8, where dz's pass and its join take 6.2.
// More elements take those as long (2048 x 1500: 11.7 and 11.9), and fp32 planes need dz's pass anyway
// (2048 x 512 x 512 57 us, 61 with db apart).  By m and n alone, since db is asked for without x and w too.
constexpr uint64_t kSplitBias = 2048, kSplitBiasElements = 1ull << 19;
constexpr uint64_t kDzAlone = 32;        // rows that one workgroup takes, without a launch for db

uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to; }

// Direct products: cut along l until there are this many workgroups.
constexpr uint64_t kSlots = 1024;
constexpr uint64_t kMostPieces = 64;

uint64_t direct_pieces(uint64_t tiles, uint64_t lines) {
    uint64_t pieces = kSlots / tiles;
    pieces = pieces > lines / 4 ? lines / 4 : pieces;
    return pieces > kMostPieces ? kMostPieces : pieces < 1 ? 1 : pieces;
}

template <Kind KIND, typename T> hipError_t direct(Product g, hipStream_t s) {
    const uint64_t lines = up(g.inner, kStep) * g.passes.count;
    g.tiles_j = (uint32_t)up(g.cols, kDirect);
    const uint64_t tiles = up(g.rows, kDirect) * g.tiles_j;
    const uint64_t pieces = direct_pieces(tiles, lines);
    g.cut = (uint32_t)tiles;
    g.pieces = (uint32_t)pieces;
    g.part_ld = (uint32_t)up(g.cols, 8) * 8;
    hipLaunchKernelGGL((direct_kernel<KIND, T>), dim3((uint32_t)(tiles * pieces)), dim3(256), 0, s, g);
    if (pieces > 1)
        hipLaunchKernelGGL((direct_join_kernel<KIND, T>), dim3((uint32_t)up(g.rows * (g.part_ld / 8), 256)),
                           dim3(256), 0, s, g);
    return hipGetLastError();
}

typedef Shape<256, 256, 128, 64, 2> Large;
typedef Shape<128, 128, 64, 64, 2> Medium;
typedef Shape<64, 64, 32, 32, 3> Small;
constexpr int kShapes = 3;

// Estimated times in us: a step takes a workgroup `alone` on its CU, or `shared` by
// as many as fit; a tile's first loads and its results take `ends`, a piece's with
// the tile of sums that it writes `piece_ends`.  From measured products whose inputs
// come from memory.
struct TileCost {
    uint64_t bm, bn, resident;
    double alone, shared, ends, piece_ends;
};
constexpr TileCost kTileCosts[kShapes] = {
    {256, 256, 1, 1.50, 1.50, 16.0, 10.0},
    {128, 128, 2, 0.60, 0.86, 7.0, 6.0},
    {64, 64, 3, 0.35, 0.70, 5.0, 4.0},
};
constexpr uint64_t kLeastSteps = 4;      // of a piece
constexpr double kJoin = 5.0, kBytesPerUs = 5e6;

struct TilePlan {
    int shape;
    uint32_t tiles_i, tiles_j, whole, cut, pieces;
    double us;
};

double rounds(const TileCost& c, uint64_t groups, double steps, double ends) {
    const uint64_t slots = kCus * c.resident, full = groups / slots, rest = groups % slots;
    double t = (double)full * (steps * c.shared + ends);
    if (rest) t += steps * (rest <= kCus ? c.alone : c.shared) + ends;
    return t;
}

// The tile's size, and how many tiles are cut into how many pieces: none, all, or
// those left after whole rounds of the CUs.  (bf16, us: 4096 x 25088 x 4096 in 256-tiles
// 710 whole, 672 with the 32 left after six rounds in 8 pieces each; 2048 x 2048 x 2048
// 68 in 256-tiles, 37 in 128; 1024 x 1024 x 1024 36, 21 and 12 in 256, 128 and 64.)
TilePlan tile_plan(uint64_t rows, uint64_t cols, uint64_t steps) {
    TilePlan best = {};
    double least = 1e300;
    for (int k = 0; k < kShapes; k++) {
        const TileCost& c = kTileCosts[k];
        const uint64_t ti = up(rows, c.bm), tj = up(cols, c.bn), n = ti * tj, slots = kCus * c.resident;
        auto consider = [&](double t, uint64_t whole, uint64_t pieces) {
            if (t >= least) return;
            least = t;
            best = {k, (uint32_t)ti, (uint32_t)tj, (uint32_t)whole, (uint32_t)(n - whole), (uint32_t)pieces, t};
        };
        consider(rounds(c, n, (double)steps, c.ends), n, 1);
        const uint64_t rest = n % slots, most = steps / kLeastSteps < kMostPieces ? steps / kLeastSteps : kMostPieces;
        if (rest == 0) continue;
        const uint64_t whole = n - rest;
        for (uint64_t room : {(uint64_t)kCus, slots}) {
            const uint64_t pieces = room / rest < most ? room / rest : most;
            if (pieces < 2) continue;
            const double t = rounds(c, whole, (double)steps, c.ends) +
                             rounds(c, rest * pieces, (double)up(steps, pieces), c.piece_ends) + kJoin +
                             4.0 * (double)(c.bm * c.bn * rest * (pieces + 1)) / kBytesPerUs;
            consider(t, whole, pieces);
        }
    }
    return best;
}

template <Kind KIND, typename T, typename V, typename S>
hipError_t tiled_shape(const Product& g, uint64_t resident, hipStream_t s) {
    const auto kernel = &tiled_kernel<KIND, T, V, S>;
    constexpr int kLds = Reads<KIND, V, S>::kLdsBytes;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kLds);
    if (e != hipSuccess) return e;
    const uint32_t all = g.whole + g.cut * g.pieces, slots = (uint32_t)(kCus * resident);
    hipLaunchKernelGGL(kernel, dim3(all < slots ? all : slots), dim3(S::kThreads), kLds, s, g);
    if (g.cut)
        hipLaunchKernelGGL((join_kernel<KIND, T, S>),
                           dim3(g.cut * (S::BM * S::BN / 512 / 4)), dim3(256), 0, s, g);
    return hipGetLastError();
}

template <Kind KIND, typename T, typename V> hipError_t tiled(Product g, hipStream_t s) {
    const TilePlan p = tile_plan(g.rows, g.cols, up(g.inner, 64) * g.passes.count);
    g.tiles_i = p.tiles_i;
    g.tiles_j = p.tiles_j;
    g.whole = p.whole;
    g.cut = p.cut;
    g.pieces = p.pieces;
    const TileCost& c = kTileCosts[p.shape];
    // as wide as Q's rows fit an XCD's L2 beside P's
    const uint64_t panel = c.bn * g.inner * 2 * g.passes.count;
    const uint64_t stripe = panel < (1u << 21) / 4 ? (1u << 21) / panel : 4;
    g.stripe = (uint32_t)(stripe < p.tiles_j ? stripe : p.tiles_j);
    const uint64_t resident = c.resident;
    if (p.shape == 0) return tiled_shape<KIND, T, V, Large>(g, resident, s);
    if (p.shape == 1) return tiled_shape<KIND, T, V, Medium>(g, resident, s);
    return tiled_shape<KIND, T, V, Small>(g, resident, s);
}

// Estimated time of a small product: a wave's four steps take 1 us, its tiles' rows
// come from L2 again and again, and four workgroups on a CU take 4 us at least.  Of an
// operand across its rows a tile reads 16 columns, and with them the 128 bytes that they
// are in: dx of 1 x 4096 x 4096 (bf16) 23 us, in tiles 12.5.
double split_cost(Kind kind, uint64_t rows, uint64_t cols, uint64_t inner, uint32_t passes, hc_type type) {
    const double tiles = (double)up(rows, kSplitTile) * (double)up(cols, kSplitTile);
    const uint64_t lines = up(inner, kStep) * passes, along = type == HC_T_F32 ? 4 : 2, across = 128 / kSplitTile;
    const uint64_t live = (rows < kSplitTile ? rows : kSplitTile) * (kind == DW ? across : along) +
                          (cols < kSplitTile ? cols : kSplitTile) * (kind == FORWARD ? along : across);
    return 1.5 + 1.0 * (double)up(lines, kSplitWaves * kSplitAhead) + tiles / (4 * kCus) * 4.0 +
           tiles * passes * (double)inner * (double)live / 9e6;
}

// And of a direct one: a step of 32 takes 0.8 us.
double direct_cost(uint64_t rows, uint64_t cols, uint64_t inner, uint32_t passes, hc_type type) {
    const uint64_t lines = up(inner, kStep) * passes, pieces = direct_pieces(up(rows, kDirect) * up(cols, kDirect), lines);
    return 3.0 + 0.8 * (double)up(lines, pieces) + (pieces > 1 ? 4.0 : 0.0) +
           2.0 * (double)(up(rows, kDirect) * kDirect) * (double)(up(cols, kDirect) * kDirect) * (double)inner * passes /
               (type == HC_T_F32 ? 75e6 : 280e6);
}

// How a product runs: operands as the tiles take them (fp32 in two planes) or as
// they are, and then in small tiles or not.
enum Way { SPLIT, DIRECT, TILED };

Way way_of(Kind kind, const Product& g, hc_type type, bool in_tiles) {
    if (g.inner == 0 || g.rows == 0) return DIRECT;
    if (in_tiles && type == HC_T_F32) return TILED;
    const uint32_t passes = g.passes.count;
    const double split = split_cost(kind, g.rows, g.cols, g.inner, passes, type);
    const double other = in_tiles ? tile_plan(g.rows, g.cols, up(g.inner, 64) * passes).us
                                  : direct_cost(g.rows, g.cols, g.inner, passes, type);
    return split < other ? SPLIT : in_tiles ? TILED : DIRECT;
}

uint32_t split_tiles(Product* g) {
    g->tiles_j = (uint32_t)up(g->cols, kSplitTile);
    return (uint32_t)up(g->rows, kSplitTile) * g->tiles_j;
}

template <typename T> hipError_t split_forward(Product g, hipStream_t s) {
    const uint32_t tiles = split_tiles(&g);
    hipLaunchKernelGGL(split_forward_kernel<T>, dim3(tiles), dim3(512), 0, s, g);
    return hipGetLastError();
}

template <typename T> hipError_t split_grad(SplitGrad g, hipStream_t s) {
    g.dx_tiles = g.dx.gradient.out ? split_tiles(&g.dx) : 0;
    g.dw_tiles = g.dw.gradient.out ? split_tiles(&g.dw) : 0;
    const uint32_t all = g.dx_tiles + g.dw_tiles + (g.dy ? (uint32_t)up(g.n, 64) : 0);
    if (all) hipLaunchKernelGGL(split_grad_kernel<T>, dim3(all), dim3(512), 0, s, g);
    return hipGetLastError();
}

template <Kind KIND> hipError_t product(const Product& g, hc_type type, Way way, hipStream_t s) {
    if (way == TILED) {
        if (type == HC_T_F32) return tiled<KIND, float, h8>(g, s);
        if (type == HC_T_BF16) return tiled<KIND, __bf16, b8>(g, s);
        return tiled<KIND, _Float16, h8>(g, s);
    }
    if (type == HC_T_F32) return direct<KIND, float>(g, s);
    if (type == HC_T_BF16) return direct<KIND, __bf16>(g, s);
    return direct<KIND, _Float16>(g, s);
}

// Most bytes of partial sums for up to this many rows of D (fewer rows may be cut
// into more pieces): pieces fill the CUs once.
size_t most_part_bytes(uint64_t rows, uint64_t cols) {
    size_t most = 0;
    auto take = [&](uint64_t bm, uint64_t bn, uint64_t groups) {
        const uint64_t tiles = up(rows, bm) * up(cols, bn);
        const uint64_t n = tiles < groups / kMostPieces ? tiles * kMostPieces : groups;
        const size_t bytes = n * bm * bn * 4;
        most = bytes > most ? bytes : most;
    };
    for (const TileCost& c : kTileCosts) take(c.bm, c.bn, kCus * c.resident);
    take(kDirect, kDirect, kSlots);
    return most;
}

// ---- which way a call goes --------------------------------------------------------------

constexpr uint64_t kStreamBytes = 32ull << 20;  // of all eight L2s
constexpr uint64_t kMostTileLd = 1ull << 22;  // a tile's rows within 2^31 bytes

// A 16-bit operand whose rows the tiles can take where they are.
bool tile_rows(const void* p, uint64_t cols, uint64_t ld) {
    return aligned(p, 16) && cols % 8 == 0 && ld % 8 == 0 && ld <= kMostTileLd;
}

// Whether operands that the tiles cannot take as they are (fp32: all) are copied
// for them, rather than multiplied directly: by estimated times that are linear in
// m, so that what is copied for m rows is room for fewer.  Direct products reach 75
// TFLOP/s in fp32 and 170 to 400 in 16 bits; tiles a third of 1000 and 1000.
bool worth_packing(const hc_linear_params& p, hc_type type, bool grad) {
    const bool fp32 = type == HC_T_F32;
    const double mk = (double)p.m * p.k, nk = (double)p.n * p.k, mn = (double)p.m * p.n;
    const double flops = 2.0 * mn * p.k * (grad ? 2.0 : 1.0);
    // what packing moves, and its launches
    const double bytes = !fp32 ? 4.0 * (mk + nk + (grad ? mn : 0.0)) : grad ? 12.0 * (mk + nk) + 24.0 * mn : 8.0 * (mk + nk);
    const double launches = !fp32 ? 15.0 : grad ? 40.0 : 15.0;
    const double gain = fp32 ? 1.0 / 75e6 - 3.0 / 1000e6 : 1.0 / 280e6 - 1.0 / 1000e6;
    return p.k <= kMostTileLd && p.n <= kMostTileLd && flops * gain > bytes / 4e6 + launches;
}

struct Layout {
    size_t x, w, dz, bias, part, bytes;
    size_t dz_rows, dz_cols;          // fp32: its planes by rows and by columns
    size_t row_most, col_most;        // the largest elements: forward of x and w; of dz,
    uint64_t x_most, w_most, most;    // and of dz, x and w by columns, from here and in all
    uint64_t k_ld, n_ld;  // of packed rows
    uint64_t per, blocks;
    uint32_t width;
    bool pack_x, pack_w;  // whether they are copied; fp32: both or none
};

size_t take(size_t& at, size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
}

// Copies of x and w: where they are worth it, and they may be needed (a pointer's
// alignment is not known here; one that is off by itself goes the direct way).  The
// gradient has them each by its own strides, since dx is the same whether x is there
// or not, and dw whether w is.
void take_packed(const hc_linear_params& p, hc_type type, bool grad, size_t& at, Layout* L) {
    const size_t size = type == HC_T_F32 ? 4 : 2;
    L->k_ld = up(p.k, 64) * 64;
    L->n_ld = up(p.n, 64) * 64;
    const bool worth = worth_packing(p, type, grad);
    auto needed = [&](uint64_t ld) { return type == HC_T_F32 || p.k % 8 || ld % 8 || ld > kMostTileLd; };
    L->pack_x = worth && (needed(p.x_ld) || (!grad && needed(p.w_ld)));
    L->pack_w = worth && (needed(p.w_ld) || (!grad && needed(p.x_ld)));
    L->x = take(at, L->pack_x ? p.m * L->k_ld * size : 0);
    L->w = take(at, L->pack_w ? p.n * L->k_ld * size : 0);
}

Layout linear_layout(const hc_linear_params& p, hc_type type) {
    Layout L = {};
    size_t at = 0;
    take_packed(p, type, false, at, &L);
    const bool planes = L.pack_x && type == HC_T_F32;
    L.row_most = take(at, planes ? p.m * 4 : 0);
    L.col_most = take(at, planes ? L.n_ld * 4 : 0);
    L.part = take(at, most_part_bytes(p.m, p.n));
    L.bytes = at;
    return L;
}

Layout grad_layout(const hc_linear_params& p, hc_type type) {
    Layout L = {};
    size_t at = 0;
    take_packed(p, type, true, at, &L);
    const uint64_t groups = L.n_ld / 8;
    // as few column blocks of up to 64 lanes as there can be, evenly wide
    const uint64_t across = up(groups, 64);
    L.width = (uint32_t)up(groups, across);
    const uint64_t step = 256 / L.width, most = across < kDzGroups ? kDzGroups / across : 1;
    L.per = p.m <= kDzAlone ? kDzAlone : up(up(p.m, most), step) * step;
    L.blocks = p.m ? up(p.m, L.per) : 0;
    L.dz = take(at, p.m * L.n_ld * (type == HC_T_BF16 ? 6 : 4));
    const bool planes = L.pack_x && type == HC_T_F32;
    L.dz_rows = take(at, planes ? p.m * L.n_ld * 4 : 0);
    L.dz_cols = take(at, planes ? p.m * L.n_ld * 4 : 0);
    L.row_most = take(at, planes ? p.m * 4 : 0);
    L.x_most = L.n_ld;
    L.w_most = L.n_ld + L.k_ld;
    L.most = L.n_ld + 2 * L.k_ld;
    L.col_most = take(at, planes ? L.most * 4 : 0);
    L.bias = take(at, (p.m < most ? p.m : most) * p.n * 4);
    const size_t a = most_part_bytes(p.m, p.k), b = most_part_bytes(p.n, p.k);
    L.part = take(at, a > b ? a : b);
    L.bytes = at;
    return L;
}

struct Operand {
    const void* p;
    uint64_t ld, cols, plane;
};

// rows x cols of a 16-bit operand in tiles' form: where it is, or packed into `to`.
hipError_t packed(hc_type type, bool pack, const void* p, uint64_t rows, uint64_t cols, uint64_t ld, void* to,
                  uint64_t to_ld, Operand* out, hipStream_t s) {
    *out = {p, ld, cols, 0};
    if (!pack) return hipSuccess;
    const PackArgs a = {p, to, rows, ld, to_ld, rows * to_ld, (uint32_t)cols};
    *out = {to, to_ld, to_ld, a.plane};
    const dim3 grid((uint32_t)up(rows * (to_ld / 8), 256));
    if (type == HC_T_BF16) hipLaunchKernelGGL(pack_kernel<__bf16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(pack_kernel<_Float16>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// An fp32 operand in planes, scaled by its rows (and again by its columns into
// cols_out), or by its columns, whose largest elements are taken first if `find`.
hipError_t split_rows(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, void* to, uint64_t to_ld, float* most,
                      void* cols_out, const float* cols_most, Operand* out, hipStream_t s) {
    const SplitRowsArgs a = {{p, to, rows, ld, to_ld, rows * to_ld, (uint32_t)cols}, most, cols_out, cols_most};
    *out = {to, to_ld, to_ld, a.pack.plane};
    hipLaunchKernelGGL(split_rows_kernel, dim3((uint32_t)(rows < 65536 ? rows : 65536)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t split_columns(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, void* to, uint64_t to_ld,
                         float* most, bool find, Operand* out, hipStream_t s) {
    const PackArgs a = {p, to, rows, ld, to_ld, rows * to_ld, (uint32_t)cols};
    *out = {to, to_ld, to_ld, a.plane};
    if (find) {
        const uint64_t per = rows > 32 * 1024 ? up(rows, 1024) : 32;
        hipLaunchKernelGGL(most_kernel, dim3((uint32_t)up(cols, 512), (uint32_t)up(rows, per)), dim3(256), 0, s, a, per,
                           most);
    }
    hipLaunchKernelGGL(split_columns_kernel, dim3((uint32_t)up(rows * (to_ld / 8), 256)), dim3(256), 0, s, a, most);
    return hipGetLastError();
}

void set(Product* g, const Operand& p, const Operand& q) {
    g->p = p.p;
    g->p_ld = p.ld;
    g->p_cols = p.cols;
    g->p_plane = p.plane;
    g->q = q.p;
    g->q_ld = q.ld;
    g->q_cols = q.cols;
    g->q_plane = q.plane;
}

}  // namespace

size_t linear_bytes(const hc_linear_params& p, hc_type type) { return linear_layout(p, type).bytes; }

hipError_t launch_linear(const hc_linear_params& p, const Dropout& d, hc_type type, const void* x,
                         const void* w, const void* bias, const void* residual, void* y, void* z,
                         void* ws_, hipStream_t s) {
    const Layout L = linear_layout(p, type);
    char* ws = static_cast<char*>(ws_);
    const bool fp32 = type == HC_T_F32;
    const bool x_fits = !fp32 && tile_rows(x, p.k, p.x_ld), w_fits = !fp32 && tile_rows(w, p.k, p.w_ld);
    const bool in_tiles = L.pack_x || (x_fits && w_fits);
    Product g = {};
    g.passes = kOnePass;
    g.rows = p.m;
    g.cols = (uint32_t)p.n;
    g.inner = p.k;
    g.part = reinterpret_cast<float*>(ws + L.part);
    // results that the L2s cannot keep leave them to the operands: 16384 x 2048 x 512 (bf16)
    // 58 -> 46 us, 4096 x 4096 x 4096 126 -> 121 (dx 32768 x 768 x 768 56 -> 60: not there)
    const bool stream = p.m * p.n * (fp32 ? 4 : 2) > kStreamBytes;
    g.forward = {bias, residual, y, z, p.residual_ld, p.y_ld, p.z_ld, p.act, stream, d};
    Operand ox, ow;
    hipError_t e;
    if (fp32 && in_tiles) {
        float *x_most = reinterpret_cast<float*>(ws + L.row_most), *w_most = reinterpret_cast<float*>(ws + L.col_most);
        e = split_rows(x, p.m, p.k, p.x_ld, ws + L.x, L.k_ld, x_most, nullptr, nullptr, &ox, s);
        if (e == hipSuccess) e = split_rows(w, p.n, p.k, p.w_ld, ws + L.w, L.k_ld, w_most, nullptr, nullptr, &ow, s);
        if (e != hipSuccess) return e;
        g.passes = kTwoPlanes;
        g.p_most = x_most;
        g.q_most = w_most;
        set(&g, ox, ow);
        return product<FORWARD>(g, type, TILED, s);
    }
    e = packed(type, L.pack_x && !x_fits, x, p.m, p.k, p.x_ld, ws + L.x, L.k_ld, &ox, s);
    if (e == hipSuccess) e = packed(type, L.pack_w && !w_fits, w, p.n, p.k, p.w_ld, ws + L.w, L.k_ld, &ow, s);
    if (e != hipSuccess) return e;
    set(&g, ox, ow);
    const Way way = way_of(FORWARD, g, type, in_tiles);
    if (way != SPLIT) return product<FORWARD>(g, type, way, s);
    if (type == HC_T_F32) return split_forward<float>(g, s);
    if (type == HC_T_BF16) return split_forward<__bf16>(g, s);
    return split_forward<_Float16>(g, s);
}

size_t linear_grad_bytes(const hc_linear_params& p, hc_type type) { return grad_layout(p, type).bytes; }

hipError_t launch_linear_grad(const hc_linear_params& p, const Dropout& d, hc_type type,
                              const LinearGrad& q, void* ws_, hipStream_t s) {
    const Layout L = grad_layout(p, type);
    char* ws = static_cast<char*>(ws_);
    const bool fp32 = type == HC_T_F32, plain = p.act == HC_ACT_NONE && d.limit == 0;
    const bool x_fits = !fp32 && tile_rows(q.x, p.k, p.x_ld), w_fits = !fp32 && tile_rows(q.w, p.k, p.w_ld);
    // dx goes by w, dw by x and db by dy: what else is wanted changes none of them
    const bool dz_fits = p.n <= kMostTileLd;
    const bool dx_in_tiles = L.pack_w || (w_fits && dz_fits), dw_in_tiles = L.pack_x || (x_fits && dz_fits);
    const bool rest = !plain && q.dw && !fp32 && (q.g_type == HC_T_F32 || q.g_type == HC_T_I32);
    Product dx = {}, dw = {};
    dx.part = dw.part = reinterpret_cast<float*>(ws + L.part);
    dx.cols = dw.cols = (uint32_t)p.k;
    const bool planes = fp32 && L.pack_x;
    dx.passes = dw.passes = planes ? kTwoPlanes : kOnePass;
    dx.rows = dw.inner = p.m;
    dx.inner = dw.rows = p.n;
    if (rest) dw.passes = type == HC_T_BF16 ? kRestBf16 : kRestF16;
    const float unit = dz_unit(p.act, d);
    const Gradient gradient = {nullptr, 0, (uint32_t)q.g_type, q.accumulate ? 1u : 0u, p.fixed, unit};
    dw.gradient = gradient;
    if (p.m) {
        dx.gradient.out = q.dx;
        dx.gradient.unit = unit;
        dx.gradient.ld = p.dx_ld;
    }
    dw.gradient.out = q.dw;
    dw.gradient.ld = p.dw_ld;
    Gradient db = gradient;
    db.out = q.db;
    const Way dx_way = way_of(DX, dx, type, dx_in_tiles), dw_way = way_of(DW, dw, type, dw_in_tiles);
    // small products go in one launch, where nothing is packed for them; db too if dz is dy
    const bool dx_split = dx.gradient.out && dx_way == SPLIT, dw_split = q.dw && dw_way == SPLIT;
    const bool db_split = q.db && plain && p.m <= kSplitBias && p.m * p.n <= kSplitBiasElements;
    // dz is dy itself where nothing changes it and the products can take it
    const bool tiles = !planes && ((dx.gradient.out && dx_way == TILED) || (q.dw && dw_way == TILED));
    const bool dy_fits = plain && (!tiles || tile_rows(q.dy, p.n, p.y_ld));
    const bool dz = !dy_fits && (q.dx || q.dw), db_pass = q.db && !db_split;
    hipError_t e = hipSuccess;
    Operand oz = {q.dy, p.y_ld, p.n, 0};
    float* col_most = reinterpret_cast<float*>(ws + L.col_most);
    if (planes && p.m) {
        e = launch_fill_u32(reinterpret_cast<uint32_t*>(col_most), L.most, 0, s);
        if (e != hipSuccess) return e;
    }
    if ((dz || db_pass || (planes && q.dw)) && p.m) {
        DzArgs a = {};
        a.dy = q.dy;
        a.z = q.z;
        a.dy_ld = p.y_ld;
        a.z_ld = p.z_ld;
        a.m = p.m;
        a.n = (uint32_t)p.n;
        a.groups = (uint32_t)(L.n_ld / 8);
        a.act = p.act;
        a.per = (uint32_t)L.per;
        a.width = L.width;
        a.drop = d;
        if (dz) {
            a.dz.out = ws + L.dz;
            a.dz.out_ld = L.n_ld;
            a.dz.plane = p.m * L.n_ld;
            a.per_unit = 1.0f / unit;
            a.planes = !rest ? 1 : type == HC_T_BF16 ? 3 : 2;
            oz = {a.dz.out, L.n_ld, L.n_ld, a.dz.plane};
        }
        a.most = planes && q.dw ? col_most : nullptr;
        a.part = db_pass ? reinterpret_cast<float*>(ws + L.bias) : nullptr;
        a.db = db;
        const dim3 grid((uint32_t)up(a.groups, L.width), (uint32_t)L.blocks);
        if (fp32) hipLaunchKernelGGL(dz_kernel<float>, grid, dim3(256), 0, s, a);
        else if (type == HC_T_BF16) hipLaunchKernelGGL(dz_kernel<__bf16>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(dz_kernel<_Float16>, grid, dim3(256), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (db_pass && L.blocks != 1) {
        hipLaunchKernelGGL(bias_kernel, dim3((uint32_t)up(p.n, 16)), dim3(1024), 0, s,
                           reinterpret_cast<const float*>(ws + L.bias), (uint32_t)L.blocks, (uint32_t)p.n, db);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (dx_split || dw_split || db_split) {
        SplitGrad g = {};
        if (dx_split) {
            g.dx = dx;
            set(&g.dx, oz, {q.w, p.w_ld, p.k, 0});
        }
        if (dw_split) {
            g.dw = dw;
            set(&g.dw, oz, {q.x, p.x_ld, p.k, 0});
        }
        if (db_split) {
            g.dy = p.m ? q.dy : ws;  // not read without rows
            g.dy_ld = p.y_ld;
            g.m = p.m;
            g.n = (uint32_t)p.n;
            g.db = db;
        }
        e = fp32 ? split_grad<float>(g, s) : type == HC_T_BF16 ? split_grad<__bf16>(g, s) : split_grad<_Float16>(g, s);
        if (e != hipSuccess) return e;
    }
    if (planes && p.m) {
        float* row_most = reinterpret_cast<float*>(ws + L.row_most);
        Operand by_rows, by_cols, ox, ow;
        by_cols = {ws + L.dz_cols, L.n_ld, L.n_ld, p.m * L.n_ld};
        if (q.dx)
            e = split_rows(oz.p, p.m, p.n, oz.ld, ws + L.dz_rows, L.n_ld, row_most,
                           q.dw ? ws + L.dz_cols : nullptr, col_most, &by_rows, s);
        else if (q.dw)
            e = split_columns(oz.p, p.m, p.n, oz.ld, ws + L.dz_cols, L.n_ld, col_most, false, &by_cols, s);
        if (e != hipSuccess) return e;
        if (q.dx) {
            e = split_columns(q.w, p.n, p.k, p.w_ld, ws + L.w, L.k_ld, col_most + L.w_most, true, &ow, s);
            if (e != hipSuccess) return e;
            set(&dx, by_rows, ow);
            dx.p_most = row_most;
            dx.q_most = col_most + L.w_most;
            e = product<DX>(dx, type, TILED, s);
            if (e != hipSuccess) return e;
        }
        if (q.dw) {
            e = split_columns(q.x, p.m, p.k, p.x_ld, ws + L.x, L.k_ld, col_most + L.x_most, true, &ox, s);
            if (e != hipSuccess) return e;
            set(&dw, by_cols, ox);
            dw.p_most = col_most;
            dw.q_most = col_most + L.x_most;
            e = product<DW>(dw, type, TILED, s);
        }
        return e;
    }
    if (dx.gradient.out && !dx_split) {
        Operand ow;
        e = packed(type, dx_way == TILED && !w_fits, q.w, p.n, p.k, p.w_ld, ws + L.w, L.k_ld, &ow, s);
        if (e != hipSuccess) return e;
        set(&dx, oz, ow);
        e = product<DX>(dx, type, dx_way, s);
        if (e != hipSuccess) return e;
    }
    if (q.dw && !dw_split) {
        Operand ox;
        e = packed(type, dw_way == TILED && !x_fits, q.x, p.m, p.k, p.x_ld, ws + L.x, L.k_ld, &ox, s);
        if (e != hipSuccess) return e;
        set(&dw, oz, ox);
        return product<DW>(dw, type, dw_way, s);
    }
    return hipSuccess;
}

}  // namespace hc
