// hc_embed.hip -- embedding lookup with scaling, and its gradient by sorted
// token ids (include/hc_train.h).
//
// The gradient of out[i] = scale * W[t_i] is dW[v] = scale * sum over t_i = v of
// dOut[i].  Sorting the pairs (t_i, i) by id, stably, puts the terms of one row
// next to each other in token order.  The sorted list is cut into chunks of
// equal length whatever the ids are, so a frequent id is shared by many
// workgroups: a run that lies inside one chunk is summed and stored at once,
// a run that crosses chunks leaves one partial sum per chunk and a second
// launch joins those in chunk order.  Every order is fixed by the ids alone.
#include "hc_device.h"
#include "hc_internal.h"
#include "hc_train_internal.h"

namespace hc {

namespace {

constexpr int kBlock = 256;

// ---- element types ---------------------------------------------------------------

// 16 bytes at the alignment of their elements (global memory takes wide
// accesses at any element alignment on gfx950)
template <typename T> struct Wide;
template <> struct Wide<float> {
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Wide<__bf16> {
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
};
template <> struct Wide<_Float16> {
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
};
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

template <typename T> __device__ __forceinline__ void unpack(v4u w, float* v) {
    typedef T TV __attribute__((ext_vector_type(kVec<T>)));
    const TV t = __builtin_bit_cast(TV, w);
#pragma unroll
    for (int j = 0; j < kVec<T>; j++) v[j] = (float)t[j];
}

// nv (1 .. kVec<T>) elements at p, the others 0
template <typename T> __device__ __forceinline__ void load_vec(const T* p, int nv, float* v) {
    if (nv == kVec<T>) {
        const typename Wide<T>::V w = *reinterpret_cast<const typename Wide<T>::V*>(p);
        unpack<T>((v4u)w, v);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<T>; j++) v[j] = j < nv ? (float)p[j] : 0.0f;
    }
}

// ---- lookup ----------------------------------------------------------------------

template <typename ID>
__device__ __forceinline__ bool valid_id(ID id, uint32_t vocab) {
    return id >= 0 && (uint64_t)id < vocab;
}

// A group of g lanes (a power of two up to a wave) takes one token's row, or 64
// lanes' worth of columns of it, one 16-byte vector a lane.
template <typename T, typename ID>
__global__ __launch_bounds__(kBlock) void embed_kernel(const T* __restrict__ table,
                                                       const ID* __restrict__ ids,
                                                       T* __restrict__ out, uint64_t units,
                                                       uint32_t vocab, uint32_t dim,
                                                       uint64_t table_ld, uint64_t out_ld,
                                                       uint32_t log2g, uint32_t slabs,
                                                       float scale) {
    constexpr int VEC = kVec<T>;
    const uint64_t first = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) >> log2g;
    const uint64_t step = ((uint64_t)gridDim.x * kBlock) >> log2g;
    for (uint64_t unit = first; unit < units; unit += step) {
        const uint64_t i = unit / slabs;
        const uint32_t slab = (uint32_t)(unit - i * slabs);
        const uint32_t col = ((slab << log2g) + (threadIdx.x & ((1u << log2g) - 1u))) * VEC;
        if (col >= dim) continue;
        const int nv = (int)min((uint32_t)VEC, dim - col);
        const ID id = ids[i];
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; j++) v[j] = 0.0f;
        if (valid_id(id, vocab)) {
            load_vec<T>(table + (uint64_t)id * table_ld + col, nv, v);
#pragma unroll
            for (int j = 0; j < VEC; j++) v[j] *= scale;
        }
        T* q = out + i * out_ld + col;
        if (nv == VEC) {
            typedef T TV __attribute__((ext_vector_type(VEC)));
            TV t;
#pragma unroll
            for (int j = 0; j < VEC; j++) t[j] = (T)v[j];
            *reinterpret_cast<typename Wide<T>::V*>(q) = __builtin_bit_cast(v4u, t);
        } else {
            for (int j = 0; j < nv; j++) q[j] = (T)v[j];
        }
    }
}

// Workgroups are at most this many: what is past them is taken in a stride.
constexpr uint64_t kMaxGroups = 1ull << 22;

// Lanes of a group: enough 16-byte vectors for a row, at most a wave.
uint32_t group_log2(uint64_t vectors) {
    uint32_t g = 0;
    while (g < 6 && (1ull << g) < vectors) g++;
    return g;
}

template <typename T, typename ID>
hipError_t embed_typed(const hc_embed_params& p, const void* table, const void* ids, void* out,
                       hipStream_t s) {
    const uint64_t vectors = (p.dim + kVec<T> - 1) / kVec<T>;
    const uint32_t log2g = group_log2(vectors);
    const uint64_t slabs = (vectors + (1ull << log2g) - 1) >> log2g;
    const uint64_t units = p.count * slabs;
    const uint64_t per_block = kBlock >> log2g;
    const uint64_t blocks = (units + per_block - 1) / per_block;
    hipLaunchKernelGGL((embed_kernel<T, ID>), dim3((uint32_t)(blocks < kMaxGroups ? blocks : kMaxGroups)), dim3(kBlock), 0, s,
                       static_cast<const T*>(table), static_cast<const ID*>(ids),
                       static_cast<T*>(out), units, (uint32_t)p.vocab, (uint32_t)p.dim, p.table_ld,
                       p.x_ld, log2g, (uint32_t)slabs, p.scale);
    return hipGetLastError();
}

// ---- gradient: sort --------------------------------------------------------------

// Stable radix sort of the pairs (id, token) by id in digits of up to 9 bits:
// per pass every workgroup counts its tile's digits, the counts are scanned per
// digit over the workgroups, and every workgroup moves its tile's pairs to
// their places.  Ids that add nothing get the key `vocab` and end up last.
constexpr int kItems = 8;
constexpr uint32_t kTile = kBlock * kItems;
constexpr uint32_t kMaxBins = 512;

struct Pair {
    uint32_t key, pos;
};

template <typename ID>
__device__ __forceinline__ uint32_t key_of(ID id, uint32_t vocab, int64_t padding) {
    return valid_id(id, vocab) && (int64_t)id != padding ? (uint32_t)id : vocab;
}

// Where a pass reads its pairs from: the ids themselves, or the last pass's.
template <typename ID> struct FromIds {
    const ID* ids;
    uint32_t vocab;
    int64_t padding;
    __device__ Pair get(uint32_t i) const { return {key_of(ids[i], vocab, padding), i}; }
};
struct FromPairs {
    const Pair* pairs;
    __device__ Pair get(uint32_t i) const { return pairs[i]; }
};

template <typename SRC>
__global__ __launch_bounds__(kBlock) void digit_count_kernel(SRC src, uint32_t count,
                                                             uint32_t shift, uint32_t bins,
                                                             uint32_t* __restrict__ hist) {
    __shared__ uint32_t s_cnt[kMaxBins];
    for (uint32_t b = threadIdx.x; b < bins; b += kBlock) s_cnt[b] = 0;
    lds_barrier();
    const uint32_t base = blockIdx.x * kTile;
#pragma unroll
    for (int it = 0; it < kItems; it++) {
        const uint32_t i = base + it * kBlock + threadIdx.x;
        if (i < count) atomicAdd(&s_cnt[(src.get(i).key >> shift) & (bins - 1u)], 1u);
    }
    lds_barrier();
    for (uint32_t b = threadIdx.x; b < bins; b += kBlock)
        hist[(uint64_t)b * gridDim.x + blockIdx.x] = s_cnt[b];
}

// One wave a digit: hist[digit][workgroup] becomes the count in earlier
// workgroups, total[digit] the count in all.
__global__ __launch_bounds__(kBlock) void digit_scan_kernel(uint32_t* __restrict__ hist,
                                                            uint32_t* __restrict__ total,
                                                            uint32_t bins, uint32_t groups) {
    const uint32_t bin = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (bin >= bins) return;
    const uint32_t lane = lane_id();
    uint32_t* h = hist + (uint64_t)bin * groups;
    uint32_t before = 0;
    for (uint32_t g0 = 0; g0 < groups; g0 += 64) {
        const uint32_t g = g0 + lane;
        const uint32_t v = g < groups ? h[g] : 0u;
        uint32_t x = v;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t y = __shfl_up(x, d);
            if (lane >= (uint32_t)d) x += y;
        }
        if (g < groups) h[g] = before + x - v;
        before += __shfl(x, 63);
    }
    if (lane == 0) total[bin] = before;
}

// A wave takes its pairs in order, 64 at a time; equal digits among the lanes
// are found with one ballot per digit bit, and the wave's own running counts in
// LDS give every pair its rank, so equal keys keep their order.
template <typename SRC>
__global__ __launch_bounds__(kBlock) void digit_move_kernel(SRC src, uint32_t count,
                                                            uint32_t shift, uint32_t log2bins,
                                                            const uint32_t* __restrict__ hist,
                                                            const uint32_t* __restrict__ total,
                                                            Pair* __restrict__ out) {
    constexpr uint32_t kWaves = kBlock / 64;
    __shared__ uint32_t s_cnt[kWaves][kMaxBins];
    __shared__ uint32_t s_tmp[kWaves];
    const uint32_t bins = 1u << log2bins;
    const uint32_t wave = threadIdx.x >> 6, lane = lane_id();
    for (uint32_t b = threadIdx.x; b < kWaves * kMaxBins; b += kBlock)
        (&s_cnt[0][0])[b] = 0;
    lds_barrier();
    Pair p[kItems];
    uint32_t rank[kItems];
    const uint32_t base = blockIdx.x * kTile + wave * (64 * kItems) + lane;
    volatile uint32_t* cnt = s_cnt[wave];
#pragma unroll
    for (int it = 0; it < kItems; it++) {
        const uint32_t i = base + it * 64;
        const bool live = i < count;
        p[it] = live ? src.get(i) : Pair{0, 0};
        const uint32_t digit = (p[it].key >> shift) & (bins - 1u);
        uint64_t same = __ballot(live);
        for (uint32_t b = 0; b < log2bins; b++) {
            const bool bit = (digit >> b) & 1u;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        const uint32_t before = lanes_below(same);
        const uint32_t seen = live ? cnt[digit] : 0u;
        rank[it] = seen + before;
        __builtin_amdgcn_wave_barrier();
        if (live && before == 0) cnt[digit] = seen + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    lds_barrier();
    // per digit: where this workgroup's pairs of earlier waves end
    uint32_t t[2], first = 0;
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const uint32_t b = threadIdx.x * 2 + j;
        t[j] = b < bins ? total[b] : 0u;
    }
    uint32_t all;
    first = block_exclusive_scan(t[0] + t[1], s_tmp, &all);
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const uint32_t b = threadIdx.x * 2 + j;
        if (b < bins) {
            uint32_t at = first + (j ? t[0] : 0u) + hist[(uint64_t)b * gridDim.x + blockIdx.x];
            for (uint32_t w = 0; w < kWaves; w++) {
                const uint32_t c = s_cnt[w][b];
                s_cnt[w][b] = at;
                at += c;
            }
        }
    }
    lds_barrier();
#pragma unroll
    for (int it = 0; it < kItems; it++) {
        const uint32_t i = base + it * 64;
        if (i < count) out[s_cnt[wave][(p[it].key >> shift) & (bins - 1u)] + rank[it]] = p[it];
    }
}

// ---- gradient: rows --------------------------------------------------------------

// First positions of runs per chunk of the sorted pairs.
__global__ __launch_bounds__(kBlock) void head_count_kernel(const Pair* __restrict__ pairs,
                                                            uint32_t count, uint32_t chunk,
                                                            uint32_t chunks, uint32_t vocab,
                                                            uint32_t* __restrict__ heads) {
    const uint32_t c = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (c >= chunks) return;
    const uint32_t lane = lane_id();
    const uint32_t i = c * chunk + lane;
    bool head = false;
    if (lane < chunk && i < count) {
        const uint32_t key = pairs[i].key;
        head = key != vocab && (i == 0 || pairs[i - 1].key != key);
    }
    const uint64_t m = __ballot(head);
    if (lane == 0) heads[c] = (uint32_t)__popcll(m);
}

// heads[c] becomes the number of runs that begin before chunk c; *touched the
// number of runs.
__global__ __launch_bounds__(1024) void head_scan_kernel(uint32_t* __restrict__ heads,
                                                         uint32_t chunks,
                                                         uint32_t* __restrict__ touched) {
    __shared__ uint32_t s_tmp[16];
    uint32_t before = 0;
    for (uint32_t c0 = 0; c0 < chunks; c0 += 4096) {
        uint32_t v[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t c = c0 + threadIdx.x * 4 + j;
            v[j] = c < chunks ? heads[c] : 0u;
            sum += v[j];
        }
        uint32_t total;
        uint32_t at = before + block_exclusive_scan(sum, s_tmp, &total);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t c = c0 + threadIdx.x * 4 + j;
            if (c < chunks) heads[c] = at;
            at += v[j];
        }
        before += total;
    }
    if (threadIdx.x == 0) *touched = before;
}

// ---- gradient: sums --------------------------------------------------------------

// How an output type sums: fp32, or 64-bit whole numbers of the fixed point.
template <typename TO> struct Sum {
    typedef float A;
    __device__ static A term(float v, float scale, float) { return v * scale; }
    __device__ static TO narrow(A a) { return (TO)a; }
    __device__ static A widen(TO o) { return (float)o; }
};
template <> struct Sum<int32_t> {
    typedef int64_t A;
    __device__ static A term(float v, float scale, float fixed) {
        const float q = rintf((v * scale) * fixed);
        if (!(q == q)) return 0;
        // the largest fp32 below 2^31 is a whole number, so only the bounds clip
        return q >= 2147483648.0f ? 2147483647 : q <= -2147483648.0f ? -2147483647 : (A)(int32_t)q;
    }
    __device__ static int32_t narrow(A a) {
        return a > 2147483647 ? 2147483647 : a < -2147483647 ? -2147483647 : (int32_t)a;
    }
    __device__ static A widen(int32_t o) { return o; }
};

template <typename TO, int VEC>
__device__ __forceinline__ void store_sum(TO* p, int nv, const typename Sum<TO>::A* acc,
                                          bool accumulate) {
    TO o[VEC];
#pragma unroll
    for (int j = 0; j < VEC; j++)
        o[j] = Sum<TO>::narrow(accumulate && j < nv ? acc[j] + Sum<TO>::widen(p[j]) : acc[j]);
    if (nv == VEC) {
        typedef TO TV __attribute__((ext_vector_type(VEC), aligned(sizeof(TO))));
        TV t;
#pragma unroll
        for (int j = 0; j < VEC; j++) t[j] = o[j];
        *reinterpret_cast<TV*>(p) = t;
    } else {
        for (int j = 0; j < nv; j++) p[j] = o[j];
    }
}

struct SumArgs {
    const Pair* pairs;
    uint32_t count, chunk, chunks, vocab, dim;
    uint64_t x_ld, dst_ld;
    uint32_t log2g, slabs;
    float scale, fixed;
    bool accumulate;
    // rows
    uint32_t* rows;
    const uint32_t* heads;
    uint64_t cap;
    // runs that cross chunks: (chunk they begin in, rank), and their partial
    // sums, two of dim elements a chunk: of the run it begins with, of the run
    // it ends with
    uint32_t* crossing_count;
    uint2* crossing;
    void* partial;
};

// One chunk's columns of one slab (a group of lanes).
template <typename TI, typename TO, bool ROWS>
__device__ __forceinline__ void sum_chunk(const SumArgs& a, const TI* __restrict__ x,
                                          TO* __restrict__ dst, uint64_t unit) {
    typedef typename Sum<TO>::A A;
    constexpr int VEC = kVec<TI>;
    constexpr int U = 4;
    const uint32_t c = (uint32_t)(unit / a.slabs);
    const uint32_t slab = (uint32_t)(unit - (uint64_t)c * a.slabs);
    const uint32_t col = ((slab << a.log2g) + (threadIdx.x & ((1u << a.log2g) - 1u))) * VEC;
    if (col >= a.dim) return;
    const int nv = (int)min((uint32_t)VEC, a.dim - col);
    const uint32_t start = c * a.chunk, end = min(start + a.chunk, a.count);
    uint32_t cur = a.pairs[start].key;
    if (cur == a.vocab) return;
    bool begins = start == 0 || a.pairs[start - 1].key != cur;
    uint32_t rank = 0;
    if constexpr (ROWS) rank = a.heads[c] - (begins ? 0u : 1u);
    A* partial = static_cast<A*>(a.partial) + (uint64_t)c * 2 * a.dim + col;
    A acc[VEC];
#pragma unroll
    for (int j = 0; j < VEC; j++) acc[j] = 0;

    auto flush = [&](bool finishes) {
        if (begins && finishes) {
            if constexpr (ROWS) {
                if (rank < a.cap) {
                    if (col == 0) a.rows[rank] = cur;
                    store_sum<TO, VEC>(dst + (uint64_t)rank * a.dst_ld + col, nv, acc, false);
                }
            } else {
                store_sum<TO, VEC>(dst + (uint64_t)cur * a.dst_ld + col, nv, acc, a.accumulate);
            }
        } else {
            A* q = partial + (begins ? a.dim : 0u);
            for (int j = 0; j < nv; j++) q[j] = acc[j];
            if (begins && col == 0) a.crossing[atomicAdd(a.crossing_count, 1u)] = make_uint2(c, rank);
        }
    };

    for (uint32_t i = start; i < end; i += U) {
        Pair p[U];
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; u++) p[u] = i + u < end ? a.pairs[i + u] : Pair{a.vocab, 0};
#pragma unroll
        for (int u = 0; u < U; u++)
            if (p[u].key != a.vocab) load_vec<TI>(x + (uint64_t)p[u].pos * a.x_ld + col, nv, v[u]);
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (p[u].key == a.vocab) break;
            if (p[u].key != cur) {
                flush(true);
                cur = p[u].key;
                begins = true;
                rank++;
#pragma unroll
                for (int j = 0; j < VEC; j++) acc[j] = 0;
            }
#pragma unroll
            for (int j = 0; j < VEC; j++) acc[j] += Sum<TO>::term(v[u][j], a.scale, a.fixed);
        }
    }
    flush(end == a.count || a.pairs[end].key != cur);
}

template <typename TI, typename TO, bool ROWS>
__global__ __launch_bounds__(kBlock) void segment_sum_kernel(SumArgs a, const TI* __restrict__ x,
                                                             TO* __restrict__ dst) {
    const uint64_t units = (uint64_t)a.chunks * a.slabs;
    const uint64_t step = ((uint64_t)gridDim.x * kBlock) >> a.log2g;
    for (uint64_t unit = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) >> a.log2g; unit < units;
         unit += step)
        sum_chunk<TI, TO, ROWS>(a, x, dst, unit);
}

// Joins the partial sums of the runs that cross chunks: a workgroup takes one
// run's columns, its groups of lanes a contiguous share of the run's chunks
// each, in order, and the groups' sums are added in order.
constexpr int kJoinBlock = 512;

template <typename TI, typename TO, bool ROWS>
__global__ __launch_bounds__(kJoinBlock) void segment_join_kernel(SumArgs a,
                                                                  TO* __restrict__ dst) {
    typedef typename Sum<TO>::A A;
    constexpr int VEC = kVec<TI>;
    __shared__ A s_sum[kJoinBlock * VEC];
    __shared__ uint32_t s_more;
    const uint32_t lanes = 1u << a.log2g, groups = kJoinBlock >> a.log2g;
    const uint32_t group = threadIdx.x >> a.log2g, li = threadIdx.x & (lanes - 1u);
    const uint32_t col = ((blockIdx.y << a.log2g) + li) * VEC;
    const int nv = col < a.dim ? (int)min((uint32_t)VEC, a.dim - col) : 0;
    const uint32_t runs = *a.crossing_count;
    for (uint32_t r = blockIdx.x; r < runs; r += gridDim.x) {
        const uint2 run = a.crossing[r];
        const uint32_t c = run.x;
        const uint32_t key = a.pairs[(uint64_t)(c + 1) * a.chunk].key;  // the run goes on there
        // chunks after c that the run reaches: those that begin with its key
        uint32_t n = 0;
        for (;;) {
            if (threadIdx.x == 0) s_more = 0;
            lds_barrier();
            const uint32_t d = c + 1 + n + threadIdx.x;
            const bool in = d < a.chunks && a.pairs[(uint64_t)d * a.chunk].key == key;
            const uint64_t m = __ballot(in);
            if (lane_id() == 0) atomicAdd(&s_more, (uint32_t)__popcll(m));
            lds_barrier();
            const uint32_t more = s_more;
            lds_barrier();
            n += more;
            if (more < (uint32_t)kJoinBlock) break;
        }
        const uint32_t items = n + 1, per = (items + groups - 1) / groups;
        const uint32_t lo = min(group * per, items), hi = min(lo + per, items);
        A acc[VEC];
#pragma unroll
        for (int j = 0; j < VEC; j++) acc[j] = 0;
        const A* base = static_cast<const A*>(a.partial) + (uint64_t)c * 2 * a.dim + col;
#pragma unroll 4
        for (uint32_t k = lo; k < hi; k++) {
            // item 0: what chunk c ends with; item k: what chunk c + k begins with
            const A* q = base + (k == 0 ? (uint64_t)a.dim : (uint64_t)k * 2 * a.dim);
#pragma unroll
            for (int j = 0; j < VEC; j++)
                if (j < nv) acc[j] += q[j];
        }
#pragma unroll
        for (int j = 0; j < VEC; j++) s_sum[threadIdx.x * VEC + j] = acc[j];
        lds_barrier();
        if (group == 0 && nv > 0) {
            const uint32_t used = (items + per - 1) / per;
            for (uint32_t g = 1; g < used; g++)
#pragma unroll
                for (int j = 0; j < VEC; j++) acc[j] += s_sum[((g << a.log2g) + li) * VEC + j];
            if constexpr (ROWS) {
                if (run.y < a.cap) {
                    if (col == 0) a.rows[run.y] = key;
                    store_sum<TO, VEC>(dst + (uint64_t)run.y * a.dst_ld + col, nv, acc, false);
                }
            } else {
                store_sum<TO, VEC>(dst + (uint64_t)key * a.dst_ld + col, nv, acc, a.accumulate);
            }
        }
        lds_barrier();
    }
}

// ---- gradient: zeros -------------------------------------------------------------

// rows x row_bytes zeros at a stride of ld_bytes (one row where the rows lie
// back to back), 16 bytes a lane where everything is 16-byte aligned.
template <typename V>
__global__ __launch_bounds__(kBlock) void zero_rows_kernel(char* __restrict__ dst, uint64_t rows,
                                                           uint64_t row_bytes, uint64_t ld_bytes) {
    const uint64_t per = row_bytes / sizeof(V);
    const V zero = {};
    if (rows == 1) {
        for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < per;
             i += (uint64_t)gridDim.x * kBlock)
            reinterpret_cast<V*>(dst)[i] = zero;
        return;
    }
    for (uint64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (uint64_t i = threadIdx.x; i < per; i += kBlock)
            reinterpret_cast<V*>(dst + r * ld_bytes)[i] = zero;
}

__global__ void clear_word_kernel(uint32_t* a, uint32_t* b) {
    if (a) *a = 0;
    if (b) *b = 0;
}

// ---- layout and launches ---------------------------------------------------------

// Pairs per chunk: 64, or fewer (down to 8) while that leaves under 4096 waves'
// worth of work for the sums.
uint32_t chunk_for(const hc_embed_params& p) {
    const uint64_t slabs = (p.dim + 255) / 256;
    uint32_t chunk = 64;
    while (chunk > 8 && p.count * slabs / chunk < 4096) chunk /= 2;
    return chunk;
}

struct GradLayout {
    uint32_t chunk, chunks, groups;
    size_t pairs[2], hist, total, heads, crossing_count, crossing, partial, bytes;
};

GradLayout grad_layout(const hc_embed_params& p) {
    GradLayout L;
    L.chunk = chunk_for(p);
    L.chunks = (uint32_t)((p.count + L.chunk - 1) / L.chunk);
    L.groups = (uint32_t)((p.count + kTile - 1) / kTile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    L.pairs[0] = take(p.count * sizeof(Pair));
    L.pairs[1] = take(p.count * sizeof(Pair));
    L.hist = take((size_t)L.groups * kMaxBins * 4);
    L.total = take(kMaxBins * 4);
    L.heads = take((size_t)L.chunks * 4);
    L.crossing_count = take(4);
    L.crossing = take((size_t)L.chunks * 8);
    L.partial = take((size_t)L.chunks * 2 * p.dim * 8);
    L.bytes = at;
    return L;
}

hipError_t zero_rows(void* dst, uint64_t rows, uint64_t row_bytes, uint64_t ld_bytes, int cus,
                     hipStream_t s) {
    if (ld_bytes == row_bytes) {
        row_bytes *= rows;
        rows = 1;
    }
    const uint64_t want = rows == 1 ? (row_bytes / 16 + kBlock - 1) / kBlock : rows;
    const uint32_t grid = (uint32_t)(want < 1 ? 1 : want < (uint64_t)cus * 16 ? want : cus * 16);
    const uintptr_t al = reinterpret_cast<uintptr_t>(dst) | row_bytes | (rows > 1 ? ld_bytes : 0);
    if (al % 16 == 0)
        hipLaunchKernelGGL(zero_rows_kernel<v4u>, dim3(grid), dim3(kBlock), 0, s,
                           static_cast<char*>(dst), rows, row_bytes, ld_bytes);
    else if (al % 4 == 0)
        hipLaunchKernelGGL(zero_rows_kernel<uint32_t>, dim3(grid), dim3(kBlock), 0, s,
                           static_cast<char*>(dst), rows, row_bytes, ld_bytes);
    else
        hipLaunchKernelGGL(zero_rows_kernel<uint16_t>, dim3(grid), dim3(kBlock), 0, s,
                           static_cast<char*>(dst), rows, row_bytes, ld_bytes);
    return hipGetLastError();
}

template <typename SRC>
hipError_t radix_pass(const SRC& src, uint32_t count, uint32_t shift, uint32_t log2bins,
                      const GradLayout& L, char* ws, Pair* out, hipStream_t s) {
    const uint32_t bins = 1u << log2bins;
    uint32_t* hist = reinterpret_cast<uint32_t*>(ws + L.hist);
    uint32_t* total = reinterpret_cast<uint32_t*>(ws + L.total);
    hipLaunchKernelGGL(digit_count_kernel<SRC>, dim3(L.groups), dim3(kBlock), 0, s, src, count,
                       shift, bins, hist);
    hipLaunchKernelGGL(digit_scan_kernel, dim3((bins + kBlock / 64 - 1) / (kBlock / 64)),
                       dim3(kBlock), 0, s, hist, total, bins, L.groups);
    hipLaunchKernelGGL(digit_move_kernel<SRC>, dim3(L.groups), dim3(kBlock), 0, s, src, count,
                       shift, log2bins, hist, total, out);
    return hipGetLastError();
}

template <typename ID>
hipError_t sort_ids(const hc_embed_params& p, const void* ids, const GradLayout& L, char* ws,
                    const Pair** sorted, hipStream_t s) {
    uint32_t bits = 1;
    while ((p.vocab >> bits) != 0) bits++;
    const uint32_t passes = (bits + 8) / 9, width = (bits + passes - 1) / passes;
    const uint32_t count = (uint32_t)p.count;
    Pair* buf[2] = {reinterpret_cast<Pair*>(ws + L.pairs[0]),
                    reinterpret_cast<Pair*>(ws + L.pairs[1])};
    for (uint32_t k = 0; k < passes; k++) {
        hipError_t e;
        if (k == 0)
            e = radix_pass(FromIds<ID>{static_cast<const ID*>(ids), (uint32_t)p.vocab, p.padding},
                           count, 0, width, L, ws, buf[0], s);
        else
            e = radix_pass(FromPairs{buf[(k - 1) & 1]}, count, k * width, width, L, ws, buf[k & 1], s);
        if (e != hipSuccess) return e;
    }
    *sorted = buf[(passes - 1) & 1];
    return hipSuccess;
}

template <typename TI, typename TO, bool ROWS>
hipError_t sum_typed(SumArgs a, const void* x, void* dst, int cus, hipStream_t s) {
    const uint64_t vectors = (a.dim + kVec<TI> - 1) / kVec<TI>;
    a.log2g = group_log2(vectors);
    a.slabs = (uint32_t)((vectors + (1ull << a.log2g) - 1) >> a.log2g);
    const uint64_t units = (uint64_t)a.chunks * a.slabs, per_block = kBlock >> a.log2g;
    const uint64_t blocks = (units + per_block - 1) / per_block;
    hipLaunchKernelGGL((segment_sum_kernel<TI, TO, ROWS>),
                       dim3((uint32_t)(blocks < kMaxGroups ? blocks : kMaxGroups)), dim3(kBlock), 0, s, a, static_cast<const TI*>(x), static_cast<TO*>(dst));
    const uint32_t grid = a.chunks < (uint32_t)cus ? a.chunks : (uint32_t)cus;
    hipLaunchKernelGGL((segment_join_kernel<TI, TO, ROWS>), dim3(grid, a.slabs), dim3(kJoinBlock),
                       0, s, a, static_cast<TO*>(dst));
    return hipGetLastError();
}

template <typename TI, bool ROWS>
hipError_t sum_to(const SumArgs& a, hc_type g_type, const void* x, void* dst, int cus,
                  hipStream_t s) {
    switch (g_type) {
        case HC_T_I32: return sum_typed<TI, int32_t, ROWS>(a, x, dst, cus, s);
        case HC_T_F32: return sum_typed<TI, float, ROWS>(a, x, dst, cus, s);
        case HC_T_BF16: return sum_typed<TI, __bf16, ROWS>(a, x, dst, cus, s);
        default: return sum_typed<TI, _Float16, ROWS>(a, x, dst, cus, s);
    }
}

template <bool ROWS>
hipError_t sum_from(const SumArgs& a, hc_type x_type, hc_type g_type, const void* x, void* dst,
                    int cus, hipStream_t s) {
    switch (x_type) {
        case HC_T_F32: return sum_to<float, ROWS>(a, g_type, x, dst, cus, s);
        case HC_T_BF16: return sum_to<__bf16, ROWS>(a, g_type, x, dst, cus, s);
        default: return sum_to<_Float16, ROWS>(a, g_type, x, dst, cus, s);
    }
}

}  // namespace

hipError_t launch_embed(const hc_embed_params& p, hc_type type, const void* table, const void* ids,
                        void* out, hipStream_t s) {
    const bool wide = p.id_bits == 64;
    switch (type) {
        case HC_T_F32:
            return wide ? embed_typed<float, int64_t>(p, table, ids, out, s)
                        : embed_typed<float, int32_t>(p, table, ids, out, s);
        case HC_T_BF16:
            return wide ? embed_typed<__bf16, int64_t>(p, table, ids, out, s)
                        : embed_typed<__bf16, int32_t>(p, table, ids, out, s);
        default:
            return wide ? embed_typed<_Float16, int64_t>(p, table, ids, out, s)
                        : embed_typed<_Float16, int32_t>(p, table, ids, out, s);
    }
}

size_t embed_grad_bytes(const hc_embed_params& p) { return grad_layout(p).bytes; }

hipError_t launch_embed_grad(const hc_embed_params& p, hc_type x_type, const void* dout,
                             const void* ids, const EmbedGradOut& out, void* ws_, hipStream_t s) {
    DeviceInfo di;
    hipError_t e = device_info(&di);
    if (e != hipSuccess) return e;
    char* ws = static_cast<char*>(ws_);
    const GradLayout L = grad_layout(p);
    uint32_t* crossing_count = reinterpret_cast<uint32_t*>(ws + L.crossing_count);
    const bool rows = out.by_rows;
    if (!rows && !out.accumulate) {
        const uint64_t size = out.type == HC_T_I32 || out.type == HC_T_F32 ? 4 : 2;
        e = zero_rows(out.dst, p.vocab, p.dim * size, p.table_ld * size, di.cus, s);
        if (e != hipSuccess) return e;
    }
    if (p.count == 0) {
        if (!rows) return hipSuccess;
        hipLaunchKernelGGL(clear_word_kernel, dim3(1), dim3(1), 0, s, out.touched,
                           static_cast<uint32_t*>(nullptr));
        return hipGetLastError();
    }
    hipLaunchKernelGGL(clear_word_kernel, dim3(1), dim3(1), 0, s, crossing_count,
                       static_cast<uint32_t*>(nullptr));
    SumArgs a = {};
    e = p.id_bits == 64 ? sort_ids<int64_t>(p, ids, L, ws, &a.pairs, s)
                        : sort_ids<int32_t>(p, ids, L, ws, &a.pairs, s);
    if (e != hipSuccess) return e;
    a.count = (uint32_t)p.count;
    a.chunk = L.chunk;
    a.chunks = L.chunks;
    a.vocab = (uint32_t)p.vocab;
    a.dim = (uint32_t)p.dim;
    a.x_ld = p.x_ld;
    a.dst_ld = p.table_ld;
    a.scale = p.scale;
    a.fixed = p.fixed;
    a.accumulate = out.accumulate;
    a.rows = out.rows;
    a.cap = out.cap;
    a.crossing_count = crossing_count;
    a.crossing = reinterpret_cast<uint2*>(ws + L.crossing);
    a.partial = ws + L.partial;
    if (!rows) return sum_from<false>(a, x_type, out.type, dout, out.dst, di.cus, s);
    uint32_t* heads = reinterpret_cast<uint32_t*>(ws + L.heads);
    a.heads = heads;
    hipLaunchKernelGGL(head_count_kernel, dim3((L.chunks + kBlock / 64 - 1) / (kBlock / 64)),
                       dim3(kBlock), 0, s, a.pairs, a.count, a.chunk, a.chunks, a.vocab, heads);
    hipLaunchKernelGGL(head_scan_kernel, dim3(1), dim3(1024), 0, s, heads, a.chunks, out.touched);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    return sum_from<true>(a, x_type, out.type, dout, out.dst, di.cus, s);
}

}  // namespace hc
