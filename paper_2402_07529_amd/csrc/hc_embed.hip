// hc_embed.hip -- embedding lookup with scaling, and its gradient by sorted
// token ids (include/hc_train.h).
//
// The gradient of out[i] = scale * W[t_i] is dW[v] = scale * sum over t_i = v of
// dOut[i].  Sorting the pairs (t_i, i) by id, stably, puts the terms of one row
// next to each other in token order.  The sorted list is cut into chunks of
// equal length whatever the ids are.  A run of equal ids is summed by the chunk
// it begins in, which follows it into the next chunk; a run that goes on past
// that (a frequent id) is shared by all chunks it reaches, one partial sum each,
// and a second launch joins those in chunk order.  Every order is fixed by the
// ids alone.  A dense gradient's zeros are written by workgroups of the sorting
// launches that have no pairs to sort.
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
template <typename T> __device__ __forceinline__ v4u load_raw(const T* p, int nv) {
    if (nv == kVec<T>) return *reinterpret_cast<const typename Wide<T>::V*>(p);
    typedef T TV __attribute__((ext_vector_type(kVec<T>)));
    TV t = {};
#pragma unroll
    for (int j = 0; j < kVec<T>; j++)
        if (j < nv) t[j] = p[j];
    return __builtin_bit_cast(v4u, t);
}

// The same for what is read once.
template <typename T> __device__ __forceinline__ v4u load_once(const T* p, int nv) {
    if (nv == kVec<T>)
        return __builtin_nontemporal_load(reinterpret_cast<const typename Wide<T>::V*>(p));
    return load_raw<T>(p, nv);
}

// ---- lookup ----------------------------------------------------------------------

template <typename ID>
__device__ __forceinline__ bool valid_id(ID id, uint32_t vocab) {
    return id >= 0 && (uint64_t)id < vocab;
}

// A unit is one token's row, or 64 lanes' worth of columns of it; a group of g
// lanes (a power of two up to a wave) takes U units, one 16-byte vector a lane
// each, all loads before the first store.  Bound by memory: 2^20 rows of 64 fp32
// from a 2^24-row table 74 us, 268 MB of them written; one unit a group 99.  Few
// tokens: by the call (2.8 us of kernel in 5.5).
template <typename T, typename ID, int U>
__global__ __launch_bounds__(kBlock) void embed_kernel(const T* __restrict__ table,
                                                       const ID* __restrict__ ids,
                                                       T* __restrict__ out, uint64_t units,
                                                       uint32_t vocab, uint32_t dim,
                                                       uint64_t table_ld, uint64_t out_ld,
                                                       uint32_t log2g, uint32_t slabs,
                                                       float scale) {
    constexpr int VEC = kVec<T>;
    const uint32_t groups = kBlock >> log2g, group = threadIdx.x >> log2g;
    const uint32_t lane_col = (threadIdx.x & ((1u << log2g) - 1u)) * VEC;
    for (uint64_t base = (uint64_t)blockIdx.x * groups * U; base < units;
         base += (uint64_t)gridDim.x * groups * U) {
        ID id[U];
        uint64_t row[U];
        uint32_t col[U];
        v4u w[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const uint64_t unit = base + u * groups + group;
            row[u] = slabs == 1 ? unit : unit / slabs;
            col[u] = unit < units ? (((uint32_t)(unit - row[u] * slabs) << log2g) * VEC + lane_col) : dim;
            id[u] = unit < units ? ids[row[u]] : (ID)-1;
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            w[u] = v4u{};
            if (col[u] < dim && valid_id(id[u], vocab))
                w[u] = load_raw<T>(table + (uint64_t)id[u] * table_ld + col[u],
                                   (int)min((uint32_t)VEC, dim - col[u]));
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (col[u] >= dim) continue;
            const bool valid = valid_id(id[u], vocab);
            float v[VEC];
            unpack<T>(w[u], v);
            T* q = out + row[u] * out_ld + col[u];
            const int nv = (int)min((uint32_t)VEC, dim - col[u]);
            typedef T TV __attribute__((ext_vector_type(VEC)));
            TV t;
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                float y = valid ? v[j] * scale : 0.0f;
                // the product in fp32 first: not fused with the rounding to fp16
                if constexpr (sizeof(T) == 2) asm("" : "+v"(y));
                t[j] = (T)y;
            }
            if (nv == VEC) {
                // from 64 MB on past the caches, which then keep the table's rows:
                // 2^20 rows of 64 fp32 91 -> 74 us
                typedef typename Wide<T>::V V;
                if constexpr (U > 1)
                    __builtin_nontemporal_store((V)__builtin_bit_cast(v4u, t), reinterpret_cast<V*>(q));
                else
                    *reinterpret_cast<V*>(q) = __builtin_bit_cast(v4u, t);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j++)
                    if (j < nv) q[j] = t[j];
            }
        }
    }
}

// Workgroups are at most this many: what is past them is taken in a stride.
constexpr uint64_t kMaxGroups = 1ull << 22;

// Lanes of a group: enough 16-byte vectors for a row, at most a wave; half a wave
// where the last of a row's groups would hold 17 to 32 vectors (30,522 x 768 bf16:
// gradient of 32,768 ids 59 -> 49 us, lookup of 262,144 95 -> 85).  With 1 to 16 of
// them half waves are faster for one thing and slower for another, and a whole
// wave stays: 640 bf16 columns 53 us (46 in half waves) and 84 (76), 320 fp32
// columns 42 (46) and 80 (77), 576 fp32 columns 60 (57) and 140 (144).
uint32_t group_log2(uint64_t vectors) {
    if (vectors > 64 && vectors % 64 > 16 && vectors % 64 <= 32) return 5;
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
    const uint64_t units = p.count * slabs, groups = kBlock >> log2g;
    auto launch = [&](auto kernel, uint64_t per_block) {
        const uint64_t blocks = (units + per_block - 1) / per_block;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(blocks < kMaxGroups ? blocks : kMaxGroups)),
                           dim3(kBlock), 0, s, static_cast<const T*>(table),
                           static_cast<const ID*>(ids), static_cast<T*>(out), units,
                           (uint32_t)p.vocab, (uint32_t)p.dim, p.table_ld, p.x_ld, log2g,
                           (uint32_t)slabs, p.scale);
        return hipGetLastError();
    };
    // four units a group once that still leaves every CU 16 workgroups (64 MB)
    if (units >= groups * 4 * 4096) return launch(&embed_kernel<T, ID, 4>, groups * 4);
    return launch(&embed_kernel<T, ID, 1>, groups);
}

// ---- gradient: zeros -------------------------------------------------------------

// A dense gradient's zeros, cut into pieces of about 4 KiB: a 16-byte store for
// each of 256 lanes, a workgroup one piece or as many as it has lanes for.  Each
// XCD's workgroups take neighbouring pieces.  4.3 GB 7.1 TB/s, 477 MB 6.6 (16 KiB
// a workgroup in the grid's order 5.9 and 5.7, with nontemporal stores 5.9 and
// 5.6), 200 MB 7.2 in any of these forms but the last.
constexpr uint64_t kPieceBytes = 4096, kPieceLanes = 256;

struct Zeros {
    char* dst;            // NULL: none
    uint64_t rows;        // rows of row_bytes at ld_bytes; one where they lie back to back
    uint64_t row_bytes, ld_bytes;
    uint64_t per;         // rows a piece (rows > 1)
    uint64_t pieces;
    uint64_t first;       // this launch's: from `first`, as many as its extra workgroups take
};

__device__ __forceinline__ void zero_bytes(char* p, uint64_t bytes, uint32_t at, uint32_t step) {
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
    const V zero = {};
    for (uint64_t i = at; i < bytes / 16; i += step) reinterpret_cast<V*>(p)[i] = zero;
    if (at < (bytes & 15) / 2) reinterpret_cast<uint16_t*>(p + (bytes & ~15ull))[at] = 0;
}

// Extra workgroup k of n.
__device__ __forceinline__ void zero_pieces(const Zeros& z, uint32_t k, uint32_t n) {
    const uint32_t per = n >> 3, each = max(blockDim.x / (uint32_t)kPieceLanes, 1u);
    const uint64_t piece = z.first + (uint64_t)(k < 8 * per ? (k & 7u) * per + (k >> 3) : k) * each;
    if (z.rows == 1) {
        const uint64_t b = piece * kPieceBytes;
        if (b < z.row_bytes)
            zero_bytes(z.dst + b, min(each * kPieceBytes, z.row_bytes - b), threadIdx.x, blockDim.x);
        return;
    }
    const uint64_t r0 = piece * z.per, r1 = min(r0 + each * z.per, z.rows);
    for (uint64_t r = r0 + (threadIdx.x >> 6); r < r1; r += blockDim.x >> 6)
        zero_bytes(z.dst + r * z.ld_bytes, z.row_bytes, threadIdx.x & 63, 64);
}

__global__ __launch_bounds__(kBlock) void zero_kernel(Zeros z) { zero_pieces(z, blockIdx.x, gridDim.x); }

// ---- gradient: sort --------------------------------------------------------------

// Stable radix sort of the pairs (id, token) by id in digits of up to 9 bits.
// Ids that add nothing get the key `vocab` and end up last.
constexpr int kItems = 8;
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

// Rank of this lane's digit among the wave's earlier lanes and, by its running
// counts `cnt`, the wave's earlier pairs, so that equal keys keep their order.
// Equal digits among the lanes are found with one ballot per digit bit.
__device__ __forceinline__ uint32_t wave_rank(volatile uint32_t* cnt, uint32_t digit, bool live,
                                              uint32_t log2bins) {
    uint64_t same = __ballot(live);
    for (uint32_t b = 0; b < log2bins; b++) {
        const bool bit = (digit >> b) & 1u;
        const uint64_t m = __ballot(bit);
        same &= bit ? m : ~m;
    }
    const uint32_t before = lanes_below(same);
    const uint32_t seen = live ? cnt[digit] : 0u;
    __builtin_amdgcn_wave_barrier();
    if (live && before == 0) cnt[digit] = seen + (uint32_t)__popcll(same);
    __builtin_amdgcn_wave_barrier();
    return seen + before;
}

// Up to kSmallCount ids: one launch.  A pair's place is the number of pairs
// before it in the order, and every workgroup counts that for kSmallOwn pairs
// against all keys, held in LDS: its lanes are kSmallOwn pairs times 64
// interleaved slices of the keys.  4099 ids, 25-bit keys: 5.8 us, where
// a radix sort by one workgroup took 23.  The other workgroups write zeros.
constexpr uint32_t kSmallThreads = 1024, kSmallCount = 6144, kSmallOwn = 16;

struct SmallSort {
    uint32_t count, groups;
    Pair* out;
    uint32_t* crossing_count;
    Zeros zeros;
};

template <typename ID>
__global__ __launch_bounds__(kSmallThreads) void small_sort_kernel(FromIds<ID> src, SmallSort a) {
    extern __shared__ __align__(16) uint32_t s_key[];  // padded to a multiple of 4 keys
    __shared__ uint32_t s_rank[kSmallOwn];
    if (blockIdx.x >= a.groups) {
        zero_pieces(a.zeros, blockIdx.x - a.groups, gridDim.x - a.groups);
        return;
    }
    const uint32_t quads = (a.count + 3) / 4;
    uint32_t keys[kSmallCount / kSmallThreads];
#pragma unroll
    for (uint32_t u = 0; u < kSmallCount / kSmallThreads; u++) {
        const uint32_t k = u * kSmallThreads + threadIdx.x;
        keys[u] = k < a.count ? src.get(k).key : ~0u;
    }
#pragma unroll
    for (uint32_t u = 0; u < kSmallCount / kSmallThreads; u++) {
        const uint32_t k = u * kSmallThreads + threadIdx.x;
        if (k < quads * 4) s_key[k] = keys[u];
    }
    if (threadIdx.x < kSmallOwn) s_rank[threadIdx.x] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.crossing_count = 0;
    lds_barrier();
    const uint32_t first = blockIdx.x * kSmallOwn, i = first + threadIdx.x % kSmallOwn;
    const uint32_t key = i < a.count ? s_key[i] : 0u;
    // smaller keys, and equal ones of earlier pairs: of workgroups before this one,
    // then (a slice each) of this one's own
    const uint32_t slice = threadIdx.x / kSmallOwn;
    uint32_t before = i < a.count && slice < i - first && s_key[first + slice] == key ? 1u : 0u;
#pragma unroll 4
    for (uint32_t q = slice; q < quads; q += kSmallThreads / kSmallOwn) {
        const v4u k = *reinterpret_cast<const v4u*>(s_key + 4 * q);
        const uint32_t bound = 4 * q < first ? key + 1 : key;
#pragma unroll
        for (uint32_t j = 0; j < 4; j++) before += k[j] < bound ? 1u : 0u;
    }
    for (uint32_t d = kSmallOwn; d < 64; d <<= 1) before += __shfl_xor(before, d);
    if (lane_id() < kSmallOwn) atomicAdd(&s_rank[lane_id()], before);
    lds_barrier();
    if (threadIdx.x < kSmallOwn && i < a.count) a.out[s_rank[threadIdx.x]] = Pair{key, i};
}

// Up to kMergeCount ids: two launches.  The first sorts blocks of kMergeBlock pairs
// as above, kBlockOwn of them a workgroup, a slice of the keys a wave.  In the
// second every workgroup holds all sorted keys in LDS, and eight lanes a pair
// search the other blocks for its place.  Both bounds as measured, the whole call
// by rows of 64: 4099 ids 20 us in one launch, 22 in two; 6000 24 and 24; 8192 27
// and 25.5; 16,384 33 in two, 67 in radix passes, and 32,768 of 768 bf16 70 and 82.
constexpr uint32_t kMergeCount = 32768, kMergeBlock = 1024, kBlockOwn = 64, kMergeOwn = 128;

struct MergeSort {
    uint32_t count, groups, blocks;
    uint32_t *keys, *pos;  // of the sorted blocks
    Pair* out;
    uint32_t* crossing_count;
    Zeros zeros;
};

template <typename ID>
__global__ __launch_bounds__(kMergeBlock) void block_sort_kernel(FromIds<ID> src, MergeSort a) {
    __shared__ __align__(16) uint32_t s_key[kMergeBlock];
    __shared__ uint32_t s_rank[kBlockOwn];
    if (blockIdx.x >= a.groups) {
        zero_pieces(a.zeros, blockIdx.x - a.groups, gridDim.x - a.groups);
        return;
    }
    constexpr uint32_t kParts = kMergeBlock / kBlockOwn, kSlices = kMergeBlock / 64;
    static_assert(kBlockOwn == 64 && kParts == kSlices, "a lane a pair; see `own` below");
    const uint32_t base = blockIdx.x / kParts * kMergeBlock, part = blockIdx.x % kParts;
    s_key[threadIdx.x] = base + threadIdx.x < a.count ? src.get(base + threadIdx.x).key : ~0u;
    if (threadIdx.x < kBlockOwn) s_rank[threadIdx.x] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.crossing_count = 0;
    lds_barrier();
    const uint32_t i = part * kBlockOwn + lane_id(), key = s_key[i];
    uint32_t before = 0;
#pragma unroll
    for (uint32_t k = 0; k < kSlices; k++) {
        const uint32_t q = k * kSlices + (threadIdx.x >> 6);
        const v4u w = *reinterpret_cast<const v4u*>(s_key + 4 * q);
        if (k == part) {  // these four may be on either side of i
#pragma unroll
            for (uint32_t j = 0; j < 4; j++)
                before += w[j] < key + (4 * q + j < i ? 1u : 0u) ? 1u : 0u;
        } else {
            const uint32_t bound = k < part ? key + 1 : key;
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) before += w[j] < bound ? 1u : 0u;
        }
    }
    atomicAdd(&s_rank[lane_id()], before);
    lds_barrier();
    if (threadIdx.x < kBlockOwn && base + i < a.count) {
        a.keys[base + s_rank[threadIdx.x]] = key;
        a.pos[base + s_rank[threadIdx.x]] = base + i;
    }
}

__global__ __launch_bounds__(1024) void merge_kernel(MergeSort a) {
    extern __shared__ __align__(16) uint32_t s_key[];  // whole blocks
    if (blockIdx.x >= a.groups) {
        zero_pieces(a.zeros, blockIdx.x - a.groups, gridDim.x - a.groups);
        return;
    }
    constexpr uint32_t kLanes = 1024 / kMergeOwn;                     // of a pair
    constexpr uint32_t kEach = kMergeCount / kMergeBlock / kLanes;    // blocks a lane searches
    constexpr uint32_t kLoads = kMergeCount / 4 / 1024;
    v4u w[kLoads];
#pragma unroll
    for (uint32_t u = 0; u < kLoads; u++) {
        const uint32_t k = (u * 1024 + threadIdx.x) * 4;
        if (k < a.count) w[u] = *reinterpret_cast<const v4u*>(a.keys + k);  // the list is padded
    }
#pragma unroll
    for (uint32_t u = 0; u < kLoads; u++) {
        const uint32_t k = (u * 1024 + threadIdx.x) * 4;
#pragma unroll
        for (uint32_t j = 0; j < 4; j++)
            if (k + j >= a.count) w[u][j] = ~0u;
        if (k < a.blocks * kMergeBlock) *reinterpret_cast<v4u*>(s_key + k) = w[u];
    }
    const uint32_t i = blockIdx.x * kMergeOwn + threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t own = i / kMergeBlock;
    const uint32_t at = i < a.count && lane == 0 ? a.pos[i] : 0;
    lds_barrier();
    const uint32_t key = i < a.count ? s_key[i] : 0;
    // pairs before this one in each block: of smaller keys, and of equal ones if the
    // block is an earlier one
    uint32_t first[kEach], found[kEach], bound[kEach];
#pragma unroll
    for (uint32_t e = 0; e < kEach; e++) {
        const uint32_t b = e * kLanes + lane;
        first[e] = b < a.blocks ? b * kMergeBlock : 0;
        bound[e] = b < own ? key + 1 : key;
        found[e] = 0;
    }
#pragma unroll
    for (uint32_t step = kMergeBlock / 2; step > 0; step /= 2)
#pragma unroll
        for (uint32_t e = 0; e < kEach; e++)
            found[e] += s_key[first[e] + found[e] + step - 1] < bound[e] ? step : 0;
    uint32_t rank = 0;
#pragma unroll
    for (uint32_t e = 0; e < kEach; e++) {
        const uint32_t b = e * kLanes + lane;
        found[e] += s_key[first[e] + found[e]] < bound[e] ? 1 : 0;
        rank += b >= a.blocks ? 0 : b == own ? i % kMergeBlock : found[e];
    }
    for (uint32_t d = 1; d < kLanes; d <<= 1) rank += __shfl_xor(rank, d);
    if (lane == 0 && i < a.count) a.out[rank] = Pair{key, at};
}

// More ids (2^20 of 25 bits: three passes of 8 + 5 + 12 us): per pass every
// workgroup counts its tile's digits, the counts are scanned per digit over the
// workgroups, and every workgroup moves its tile's pairs to their places.  Each
// launch's workgroups past its own write zeros.
template <uint32_t THREADS, typename SRC>
__global__ __launch_bounds__(THREADS) void digit_count_kernel(SRC src, uint32_t count,
                                                              uint32_t groups, uint32_t shift,
                                                              uint32_t bins,
                                                              uint32_t* __restrict__ hist,
                                                              uint32_t* __restrict__ crossing_count,
                                                              Zeros zeros) {
    __shared__ uint32_t s_cnt[kMaxBins];
    if (blockIdx.x >= groups) {
        zero_pieces(zeros, blockIdx.x - groups, gridDim.x - groups);
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *crossing_count = 0;
    const uint32_t base = blockIdx.x * (THREADS * kItems) + threadIdx.x;
    uint32_t key[kItems];
#pragma unroll
    for (int it = 0; it < kItems; it++)
        key[it] = base + it * THREADS < count ? src.get(base + it * THREADS).key : 0u;
    for (uint32_t b = threadIdx.x; b < bins; b += THREADS) s_cnt[b] = 0;
    lds_barrier();
#pragma unroll
    for (int it = 0; it < kItems; it++)
        if (base + it * THREADS < count) atomicAdd(&s_cnt[(key[it] >> shift) & (bins - 1u)], 1u);
    lds_barrier();
    for (uint32_t b = threadIdx.x; b < bins; b += THREADS)
        hist[(uint64_t)b * groups + blockIdx.x] = s_cnt[b];
}

// One wave a digit: hist[digit][workgroup] becomes the count in earlier
// workgroups, total[digit] the count in all.
__global__ __launch_bounds__(kBlock) void digit_scan_kernel(uint32_t* __restrict__ hist,
                                                            uint32_t* __restrict__ total,
                                                            uint32_t bins, uint32_t groups,
                                                            Zeros zeros) {
    const uint32_t own = (bins + kBlock / 64 - 1) / (kBlock / 64);
    if (blockIdx.x >= own) {
        zero_pieces(zeros, blockIdx.x - own, gridDim.x - own);
        return;
    }
    const uint32_t bin = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (bin >= bins) return;
    const uint32_t lane = lane_id();
    uint32_t* h = hist + (uint64_t)bin * groups;
    uint32_t before = 0;
    for (uint32_t g0 = 0; g0 < groups; g0 += 256) {  // 4 consecutive workgroups a lane
        uint32_t v[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t g = g0 + lane * 4 + j;
            v[j] = g < groups ? h[g] : 0u;
            sum += v[j];
        }
        uint32_t x = sum;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t y = __shfl_up(x, d);
            if (lane >= (uint32_t)d) x += y;
        }
        uint32_t at = before + x - sum;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t g = g0 + lane * 4 + j;
            if (g < groups) h[g] = at;
            at += v[j];
        }
        before += __shfl(x, 63);
    }
    if (lane == 0) total[bin] = before;
}

template <uint32_t THREADS, typename SRC>
__global__ __launch_bounds__(THREADS) void digit_move_kernel(SRC src, uint32_t count,
                                                             uint32_t groups, uint32_t shift,
                                                             uint32_t log2bins,
                                                             const uint32_t* __restrict__ hist,
                                                             const uint32_t* __restrict__ total,
                                                             Pair* __restrict__ out, Zeros zeros) {
    constexpr uint32_t kWaves = THREADS / 64, kPer = kMaxBins / THREADS > 0 ? kMaxBins / THREADS : 1;
    __shared__ uint32_t s_cnt[kWaves][kMaxBins];
    __shared__ uint32_t s_tmp[kWaves];
    if (blockIdx.x >= groups) {
        zero_pieces(zeros, blockIdx.x - groups, gridDim.x - groups);
        return;
    }
    const uint32_t bins = 1u << log2bins;
    const uint32_t wave = threadIdx.x >> 6, lane = lane_id();
    const uint32_t base = blockIdx.x * (THREADS * kItems) + wave * (64 * kItems) + lane;
    Pair p[kItems];
    uint32_t rank[kItems];
#pragma unroll
    for (int it = 0; it < kItems; it++)
        p[it] = base + it * 64 < count ? src.get(base + it * 64) : Pair{0, 0};
    // per digit: its pairs in all, and in earlier workgroups
    uint32_t t[kPer], h[kPer], sum = 0;
#pragma unroll
    for (uint32_t j = 0; j < kPer; j++) {
        const uint32_t b = threadIdx.x * kPer + j;
        t[j] = b < bins ? total[b] : 0u;
        h[j] = b < bins ? hist[(uint64_t)b * groups + blockIdx.x] : 0u;
        sum += t[j];
    }
    for (uint32_t b = threadIdx.x; b < kWaves * kMaxBins; b += THREADS) (&s_cnt[0][0])[b] = 0;
    lds_barrier();
#pragma unroll
    for (int it = 0; it < kItems; it++)
        rank[it] = wave_rank(s_cnt[wave], (p[it].key >> shift) & (bins - 1u),
                                       base + it * 64 < count, log2bins);
    lds_barrier();
    uint32_t all;
    uint32_t first = block_exclusive_scan(sum, s_tmp, &all);
#pragma unroll
    for (uint32_t j = 0; j < kPer; j++) {
        const uint32_t b = threadIdx.x * kPer + j;
        if (b < bins) {
            uint32_t at = first + h[j];
            for (uint32_t w = 0; w < kWaves; w++) {
                const uint32_t c = s_cnt[w][b];
                s_cnt[w][b] = at;
                at += c;
            }
        }
        first += t[j];
    }
    lds_barrier();
#pragma unroll
    for (int it = 0; it < kItems; it++)
        if (base + it * 64 < count)
            out[s_cnt[wave][(p[it].key >> shift) & (bins - 1u)] + rank[it]] = p[it];
}

// ---- gradient: rows --------------------------------------------------------------

// First positions of runs per chunk of the sorted pairs.
__global__ __launch_bounds__(kBlock) void head_count_kernel(const Pair* __restrict__ pairs,
                                                            uint32_t count, uint32_t chunk,
                                                            uint32_t vocab,
                                                            uint32_t* __restrict__ heads) {
    const uint32_t lane = lane_id();
    const uint32_t i = (blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)) * 64 + lane;
    bool head = false;
    if (i < count) {
        const uint32_t key = pairs[i].key;
        head = key != vocab && (i == 0 || pairs[i - 1].key != key);
    }
    const uint64_t m = __ballot(head);
    if (i < count && lane % chunk == 0)
        heads[i / chunk] = (uint32_t)__popcll((m >> lane) & (~0ull >> (64 - chunk)));
}

// heads[c] becomes the number of runs that begin before chunk c; *touched the
// number of runs.  One workgroup, 16 chunks a lane at a time.
__global__ __launch_bounds__(1024) void head_scan_kernel(uint32_t* __restrict__ heads,
                                                         uint32_t chunks,
                                                         uint32_t* __restrict__ touched) {
    constexpr int N = 16;
    __shared__ uint32_t s_tmp[16];
    uint32_t before = 0;
    for (uint64_t c0 = 0; c0 < chunks; c0 += 1024 * N) {
        uint32_t v[N], sum = 0;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const uint64_t c = c0 + threadIdx.x * N + j;
            v4u w = {};
            if (c < chunks) w = *reinterpret_cast<const v4u*>(heads + c);  // padded to 16
#pragma unroll
            for (int k = 0; k < 4; k++) {
                v[j + k] = c + k < chunks ? w[k] : 0u;
                sum += v[j + k];
            }
        }
        uint32_t total;
        uint32_t at = before + block_exclusive_scan(sum, s_tmp, &total);
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const uint64_t c = c0 + threadIdx.x * N + j;
            v4u w;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                w[k] = at;
                at += v[j + k];
            }
            if (c < chunks) *reinterpret_cast<v4u*>(heads + c) = w;
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
#pragma unroll
        for (int j = 0; j < VEC; j++)
            if (j < nv) p[j] = o[j];
    }
}

constexpr uint32_t kCountedHeads = 8192;  // 4096 pairs a round of loads

struct SumArgs {
    const Pair* pairs;
    uint32_t count, chunk, chunks, vocab, dim, dim8;
    uint64_t x_ld, dst_ld;
    uint32_t log2g, slabs;
    float scale, fixed;
    bool accumulate;
    // by rows; heads: runs that begin before each chunk (NULL, for up to
    // kCountedHeads pairs: counted by the sums, which then set *touched)
    uint32_t* rows;
    const uint32_t* heads;
    uint32_t* touched;
    uint64_t cap;
    // shared runs: (chunk they begin in, rank), and their partial sums, two of
    // dim8 (dim rounded up to 8) elements a chunk: of the run it begins with, of
    // the run it ends with
    uint32_t* crossing_count;
    uint2* crossing;
    void* partial;
};

// Sums of the sorted pairs.  Bound by the random rows that they read: 2^20 rows
// of 64 fp32 in 84 us, 279 MB read and 61 MB written.
//
// The pairs that a workgroup's chunks look at lie in LDS: positions from p0.  (A
// pair read from memory would wait for the stores of the sums before it, as all
// vector memory of a wave completes in order.)
constexpr uint32_t kGroupPairs = 2048;  // of the chunks themselves, see chunk_for
struct NearPairs {
    const Pair* s;
    uint32_t p0;
    __device__ __forceinline__ Pair operator[](uint32_t i) const { return s[i - p0]; }
};

// One chunk's columns of one slab (a group of lanes).  A run of pairs covers
// boundary c if it holds the pairs on both sides of chunk c's start.  A run that
// covers two boundaries is shared by the chunks that it reaches; any other is
// summed whole by the chunk it begins in.
template <typename TI, typename TO, bool ROWS>
__device__ __forceinline__ void sum_chunk(const SumArgs& a, const NearPairs& pairs,
                                          const TI* __restrict__ x, TO* __restrict__ dst, uint32_t c,
                                          uint32_t slab, uint32_t heads) {
    typedef typename Sum<TO>::A A;
    constexpr int VEC = kVec<TI>;
    constexpr int U = 4;  // two batches in flight; 8 is 4 % slower by rows of 2^20 ids and for BERT's
    const uint32_t col = ((slab << a.log2g) + (threadIdx.x & ((1u << a.log2g) - 1u))) * VEC;
    if (col >= a.dim) return;
    const int nv = (int)min((uint32_t)VEC, a.dim - col);
    const uint32_t C = a.chunk, n = a.count;
    uint32_t start = c * C;
    const uint32_t end = min(start + C, n);
    const uint32_t k_first = pairs[start].key, k_last = pairs[end - 1].key;
    const uint32_t k_before = c > 0 ? pairs[start - 1].key : a.vocab;
    const uint32_t k_earlier = c > 1 ? pairs[start - C - 1].key : a.vocab;
    const uint32_t k_next = end < n ? pairs[end].key : a.vocab;
    const uint32_t k_later = (uint64_t)end + C < n ? pairs[end + C].key : a.vocab;
    if (k_first == a.vocab) return;
    uint32_t rank = heads;
    bool begins = k_before != k_first;
    if (!begins) {
        const bool shared = k_earlier == k_first || (end < n && k_next == k_first);
        if (!shared) {  // an earlier chunk sums it: on to the next run
            uint32_t lo = start, hi = end;  // first position with another key
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (pairs[mid].key == k_first) lo = mid + 1; else hi = mid;
            }
            if (lo == end) return;
            start = lo;
            begins = true;
        } else if constexpr (ROWS) {
            rank--;
        }
    }
    uint32_t cur = pairs[start].key;
    if (cur == a.vocab) return;
    // the last run goes on: shared if it covers the boundary after the next too,
    // else followed to its end
    const bool goes_on = end < n && k_next == k_last && k_last != a.vocab;
    const bool covers = goes_on && (k_later == k_last || (k_first == k_last && !begins));
    const uint32_t limit = goes_on && !covers ? min(end + C, n) : end;

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
            A* q = static_cast<A*>(a.partial) + ((uint64_t)c * 2 + (begins ? 1 : 0)) * a.dim8 + col;
#pragma unroll
            for (int j = 0; j < VEC; j++) q[j] = acc[j];
            if (begins && col == 0) a.crossing[atomicAdd(a.crossing_count, 1u)] = make_uint2(c, rank);
        }
    };
    // keys (vocab: nothing) and rows of U positions
    auto ask = [&](uint32_t i, uint32_t (&key)[U], v4u (&w)[U]) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const Pair p = i + u < limit ? pairs[i + u] : Pair{a.vocab, 0};
            key[u] = i + u >= end && p.key != k_last ? a.vocab : p.key;
            if (key[u] != a.vocab) w[u] = load_once<TI>(x + (uint64_t)p.pos * a.x_ld + col, nv);
        }
    };
    uint32_t key[U], next_key[U];
    v4u w[U], next_w[U];
    ask(start, next_key, next_w);
    for (uint32_t i = start; i < limit; i += U) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            key[u] = next_key[u];
            w[u] = next_w[u];
        }
        ask(i + U, next_key, next_w);  // before this batch's stores
        bool done = false;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (key[u] == a.vocab) {
                done = true;
                break;
            }
            if (key[u] != cur) {
                flush(true);
                cur = key[u];
                begins = true;
                if constexpr (ROWS) rank++;
#pragma unroll
                for (int j = 0; j < VEC; j++) acc[j] = 0;
            }
            float v[VEC];
            unpack<TI>(w[u], v);
#pragma unroll
            for (int j = 0; j < VEC; j++) acc[j] += Sum<TO>::term(v[j], a.scale, a.fixed);
        }
        if (done) break;
    }
    flush(!covers);
}

// This wave's share of the runs that begin at positions below `hi` (all lanes of
// a workgroup call it, at most kCountedHeads positions): two pairs a lane and load,
// 8 loads in flight.
__device__ __forceinline__ uint32_t count_begins(const SumArgs& a, uint32_t hi) {
    uint32_t found = 0;
    for (uint32_t i0 = 0; i0 < hi; i0 += kBlock * 2 * 8) {
        v4u w[8];
        uint32_t before[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; u++) {
            const uint32_t i = i0 + (u * kBlock + threadIdx.x) * 2;  // the list is padded to 256 bytes
            w[u] = i < hi ? *reinterpret_cast<const v4u*>(a.pairs + i) : v4u{};
            before[u] = lane_id() == 0 && i > 0 && i < hi ? a.pairs[i - 1].key : a.vocab;
        }
#pragma unroll
        for (uint32_t u = 0; u < 8; u++) {
            const uint32_t i = i0 + (u * kBlock + threadIdx.x) * 2;
            const uint32_t up = __shfl_up(w[u].z, 1);
            const uint32_t prev = lane_id() == 0 ? before[u] : up;
            if (i < hi && w[u].x != a.vocab && (i == 0 || prev != w[u].x)) found++;
            if (i + 1 < hi && w[u].z != a.vocab && w[u].z != w[u].x) found++;
        }
    }
    for (int d = 32; d > 0; d >>= 1) found += __shfl_xor(found, d);
    return found;
}

template <typename TI, typename TO, bool ROWS>
__global__ __launch_bounds__(kBlock) void segment_sum_kernel(SumArgs a, const TI* __restrict__ x,
                                                             TO* __restrict__ dst) {
    const uint64_t units = (uint64_t)a.chunks * a.slabs;
    const uint32_t groups = kBlock >> a.log2g;
    __shared__ Pair s_pairs[kGroupPairs + 2 * 64 + 2];
    __shared__ uint32_t s_heads[kBlock + 1];  // before the workgroup's chunks, then in each
    const bool count_heads = ROWS && a.heads == nullptr;
    for (uint64_t first = (uint64_t)blockIdx.x * groups; first < units;
         first += (uint64_t)gridDim.x * groups) {
        const uint32_t c0 = (uint32_t)(first / a.slabs);
        const uint32_t c1 = (uint32_t)((min(first + groups, units) - 1) / a.slabs);
        const uint32_t lo = c0 * a.chunk, hi = min((c1 + 1) * a.chunk, a.count);
        NearPairs pairs = {s_pairs, lo > a.chunk ? lo - a.chunk - 1 : 0u};
        const uint32_t near = min(hi + a.chunk + 1, a.count) - pairs.p0;
        uint32_t before = 0;
        lds_barrier();
        {
            constexpr int N = (kGroupPairs + 2 * 64 + 2 + kBlock - 1) / kBlock;
            Pair p[N];
#pragma unroll
            for (int k = 0; k < N; k++)
                if (k * kBlock + threadIdx.x < near) p[k] = a.pairs[pairs.p0 + k * kBlock + threadIdx.x];
            if (count_heads) {
                for (uint32_t i = threadIdx.x; i <= kBlock; i += kBlock) s_heads[i] = 0;
                before = count_begins(a, lo);
            }
#pragma unroll
            for (int k = 0; k < N; k++)
                if (k * kBlock + threadIdx.x < near) s_pairs[k * kBlock + threadIdx.x] = p[k];
        }
        if (count_heads) {
            lds_barrier();
            if (lane_id() == 0 && before) atomicAdd(&s_heads[0], before);
            for (uint32_t i = lo + threadIdx.x; i < hi; i += kBlock) {
                const uint32_t key = pairs[i].key;
                if (key != a.vocab && (i == 0 || pairs[i - 1].key != key))
                    atomicAdd(&s_heads[1 + i / a.chunk - c0], 1u);
            }
        }
        lds_barrier();
        if (count_heads && c1 + 1 == a.chunks && threadIdx.x == 0) {
            uint32_t all = 0;
            for (uint32_t k = 0; k <= c1 - c0 + 1; k++) all += s_heads[k];
            *a.touched = all;
        }
        const uint64_t unit = first + (threadIdx.x >> a.log2g);
        if (unit < units) {
            const uint32_t c = (uint32_t)(unit / a.slabs);
            uint32_t heads = 0;
            if (count_heads)
                for (uint32_t k = 0; k <= c - c0; k++) heads += s_heads[k];
            else if (ROWS)
                heads = a.heads[c];
            sum_chunk<TI, TO, ROWS>(a, pairs, x, dst, c, (uint32_t)(unit - (uint64_t)c * a.slabs), heads);
        }
    }
}

// Joins the partial sums of the shared runs (a chain of a few loads: 4 us with
// none, 9 to 16 with the 1 % most frequent of Zipf(1.1) ids): a workgroup takes one
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
        if (nv > 0) {
            typedef A AV __attribute__((ext_vector_type(VEC)));
            const A* base = static_cast<const A*>(a.partial) + (uint64_t)c * 2 * a.dim8 + col;
            for (uint32_t k = lo; k < hi; k += 8) {
                AV w[8];
#pragma unroll
                for (uint32_t u = 0; u < 8; u++)
                    // item 0: what chunk c ends with; item k: what chunk c + k begins with
                    if (k + u < hi)
                        w[u] = *reinterpret_cast<const AV*>(
                            base + (k + u == 0 ? (uint64_t)a.dim8 : (uint64_t)(k + u) * 2 * a.dim8));
#pragma unroll
                for (uint32_t u = 0; u < 8; u++)
                    if (k + u < hi)
#pragma unroll
                        for (int j = 0; j < VEC; j++) acc[j] += w[u][j];
            }
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

__global__ void clear_word_kernel(uint32_t* a) { *a = 0; }

// ---- layout and launches ---------------------------------------------------------

// Pairs per chunk: 64, or fewer (down to 4) while that leaves under kFewWaves
// waves of sums (a lane takes four columns, a wave up to 64 lanes of one row).
// Half and twice as many waves: 30,522 x 768 bf16 with 32,768 ids 57 and 58 us
// (49), 2^24 x 64 with 2^20 ids by rows 179 and 188 us (179).  Down to 4: 4099
// ids by rows of 64 24.7 us, 26.6 with 8 at least.
constexpr uint64_t kFewWaves = 4096;

// A workgroup's chunks (256 lanes' worth, 8 columns a lane at least) hold at most
// kGroupPairs pairs.
uint32_t most_chunk(uint64_t dim) {
    uint32_t chunk = 64;
    while (chunk > 8 && (chunk * kBlock) >> group_log2((dim + 7) / 8) > kGroupPairs) chunk /= 2;
    return chunk;
}

// Lanes that a row's sums take, 64 a slab.
uint64_t lanes_of_row(uint64_t dim) {
    const uint64_t vectors = (dim + 3) / 4;
    const uint32_t log2g = group_log2(vectors);
    return ((vectors + (1ull << log2g) - 1) >> log2g) << log2g;
}

uint32_t chunk_for(const hc_embed_params& p) {
    const uint64_t lanes = lanes_of_row(p.dim);
    uint32_t chunk = most_chunk(p.dim);
    while (chunk > 4 && p.count / chunk * lanes / 64 < kFewWaves) chunk /= 2;
    return chunk;
}

// Chunks and sorting workgroups of up to `count` ids: more ids can make fewer of
// either, and a workspace for more ids has to do for fewer.
uint64_t most_chunks(uint64_t dim, uint64_t count) {
    // a chunk is halved while it leaves fewer than kFewWaves waves, so the halves
    // make fewer than twice as many
    const uint64_t few = 2 * kFewWaves * 64 / lanes_of_row(dim) + 2, c = most_chunk(dim);
    const uint64_t small = (count + 3) / 4 < few ? (count + 3) / 4 : few, large = (count + c - 1) / c;
    return small > large ? small : large;
}

// Digits of the keys 0 .. vocab.
void digits_for(uint64_t vocab, uint32_t* passes, uint32_t* log2bins) {
    uint32_t bits = 1;
    while ((vocab >> bits) != 0) bits++;
    *passes = (bits + 8) / 9;
    *log2bins = (bits + *passes - 1) / *passes;
}

// Lanes of a sorting workgroup (8 pairs each): few enough pairs a workgroup to
// spread them over the CUs, many enough that the counts stay few.
constexpr uint64_t kManyIds = 1u << 19;
uint32_t sort_threads(uint64_t count) { return count >= kManyIds ? 512 : 256; }

uint64_t most_groups(uint64_t count) {
    const uint64_t few = count < kManyIds ? count : kManyIds;
    const uint64_t small = (few + 256 * kItems - 1) / (256 * kItems);
    const uint64_t large = (count + 512 * kItems - 1) / (512 * kItems);
    return small > large ? small : large;
}

struct GradLayout {
    uint32_t chunk, chunks, groups;
    bool small, merge;  // how ids are sorted; neither: radix passes
    size_t pairs[2], hist, total, heads, crossing_count, crossing, partial, bytes;
};

GradLayout grad_layout(const hc_embed_params& p) {
    GradLayout L;
    L.chunk = chunk_for(p);
    L.chunks = (uint32_t)((p.count + L.chunk - 1) / L.chunk);
    const uint64_t tile = sort_threads(p.count) * kItems;
    L.groups = (uint32_t)((p.count + tile - 1) / tile);
    L.small = p.count <= kSmallCount;
    L.merge = !L.small && p.count <= kMergeCount;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    L.pairs[0] = take(p.count * sizeof(Pair));
    L.pairs[1] = take(L.small ? 0 : L.merge ? 2 * align256(p.count * 4) : p.count * sizeof(Pair));
    const size_t chunks = most_chunks(p.dim, p.count);
    L.hist = take(L.small || L.merge ? 0 : most_groups(p.count) * kMaxBins * 4);
    L.total = take(kMaxBins * 4);
    L.heads = take(chunks * 4);
    L.crossing_count = take(4);
    L.crossing = take(chunks * 8);
    L.partial = take(chunks * 2 * ((p.dim + 7) / 8 * 8) * 8);
    L.bytes = at;
    return L;
}

Zeros zeros_for(void* dst, uint64_t rows, uint64_t row_bytes, uint64_t ld_bytes) {
    Zeros z = {};
    z.dst = static_cast<char*>(dst);
    if (ld_bytes == row_bytes || rows == 1) {
        z.rows = 1;
        z.row_bytes = rows * row_bytes;
        z.pieces = (z.row_bytes + kPieceBytes - 1) / kPieceBytes;
    } else {
        z.rows = rows;
        z.row_bytes = row_bytes;
        z.ld_bytes = ld_bytes;
        z.per = row_bytes >= kPieceBytes ? 1 : kPieceBytes / row_bytes;
        z.pieces = (rows + z.per - 1) / z.per;
    }
    return z;
}

// Workgroups of `threads` for the launch's share of the pieces, beyond its own;
// `next` is where the launches after it go on.  The grid's lanes stay below 2^32,
// so what does not fit is written by launches of its own.
constexpr uint64_t kMaxZeroGroups = 1ull << 20;

uint32_t share(const Zeros& z, uint64_t launches_left, uint32_t threads, Zeros* next) {
    const uint64_t each = threads / kPieceLanes;
    const uint64_t left = z.first < z.pieces ? z.pieces - z.first : 0;
    uint64_t n = ((left + launches_left - 1) / launches_left + each - 1) / each;
    if (n > kMaxZeroGroups) n = kMaxZeroGroups;
    *next = z;
    next->first += n * each;
    return (uint32_t)n;
}

hipError_t zero_rest(Zeros z, hipStream_t s) {
    while (z.first < z.pieces) {
        Zeros next;
        const uint32_t n = share(z, 1, kBlock, &next);
        hipLaunchKernelGGL(zero_kernel, dim3(n), dim3(kBlock), 0, s, z);
        z = next;
    }
    return hipGetLastError();
}

template <uint32_t THREADS, typename SRC>
void radix_pass(const SRC& src, uint32_t count, uint32_t shift, uint32_t log2bins,
                const GradLayout& L, char* ws, Pair* out, Zeros* z, uint32_t launches_left,
                hipStream_t s) {
    const uint32_t bins = 1u << log2bins;
    uint32_t* hist = reinterpret_cast<uint32_t*>(ws + L.hist);
    uint32_t* total = reinterpret_cast<uint32_t*>(ws + L.total);
    Zeros next;
    uint32_t n = share(*z, launches_left, THREADS, &next);
    hipLaunchKernelGGL((digit_count_kernel<THREADS, SRC>), dim3(L.groups + n), dim3(THREADS), 0, s,
                       src, count, L.groups, shift, bins, hist,
                       reinterpret_cast<uint32_t*>(ws + L.crossing_count), *z);
    *z = next;
    n = share(*z, launches_left - 1, kBlock, &next);
    hipLaunchKernelGGL(digit_scan_kernel, dim3((bins + kBlock / 64 - 1) / (kBlock / 64) + n),
                       dim3(kBlock), 0, s, hist, total, bins, L.groups, *z);
    *z = next;
    n = share(*z, launches_left - 2, THREADS, &next);
    hipLaunchKernelGGL((digit_move_kernel<THREADS, SRC>), dim3(L.groups + n), dim3(THREADS), 0, s,
                       src, count, L.groups, shift, log2bins, hist, total, out, *z);
    *z = next;
}

template <uint32_t THREADS, typename ID>
hipError_t sort_large(const hc_embed_params& p, const FromIds<ID>& ids, const GradLayout& L,
                      char* ws, const Pair** sorted, Zeros z, hipStream_t s) {
    uint32_t passes, log2bins;
    digits_for(p.vocab, &passes, &log2bins);
    Pair* buf[2] = {reinterpret_cast<Pair*>(ws + L.pairs[0]),
                    reinterpret_cast<Pair*>(ws + L.pairs[1])};
    for (uint32_t k = 0; k < passes; k++) {
        const uint32_t left = 3 * (passes - k);
        if (k == 0)
            radix_pass<THREADS>(ids, (uint32_t)p.count, 0, log2bins, L, ws, buf[0], &z, left, s);
        else
            radix_pass<THREADS>(FromPairs{buf[(k - 1) & 1]}, (uint32_t)p.count, k * log2bins, log2bins,
                                L, ws, buf[k & 1], &z, left, s);
    }
    *sorted = buf[(passes - 1) & 1];
    return zero_rest(z, s);
}

template <typename ID>
hipError_t sort_ids(const hc_embed_params& p, const void* ids, const GradLayout& L, char* ws,
                    const Pair** sorted, Zeros z, hipStream_t s) {
    const FromIds<ID> src = {static_cast<const ID*>(ids), (uint32_t)p.vocab, p.padding};
    if (L.merge) {
        MergeSort a = {};
        a.count = (uint32_t)p.count;
        a.blocks = (a.count + kMergeBlock - 1) / kMergeBlock;
        a.keys = reinterpret_cast<uint32_t*>(ws + L.pairs[1]);
        a.pos = reinterpret_cast<uint32_t*>(ws + L.pairs[1] + align256(p.count * 4));
        a.out = reinterpret_cast<Pair*>(ws + L.pairs[0]);
        a.crossing_count = reinterpret_cast<uint32_t*>(ws + L.crossing_count);
        *sorted = a.out;
        const int lds = (int)(a.blocks * kMergeBlock * 4);
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&merge_kernel), lds);
        if (e != hipSuccess) return e;
        Zeros next;
        uint32_t n = share(z, 2, kMergeBlock, &next);
        a.zeros = z;
        a.groups = a.blocks * (kMergeBlock / kBlockOwn);
        hipLaunchKernelGGL(block_sort_kernel<ID>, dim3(a.groups + n), dim3(kMergeBlock), 0, s, src, a);
        z = next;
        n = share(z, 1, 1024, &next);
        a.zeros = z;
        a.groups = (a.count + kMergeOwn - 1) / kMergeOwn;
        hipLaunchKernelGGL(merge_kernel, dim3(a.groups + n), dim3(1024), lds, s, a);
        return zero_rest(next, s);
    }
    if (!L.small) {
        if (sort_threads(p.count) == 512) return sort_large<512>(p, src, L, ws, sorted, z, s);
        return sort_large<256>(p, src, L, ws, sorted, z, s);
    }
    SmallSort a = {};
    a.count = (uint32_t)p.count;
    a.groups = (a.count + kSmallOwn - 1) / kSmallOwn;
    a.out = reinterpret_cast<Pair*>(ws + L.pairs[0]);
    a.crossing_count = reinterpret_cast<uint32_t*>(ws + L.crossing_count);
    a.zeros = z;
    Zeros next;
    const uint32_t n = share(z, 1, kSmallThreads, &next);
    hipLaunchKernelGGL(small_sort_kernel<ID>, dim3(a.groups + n), dim3(kSmallThreads),
                       (a.count + 3) / 4 * 16, s, src, a);
    *sorted = a.out;
    return zero_rest(next, s);
}

template <typename TI, typename TO, bool ROWS>
hipError_t sum_typed(SumArgs a, const void* x, void* dst, int cus, hipStream_t s) {
    const uint64_t vectors = (a.dim + kVec<TI> - 1) / kVec<TI>;
    a.log2g = group_log2(vectors);
    a.slabs = (uint32_t)((vectors + (1ull << a.log2g) - 1) >> a.log2g);
    const uint64_t units = (uint64_t)a.chunks * a.slabs, per_block = kBlock >> a.log2g;
    const uint64_t blocks = (units + per_block - 1) / per_block;
    hipLaunchKernelGGL((segment_sum_kernel<TI, TO, ROWS>),
                       dim3((uint32_t)(blocks < kMaxGroups ? blocks : kMaxGroups)), dim3(kBlock), 0, s, a,
                       static_cast<const TI*>(x), static_cast<TO*>(dst));
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
    const bool rows = out.by_rows;
    Zeros z = {};
    if (!rows && !out.accumulate) {
        const uint64_t size = out.type == HC_T_I32 || out.type == HC_T_F32 ? 4 : 2;
        z = zeros_for(out.dst, p.vocab, p.dim * size, p.table_ld * size);
    }
    if (p.count == 0) {
        if (!rows) return zero_rest(z, s);
        hipLaunchKernelGGL(clear_word_kernel, dim3(1), dim3(1), 0, s, out.touched);
        return hipGetLastError();
    }
    SumArgs a = {};
    e = p.id_bits == 64 ? sort_ids<int64_t>(p, ids, L, ws, &a.pairs, z, s)
                        : sort_ids<int32_t>(p, ids, L, ws, &a.pairs, z, s);
    if (e != hipSuccess) return e;
    a.count = (uint32_t)p.count;
    a.chunk = L.chunk;
    a.chunks = L.chunks;
    a.vocab = (uint32_t)p.vocab;
    a.dim = (uint32_t)p.dim;
    a.dim8 = (a.dim + 7) / 8 * 8;
    a.x_ld = p.x_ld;
    a.dst_ld = p.table_ld;
    a.scale = p.scale;
    a.fixed = p.fixed;
    a.accumulate = out.accumulate;
    a.rows = out.rows;
    a.cap = out.cap;
    a.crossing_count = reinterpret_cast<uint32_t*>(ws + L.crossing_count);
    a.crossing = reinterpret_cast<uint2*>(ws + L.crossing);
    a.partial = ws + L.partial;
    if (!rows) return sum_from<false>(a, x_type, out.type, dout, out.dst, di.cus, s);
    a.touched = out.touched;
    if (p.count > kCountedHeads) {
        uint32_t* heads = reinterpret_cast<uint32_t*>(ws + L.heads);
        a.heads = heads;
        hipLaunchKernelGGL(head_count_kernel, dim3((uint32_t)((p.count + kBlock - 1) / kBlock)),
                           dim3(kBlock), 0, s, a.pairs, a.count, a.chunk, a.vocab, heads);
        hipLaunchKernelGGL(head_scan_kernel, dim3(1), dim3(1024), 0, s, heads, a.chunks, out.touched);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return sum_from<true>(a, x_type, out.type, dout, out.dst, di.cus, s);
}

}  // namespace hc
