// hc_tiles.h -- tiles of a matrix product on the matrix cores: how a workgroup
// holds them in LDS, reads fragments and multiplies.  Shared by the
// orthogonalisation and the layers.
//
// D[i][j] = sum over l of P[i][l] Q[j][l], 16-bit operands, fp32 sums, in steps of
// 64 values of l.
#pragma once

#include "hc_device.h"

namespace hc {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

// Value (i, j) of a block in LDS, [i][EN]: its 4-value group is turned by i so
// that rows written and columns read are spread over the banks.
template <int EN> __device__ __forceinline__ uint32_t staged(uint32_t i, uint32_t j) {
    return i * EN + ((((j >> 2) ^ i ^ (i >> 3)) & (EN / 4 - 1)) << 2) + (j & 3u);
}

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
__device__ __forceinline__ f4 product16(b8 a, b8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Fragments: 16 rows of an operand by 32 values of l, half h of a step.  A lane
// holds row lane % 16, values 8 (lane / 16) .. + 7 of the half.  kBlock: bytes in
// LDS from one load instruction's 1024 bytes to the next.

// An operand stored by rows along l: a tile is [row][64], 128 bytes a row.
template <typename V> struct AlongRows {
    static constexpr uint32_t kBlock = 1024;
    static constexpr bool kWaits = false;
    template <int N>
    __device__ __forceinline__ static void read(V (&f)[N], int first, int count, const char* tile,
                                                uint32_t row0, uint32_t h, uint32_t lane) {
#pragma unroll
        for (int u = 0; u < N; u++)
            if (u >= first && u < first + count)
                f[u] = *reinterpret_cast<const V*>(tile + 2 * swizzled(row0 + 16 * u + (lane & 15), 4 * h + (lane >> 4)));
    }
};

// An operand stored by l, its rows' index contiguous: a tile is [64 of l][ROWS].
// The transposing load gives lane t of 16 column t of the four lines that lanes
// 4 r .. 4 r + 3 point to, 32 bytes of each; two loads make a fragment.  Chunk c (16
// bytes) of line l lies at c ^ turn(l) and blocks are padded, so that the 32 bytes
// of the four lines, and those of the lanes 16 on (8 lines further), are in
// different banks: with a pitch of 512 bytes two lines are in a block and the pad
// moves the next two by 32 bytes, with 256 four and with 128 eight are.
//
// The loads are written in assembly, with their wait: before a builtin one the
// compiler waits for all loads from memory to LDS that are on their way, also those
// of the next step.
template <int ROWS> struct Across {
    static constexpr uint32_t kLines = 512 / ROWS;  // of a block
    static constexpr uint32_t kBlock = 1024 + (ROWS == 256 ? 32 : 64);
    __device__ __forceinline__ static uint32_t turn(uint32_t l) {
        return ROWS == 256 ? (l & 1u) << 2 : ROWS == 128 ? (l & 3u) << 1 : (l & 2u);
    }
    // of line l, chunk c
    __device__ __forceinline__ static uint32_t place(uint32_t l, uint32_t c) {
        return l / kLines * kBlock + l % kLines * (2 * ROWS) + ((c ^ turn(l)) << 4);
    }
};

template <typename V, int ROWS> struct AcrossRows {
    static constexpr uint32_t kBlock = Across<ROWS>::kBlock;
    static constexpr bool kWaits = true;
    // from a load to the one of the next four lines
    static constexpr uint32_t kFour = ROWS == 256 ? 2 * kBlock : ROWS == 128 ? kBlock : 4 * 2 * ROWS;
    typedef short s4 __attribute__((ext_vector_type(4)));

    __device__ __forceinline__ static V joined(s4 lo, s4 hi) {
        return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // all N of them; every load that was asked for before has landed too
    template <int N>
    __device__ __forceinline__ static void read(V (&f)[N], int, int, const char* tile, uint32_t row0,
                                                uint32_t h, uint32_t lane) {
        static_assert((ROWS == 256 && (N == 8 || N == 4)) || (ROWS == 128 && N == 4) || (ROWS == 64 && N == 2), "");
        const uint32_t t = lane & 15, l = 32 * h + 8 * (lane >> 4) + (t >> 2), c = row0 / 8 + (t >> 1 & 1u);
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)tile + ((t & 1u) << 3);
        // fragment u is 2 u chunks on, which turn() mixes with bits of u
        auto at = [&](uint32_t u) { return base + Across<ROWS>::place(l, c + 2 * u); };
        s4 a[N], b[N];
        if constexpr (N == 8) {
            asm volatile(
                "ds_read_b64_tr_b16 %0, %16\n\t"
                "ds_read_b64_tr_b16 %8, %16 offset:%18\n\t"
                "ds_read_b64_tr_b16 %1, %16 offset:32\n\t"
                "ds_read_b64_tr_b16 %9, %16 offset:%18+32\n\t"
                "ds_read_b64_tr_b16 %2, %17\n\t"
                "ds_read_b64_tr_b16 %10, %17 offset:%18\n\t"
                "ds_read_b64_tr_b16 %3, %17 offset:32\n\t"
                "ds_read_b64_tr_b16 %11, %17 offset:%18+32\n\t"
                "ds_read_b64_tr_b16 %4, %16 offset:128\n\t"
                "ds_read_b64_tr_b16 %12, %16 offset:%18+128\n\t"
                "ds_read_b64_tr_b16 %5, %16 offset:160\n\t"
                "ds_read_b64_tr_b16 %13, %16 offset:%18+160\n\t"
                "ds_read_b64_tr_b16 %6, %17 offset:128\n\t"
                "ds_read_b64_tr_b16 %14, %17 offset:%18+128\n\t"
                "ds_read_b64_tr_b16 %7, %17 offset:160\n\t"
                "ds_read_b64_tr_b16 %15, %17 offset:%18+160\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(a[4]), "=&v"(a[5]), "=&v"(a[6]),
                  "=&v"(a[7]), "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]), "=&v"(b[3]), "=&v"(b[4]), "=&v"(b[5]),
                  "=&v"(b[6]), "=&v"(b[7])
                : "v"(at(0)), "v"(at(2)), "n"(kFour)
                : "memory");
        } else if constexpr (N == 4 && ROWS == 256) {
            asm volatile(
                "ds_read_b64_tr_b16 %0, %8\n\t"
                "ds_read_b64_tr_b16 %4, %8 offset:%10\n\t"
                "ds_read_b64_tr_b16 %1, %8 offset:32\n\t"
                "ds_read_b64_tr_b16 %5, %8 offset:%10+32\n\t"
                "ds_read_b64_tr_b16 %2, %9\n\t"
                "ds_read_b64_tr_b16 %6, %9 offset:%10\n\t"
                "ds_read_b64_tr_b16 %3, %9 offset:32\n\t"
                "ds_read_b64_tr_b16 %7, %9 offset:%10+32\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]),
                  "=&v"(b[3])
                : "v"(at(0)), "v"(at(2)), "n"(kFour)
                : "memory");
        } else if constexpr (N == 4) {
            asm volatile(
                "ds_read_b64_tr_b16 %0, %8\n\t"
                "ds_read_b64_tr_b16 %4, %8 offset:%12\n\t"
                "ds_read_b64_tr_b16 %1, %9\n\t"
                "ds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
                "ds_read_b64_tr_b16 %2, %10\n\t"
                "ds_read_b64_tr_b16 %6, %10 offset:%12\n\t"
                "ds_read_b64_tr_b16 %3, %11\n\t"
                "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]),
                  "=&v"(b[3])
                : "v"(at(0)), "v"(at(1)), "v"(at(2)), "v"(at(3)), "n"(kFour)
                : "memory");
        } else {
            asm volatile(
                "ds_read_b64_tr_b16 %0, %4\n\t"
                "ds_read_b64_tr_b16 %2, %4 offset:%6\n\t"
                "ds_read_b64_tr_b16 %1, %5\n\t"
                "ds_read_b64_tr_b16 %3, %5 offset:%6\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(a[0]), "=&v"(a[1]), "=&v"(b[0]), "=&v"(b[1])
                : "v"(at(0)), "v"(at(1)), "n"(kFour)
                : "memory");
        }
#pragma unroll
        for (int u = 0; u < N; u++) f[u] = joined(a[u], b[u]);
    }
};

// Bytes of a step's tiles in LDS.
template <typename S, typename RP, typename RQ> struct Stage {
    static constexpr uint32_t kQ = S::BM / 8 * RP::kBlock, kBytes = kQ + S::BN / 8 * RQ::kBlock;
};

// Fragments and products of the steps.  The first operand of the instruction gives
// a lane's 4 consecutive results: Q, so that they lie along j.  RP and RQ read the
// fragments.  Two planes: a step is 32 high parts and their 32 low parts.
template <int PLANES, typename S, typename V, typename RP, typename RQ, typename F>
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
        const char* sp = s_mem + buf * Stage<S, RP, RQ>::kBytes;
        buf = buf + 1 == N ? 0 : buf + 1;
        const char* sq = sp + Stage<S, RP, RQ>::kQ;
        V fp[2][FM], fq[2][FN];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            RP::read(fp[h], 0, FM, sp, wi, h, lane);
            RQ::read(fq[h], 0, FN, sq, wj, h, lane);
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
template <int PLANES, typename S, typename V, typename RP, typename RQ, typename F>
__device__ __forceinline__ void main_loop_paired(f4 (&acc)[S::WM / 16][S::WN / 16], const F& fetch,
                                                 const char* s_mem, uint32_t lines, uint32_t wi,
                                                 uint32_t wj, uint32_t lane, uint32_t wave) {
    constexpr int FM = S::WM / 16, FN = S::WN / 16;
    // reads that wait for themselves come after the step's loads were asked for
    constexpr bool kFetchFirst = RP::kWaits || RQ::kWaits;
    const bool second = wave >= 4;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    phase_barrier();
    if (second) phase_barrier();
    for (uint32_t l = 0; l < lines; l++) {
        const char* sp = s_mem + (l & 1) * Stage<S, RP, RQ>::kBytes;
        const char* sq = sp + Stage<S, RP, RQ>::kQ;
        V fp[2][FM], fq[2][FN];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            // one plane: a half is 32 of the 64 values of l.  Two planes: a half is
            // half of the rows, with all of Q read in the first
#pragma unroll
            for (int c2 = 0; c2 < 2; c2++) {
                if (PLANES == 1 && c2 != h) continue;
                if (kFetchFirst && h == 0 && l + 1 < lines) fetch(l + 1, (l + 1) & 1);
                if (RQ::kWaits) {
                    RP::read(fp[c2], 0, FM, sp, wi, c2, lane);
                    RQ::read(fq[c2], 0, FN, sq, wj, c2, lane);
                } else {
                    if (PLANES == 1 || h == 0) RQ::read(fq[c2], 0, FN, sq, wj, c2, lane);
                    RP::read(fp[c2], PLANES == 1 ? 0 : h * FM / 2, PLANES == 1 ? FM : FM / 2, sp, wi, c2, lane);
                }
            }
            if (!kFetchFirst && h == 0 && l + 1 < lines) fetch(l + 1, (l + 1) & 1);
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

// Workgroups go to the 8 XCDs in turn; each XCD takes a contiguous share of the
// tiles, so that what neighbouring tiles read is shared in its L2.
__device__ __forceinline__ uint32_t by_xcd(uint32_t block, uint32_t blocks) {
    const uint32_t xcd = block & 7u, k = block >> 3, per = blocks >> 3, more = blocks & 7u;
    return xcd * per + min(xcd, more) + k;
}

}  // namespace hc
