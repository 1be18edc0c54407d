// hc_dropout.hip -- dropout and its gradient (include/hc_train.h).
//
// A lane takes eight elements of a row, one call of the generator, four times 256
// groups apart.  Memory bounds it: a call for 393216 x 512 (fp16) takes 137 us, 5.9 TB/s
// of reads and writes; for 32768 x 768 (bf16) with a residual 26, 5.7 (a plain copy 4.4 to 4.8).
// The generator alone would take 86 and 11 us of the vector units.
#include "hc_layer.h"

namespace hc {

namespace {

constexpr int kBlock = 256;
// Groups of a lane: four, or one where that leaves CUs without a workgroup (700 x 1500
// in fp32: 129 workgroups of four).
constexpr uint32_t kPer = 4;
constexpr uint64_t kFewGroups = 1024ull * kBlock;
// Results that the L2s cannot keep pass them by, and so does what is read for them:
// 32768 x 768 (bf16) with a residual 29.5 -> 26 us, 393216 x 512 (fp16) 141 -> 137.
constexpr uint64_t kPastBytes = 32ull << 20;

struct DropoutArgs {
    const void *x, *residual;
    void* out;
    uint64_t x_ld, residual_ld, out_ld;
    uint64_t rows;
    uint32_t cols, groups;           // columns of a row, and groups of eight of them
    uint32_t step_rows, step_groups; // 256 groups on: whole rows and the rest
    Dropout drop;
};

// Rows and groups are found by one division a workgroup and steps of 256 groups.
template <typename T, bool RESIDUAL, uint32_t PER, bool PAST>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutArgs a) {
    const Masks masks = masks_of(a.drop);
    const uint64_t first = (uint64_t)blockIdx.x * (kBlock * PER);
    uint64_t row = first / a.groups;
    uint32_t group = (uint32_t)(first - row * a.groups) + threadIdx.x;
    row += group / a.groups;
    group %= a.groups;
#pragma unroll
    for (uint32_t k = 0; k < PER; k++) {
        if (row < a.rows) {
            const uint32_t col = group * 8, count = a.cols - col;
            float v[8], r[8];
            auto load = [&](const void* p, uint64_t ld, float (&w)[8]) {
                const T* at = static_cast<const T*>(p) + row * ld + col;
                if constexpr (PAST) load8_past(at, count, w);
                else load8(at, count, w);
            };
            load(a.x, a.x_ld, v);
            if constexpr (RESIDUAL) load(a.residual, a.residual_ld, r);
            if (masks.limit) drop8(masks, (uint32_t)row, group, v);
            if constexpr (RESIDUAL)
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] += r[e];
            T* out = static_cast<T*>(a.out) + row * a.out_ld + col;
            if constexpr (PAST) store8_past(out, count, v);
            else store8(out, count, v);
        }
        row += a.step_rows;
        group += a.step_groups;
        if (group >= a.groups) {
            group -= a.groups;
            row++;
        }
    }
}

template <typename T, bool RESIDUAL, uint32_t PER, bool PAST>
hipError_t launch_variant(const DropoutArgs& a, hipStream_t s) {
    const uint64_t per = (uint64_t)kBlock * PER, blocks = (a.rows * a.groups + per - 1) / per;
    hipLaunchKernelGGL((dropout_kernel<T, RESIDUAL, PER, PAST>), dim3((uint32_t)blocks), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

template <typename T, bool RESIDUAL> hipError_t launch_typed(const DropoutArgs& a, hipStream_t s) {
    if (a.rows * a.groups <= kFewGroups) return launch_variant<T, RESIDUAL, 1, false>(a, s);
    if (a.rows * a.cols * sizeof(T) <= kPastBytes) return launch_variant<T, RESIDUAL, kPer, false>(a, s);
    return launch_variant<T, RESIDUAL, kPer, true>(a, s);
}

template <typename T> hipError_t launch_type(const DropoutArgs& a, hipStream_t s) {
    return a.residual ? launch_typed<T, true>(a, s) : launch_typed<T, false>(a, s);
}

}  // namespace

hipError_t launch_dropout(const hc_dropout_params& p, const Dropout& d, hc_type type, const void* x,
                          const void* residual, void* out, hipStream_t s) {
    DropoutArgs a = {};
    a.x = x;
    a.residual = residual;
    a.out = out;
    a.x_ld = p.x_ld;
    a.residual_ld = p.residual_ld;
    a.out_ld = p.out_ld;
    a.rows = p.rows;
    a.cols = (uint32_t)p.cols;
    a.groups = (uint32_t)((p.cols + 7) / 8);
    a.step_rows = kBlock / a.groups;
    a.step_groups = kBlock % a.groups;
    a.drop = d;
    if (type == HC_T_F32) return launch_type<float>(a, s);
    if (type == HC_T_BF16) return launch_type<__bf16>(a, s);
    return launch_type<_Float16>(a, s);
}

}  // namespace hc
