// hc_dropout.hip -- dropout and its gradient (include/hc_train.h).
//
// A lane takes eight elements of a row, one call of the generator, four times 256
// groups apart.  Memory bounds it: 393216 x 512 (fp16) 141 us, 5.7 TB/s of reads and
// writes; 32768 x 768 (bf16) with a residual 29, 5.1 TB/s (a plain copy 4.4 to 4.8).
// The generator alone would take 86 and 11 us of the vector units.
#include "hc_layer.h"

namespace hc {

namespace {

constexpr int kBlock = 256;
// Groups of a lane: four, or one where that leaves CUs without a workgroup (700 x 1500
// in fp32: 129 workgroups of four).
constexpr uint32_t kPer = 4;
constexpr uint64_t kFewGroups = 1024ull * kBlock;

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
template <typename T, bool RESIDUAL, uint32_t PER>
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
            load8(static_cast<const T*>(a.x) + row * a.x_ld + col, count, v);
            if constexpr (RESIDUAL)
                load8(static_cast<const T*>(a.residual) + row * a.residual_ld + col, count, r);
            if (masks.limit) drop8(masks, (uint32_t)row, group, v);
            if constexpr (RESIDUAL)
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] += r[e];
            store8(static_cast<T*>(a.out) + row * a.out_ld + col, count, v);
        }
        row += a.step_rows;
        group += a.step_groups;
        if (group >= a.groups) {
            group -= a.groups;
            row++;
        }
    }
}

template <typename T, bool RESIDUAL> hipError_t launch_typed(const DropoutArgs& a, hipStream_t s) {
    const uint64_t groups = a.rows * a.groups;
    if (groups <= kFewGroups)
        hipLaunchKernelGGL((dropout_kernel<T, RESIDUAL, 1>), dim3((uint32_t)((groups + kBlock - 1) / kBlock)),
                           dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((dropout_kernel<T, RESIDUAL, kPer>),
                           dim3((uint32_t)((groups + kBlock * kPer - 1) / (kBlock * kPer))), dim3(kBlock), 0, s, a);
    return hipGetLastError();
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
