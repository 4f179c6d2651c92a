// Entry point of the products with 4-bit weights (kernels: w4_matvec.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "coral_lmhead.h"
#include "device_utils.h"
#include "w4_kernels.h"

namespace {

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + b_bytes && y < x + a_bytes;
}

}  // namespace

extern "C" coral_status coral_matvec_w4(const void* x, const void* codes, const void* scales, const void* zeros,
                                        const float* bias, const void* residual, int M, int N, int K, int group,
                                        coral_w4_code code, coral_dtype dt, coral_activation act, coral_dtype out_dt,
                                        void* y, void* hip_stream) {
    if (!x || !codes || !scales || !y) return CORAL_ERR_NULL;
    if (dt != CORAL_F32 && dt != CORAL_BF16 && dt != CORAL_F16) return CORAL_ERR_SHAPE;
    if (out_dt != CORAL_F32 && out_dt != dt) return CORAL_ERR_SHAPE;
    if (act != CORAL_ACT_SILU && act != CORAL_ACT_RELU && act != CORAL_ACT_IDENTITY) return CORAL_ERR_SHAPE;
    if (code != CORAL_W4_INT && code != CORAL_W4_E2M1) return CORAL_ERR_SHAPE;
    if (code == CORAL_W4_E2M1 && zeros) return CORAL_ERR_SHAPE;
    if (M < 1 || N < 1 || K < 1 || group < 1) return CORAL_ERR_SHAPE;
    if (M > kMaxM || K % 8 != 0 || K > CORAL_W4_MAX_K) return CORAL_ERR_UNSUPPORTED;
    if (group != 32 && group != 64 && group % 128 != 0) return CORAL_ERR_UNSUPPORTED;
    if (((uintptr_t)x | (uintptr_t)codes) & 15u) return CORAL_ERR_UNSUPPORTED;
    const size_t w = dt == CORAL_F32 ? 4 : 2, out_w = out_dt == CORAL_F32 ? 4 : 2;
    if (((uintptr_t)scales & (w - 1)) || ((uintptr_t)residual & (w - 1)) || ((uintptr_t)bias & 3u) || ((uintptr_t)y & (out_w - 1)))
        return CORAL_ERR_UNSUPPORTED;
    W4Params p = {};
    p.n_groups = (int)(((int64_t)K + group - 1) / group);
    const size_t y_bytes = (size_t)M * N * out_w, n_scales = (size_t)N * p.n_groups;
    // results are written while other workgroups still read the operands; the residual is read and
    // its place written by the same thread, so y may be the residual itself
    if (overlap(y, y_bytes, x, (size_t)M * K * w) || overlap(y, y_bytes, codes, (size_t)N * (K / 2)) ||
        overlap(y, y_bytes, scales, n_scales * w) || overlap(y, y_bytes, zeros, n_scales) ||
        overlap(y, y_bytes, bias, (size_t)N * 4) ||
        (overlap(y, y_bytes, residual, (size_t)M * N * w) && (y != residual || out_w != w)))
        return CORAL_ERR_UNSUPPORTED;
    p.x = x;
    p.codes = static_cast<const unsigned char*>(codes);
    p.scales = scales;
    p.zeros = static_cast<const unsigned char*>(zeros);
    p.bias = bias;
    p.residual = residual;
    p.y = y;
    p.M = M; p.N = N; p.K = K; p.group = group; p.act = (int)act;
    p.out_f32 = out_dt == CORAL_F32;
    p.per_group = group < kW4UnitCols ? 1 : group / kW4UnitCols;
    p.per_group_inv = (unsigned)((((uint64_t)1 << 32) + p.per_group - 1) / p.per_group);
    const int kind = code == CORAL_W4_E2M1 ? kW4E2M1 : zeros ? kW4Zero : kW4Sym;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const int slots = group < kW4UnitCols ? kW4UnitCols / group : 1;
    const bool f32 = dt == CORAL_F32;
    if (w4_plan_rows(M, N, f32)) {
        const void* rows = dt == CORAL_BF16 ? coral_w4_rows_bf16(kind, slots) : coral_w4_rows_f16(kind, slots);
        hipLaunchKernelGGL(reinterpret_cast<w4_fn>(const_cast<void*>(rows)), dim3((N - 1) / kW4RowsRows + 1), dim3(kW4Block), 0, stream, p);
        return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
    }
    const W4Plan plan = w4_plan_held(M, K, f32);
    const void* held = dt == CORAL_F32    ? coral_w4_held_f32(kind, slots, plan.t, plan.nb, plan.passes, plan.spread)
                       : dt == CORAL_BF16 ? coral_w4_held_bf16(kind, slots, plan.t, plan.nb, plan.passes, plan.spread)
                                          : coral_w4_held_f16(kind, slots, plan.t, plan.nb, plan.passes, plan.spread);
    const W4Grid grid = w4_held_grid(plan, M, N, f32);
    hipLaunchKernelGGL(reinterpret_cast<w4_fn>(const_cast<void*>(held)), dim3(grid.x, grid.y), dim3(kW4Block), 0, stream, p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}
