// Entry point of the products with 4-bit weights (kernels: w4_matvec.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "coral_lmhead.h"
#include "device_utils.h"
#include "w4_kernels.h"

namespace {

struct W4Plan {
    int t, nb;                  // k_w4_held's parameters
    bool passes, spread;
};

// More than 16 tokens are taken 32 at a time (a workgroup for each 32): all 64 at once need fewer reads of the
// codes and four times the activations a workgroup.  Measured with 64 tokens, bf16 (us), 64, 32 and 16 at a
// time: 4096 x 4096 18, 11, 12; 16384 x 4096 30, 23, 28; 50257 x 4096 62, 60, 73; 4096 x 14336 48, 34, 33.
// fp32 activations are spread over three rows of the products, five or ten tokens at a time, or taken as
// three products one after the other, 16 tokens at a time, where their parts fit the registers (up to 24
// units of columns) and more than five tokens share them.  Measured (us), chained and spread: one token, 128256 x 4096
// 144, 55; 4096 x 4096 12, 8; 8 tokens, 32000 x 4096 46, 27; 7 tokens, 50257 x 2568 33, 49.
// Registers hold eight units of 128 columns a wave for 16 rows of activations, four for 32; four of fp32
// ones (LDS for their scales).  More columns are taken in passes.
W4Plan plan_held(const W4Params& p, coral_dtype dt) {
    const int units = (p.K + kW4UnitCols - 1) / kW4UnitCols;
    int nb = (units + kW4Held - 1) / kW4Held;
    if (dt == CORAL_F32) {
        const bool spread = p.M <= w4_held_tokens(true, 1) || nb > 3;
        const int t = !spread || p.M <= w4_held_tokens(true, 1) ? 1 : 2;
        return {t, nb > 4 || t == 2 ? 4 : nb, nb > 4, spread};
    }
    const int t = p.M <= 16 ? 1 : 2, most = 8 / t;
    if (nb > most) return {t, most, true, false};
    nb = nb == 5 ? 6 : nb == 7 ? 8 : nb;
    return {t, nb, false, false};
}

// Whether k_w4_rows is taken: for more than 32 tokens, where the rows fill its rounds of workgroups (one of 512
// rows for each of 256 compute units), which take as long as 6000 tiles of k_w4_held.  Measured with 64
// tokens, bf16 (us), held and shared: 128256 rows of 1024 columns 58, 42; 2048 80, 67; 4096 126, 109 (48 tokens 127,
// 103; e2m1, groups of 32: 138, 119); 8192 245, 208.  100000 x 2048 61, 56; x 4096 100, 99; x 14336 377, 305;
// 65536 x 2048 44, 52; x 4096 72, 92; 152064 x 1024 62, 67; x 3584 143, 167.  32 tokens, 128256 x 4096 75, 82.
bool plan_rows(const W4Params& p, coral_dtype dt) {
    const int tiles = (p.N - 1) / 16 + 1, rounds = (p.N - 1) / (256 * kW4RowsRows) + 1;
    return dt != CORAL_F32 && p.M > 32 && (int64_t)rounds * 6000 < tiles;
}

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
    if (plan_rows(p, dt)) {
        const void* rows = dt == CORAL_BF16 ? coral_w4_rows_bf16(kind, slots) : coral_w4_rows_f16(kind, slots);
        hipLaunchKernelGGL(reinterpret_cast<w4_fn>(const_cast<void*>(rows)), dim3((N - 1) / kW4RowsRows + 1), dim3(kW4Block), 0, stream, p);
        return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
    }
    const W4Plan plan = plan_held(p, dt);
    const void* held = dt == CORAL_F32    ? coral_w4_held_f32(kind, slots, plan.t, plan.nb, plan.passes, plan.spread)
                       : dt == CORAL_BF16 ? coral_w4_held_bf16(kind, slots, plan.t, plan.nb, plan.passes, plan.spread)
                                          : coral_w4_held_f16(kind, slots, plan.t, plan.nb, plan.passes, plan.spread);
    // as many workgroups as stay resident: their registers allow four, two or one a compute unit (one token,
    // 128256 rows, one, two and four (us): 1024 columns 33, 22, 20; 4096 57, 52, 54; 8192 94, 98, 105)
    const int regs = w4_held_regs(dt == CORAL_F32 && !plan.spread, plan.t, plan.nb);
    const int tiles = (N - 1) / 16 + 1, groups = (M - 1) / w4_held_tokens(plan.spread, plan.t) + 1, most = 256 * (regs <= 2 ? 4 : regs <= 4 ? 2 : 1) / groups;
    hipLaunchKernelGGL(reinterpret_cast<w4_fn>(const_cast<void*>(held)), dim3(tiles < most ? tiles : most, groups), dim3(kW4Block), 0, stream, p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}
