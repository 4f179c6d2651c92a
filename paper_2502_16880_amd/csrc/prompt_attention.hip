// Entry point of causal attention over whole prompts (kernels: prompt_attention.h).
#include "prompt_attention.h"

#include <math.h>

namespace {

constexpr int64_t kMostStride = 1 << 24;         // bytes: a tile's rows are addressed by 32-bit offsets

using prompt_fn = void (*)(PromptParams);
prompt_fn prompt_kernel(coral_dtype dt, int d) {
    if (dt == CORAL_F32) return d == 64 ? k_prompt_f32<64> : d == 128 ? k_prompt_f32<128> : k_prompt_f32<256>;
    if (dt == CORAL_BF16) return d == 64 ? k_prompt<kBF16, 64> : d == 128 ? k_prompt<kBF16, 128> : k_prompt<kBF16, 256>;
    return d == 64 ? k_prompt<kF16, 64> : d == 128 ? k_prompt<kF16, 128> : k_prompt<kF16, 256>;
}

}  // namespace

extern "C" coral_status coral_attention_prompt(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                               const int32_t* q_offsets, const int32_t* k_offsets, int T, int keys, int S, int q_heads,
                                               int kv_heads, int head_dim, float scale, coral_dtype dt, void* out, void* hip_stream) {
    if (!storage_known(dt) || T < 0 || keys < 0 || S < 1 || q_heads < 1 || kv_heads < 1 || head_dim < 1 || !isfinite(scale)) return CORAL_ERR_SHAPE;
    if (q_heads % kv_heads || (!k_offsets && keys != T)) return CORAL_ERR_SHAPE;
    if (!head_dim_known(head_dim) || q_heads > kMostHeads) return CORAL_ERR_UNSUPPORTED;
    if (T == 0) return CORAL_OK;
    PromptParams p = {};
    Rows in_q, in_k = {}, in_v = {}, out_rows;
    coral_status st;
    if ((st = check_rows(q, q_stride, q_heads, head_dim, dt, T, &in_q)) != CORAL_OK) return st;
    if ((st = check_rows(out, (int64_t)q_heads * head_dim, q_heads, head_dim, dt, T, &out_rows)) != CORAL_OK) return st;
    if (keys > 0) {
        if ((st = check_rows(k, k_stride, kv_heads, head_dim, dt, keys, &in_k)) != CORAL_OK) return st;
        if ((st = check_rows(v, v_stride, kv_heads, head_dim, dt, keys, &in_v)) != CORAL_OK) return st;
        if (in_k.stride > kMostStride || in_v.stride > kMostStride) return CORAL_ERR_UNSUPPORTED;
    }
    if (!q_offsets) return CORAL_ERR_NULL;
    if (((uintptr_t)q_offsets | (uintptr_t)k_offsets) & 3u) return CORAL_ERR_UNSUPPORTED;
    const int64_t offsets = (S + 1ll) * 4;
    if (rows_overlap(out_rows, in_q) || rows_overlap(out_rows, in_k) || rows_overlap(out_rows, in_v) ||
        rows_overlap(out_rows, {q_offsets, offsets, offsets, 1}) || rows_overlap(out_rows, {k_offsets, offsets, offsets, 1}))
        return CORAL_ERR_UNSUPPORTED;
    const int rows = dt == CORAL_F32 ? 64 : 128;
    const int64_t tiles = T / rows + (S < T ? S : T);        // each sequence has at most one tile that is not full
    int parts = 1;
    while (q_heads * parts % kXcds) parts *= 2;
    const int64_t units = (tiles + parts - 1) / parts * q_heads * parts;
    if (units > INT32_MAX - 64) return CORAL_ERR_UNSUPPORTED;
    p.q = static_cast<const char*>(q); p.k = static_cast<const char*>(k); p.v = static_cast<const char*>(v);
    p.out = static_cast<char*>(out);
    p.q_stride = in_q.stride; p.k_stride = in_k.stride; p.v_stride = in_v.stride; p.out_stride = out_rows.stride;
    p.q_offsets = q_offsets; p.k_offsets = k_offsets;
    p.T = T; p.keys = keys; p.S = S; p.q_heads = q_heads; p.group = q_heads / kv_heads; p.tiles = (int)tiles; p.parts = parts;
    p.scale_log2 = score_scale(scale);
    p.q_sign = score_sign(scale, dt);
    hipLaunchKernelGGL(prompt_kernel(dt, head_dim), dim3((unsigned)units), dim3(kPromptThreads), 0,
                       static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}
