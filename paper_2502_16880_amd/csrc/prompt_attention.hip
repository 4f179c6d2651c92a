// Entry point of causal attention over whole prompts (kernels: prompt_attention.h).
#include "prompt_attention.h"

#include <math.h>

namespace {

// Groups of waves share a workgroup's keys where the card has few rows, which do not see very few keys: where each compute unit has a
// tile of rows at most, and for one prompt, whose long tiles go with short ones, where it has up to about two.  Measured by tiles of 128
// (fp32: 64) rows over all heads, us with one group and with several:
//   16 bits, one prompt, D = 64   192 30.0 23.7   384 54.7 43.2   441 82.8 72.4   480 72.0 60.6   560 78 75   756 138 144
//                        D = 128  96 11.8 11.7   256 25.8 22.9   384 38.3 34.5   420 47.2 45.6   544 55.4 60.6   1056 170 180
//                        D = 256  136 76 56   256 135 109   280 148 136   304 161 160   336 179 193   504 304 376
//            several, D = 64      576 20.9 23.5, D = 128 480 20.6 22.7, behind older keys 352 37.6 39.8, D = 256 232 61.7 43.7   328 63.7 61.9
//   fp32, one prompt, D = 64      182 45.6 28.7   288 89 53   756 315 242   1512 933 887
//                     D = 128     160 33.5 22.2   352 79 66   520 479 369   768 196 225
//                     D = 256     32 39.8 31.5   128 167 105   272 345 264   504 694 809
// (two groups of as many rows for 16 bits, of 64 for D = 256; for fp32 four of 32, two for D = 256).  A prompt of 100 tokens took 10.2
// for 9.8 us in two groups, twenty of 200 in fp32 42 for 29, where a group of most has no keys.
constexpr int64_t kFewUnits = 256, kFewUnitsOnePrompt = 400, kFewUnitsOnePromptNarrow = 600, kFewUnitsOnePromptWide = 300;
constexpr int kFewKeys = 128;
bool few_rows(int64_t units, int T, int keys, int S, int head_dim, bool f32) {
    if (keys / S < kFewKeys) return false;
    if (S > 1 || keys / 2 >= T) return units <= kFewUnits;
    if (head_dim == 256 && !f32) return units <= kFewUnitsOnePromptWide;
    return units <= (head_dim == 64 || (f32 && head_dim == 128) ? kFewUnitsOnePromptNarrow : kFewUnitsOnePrompt);
}
constexpr int64_t kMostStride = 1 << 24;         // bytes: a tile's rows are addressed by 32-bit offsets

using prompt_fn = void (*)(PromptParams);
struct PromptForm {
    prompt_fn fn;
    int rows, threads;
};
template <int DT>
PromptForm prompt_form(int d, bool few) {
    if (d == 64) return few ? PromptForm{k_prompt<DT, 64, 4, 2>, 128, 512} : PromptForm{k_prompt<DT, 64, 4, 1>, 128, 256};
    if (d == 128) return few ? PromptForm{k_prompt<DT, 128, 4, 2>, 128, 512} : PromptForm{k_prompt<DT, 128, 4, 1>, 128, 256};
    return few ? PromptForm{k_prompt<DT, 256, 2, 2>, 64, 256} : PromptForm{k_prompt<DT, 256, 4, 1>, 128, 256};
}
PromptForm prompt_form(coral_dtype dt, int d, bool few) {
    if (dt == CORAL_F32) {
        if (few) return d == 64 ? PromptForm{k_prompt_f32<64, 2, 4>, 32, 512} : d == 128 ? PromptForm{k_prompt_f32<128, 2, 4>, 32, 512} : PromptForm{k_prompt_f32<256, 2, 2>, 32, 256};
        return {d == 64 ? k_prompt_f32<64, 4, 1> : d == 128 ? k_prompt_f32<128, 4, 1> : k_prompt_f32<256, 4, 1>, 64, 256};
    }
    return dt == CORAL_BF16 ? prompt_form<kBF16>(d, few) : prompt_form<kF16>(d, few);
}

}  // namespace

extern "C" coral_status coral_attention_prompt(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                               const int32_t* q_offsets, const int32_t* k_offsets, int T, int keys, int S, int q_heads,
                                               int kv_heads, int head_dim, float scale, coral_dtype dt, void* out, void* hip_stream) {
    if (!storage_known(dt) || T < 0 || keys < 0 || S < 1 || q_heads < 1 || kv_heads < 1 || head_dim < 1 || !isfinite(scale)) return CORAL_ERR_SHAPE;
    if (q_heads % kv_heads || (!k_offsets && keys != T)) return CORAL_ERR_SHAPE;
    if (!head_dim_known(head_dim) || q_heads > kMostHeads || S > kMostSequences) return CORAL_ERR_UNSUPPORTED;
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
    const int not_full = S < T || S > kPromptLevelled ? S : T;       // each sequence has at most one tile that is not full
    const bool f32 = dt == CORAL_F32;
    const bool few = few_rows((T / (f32 ? 64ll : 128ll) + not_full) * q_heads, T, keys, S, head_dim, f32);
    const PromptForm form = prompt_form(dt, head_dim, few);
    const int rows = form.rows;
    const int64_t tiles = T / rows + not_full;
    int parts = 1;
    while (q_heads * parts % kXcds) parts *= 2;
    const int64_t units = (tiles + parts - 1) / parts * q_heads * parts;
    if (units * form.threads > UINT32_MAX) return CORAL_ERR_UNSUPPORTED;
    p.q = static_cast<const char*>(q); p.k = static_cast<const char*>(k); p.v = static_cast<const char*>(v);
    p.out = static_cast<char*>(out);
    p.q_stride = in_q.stride; p.k_stride = in_k.stride; p.v_stride = in_v.stride; p.out_stride = out_rows.stride;
    p.q_offsets = q_offsets; p.k_offsets = k_offsets;
    p.T = T; p.keys = keys; p.S = S; p.q_heads = q_heads; p.group = q_heads / kv_heads; p.tiles = (int)tiles; p.parts = parts;
    p.scale_log2 = score_scale(scale);
    p.q_sign = score_sign(scale, dt);
    hipLaunchKernelGGL(form.fn, dim3((unsigned)units), dim3(form.threads), 0,
                       static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}
