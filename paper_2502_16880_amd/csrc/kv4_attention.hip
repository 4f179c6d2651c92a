// Entry point of attention over the 4-bit cache (kernels: kv4_attention.h).
#include "kv4_attention.h"

#include <math.h>

#include <initializer_list>

#include "kv4_kernels.h"

namespace {

// Sizes that the plan is made of; false where one is out of range.
coral_status check_kv4_sizes(int T, int S, int max_rows, int max_length, int q_heads, int kv_heads, int head_dim, coral_dtype dt) {
    if (!storage_known(dt) || T < 0 || S < 1 || max_rows < 1 || max_length < 0 || q_heads < 1 || kv_heads < 1 || head_dim < 1) return CORAL_ERR_SHAPE;
    if (q_heads % kv_heads) return CORAL_ERR_SHAPE;
    if (!head_dim_known(head_dim) || q_heads > kMostHeads || S > kMostSequences || max_rows > kKv4MostRows) return CORAL_ERR_UNSUPPORTED;
    return CORAL_OK;
}
int query_terms(coral_dtype dt) { return dt == CORAL_F32 ? 3 : 1; }

}  // namespace

extern "C" size_t coral_attention_kv4_workspace_bytes(int S, int max_rows, int max_length, int q_heads, int kv_heads, int head_dim,
                                                      coral_dtype dt) {
    if (check_kv4_sizes(0, S, max_rows, max_length, q_heads, kv_heads, head_dim, dt) != CORAL_OK) return 0;
    const size_t n = kv4_workspace(kv4_plan(S, max_rows, max_length, q_heads, kv_heads, head_dim, query_terms(dt)), head_dim);
    return n < 256 ? 256 : (n + 255) / 256 * 256;
}

extern "C" coral_status coral_attention_kv4(const void* q, int64_t q_stride, const coral_kv4_cache* cache, const int32_t* page_table,
                                            int max_pages, const int32_t* lengths, const int32_t* q_offsets, const int32_t* history,
                                            const uint64_t* tree, int T, int S, int max_rows, int max_length, int q_heads, float scale,
                                            coral_dtype dt, void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
    Kv4AttnParams p = {};
    coral_status st = check_kv4(cache, &p.cache);
    if (st != CORAL_OK) return st;
    const int kv_heads = cache->kv_heads, head_dim = cache->head_dim;
    if ((st = check_kv4_sizes(T, S, max_rows, max_length, q_heads, kv_heads, head_dim, dt)) != CORAL_OK) return st;
    if (max_pages < 0 || !isfinite(scale)) return CORAL_ERR_SHAPE;
    if ((tree == nullptr) != (history == nullptr)) return CORAL_ERR_NULL;
    if (T == 0) return CORAL_OK;
    Rows in_q, out_rows, parts[4];
    if ((st = check_rows(q, q_stride, q_heads, head_dim, dt, T, &in_q)) != CORAL_OK) return st;
    if ((st = check_rows(out, (int64_t)q_heads * head_dim, q_heads, head_dim, dt, T, &out_rows)) != CORAL_OK) return st;
    if ((max_pages > 0 && !page_table) || !lengths || !q_offsets) return CORAL_ERR_NULL;
    if (((uintptr_t)page_table | (uintptr_t)lengths | (uintptr_t)q_offsets | (uintptr_t)history) & 3u) return CORAL_ERR_UNSUPPORTED;
    if ((uintptr_t)tree & 7u) return CORAL_ERR_UNSUPPORTED;
    const Kv4Plan plan = kv4_plan(S, max_rows, max_length, q_heads, kv_heads, head_dim, query_terms(dt));
    if ((int64_t)kv_heads * plan.row_blocks > 65535) return CORAL_ERR_UNSUPPORTED;
    const size_t need = kv4_workspace(plan, head_dim);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return CORAL_ERR_WORKSPACE;
    kv4_parts(cache, parts);
    auto whole = [](const void* base, int64_t bytes) { return Rows{base, bytes, bytes, 1}; };
    const Rows inputs[10] = {in_q, parts[0], parts[1], parts[2], parts[3], whole(page_table, (int64_t)S * max_pages * 4), whole(lengths, S * 4ll),
                             whole(q_offsets, (S + 1) * 4ll), whole(history, S * 4ll), whole(tree, T * 8ll)};
    const Rows scratch = whole(need ? workspace : nullptr, (int64_t)need);
    for (const Rows& r : inputs)
        if (rows_overlap(out_rows, r) || rows_overlap(scratch, r)) return CORAL_ERR_UNSUPPORTED;
    if (rows_overlap(out_rows, scratch)) return CORAL_ERR_UNSUPPORTED;
    p.q = static_cast<const char*>(q);
    p.out = static_cast<char*>(out);
    p.q_stride = in_q.stride;
    p.out_stride = out_rows.stride;
    p.page_table = page_table; p.lengths = lengths; p.q_offsets = q_offsets; p.history = history; p.tree = tree;
    p.max_pages = max_pages; p.T = T; p.S = S; p.max_rows = max_rows; p.group = q_heads / kv_heads; p.kv_heads = kv_heads;
    p.workgroups = plan.workgroups; p.apart = plan.apart; p.join_inside = plan.join_inside;
    p.scale_log2 = score_scale(scale);
    p.q_sign = score_sign(scale, dt);
    if (need) {
        const size_t rows = (size_t)plan.workgroups * 2 * 16 * plan.tiles;
        static_assert(kKv4Control == coral_ctrl::kPreparedWords * sizeof(unsigned) && kKv4Control % 256 == 0, "");
        static_assert(kKv4Units * 3 * kKv4ArrivalStride <= coral_ctrl::kGateScoreWords, "a counter for each workgroup");
        p.arrived = static_cast<unsigned*>(workspace) + coral_ctrl::kGateScores;
        p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kKv4Control);
        p.part_stats = reinterpret_cast<float2*>(p.part + rows * head_dim);
    }
    const void* fn = dt == CORAL_F32 ? coral_kv4_kernel_f32(head_dim, plan.tiles) : dt == CORAL_BF16 ? coral_kv4_kernel_bf16(head_dim, plan.tiles)
                                                                                                    : coral_kv4_kernel_f16(head_dim, plan.tiles);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid = plan.apart ? dim3(kv_heads * plan.row_blocks, S) : dim3(plan.workgroups);
    hipLaunchKernelGGL(reinterpret_cast<kv4_attn_fn>(const_cast<void*>(fn)), grid, dim3(kKv4Threads), 0, stream, p);
    if (hipGetLastError() != hipSuccess) return CORAL_ERR_HIP;
    if (need && !plan.join_inside) {
        const bool one = plan.wave_a_row;
        const void* join = dt == CORAL_F32 ? coral_kv4_join_f32(head_dim, plan.tiles, one) : dt == CORAL_BF16 ? coral_kv4_join_bf16(head_dim, plan.tiles, one)
                                                                                                             : coral_kv4_join_f16(head_dim, plan.tiles, one);
        // where there are more rows than the chip holds waves, a wave takes several heads of a token, whose place it has looked up once
        const int at_once = one ? kKv4Waves : 1, groups = (q_heads + at_once - 1) / at_once;
        const int64_t heads = one ? (int64_t)T * groups / (kKv4Units * 8) : 1;
        p.join_heads = (int)(heads < 1 ? 1 : heads < groups ? heads : groups);
        hipLaunchKernelGGL(reinterpret_cast<kv4_join_fn>(const_cast<void*>(join)), dim3(T, (groups + p.join_heads - 1) / p.join_heads), dim3(kKv4Threads), 0, stream, p);
        if (hipGetLastError() != hipSuccess) return CORAL_ERR_HIP;
    }
    return CORAL_OK;
}
