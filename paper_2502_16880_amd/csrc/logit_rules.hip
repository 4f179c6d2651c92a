// Entry points of the rules on logits (kernels: logit_rules.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "control_words.h"
#include "coral_lmhead.h"
#include "device_utils.h"
#include "logit_rules.h"

namespace {

constexpr size_t kLists = coral_ctrl::kPreparedWords * sizeof(unsigned);     // published lists start behind the control words
constexpr int kMaxList = 1 << 29;                                            // entries of the flat lists

size_t align_256(size_t x) { return (x + 255) / 256 * 256; }

int slices(int V) { return (V + 7 + kRuleSlice - 1) / kRuleSlice; }          // up to seven values lead a row

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + b_bytes && y < x + a_bytes;
}

coral_status check_rules(const void* logits, const coral_logit_rules* r, int M, int V, coral_dtype dt, RuleParams* p) {
    if (!logits) return CORAL_ERR_NULL;
    if (dt != CORAL_F32 && dt != CORAL_BF16 && dt != CORAL_F16) return CORAL_ERR_SHAPE;
    if (M < 1 || V < 1) return CORAL_ERR_SHAPE;
    if (M > kMaxM || V > CORAL_LOGITS_MAX_V) return CORAL_ERR_UNSUPPORTED;
    if ((uintptr_t)logits & 15u) return CORAL_ERR_UNSUPPORTED;
    *p = RuleParams{};
    p->logits = logits;
    p->M = M;
    p->V = V;
    if (!r) return CORAL_OK;
    if (r->n_history < 0 || r->n_biases < 0) return CORAL_ERR_SHAPE;
    if (r->history_ranges) {
        if (!r->penalties || (r->n_history > 0 && !r->history)) return CORAL_ERR_NULL;
        if (((uintptr_t)r->history | (uintptr_t)r->history_ranges | (uintptr_t)r->penalties) & 3u) return CORAL_ERR_UNSUPPORTED;
        if (r->n_history > kMaxList) return CORAL_ERR_UNSUPPORTED;
        p->history = r->history;
        p->ranges = r->history_ranges;
        p->penalties = r->penalties;
        p->n_history = r->n_history;
    } else if (r->history || r->penalties) {
        return CORAL_ERR_NULL;
    }
    if (r->bias_ranges) {
        if (r->n_biases > 0 && (!r->bias_ids || !r->bias_values)) return CORAL_ERR_NULL;
        if (((uintptr_t)r->bias_ids | (uintptr_t)r->bias_values | (uintptr_t)r->bias_ranges) & 3u) return CORAL_ERR_UNSUPPORTED;
        if (r->n_biases > kMaxList) return CORAL_ERR_UNSUPPORTED;
        p->bias_ids = r->bias_ids;
        p->bias_values = r->bias_values;
        p->bias_ranges = r->bias_ranges;
        p->n_biases = r->n_biases;
    } else if (r->bias_ids || r->bias_values) {
        return CORAL_ERR_NULL;
    }
    if (r->mask) {
        if ((uintptr_t)r->mask & 3u) return CORAL_ERR_UNSUPPORTED;
        p->mask = r->mask;
        p->mask_words = (V + 31) / 32;
    }
    return CORAL_OK;
}

// Whether [at, at + bytes) touches memory that the rules are read from.
bool touches_rules(const RuleParams& p, const void* at, size_t bytes) {
    return overlap(at, bytes, p.history, (size_t)p.n_history * 4) || overlap(at, bytes, p.ranges, (size_t)p.M * 16) ||
           overlap(at, bytes, p.penalties, (size_t)p.M * 12) || overlap(at, bytes, p.bias_ids, (size_t)p.n_biases * 4) ||
           overlap(at, bytes, p.bias_values, (size_t)p.n_biases * 4) || overlap(at, bytes, p.bias_ranges, (size_t)p.M * 8) ||
           overlap(at, bytes, p.mask, (size_t)p.M * p.mask_words * 4);
}

struct TopkLayout {
    size_t sums, total;
};
TopkLayout topk_layout(int M, int n_slices, int k) {
    const size_t sums = align_256(kLists + (size_t)M * n_slices * k * sizeof(Cand));
    return {sums, align_256(sums + (size_t)M * n_slices * sizeof(unsigned long long))};
}

}  // namespace

static_assert(coral_ctrl::kRowArrivalStride * kMaxM <= coral_ctrl::kGateScoreWords, "one arrival counter per row");
static_assert((CORAL_LOGITS_MAX_V + 7 + kRuleSlice - 1) / (kRuleSlice) <= kMaxSlices, "");

extern "C" coral_status coral_logits_adjust(const void* logits, const coral_logit_rules* rules, int M, int V,
                                            coral_dtype dt, void* out, void* hip_stream) {
    RuleParams p;
    const coral_status st = check_rules(logits, rules, M, V, dt, &p);
    if (st != CORAL_OK) return st;
    if (!out) return CORAL_ERR_NULL;
    if ((uintptr_t)out & 15u) return CORAL_ERR_UNSUPPORTED;
    const size_t bytes = (size_t)M * V * (dt == CORAL_F32 ? 4 : 2);
    if ((out != logits && overlap(out, bytes, logits, bytes)) || touches_rules(p, out, bytes)) return CORAL_ERR_UNSUPPORTED;
    const dim3 grid(slices(V), M), block(kRuleThreads);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == CORAL_F32) hipLaunchKernelGGL(k_logits_adjust<kF32>, grid, block, 0, stream, p, out);
    else if (dt == CORAL_BF16) hipLaunchKernelGGL(k_logits_adjust<kBF16>, grid, block, 0, stream, p, out);
    else hipLaunchKernelGGL(k_logits_adjust<kF16>, grid, block, 0, stream, p, out);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}

extern "C" size_t coral_logits_topk_workspace_bytes(int M, int V, int k) {
    if (M < 1 || V < 1 || k < 1 || k > V || M > kMaxM || k > kMaxK || V > CORAL_LOGITS_MAX_V) return 0;
    return topk_layout(M, slices(V), k).total;               // it serves fewer rows too
}

extern "C" coral_status coral_logits_topk(const void* logits, const coral_logit_rules* rules, int M, int V, int k,
                                          coral_dtype dt, int32_t* topk_ids, float* topk_logprob, void* workspace,
                                          size_t workspace_bytes, void* hip_stream) {
    RuleParams p;
    const coral_status st = check_rules(logits, rules, M, V, dt, &p);
    if (st != CORAL_OK) return st;
    if (!topk_ids || !topk_logprob) return CORAL_ERR_NULL;
    if (k < 1 || k > V) return CORAL_ERR_SHAPE;
    if (k > kMaxK) return CORAL_ERR_UNSUPPORTED;
    if (((uintptr_t)topk_ids | (uintptr_t)topk_logprob) & 3u) return CORAL_ERR_UNSUPPORTED;
    const int n_slices = slices(V);
    const TopkLayout L = topk_layout(M, n_slices, k);
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < L.total) return CORAL_ERR_WORKSPACE;
    const size_t out_bytes = (size_t)M * k * 4, in_bytes = (size_t)M * V * (dt == CORAL_F32 ? 4 : 2);
    for (const void* o : {(const void*)topk_ids, (const void*)topk_logprob})
        if (overlap(o, out_bytes, logits, in_bytes) || touches_rules(p, o, out_bytes) || overlap(o, out_bytes, workspace, L.total))
            return CORAL_ERR_UNSUPPORTED;
    if (overlap(topk_ids, out_bytes, topk_logprob, out_bytes) || overlap(workspace, L.total, logits, in_bytes) ||
        touches_rules(p, workspace, L.total))
        return CORAL_ERR_UNSUPPORTED;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    TopkParams t = {};
    t.part = reinterpret_cast<Cand*>(ws + kLists);
    t.sums = reinterpret_cast<unsigned long long*>(ws + L.sums);
    t.arrived = reinterpret_cast<unsigned*>(ws) + coral_ctrl::kRowArrival;
    t.ids = topk_ids;
    t.logprob = topk_logprob;
    t.k = k;
    t.slices = n_slices;
    const dim3 grid(n_slices, M), block(kRuleThreads);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == CORAL_F32) hipLaunchKernelGGL(k_logits_topk<kF32>, grid, block, 0, stream, p, t);
    else if (dt == CORAL_BF16) hipLaunchKernelGGL(k_logits_topk<kBF16>, grid, block, 0, stream, p, t);
    else hipLaunchKernelGGL(k_logits_topk<kF16>, grid, block, 0, stream, p, t);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}
