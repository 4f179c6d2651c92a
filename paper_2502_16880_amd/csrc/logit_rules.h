// Rules on a step's logits, and the k best tokens under them.
//
// For every token id of a row, in this order and each operation rounded to fp32 by itself:
//   repetition  z > 0 ? z / r : z * r     where the id is in the row's prompt or output
//   frequency   z - count * f             count: how often the id is in the row's output
//   presence    z - p                     where count > 0
//   bias        z + b                     the last entry of the id in the row's list of biases
//   mask        -inf                      where the id's bit is 0
// A workgroup takes a slice of a row.  Its logits go to registers; the row's tokens are read once and
// those of the slice counted in LDS with integer atomics (their order does not matter), then the
// biases' places are marked the same way.  So neither a count array in memory nor a second pass over
// the logits is needed, and rows of any number share their prompts by reading the same range.
#pragma once
#include "buffer_loads.h"
#include "wave_topk.h"

namespace {

struct RuleParams {
    const void* logits;         // [M,V] storage type
    const int32_t* history;     // [n_history]
    const int32_t* ranges;      // [M,4]: prompt begin, end, output begin, end
    const float* penalties;     // [M,3]: repetition, frequency, presence
    const int32_t* bias_ids;    // [n_biases]
    const float* bias_values;   // [n_biases]
    const int32_t* bias_ranges; // [M,2]
    const unsigned* mask;       // [M,mask_words]
    int n_history, n_biases, mask_words;
    int M, V;
};

constexpr int kRuleWaves = 4;
constexpr int kRuleThreads = kRuleWaves * kWave;
constexpr int kRulePerLane = 16;                            // values a lane holds of a batch
constexpr int kRuleBatch = kRulePerLane * kWave;            // 1024
constexpr int kRuleAhead = 4;                               // loads of four tokens that a thread has on their way
constexpr unsigned kInPrompt = 0x80000000u;                 // the rest of a word counts the output

template <int DT>
constexpr int kRuleVec = DT == kF32 ? 4 : 8;                // values of a 16-byte vector

// A row's values are dealt in whole 16-byte vectors of memory: place j of a row is token id j - lead,
// where lead values before the row's first share its first vector.
template <int DT>
__device__ __forceinline__ int row_lead(int m, int V) {
    return (int)(((size_t)m * V) % kRuleVec<DT>);
}

// First place of vector u of a lane: batch by batch, consecutive lanes on consecutive vectors.
template <int DT, int NB>
__device__ __forceinline__ int vec_place(int first, int wave, int lane, int u) {
    constexpr int E = kRuleVec<DT>, U = kRulePerLane / E;
    return first + ((wave * NB + u / U) * U + u % U) * (kWave * E) + lane * E;
}

// The lane's logits of the slice, as they lie in memory, and the mask bits that go with them (the words
// of a vector's first and last value; values of the row's neighbours among them are dropped later).
template <int DT, int NB>
struct SliceData {
    static constexpr int kVecs = NB * kRulePerLane / kRuleVec<DT>;
    uint4 v[kVecs];
    unsigned lo[kVecs], hi[kVecs];
};
template <int DT, int NB>
__device__ __forceinline__ void load_slice(const RuleParams& p, int m, int lead, int first, int wave, int lane, SliceData<DT, NB>& d) {
    constexpr size_t W = DT == kF32 ? 4 : 2;
    const Buffer logits = buffer_view(p.logits, ((size_t)m * p.V - lead) * W, (size_t)p.M * p.V * W);
#pragma unroll
    for (int u = 0; u < d.kVecs; ++u) d.v[u] = buffer_read16<kBufferStream>(logits, (unsigned)(vec_place<DT, NB>(first, wave, lane, u) * W));
    if (p.mask) {                                            // uniform
        const Buffer mask = buffer_view(p.mask, (size_t)m * p.mask_words * 4, (size_t)p.M * p.mask_words * 4);
#pragma unroll
        for (int u = 0; u < d.kVecs; ++u) {
            const int id = vec_place<DT, NB>(first, wave, lane, u) - lead;       // (before the row: dropped, as behind the end)
            d.lo[u] = buffer_read4(mask, (unsigned)(id >> 5) * 4u);
            d.hi[u] = buffer_read4(mask, (unsigned)((id + kRuleVec<DT> - 1) >> 5) * 4u);
        }
    }
}

// The values as fp32; -inf for those that are not the row's.
template <int DT, int NB>
__device__ __forceinline__ void slice_values(const RuleParams& p, int m, int lead, int first, int wave, int lane, const SliceData<DT, NB>& d,
                                             float (&z)[NB * kRulePerLane]) {
    constexpr int E = kRuleVec<DT>, SLICE = NB * kRuleBatch * kRuleWaves;
#pragma unroll
    for (int u = 0; u < d.kVecs; ++u) {
        const unsigned w[4] = {d.v[u].x, d.v[u].y, d.v[u].z, d.v[u].w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (DT == kF32) z[u * E + e] = __uint_as_float(w[e]);
            else z[u * E + e] = widen16<DT>((unsigned short)(w[e / 2] >> (e % 2 * 16)));
        }
    }
    if (first < lead || first + SLICE > p.V + lead) {        // uniform: the row's first or last slice
        // (half a dword at the very end of the operand is dropped by the load of a vector)
        float end = 0.f;
        if constexpr (DT != kF32) end = widen16<DT>(static_cast<const unsigned short*>(p.logits)[(size_t)p.M * p.V - 1]);
#pragma unroll
        for (int u = 0; u < d.kVecs; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int id = vec_place<DT, NB>(first, wave, lane, u) - lead + e;
                if (DT != kF32 && id == p.V - 1 && m == p.M - 1) z[u * E + e] = end;
                z[u * E + e] = id >= 0 && id < p.V ? z[u * E + e] : -INFINITY;
            }
    }
}

// A range of a flat array of n <= 2^30 entries, cut to it: 0 <= begin <= end <= n whatever the caller's
// arrays hold (a begin beyond the array would overflow where threads count on from it).
struct Span {
    int begin, end;
};
__device__ __forceinline__ Span clamp_span(int begin, int end, int n) {
    begin = begin < 0 ? 0 : begin > n ? n : begin;
    end = end > n ? n : end < begin ? begin : end;
    return {begin, end};
}

__device__ __forceinline__ float rule_penalty(float z, unsigned seen, float rep, float freq, float pres) {
#pragma clang fp contract(off)
    if (seen == 0u) return z;
    z = z > 0.f ? z / rep : z * rep;
    const unsigned count = seen & ~kInPrompt;
    const float taken = (float)count * freq;
    z = z - taken;
    return count != 0u ? z - pres : z;
}

// Applies the rules to the lane's values.  words: one LDS word per place of the slice.  Every thread
// of the workgroup comes here; barriers are reached by all.
template <int DT, int NB>
__device__ __forceinline__ void apply_rules(const RuleParams& p, int m, int lead, int first, int wave, int lane,
                                            unsigned* words, const SliceData<DT, NB>& d, float (&z)[NB * kRulePerLane]) {
    constexpr int E = kRuleVec<DT>, VECS = NB * kRulePerLane / E, SLICE = NB * kRuleBatch * kRuleWaves;
    auto clear = [&]() {
        for (int i = threadIdx.x; i < SLICE; i += kRuleThreads) words[i] = 0u;
        __syncthreads();
    };
    if (p.ranges) {                                          // uniform
        clear();
        const int32_t* r = p.ranges + (size_t)m * 4;
        const float rep = p.penalties[m * 3], freq = p.penalties[m * 3 + 1], pres = p.penalties[m * 3 + 2];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            // the tokens four at a time, several loads on their way; behind the range: token -1
            const Span s = clamp_span(r[2 * which], r[2 * which + 1], p.n_history);
            const Buffer tokens = buffer_view(p.history, (size_t)s.begin * 4, (size_t)s.end * 4);
            const int n = s.end - s.begin;
            for (int i = 0; i < n; i += kRuleThreads * 4 * kRuleAhead) {         // uniform
                uint4 t[kRuleAhead];
#pragma unroll
                for (int a = 0; a < kRuleAhead; ++a) t[a] = buffer_read16(tokens, (unsigned)(i + (a * kRuleThreads + (int)threadIdx.x) * 4) * 4u);
#pragma unroll
                for (int a = 0; a < kRuleAhead; ++a) {
                    const unsigned id[4] = {t[a].x, t[a].y, t[a].z, t[a].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned at = id[e] + (unsigned)(lead - first);
                        const bool in = i + (a * kRuleThreads + (int)threadIdx.x) * 4 + e < n;
                        if (in && at < (unsigned)SLICE && id[e] < (unsigned)p.V) {
                            if (which == 0) atomicOr(words + at, kInPrompt);
                            else atomicAdd(words + at, 1u);
                        }
                    }
                }
            }
        }
        __syncthreads();
        slice_values<DT, NB>(p, m, lead, first, wave, lane, d, z);
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int at = vec_place<DT, NB>(0, wave, lane, u);
#pragma unroll
            for (int e = 0; e < E; ++e) z[u * E + e] = rule_penalty(z[u * E + e], words[at + e], rep, freq, pres);
        }
        __syncthreads();
    } else {
        slice_values<DT, NB>(p, m, lead, first, wave, lane, d, z);
    }
    if (p.bias_ranges) {                                     // uniform
        clear();
        const Span s = clamp_span(p.bias_ranges[(size_t)m * 2], p.bias_ranges[(size_t)m * 2 + 1], p.n_biases);
        for (int i = s.begin + (int)threadIdx.x; i < s.end; i += kRuleThreads) {
            const int id = p.bias_ids[i];
            const unsigned at = (unsigned)id + (unsigned)(lead - first);
            if (id >= 0 && id < p.V && at < (unsigned)SLICE) atomicMax(words + at, (unsigned)(i + 1));    // the last entry stays
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int at = vec_place<DT, NB>(0, wave, lane, u);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const unsigned w = words[at + e];
                if (w != 0u) z[u * E + e] += p.bias_values[w - 1u];
            }
        }
    }
    if (p.mask) {                                            // uniform
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int id = vec_place<DT, NB>(first, wave, lane, u) - lead;
            const unsigned bits = __builtin_amdgcn_alignbit(d.hi[u], d.lo[u], (unsigned)(id & 31));
#pragma unroll
            for (int e = 0; e < E; ++e) z[u * E + e] = bits >> e & 1u ? z[u * E + e] : -INFINITY;
        }
    }
}

// The logits under their rules, rounded to the storage type.
template <int DT, int NB>
__global__ __launch_bounds__(kRuleThreads) void k_logits_adjust(RuleParams p, void* out) {
    constexpr int E = kRuleVec<DT>, VECS = NB * kRulePerLane / E, SLICE = NB * kRuleBatch * kRuleWaves;
    __shared__ __attribute__((aligned(16))) unsigned words[SLICE];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int m = blockIdx.y, lead = row_lead<DT>(m, p.V), first = blockIdx.x * SLICE;
    SliceData<DT, NB> d;
    load_slice<DT, NB>(p, m, lead, first, wave, lane, d);
    float z[NB * kRulePerLane];
    apply_rules<DT, NB>(p, m, lead, first, wave, lane, words, d, z);
    const size_t row = (size_t)m * p.V;
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        const int id = vec_place<DT, NB>(first, wave, lane, u) - lead;
        if (id >= 0 && id + E <= p.V) {
            uint4 v;
            if constexpr (DT == kF32) {
                v = make_uint4(__float_as_uint(z[u * 4]), __float_as_uint(z[u * 4 + 1]), __float_as_uint(z[u * 4 + 2]),
                               __float_as_uint(z[u * 4 + 3]));
                store_vec(reinterpret_cast<uint4*>(static_cast<float*>(out) + row + id), v);
            } else {
                unsigned w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = (unsigned)narrow16<DT>(z[u * 8 + 2 * e]) | (unsigned)narrow16<DT>(z[u * 8 + 2 * e + 1]) << 16;
                v = make_uint4(w[0], w[1], w[2], w[3]);
                store_vec(reinterpret_cast<uint4*>(static_cast<unsigned short*>(out) + row + id), v);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (id + e >= 0 && id + e < p.V) {
                    if constexpr (DT == kF32) static_cast<float*>(out)[row + id + e] = z[u * E + e];
                    else static_cast<unsigned short*>(out)[row + id + e] = narrow16<DT>(z[u * E + e]);
                }
        }
    }
}

// ---------------------------------------------------------------- k best tokens
// Running log-sum-exp: the largest value and the sum of exp(z - largest); (-inf, 0) for no value.
struct ExpSum {
    float top, sum;
};
__device__ __forceinline__ ExpSum join(ExpSum a, ExpSum b) {
    const float top = fmaxf(a.top, b.top);
    if (top == -INFINITY) return {top, 0.f};
    return {top, a.sum * expf(a.top - top) + b.sum * expf(b.top - top)};
}

struct TopkParams {
    Cand* part;                 // [M][slices][k] published lists
    unsigned long long* sums;   // [M][slices] published (largest, sum)
    unsigned* arrived;          // [M] counters, zero between calls
    int32_t* ids;               // [M,k]
    float* logprob;             // [M,k]
    int k, slices;
};

constexpr int kRuleMaxBatches = 2;
constexpr int kTopkLists = kRuleWaves * kRuleMaxBatches;

template <int DT, int NB>
__global__ __launch_bounds__(kRuleThreads) void k_logits_topk(RuleParams p, TopkParams t) {
    constexpr int SLICE = NB * kRuleBatch * kRuleWaves;
    __shared__ union {
        __attribute__((aligned(16))) unsigned words[SLICE];
        struct {
            __attribute__((aligned(16))) unsigned long long buf[kRuleWaves][kWave];
            unsigned long long lists[NB * kRuleWaves * kMaxK];
            MergeScratch merge;
        } s;
    } lds;
    __shared__ ExpSum wave_sums[kRuleWaves];
    __shared__ ExpSum row_sum;
    __shared__ int last;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int m = blockIdx.y, lead = row_lead<DT>(m, p.V), slice = blockIdx.x, first = slice * SLICE, k = t.k;
    SliceData<DT, NB> d;
    load_slice<DT, NB>(p, m, lead, first, wave, lane, d);
    float z[NB * kRulePerLane];
    apply_rules<DT, NB>(p, m, lead, first, wave, lane, lds.words, d, z);
    __syncthreads();                                         // the words' memory is taken again below
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NB * kRulePerLane; ++i) {
        z[i] = z[i] != z[i] ? -INFINITY : z[i];              // NaN is no candidate
        top = fmaxf(top, z[i]);
    }
    top = wave_max(top);
    float sum = 0.f;
    if (top != -INFINITY) {                                  // wave-uniform
#pragma unroll
        for (int i = 0; i < NB * kRulePerLane; ++i) sum += expf(z[i] - top);
    }
    sum = wave_sum(sum);
    if (lane == 0) wave_sums[wave] = {top, sum};
    constexpr int E = kRuleVec<DT>;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        unsigned long long key[kRulePerLane];
#pragma unroll
        for (int i = 0; i < kRulePerLane; ++i) {
            const int at = b * kRulePerLane + i;
            const int id = vec_place<DT, NB>(first, wave, lane, at / E) - lead + at % E;
            key[i] = z[at] != -INFINITY ? cand_key(z[at], id) : 0ull;
        }
        unsigned long long* list = lds.s.lists + (wave * NB + b) * k;
        wave_topk<kRulePerLane>(key, k, lane, lds.s.buf[wave], [&](int r, unsigned long long c) { list[r] = c; });
    }
    __syncthreads();
    Cand* part = t.part + ((size_t)m * t.slices) * k;
    if (wave == 0) {
        wave_topk_lds(lds.s.lists, kRuleWaves * NB * k, k, lane, lds.s.buf[0], [&](int r, unsigned long long c) {
            const Cand cand = key_cand(c);
            publish_cand(part + (size_t)slice * k + r, cand.v, cand.id);
        });
        if (lane == 0) {
            ExpSum s = wave_sums[0];
#pragma unroll
            for (int w = 1; w < kRuleWaves; ++w) s = join(s, wave_sums[w]);
            const unsigned long long bits =
                (unsigned long long)__float_as_uint(s.top) << 32 | (unsigned long long)__float_as_uint(s.sum);
            __hip_atomic_store(t.sums + (size_t)m * t.slices + slice, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wave's stores are out
        asm volatile("" ::: "memory");
        if (lane == 0) {
            const unsigned old = __hip_atomic_fetch_add(t.arrived + m, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = old == (unsigned)t.slices - 1u ? 1 : 0;
        }
    }
    __syncthreads();
    if (!last) return;                                       // uniform
    if (wave == 1) {                                         // the row's log-sum-exp, in an order of its own
        ExpSum s = {-INFINITY, 0.f};
        for (int i = lane; i < t.slices; i += kWave) {
            const unsigned long long bits =
                __hip_atomic_load(t.sums + (size_t)m * t.slices + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s = join(s, {__uint_as_float((unsigned)(bits >> 32)), __uint_as_float((unsigned)bits)});
        }
        const float row_top = wave_max(s.top);
        const float row = wave_sum(s.top == -INFINITY ? 0.f : s.sum * expf(s.top - row_top));
        if (lane == 0) row_sum = {row_top, row};
    }
    __syncthreads();
    if (wave != 0) return;
    // (z - largest) - log(sum): z - (largest + log(sum)) would lose the sum where values are far from zero
    const float row_top = row_sum.top, log_sum = logf(row_sum.sum);
    if (lane == 0) __hip_atomic_store(t.arrived + m, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    wave_merge_lists(t.slices, k, lane, &lds.s.merge, [&](int l, int i) { return fetch_cand(part + (size_t)l * k + i); },
                     [&](int r, unsigned long long c) {
                         const Cand cand = key_cand(c);
                         t.ids[(size_t)m * k + r] = is_real(cand) ? cand.id : -1;
                         t.logprob[(size_t)m * k + r] = is_real(cand) ? (cand.v - row_top) - log_sum : -INFINITY;
                     });
}

}  // namespace
