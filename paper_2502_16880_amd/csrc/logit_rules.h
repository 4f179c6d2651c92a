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
constexpr int kRuleAhead = 2;                               // loads of four tokens of each kind that a thread has on their way
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

// A range of a flat array of n <= 2^29 entries, cut to it: 0 <= begin <= end <= n whatever the caller's
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

// The lane's values under the rules.  words: one LDS word per place of the slice.  Every thread of the
// workgroup comes here; barriers are reached by all.
template <int DT, int NB>
__device__ __forceinline__ void slice_under_rules(const RuleParams& p, int m, int lead, int first, int wave, int lane,
                                                  unsigned* words, float (&z)[NB * kRulePerLane]) {
    constexpr int E = kRuleVec<DT>, VECS = NB * kRulePerLane / E, SLICE = NB * kRuleBatch * kRuleWaves;
    const int tid = threadIdx.x;
    // What is read depends on nothing but the ranges, and is all requested before anything is waited for.
    Span prompt = {0, 0}, output = {0, 0}, biases = {0, 0};
    float rep = 1.f, freq = 0.f, pres = 0.f;
    if (p.ranges) {                                          // uniform
        const int32_t* r = p.ranges + (size_t)m * 4;
        prompt = clamp_span(r[0], r[1], p.n_history);
        output = clamp_span(r[2], r[3], p.n_history);
        rep = p.penalties[m * 3];
        freq = p.penalties[m * 3 + 1];
        pres = p.penalties[m * 3 + 2];
    }
    if (p.bias_ranges) biases = clamp_span(p.bias_ranges[(size_t)m * 2], p.bias_ranges[(size_t)m * 2 + 1], p.n_biases);
    SliceData<DT, NB> d;
    load_slice<DT, NB>(p, m, lead, first, wave, lane, d);
    // tokens four at a time, the first ones of prompt and output together; behind the range a thread has none
    const int n_prompt = prompt.end - prompt.begin, n_output = output.end - output.begin, n_bias = biases.end - biases.begin;
    const Buffer prompts = buffer_view(p.history, (size_t)prompt.begin * 4, (size_t)prompt.end * 4);
    const Buffer outputs = buffer_view(p.history, (size_t)output.begin * 4, (size_t)output.end * 4);
    constexpr int A = kRuleAhead, TRIP = kRuleThreads * 4 * A;
    uint4 in_prompt[A], in_output[A];
    auto fetch = [&](const Buffer& tokens, int i, uint4 (&t)[A]) {
#pragma unroll
        for (int a = 0; a < A; ++a) t[a] = buffer_read16(tokens, (unsigned)(i + (a * kRuleThreads + tid) * 4) * 4u);
    };
    auto count = [&](bool is_output, int n, int i, const uint4 (&t)[A]) {
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const unsigned id[4] = {t[a].x, t[a].y, t[a].z, t[a].w};
            const int have = n - (i + (a * kRuleThreads + tid) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned at = id[e] + (unsigned)(lead - first);
                if (e < have && at < (unsigned)SLICE && id[e] < (unsigned)p.V) {
                    if (is_output) atomicAdd(words + at, 1u);
                    else atomicOr(words + at, kInPrompt);
                }
            }
        }
    };
    const bool counts = n_prompt + n_output > 0;             // uniform, as all of these
    if (counts) {
        fetch(prompts, 0, in_prompt);
        fetch(outputs, 0, in_output);
    }
    // a thread's bias (further ones of a long list are read again where they are needed)
    unsigned bias_id = 0xffffffffu, bias_at = 0xffffffffu;
    float bias = 0.f;
    if (n_bias > 0) {
        const int i = tid < n_bias ? biases.begin + tid : biases.begin;
        bias_id = (unsigned)p.bias_ids[i];
        bias = p.bias_values[i];
    }
    if (counts || n_bias > 0) {
        for (int i = tid; i < SLICE / 4; i += kRuleThreads) store_vec(reinterpret_cast<uint4*>(words) + i, make_uint4(0u, 0u, 0u, 0u));
        __syncthreads();
    }
    if (counts) {
        count(false, n_prompt, 0, in_prompt);
        count(true, n_output, 0, in_output);
        for (int i = TRIP; i < n_prompt; i += TRIP) {
            fetch(prompts, i, in_prompt);
            count(false, n_prompt, i, in_prompt);
        }
        for (int i = TRIP; i < n_output; i += TRIP) {
            fetch(outputs, i, in_output);
            count(true, n_output, i, in_output);
        }
        __syncthreads();
    }
    slice_values<DT, NB>(p, m, lead, first, wave, lane, d, z);
    if (counts) {
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            uint4* at = reinterpret_cast<uint4*>(words + vec_place<DT, NB>(0, wave, lane, u));
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
                const uint4 w = load_vec(at + h);
                const int i = u * E + h * 4;
                if ((w.x | w.y | w.z | w.w) != 0u) {         // few places are
                    z[i] = rule_penalty(z[i], w.x, rep, freq, pres);
                    z[i + 1] = rule_penalty(z[i + 1], w.y, rep, freq, pres);
                    z[i + 2] = rule_penalty(z[i + 2], w.z, rep, freq, pres);
                    z[i + 3] = rule_penalty(z[i + 3], w.w, rep, freq, pres);
                    if (n_bias > 0) store_vec(at + h, make_uint4(0u, 0u, 0u, 0u));
                }
            }
        }
        if (n_bias > 0) __syncthreads();
    }
    if (n_bias > 0) {
        // The last entry of an id is the one that counts: the places in the list compete.
        if (tid < n_bias && bias_id < (unsigned)p.V) bias_at = bias_id + (unsigned)(lead - first);
        if (bias_at < (unsigned)SLICE) atomicMax(words + bias_at, (unsigned)tid + 1u);
        for (int i = tid + kRuleThreads; i < n_bias; i += kRuleThreads) {
            const unsigned id = (unsigned)p.bias_ids[biases.begin + i], at = id + (unsigned)(lead - first);
            if (id < (unsigned)p.V && at < (unsigned)SLICE) atomicMax(words + at, (unsigned)i + 1u);
        }
        __syncthreads();
        if (n_bias <= kRuleThreads) {                        // who has won leaves the bias itself (0 changes nothing)
            const bool won = bias_at < (unsigned)SLICE && words[bias_at] == (unsigned)tid + 1u;
            __syncthreads();
            if (won) words[bias_at] = __float_as_uint(bias);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const uint4* at = reinterpret_cast<const uint4*>(words + vec_place<DT, NB>(0, wave, lane, u));
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
                const uint4 v = load_vec(at + h);
                const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (w[e] != 0u) z[u * E + h * 4 + e] += n_bias <= kRuleThreads ? __uint_as_float(w[e]) : p.bias_values[biases.begin + (int)(w[e] - 1u)];
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
    float z[NB * kRulePerLane];
    slice_under_rules<DT, NB>(p, m, lead, first, wave, lane, words, z);
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

// Candidates that a workgroup looks at: of at most 84 lanes (see candidate_bound), all their values.
constexpr int kBoundSpare = 20;
template <int NB>
constexpr int kMostCandidates = (kMaxK + kBoundSpare) * NB * kRulePerLane;

// A key that at least k of the workgroup's candidates reach, and the candidates of few lanes beside
// theirs: of the lanes' best keys (one per lane of the workgroup, in LDS; 0 for none) k to k + 20 reach
// it, or fewer than k lanes have one and it is 1.  By bisection, every wave for itself; the keys are
// distinct, so it ends.
__device__ __forceinline__ unsigned long long candidate_bound(const unsigned long long* best, int k, int lane) {
    unsigned long long key[kRuleWaves];
#pragma unroll
    for (int i = 0; i < kRuleWaves; ++i) key[i] = best[i * kWave + lane];
    if (count_reach<kRuleWaves>(key, 1ull) < k) return 1ull;                     // wave-uniform
    unsigned high = 0u;
#pragma unroll
    for (int i = 0; i < kRuleWaves; ++i) high = (unsigned)(key[i] >> 32) > high ? (unsigned)(key[i] >> 32) : high;
    const unsigned top = wave_max_u32(high);
    unsigned long long lo = 1ull, hi = top == 0xffffffffu ? ~0ull : (unsigned long long)(top + 1u) << 32;    // reached by none
    while (hi - lo > 1ull) {
        const unsigned long long mid = lo + ((hi - lo) >> 1);
        const int c = count_reach<kRuleWaves>(key, mid);
        if (c >= k) {
            lo = mid;
            if (c <= k + kBoundSpare) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// The k best of n keys in LDS, n > 0 of any size: put(rank, key).  They are cut down from the front, the k
// best so far before the next ones.
template <class Put>
__device__ __forceinline__ void topk_of_many(unsigned long long* keys, int n, int k, int lane, unsigned long long* buf, Put put) {
    int from = 0;
    while (n - from > kTopkLdsMax) {                                             // wave-uniform
        unsigned long long* kept = keys + from + kTopkLdsMax - k;
        wave_topk_lds(keys + from, kTopkLdsMax, k, lane, buf, [&](int r, unsigned long long c) { kept[r] = c; });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        from += kTopkLdsMax - k;
    }
    wave_topk_lds(keys + from, n - from, k, lane, buf, put);
}

// A workgroup's slice: its candidates are the values that reach a bound, found from the lanes' best
// values, of which there are little more than k; one wave ranks these and publishes the k best, and
// the row's last workgroup merges the lists.
template <int DT, int NB>
__global__ __launch_bounds__(kRuleThreads) void k_logits_topk(RuleParams p, TopkParams t) {
    constexpr int SLICE = NB * kRuleBatch * kRuleWaves, E = kRuleVec<DT>, N = NB * kRulePerLane;
    __shared__ union {
        __attribute__((aligned(16))) unsigned words[SLICE];
        __attribute__((aligned(16))) unsigned long long keys[kMostCandidates<NB>];
        MergeScratch merge;
    } lds;
    __shared__ __attribute__((aligned(16))) unsigned long long best[kRuleThreads];
    __shared__ __attribute__((aligned(16))) unsigned long long buf[kWave];
    __shared__ ExpSum wave_sums[kRuleWaves];
    __shared__ ExpSum row_sum;
    __shared__ int n_keys, last;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int m = blockIdx.y, lead = row_lead<DT>(m, p.V), slice = blockIdx.x, first = slice * SLICE, k = t.k;
    float z[N];
    slice_under_rules<DT, NB>(p, m, lead, first, wave, lane, lds.words, z);
    // the lane's best value, of equal ones the first (ids grow with the index)
    float top = -INFINITY;
    int top_at = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        z[i] = z[i] != z[i] ? -INFINITY : z[i];              // NaN is no candidate
        top_at = z[i] >= top ? i : top_at;
        top = fmaxf(top, z[i]);
    }
    auto id_of = [&](int i) { return vec_place<DT, NB>(first, wave, lane, i / E) - lead + i % E; };
    best[threadIdx.x] = top != -INFINITY ? cand_key(top, id_of(top_at)) : 0ull;
    if (threadIdx.x == 0) n_keys = 0;
    const float wave_top = wave_max(top);
    float sum = 0.f;
    if (wave_top != -INFINITY) {                             // wave-uniform
#pragma unroll
        for (int i = 0; i < N; ++i) sum += exp2f((z[i] - wave_top) * 1.44269504f);
    }
    sum = wave_sum(sum);
    if (lane == 0) wave_sums[wave] = {wave_top, sum};
    __syncthreads();                                         // (and the words' memory is taken again from here on)
    const unsigned long long bound = candidate_bound(best, k, lane);
    const float bound_value = bound > 1ull ? key_value(bound) : -INFINITY;
    if (top >= bound_value && top != -INFINITY) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (z[i] >= bound_value && z[i] != -INFINITY) {
                const unsigned long long key = cand_key(z[i], id_of(i));
                if (key >= bound) lds.keys[atomicAdd(&n_keys, 1)] = key;         // (their order does not matter)
            }
        }
    }
    __syncthreads();
    Cand* part = t.part + ((size_t)m * t.slices) * k;
    if (wave == 0) {
        topk_of_many(lds.keys, n_keys, k, lane, buf, [&](int r, unsigned long long c) {
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
    // (the other waves' candidates are read by now: the merge takes their memory)
    if (wave == 0) {
        if (lane == 0) __hip_atomic_store(t.arrived + m, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wave_merge_lists(t.slices, k, lane, &lds.merge, [&](int l, int i) { return fetch_cand(part + (size_t)l * k + i); },
                         [&](int r, unsigned long long c) { best[r] = c; });
    }
    __syncthreads();
    if (threadIdx.x < (unsigned)k) {
        // (z - largest) - log(sum): z - (largest + log(sum)) would lose the sum where values are far from zero
        const Cand cand = key_cand(best[threadIdx.x]);
        t.ids[(size_t)m * k + threadIdx.x] = is_real(cand) ? cand.id : -1;
        t.logprob[(size_t)m * k + threadIdx.x] = is_real(cand) ? (cand.v - row_sum.top) - logf(row_sum.sum) : -INFINITY;
    }
}

}  // namespace
