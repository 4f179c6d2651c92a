// Rules on a step's logits, and the k best tokens under them.
//
// For every token id of a row, in this order and each operation rounded to fp32 by itself:
//   repetition  z > 0 ? z / r : z * r     where the id is in the row's prompt or output
//   frequency   z - count * f             where count > 0: how often the id is in the row's output
//   presence    z - p                     where count > 0
//   bias        z + b                     the last entry of the id in the row's list of biases
//   mask        -inf                      where the id's bit is 0
// A workgroup takes a slice of a row.  Its logits go to registers; the row's tokens are read once and
// those of the slice counted in LDS with integer atomics (their order does not matter), then the
// biases' places are marked the same way.  So neither a count array in memory nor a second pass over
// the logits is needed, and rows of any number share their prompts by reading the same range.
//
// Measured: written back, 64 rows of 151665 bf16 values with prompts of 8000, outputs of 1000, 100 biases and
// masks: 20 us (39 MB of logits: 8 us); without rules 9.7 us.  One row of 128256 fp32: 6 us, most of it
// the launch and two trips to memory.  The k best: 64 rows of 152064 fp32, every rule, k = 64: 33 us, without
// rules 22 us, k = 10 17 us (the reading alone: 6 us); one row, k = 10: 9.0 us.  What bounds the large ones
// is the instructions of a value (words of LDS read, rules, comparisons, 2^x) and that 64 rows are 2432 workgroups for
// 2048 places (62 registers, 19 KB of LDS): the chain of one is run twice.  The small ones are the chain of
// the steps, from the launch to the last workgroup's merge.  24 rows over one prompt of 60000 tokens: 20 us,
// of which 7 are the prompt's reading by each of 13 slices.
// A slice of 8192 values, two batches a wave, instead of 4096 took 24 us for 21 and 42 for 41; one streamed by
// eight waves in tiles, with notes of 16 bits in LDS, 29 and 48.
#pragma once
#include "buffer_loads.h"
#include "control_words.h"
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
constexpr int kRulePerLane = 16;                            // values a lane holds
constexpr int kRuleSlice = kRulePerLane * kRuleThreads;     // values of a workgroup
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

// First place of vector u of a lane: consecutive lanes on consecutive vectors.
template <int DT>
__device__ __forceinline__ int vec_place(int first, int wave, int lane, int u) {
    constexpr int E = kRuleVec<DT>, U = kRulePerLane / E;
    return first + (wave * U + u) * (kWave * E) + lane * E;
}

// The lane's logits of the slice, as they lie in memory, and the mask bits that go with them (the words
// of a vector's first and last value; values of the row's neighbours among them are dropped later).
template <int DT>
struct SliceData {
    static constexpr int kVecs = kRulePerLane / kRuleVec<DT>;
    uint4 v[kVecs];
    unsigned lo[kVecs], hi[kVecs];
};
template <int DT>
__device__ __forceinline__ void load_slice(const RuleParams& p, int m, int lead, int first, int wave, int lane, SliceData<DT>& d) {
    constexpr size_t W = DT == kF32 ? 4 : 2;
    const Buffer logits = buffer_view(p.logits, ((size_t)m * p.V - lead) * W, (size_t)p.M * p.V * W);
#pragma unroll
    for (int u = 0; u < d.kVecs; ++u) d.v[u] = buffer_read16<kBufferStream>(logits, (unsigned)(vec_place<DT>(first, wave, lane, u) * W));
    if (p.mask) {                                            // uniform
        const Buffer mask = buffer_view(p.mask, (size_t)m * p.mask_words * 4, (size_t)p.M * p.mask_words * 4);
#pragma unroll
        for (int u = 0; u < d.kVecs; ++u) {
            const int id = vec_place<DT>(first, wave, lane, u) - lead;       // (before the row: dropped, as behind the end)
            d.lo[u] = buffer_read4(mask, (unsigned)(id >> 5) * 4u);
            d.hi[u] = buffer_read4(mask, (unsigned)((id + kRuleVec<DT> - 1) >> 5) * 4u);
        }
    }
}

// The values as fp32; -inf for those that are not the row's.
template <int DT>
__device__ __forceinline__ void slice_values(const RuleParams& p, int m, int lead, int first, int wave, int lane, const SliceData<DT>& d,
                                             float (&z)[kRulePerLane]) {
    constexpr int E = kRuleVec<DT>;
#pragma unroll
    for (int u = 0; u < d.kVecs; ++u) {
        const unsigned w[4] = {d.v[u].x, d.v[u].y, d.v[u].z, d.v[u].w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (DT == kF32) z[u * E + e] = __uint_as_float(w[e]);
            else z[u * E + e] = widen16<DT>((unsigned short)(w[e / 2] >> (e % 2 * 16)));
        }
    }
    if (first < lead || first + kRuleSlice > p.V + lead) {        // uniform: the row's first or last slice
        // (half a dword at the very end of the operand is dropped by the load of a vector)
        float end = 0.f;
        if constexpr (DT != kF32) end = widen16<DT>(static_cast<const unsigned short*>(p.logits)[(size_t)p.M * p.V - 1]);
#pragma unroll
        for (int u = 0; u < d.kVecs; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int id = vec_place<DT>(first, wave, lane, u) - lead + e;
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
    if (count == 0u) return z;                               // (infinite penalties times nothing)
    const float taken = (float)count * freq;
    z = z - taken;
    return z - pres;
}

// The lane's values under the rules.  words: one LDS word per place of the slice.  Every thread of the
// workgroup comes here; barriers are reached by all.
template <int DT>
__device__ __forceinline__ void slice_under_rules(const RuleParams& p, int m, int lead, int first, int wave, int lane,
                                                  unsigned* words, float (&z)[kRulePerLane]) {
    constexpr int E = kRuleVec<DT>, VECS = kRulePerLane / E;
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
    SliceData<DT> d;
    load_slice<DT>(p, m, lead, first, wave, lane, d);
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
    // the slice's ids of the row: first_id ... + n_ids, from word first_word on
    const unsigned first_id = (unsigned)(first > lead ? first - lead : 0), first_word = (unsigned)(first > lead ? 0 : lead - first);
    const unsigned in_slice = (unsigned)kRuleSlice - first_word, in_row = first_id < (unsigned)p.V ? (unsigned)p.V - first_id : 0u;
    const unsigned n_ids = in_slice < in_row ? in_slice : in_row;
    unsigned* const row_words = words + first_word;
    auto count = [&](bool is_output, bool whole, int n, int i, const uint4 (&t)[A]) CORAL_INLINE {
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const unsigned id[4] = {t[a].x, t[a].y, t[a].z, t[a].w};
            const int have = n - (i + (a * kRuleThreads + tid) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned at = id[e] - first_id;
                if (at < n_ids && (whole || e < have)) {
                    if (is_output) atomicAdd(row_words + at, 1u);
                    else atomicOr(row_words + at, kInPrompt);
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
        for (int i = tid; i < kRuleSlice / 4; i += kRuleThreads) store_vec(reinterpret_cast<uint4*>(words) + i, make_uint4(0u, 0u, 0u, 0u));
        __syncthreads();
    }
    if (counts) {
        count(false, false, n_prompt, 0, in_prompt);
        count(true, false, n_output, 0, in_output);
        if (TRIP < n_prompt) {                               // a long prompt: the next tokens on their way
            fetch(prompts, TRIP, in_prompt);
            int i = TRIP;
            for (; i + TRIP <= n_prompt; i += TRIP) {
                uint4 next[A];
                fetch(prompts, i + TRIP, next);              // (behind the range there is none)
                count(false, true, n_prompt, i, in_prompt);
#pragma unroll
                for (int a = 0; a < A; ++a) in_prompt[a] = next[a];
            }
            count(false, false, n_prompt, i, in_prompt);
        }
        for (int i = TRIP; i < n_output; i += TRIP) {
            fetch(outputs, i, in_output);
            count(true, false, n_output, i, in_output);
        }
        __syncthreads();
    }
    slice_values<DT>(p, m, lead, first, wave, lane, d, z);
    if (counts) {
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            uint4* at = reinterpret_cast<uint4*>(words + vec_place<DT>(0, wave, lane, u));
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
        if (bias_at < (unsigned)kRuleSlice) atomicMax(words + bias_at, (unsigned)tid + 1u);
        for (int i = tid + kRuleThreads; i < n_bias; i += kRuleThreads) {
            const unsigned id = (unsigned)p.bias_ids[biases.begin + i], at = id + (unsigned)(lead - first);
            if (id < (unsigned)p.V && at < (unsigned)kRuleSlice) atomicMax(words + at, (unsigned)i + 1u);
        }
        __syncthreads();
        if (n_bias <= kRuleThreads) {                        // who has won leaves the bias itself (0 changes nothing)
            const bool won = bias_at < (unsigned)kRuleSlice && words[bias_at] == (unsigned)tid + 1u;
            __syncthreads();
            if (won) words[bias_at] = __float_as_uint(bias);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const uint4* at = reinterpret_cast<const uint4*>(words + vec_place<DT>(0, wave, lane, u));
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
            const int id = vec_place<DT>(first, wave, lane, u) - lead;
            const unsigned bits = __builtin_amdgcn_alignbit(d.hi[u], d.lo[u], (unsigned)(id & 31));
#pragma unroll
            for (int e = 0; e < E; ++e) z[u * E + e] = bits >> e & 1u ? z[u * E + e] : -INFINITY;
        }
    }
}

// The logits under their rules, rounded to the storage type.
template <int DT>
__global__ __launch_bounds__(kRuleThreads) void k_logits_adjust(RuleParams p, void* out) {
    constexpr int E = kRuleVec<DT>, VECS = kRulePerLane / E;
    __shared__ __attribute__((aligned(16))) unsigned words[kRuleSlice];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int m = blockIdx.y, lead = row_lead<DT>(m, p.V), first = blockIdx.x * kRuleSlice;
    float z[kRulePerLane];
    slice_under_rules<DT>(p, m, lead, first, wave, lane, words, z);
    const size_t row = (size_t)m * p.V;
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        const int id = vec_place<DT>(first, wave, lane, u) - lead;
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
    unsigned* arrived;          // [M] counters, kRowArrivalStride words apart, zero between calls
    int32_t* ids;               // [M,k]
    float* logprob;             // [M,k]
    int k, slices;
};

// Candidates that a workgroup looks at: of at most 84 lanes (see candidate_bound), all their values.
constexpr int kBoundSpare = 20;
constexpr int kMaxSlices = 256;                             // lists that a merge takes
constexpr int kMostCandidates = (kMaxK + kBoundSpare) * kRulePerLane;
constexpr unsigned kLeastKey = 0x00800000u;                 // upper half of the lowest finite value's key

// A key that at least k of the workgroup's candidates reach, and the candidates of few lanes beside
// theirs: of the lanes' best keys (one per lane of the workgroup, in LDS; 0 for none) k to k + 20 reach
// it, or fewer than k lanes have one and it is 1.  By bisection, every wave for itself; the keys are
// distinct, so it ends.
__device__ __forceinline__ unsigned long long candidate_bound(const unsigned long long* best, int k, int lane) {
    unsigned long long key[kRuleWaves];
#pragma unroll
    for (int i = 0; i < kRuleWaves; ++i) key[i] = best[i * kWave + lane];
    if (count_reach<kRuleWaves>(key, 1ull) < k) return 1ull;                     // wave-uniform
    unsigned high = 0u, low = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < kRuleWaves; ++i) {
        const unsigned v = (unsigned)(key[i] >> 32);
        high = v > high ? v : high;
        low = v < low ? v : low;
    }
    // by value first: half the bits
    const unsigned top = wave_max_u32(high);
    // The least is reached by all, the lowest value's by all that have a candidate; top + 1 by none.  (Not from the
    // zero of a lane that has none: halfway to it lie the keys of -inf and NaN, which no value compares with.)
    const unsigned least = wave_min_u32(low);
    unsigned below = least > kLeastKey ? least : kLeastKey, above = top;
    while (below < above) {                                  // wave-uniform; at most 32 steps
        const unsigned mid = below + (above - below) / 2u + 1u;
        int c = 0;
#pragma unroll
        for (int i = 0; i < kRuleWaves; ++i) c += __popcll(__ballot((unsigned)(key[i] >> 32) >= mid));
        if (c >= k) {
            below = mid;
            if (c <= k + kBoundSpare) return (unsigned long long)mid << 32;
        } else {
            above = mid - 1u;
        }
    }
    // more than the spare have the same one: by ids
    unsigned long long lo = (unsigned long long)below << 32;
    unsigned long long hi = below == 0xffffffffu ? ~0ull : (unsigned long long)(below + 1u) << 32;
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

// Number of the workgroup's lanes before this one whose best key reaches the bound.
__device__ __forceinline__ int wave_slots(const unsigned long long* best, unsigned long long bound, int wave, int lane) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kRuleWaves; ++i) {
        const unsigned long long who = __ballot(best[i * kWave + lane] >= bound);
        if (i < wave) n += __popcll(who);
        else if (i == wave) n += __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0u));
    }
    return n;
}

// Appends the candidates of a lane's N values, the bits of `reach`, to the workgroup's: key(i) by index, which
// reads it from LDS.  One atomic addition a wave, as one for every key is waited for each time.  Their
// order does not matter.
template <int N, class Key>
__device__ __forceinline__ void append_candidates(unsigned reach, unsigned long long* keys, int* n_keys, int lane, Key key) {
    const unsigned mine = (unsigned)__popc(reach);
    int before = 0, all = 0;
#pragma unroll
    for (int b = 0; 1 << b <= N; ++b) {
        const unsigned long long who = __ballot((mine >> b & 1u) != 0u);
        before += __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0u)) << b;
        all += __popcll(who) << b;
    }
    if (all == 0) return;                                    // wave-uniform
    int at = 0;
    if (lane == 0) at = atomicAdd(n_keys, all);
    at = __builtin_amdgcn_readfirstlane(at) + before;
    while (reach != 0u) {
        const int i = __ffs(reach) - 1;
        reach &= reach - 1u;
        keys[at++] = key(i);
    }
}

// Sum over four neighbouring lanes.
__device__ __forceinline__ int quad_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false);               // the neighbour's
    return x + __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false);         // the other pair's
}

// Of the workgroup's keys, N a thread (0: none), those that reach a bound go to keys[0, *n_keys): the k best among
// them, and those of at most k + 20 threads.  All threads, which have read *n_keys and keys by then.
template <int N>
__device__ __forceinline__ void reduce_keys(const unsigned long long (&key)[N], int k, int lane, unsigned long long* best,
                                            unsigned long long* keys, int* n_keys) {
    unsigned long long top = 0ull;
#pragma unroll
    for (int i = 0; i < N; ++i) top = key[i] > top ? key[i] : top;
    best[threadIdx.x] = top;
    __syncthreads();
    if (threadIdx.x == 0) *n_keys = 0;
    const unsigned long long bound = candidate_bound(best, k, lane);
    __syncthreads();
    if (top >= bound) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (key[i] >= bound) keys[atomicAdd(n_keys, 1)] = key[i];            // (their order does not matter)
    }
    __syncthreads();
}

// The k best of the workgroup's candidates: put(rank, key) once for every rank < k (key 0 past the last one).
// Called by all threads behind a barrier.  Up to 256 are ranked by counting: of four threads each counts a
// quarter of the keys above two of them.  More than that, where a slice's values are few lanes' or equal, are
// dealt to the threads anew: of 84 threads' ceil(n / 256) the next time, so at most two times.
template <class Put>
__device__ __forceinline__ void slice_topk(unsigned long long* keys, int* n_keys, int k, int lane, int wave, unsigned long long* best, Put put) {
    int n = *n_keys;
    while (n > kRuleThreads) {                               // uniform
        constexpr int N = (kMostCandidates + kRuleThreads - 1) / kRuleThreads;
        unsigned long long key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = i * kRuleThreads + (int)threadIdx.x;
            key[i] = at < n ? keys[at] : 0ull;
        }
        reduce_keys<N>(key, k, lane, best, keys, n_keys);
        n = *n_keys;
    }
    const int part = lane & 3, whole = (n + 15) & ~15;   // (filled up: all threads read as many)
    if ((int)threadIdx.x < whole - n) keys[n + (int)threadIdx.x] = 0ull;
    __syncthreads();
    for (int from = 0; from < n; from += kRuleThreads / 2) {                 // uniform; two keys a thread
        const int i = from + (int)threadIdx.x / 4, i2 = i + kRuleThreads / 4;
        const unsigned long long mine = i < n ? keys[i] : ~0ull, mine2 = i2 < n ? keys[i2] : ~0ull;
        int above = 0, above2 = 0;
#pragma unroll 2
        for (int j = 0; j < whole; j += 16) {            // uniform
            const ulonglong2* at = reinterpret_cast<const ulonglong2*>(keys + j + part * 4);
            const ulonglong2 one = at[0], two = at[1];
            above += (one.x > mine ? 1 : 0) + (one.y > mine ? 1 : 0) + (two.x > mine ? 1 : 0) + (two.y > mine ? 1 : 0);
            above2 += (one.x > mine2 ? 1 : 0) + (one.y > mine2 ? 1 : 0) + (two.x > mine2 ? 1 : 0) + (two.y > mine2 ? 1 : 0);
        }
        above = quad_sum(above);
        above2 = quad_sum(above2);
        if (i < n && part == 0 && above < k) put(above, mine);
        if (i2 < n && part == 0 && above2 < k) put(above2, mine2);
    }
    if (wave == 0 && lane >= n && lane < k) put(lane, 0ull);
}

// The k best of n_e published candidates, of up to N a thread, all fetched in one trip: put(rank, key).
// meanwhile() runs while they are on their way.  Called by all threads.
// (One row of 128256, k = 64, 2048 candidates: 11.0 us, against 14.4 by one wave a few of each list at a time,
// which is left for more than 4096.)
constexpr int kMergeAll = 16 * kRuleThreads;
template <int N, class Meanwhile, class Put>
__device__ __forceinline__ void merge_all(const Cand* part, int n_e, int k, int lane, int wave, unsigned long long* best,
                                          unsigned long long* keys, int* n_keys, Meanwhile meanwhile, Put put) {
    static_assert(N <= kRulePerLane, "the candidates fit");
    // A thread's entries are of different ranks in their lists, or few threads would have all the best ones,
    // whose bound lets many through (k = 64, 38 lists, without the turn: 28 us for 8 rows, 13 us with it).
    auto entry = [&](int i) CORAL_INLINE { return i * kRuleThreads + (((int)threadIdx.x + 27 * i) & (kRuleThreads - 1)); };
    Cand c[N];
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = fetch_cand(part + (entry(i) < n_e ? entry(i) : n_e - 1));     // (unconditional, from clamped places)
    meanwhile();
    unsigned long long key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = entry(i) < n_e ? real_key(c[i]) : 0ull;
    reduce_keys<N>(key, k, lane, best, keys, n_keys);
    slice_topk(keys, n_keys, k, lane, wave, best, put);
}

// A workgroup's slice: its candidates are the values that reach a bound, found from the lanes' best
// values, of which there are little more than k; one wave ranks these and publishes the k best, and
// the row's last workgroup merges the lists.
template <int DT>
__global__ __launch_bounds__(kRuleThreads) void k_logits_topk(RuleParams p, TopkParams t) {
    constexpr int E = kRuleVec<DT>, N = kRulePerLane;
    __shared__ union {
        __attribute__((aligned(16))) unsigned words[kRuleSlice];
        struct {
            __attribute__((aligned(16))) unsigned long long keys[kMostCandidates];
            float values[kMaxK + kBoundSpare][kRulePerLane];
        } pick;
        MergeScratch merge;
    } lds;
    __shared__ __attribute__((aligned(16))) unsigned long long best[kRuleThreads];
    __shared__ unsigned long long sorted[kMaxK];
    __shared__ ExpSum wave_sums[kRuleWaves];
    __shared__ ExpSum row_sum;
    __shared__ int n_keys, last;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int m = blockIdx.y, lead = row_lead<DT>(m, p.V), slice = blockIdx.x, first = slice * kRuleSlice, k = t.k;
    float z[N];
    slice_under_rules<DT>(p, m, lead, first, wave, lane, lds.words, z);
    // the lane's best value, of equal ones the first (ids grow with the index)
    float top = -INFINITY;
    int top_at = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        z[i] = fmaxf(z[i], -INFINITY);                       // NaN is no candidate
        top_at = z[i] >= top ? i : top_at;
        top = fmaxf(top, z[i]);
    }
    auto id_of = [&](int i) { return vec_place<DT>(first, wave, lane, i / E) - lead + i % E; };
    const unsigned long long mine = top != -INFINITY ? cand_key(top, id_of(top_at)) : 0ull;
    best[threadIdx.x] = mine;
    if (threadIdx.x == 0) n_keys = 0;
    const float wave_top = wave_max(top);
    float sum = 0.f;
    if (wave_top != -INFINITY) {                             // wave-uniform
#pragma unroll
        for (int i = 0; i < N; ++i) sum += __builtin_amdgcn_exp2f((z[i] - wave_top) * 1.44269504f);
    }
    sum = wave_sum(sum);
    if (lane == 0) wave_sums[wave] = {wave_top, sum};
    __syncthreads();                                         // (and the words' memory is taken again from here on)
    const unsigned long long bound = candidate_bound(best, k, lane);
    // Lanes with a candidate, few of the workgroup's, leave their values in LDS, where they are picked out by index.
    const bool some = mine >= bound;
    const int slot = wave_slots(best, bound, wave, lane);
    unsigned reach = 0u;
    if (some) {
        const float least = bound > 1ull ? key_value(bound) : -3.402823466e38f;  // (-inf is no candidate)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            lds.pick.values[slot][i] = z[i];
            reach |= z[i] >= least ? 1u << i : 0u;
        }
    }
    auto key_of = [&](int i) CORAL_INLINE { return cand_key(lds.pick.values[slot][i], id_of(i)); };
    if ((unsigned)bound > 1u) {                              // uniform: not all that have the bound's value
        unsigned among = 0u;
        for (; reach != 0u; reach &= reach - 1u) {
            const int i = __ffs(reach) - 1;
            if (key_of(i) >= bound) among |= 1u << i;
        }
        reach = among;
    }
    append_candidates<N>(reach, lds.pick.keys, &n_keys, lane, key_of);
    __syncthreads();
    slice_topk(lds.pick.keys, &n_keys, k, lane, wave, best, [&](int r, unsigned long long c) { sorted[r] = c; });
    __syncthreads();
    Cand* part = t.part + ((size_t)m * t.slices) * k;
    if (wave == 0) {
        ExpSum s = wave_sums[0];
#pragma unroll
        for (int w = 1; w < kRuleWaves; ++w) s = join(s, wave_sums[w]);
        if (t.slices == 1) {                                 // uniform: there is nothing to wait for
            if (lane == 0) {
                row_sum = s;
                last = 1;
            }
        } else {
            if (lane < k) {
                const Cand cand = key_cand(sorted[lane]);
                publish_cand(part + (size_t)slice * k + lane, cand.v, cand.id);
            }
            if (lane == 0) {
                const unsigned long long bits =
                    (unsigned long long)__float_as_uint(s.top) << 32 | (unsigned long long)__float_as_uint(s.sum);
                __hip_atomic_store(t.sums + (size_t)m * t.slices + slice, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0): this wave's stores are out
            asm volatile("" ::: "memory");
            if (lane == 0) {
                const unsigned old = __hip_atomic_fetch_add(t.arrived + m * coral_ctrl::kRowArrivalStride, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last = old == (unsigned)t.slices - 1u ? 1 : 0;
            }
        }
    }
    __syncthreads();
    if (!last) return;                                       // uniform
    if (t.slices > 1) {
        if (threadIdx.x == 0) __hip_atomic_store(t.arrived + m * coral_ctrl::kRowArrivalStride, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // the row's log-sum-exp, in an order of its own: a slice a thread
        static_assert(kMaxSlices <= kRuleThreads, "");
        const int i = (int)threadIdx.x < t.slices ? (int)threadIdx.x : t.slices - 1;
        const unsigned long long bits = __hip_atomic_load(t.sums + (size_t)m * t.slices + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        auto join_sums = [&]() CORAL_INLINE {
            const float top = (int)threadIdx.x < t.slices ? __uint_as_float((unsigned)(bits >> 32)) : -INFINITY;
            const float wave_top = wave_max(top);
            const float sum = wave_sum(top == -INFINITY ? 0.f : __uint_as_float((unsigned)bits) * expf(top - wave_top));
            if (lane == 0) wave_sums[wave] = {wave_top, sum};
        };
        const int n_e = t.slices * k;
        auto put = [&](int r, unsigned long long c) CORAL_INLINE { sorted[r] = c; };
        if (n_e <= kMergeAll) {                              // uniform
            if (n_e <= 4 * kRuleThreads) merge_all<4>(part, n_e, k, lane, wave, best, lds.pick.keys, &n_keys, join_sums, put);
            else merge_all<kMergeAll / kRuleThreads>(part, n_e, k, lane, wave, best, lds.pick.keys, &n_keys, join_sums, put);
        } else {
            join_sums();
            if (wave == 0) wave_merge_lists(t.slices, k, lane, &lds.merge, [&](int l, int e) { return fetch_cand(part + (size_t)l * k + e); }, put);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            ExpSum s = wave_sums[0];
#pragma unroll
            for (int w = 1; w < kRuleWaves; ++w) s = join(s, wave_sums[w]);
            row_sum = s;
        }
    }
    __syncthreads();
    if (threadIdx.x < (unsigned)k) {
        // (z - largest) - log(sum): z - (largest + log(sum)) would lose the sum where values are far from zero
        const Cand cand = key_cand(sorted[threadIdx.x]);
        t.ids[(size_t)m * k + threadIdx.x] = is_real(cand) ? cand.id : -1;
        t.logprob[(size_t)m * k + threadIdx.x] = is_real(cand) ? (cand.v - row_sum.top) - logf(row_sum.sum) : -INFINITY;
    }
}

}  // namespace
