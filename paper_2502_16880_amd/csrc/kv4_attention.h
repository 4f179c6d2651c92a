// Attention over a cache of 4-bit floats.
//
//   out[t,h] = sum_j p_j v_j,  p = softmax_j(scale * q[t,h] . k_j)  over the cached tokens j that row t sees
//
// Codes become 16-bit operands of the matrix cores exactly (one conversion instruction for two values, the
// unit of their 32 included), so scores and sums have exact products and fp32 sums.  A wave takes 32
// tokens a step: 16 bytes of a token's key a lane, in the order of memory (D = 128: the whole KB of 16 keys
// in one load); which of the lane's values goes with which column of a product is free as long as the
// query's operand has the same order.  Scores come out with the token along a lane's registers, which is
// how the second product wants the weights; the values' operand needs eight tokens of one column in a
// lane, so converted values pass through the wave's part of LDS and come back transposed
// (ds_read_b64_tr_b16).  Softmax is taken in one pass: sums are kept relative to a reference of each
// row that is moved up only when a score passes it by some powers of two (kWeightsUpTo), so most steps do not touch the sums.
// Operands of fp16 calls are fp16 (an append of fp16 values has no others), those of fp32 calls three bf16 values for
// one; so are the weights p.
#pragma once
#include "attention_tiles.h"
#include "control_words.h"
#include "kv4_plan.h"

namespace {

constexpr int kKv4Threads = 256;
constexpr int kKv4ArrivalStride = 4;
constexpr int kKv4Waves = kKv4Threads / kWave;
constexpr int kKv4WaveStep = kKv4Step / kKv4Waves;          // 32 tokens

struct Kv4AttnParams {
    const char* q;
    char* out;
    int64_t q_stride, out_stride;       // bytes from token to token
    Kv4 cache;
    const int32_t *page_table, *lengths, *q_offsets, *history;
    const uint64_t* tree;
    float* part;                        // [workgroup][2][row][D] sums, then [workgroup][2][row] (largest, sum) pairs
    float2* part_stats;
    unsigned* arrived;                  // [workgroup] counters, kKv4ArrivalStride words apart, zero between calls
    int max_pages, T, S, max_rows, group, kv_heads, workgroups;
    int join_heads;                     // of a wave in k_kv4_join, one after the other
    bool apart, join_inside;
    float scale_log2;                   // scores are kept in powers of two; above zero, the sign is taken by q
    unsigned q_sign;                    // bit to flip in every value of q
};

// What the arguments say about a sequence, cut to the arrays, and what it takes: its items (a block of ROWS rows for
// one head of keys) times their steps of 128 tokens and what an item takes before and behind its steps (pages,
// queries, sums).  Among others an item of n steps, four or more, takes 4.1 + 2.1 n us (one tile of rows, D = 128, bf16), 3.6 + 1.5 n
// (D = 64), 7.7 + 1.5 n (D = 256), 4.7 + 1.7 n (fp32), 11 + 1.6 n (two tiles): as much as two to seven steps, of which three stand for
// all (without them a share of short sequences took 82 us where others took 47).  One sequence a lane.
// `rows` are those taken, max_rows at most; `old` tokens are seen by all of them: with a tree the history's, without one row i of
// all n rows that the offsets give sees old + i of them (old = length - n + 1, which may be below zero).
constexpr unsigned kKv4ItemSteps = 3;
struct Kv4Seq {
    int row0, rows, length, old;
    unsigned steps;
    unsigned long long cost;
};
template <int ROWS>
__device__ __forceinline__ Kv4Seq kv4_sequence(const Kv4AttnParams& p, int s) {
    Kv4Seq q = {};
    if (s >= p.S) return q;
    int length = p.lengths[s];
    const int h = p.tree ? p.history[s] : 0;
    q.row0 = cut_offset(p.q_offsets[s], p.T);
    const int n = cut_offset(p.q_offsets[s + 1], p.T) - q.row0;
    q.rows = n < 0 ? 0 : n < p.max_rows ? n : p.max_rows;
    const int64_t room = (int64_t)p.max_pages << p.cache.page_shift;
    length = length < 0 ? 0 : length > room ? (int)room : length;
    q.old = !p.tree ? length - (n > 0 ? n - 1 : 0) : h < 0 ? 0 : h > length ? length : h;
    q.length = p.tree && length - q.old > 64 ? q.old + 64 : length;
    q.steps = q.length > kKv4Step ? ((unsigned)q.length + kKv4Step - 1) / kKv4Step : 1;       // (rows that see nothing are written too)
    q.cost = (unsigned long long)((q.rows * p.group + ROWS - 1) / ROWS) * p.kv_heads * (q.steps + kKv4ItemSteps);
    return q;
}
// Sum over the lanes up to each: sums of 64 numbers below 2^46 in two halves.
__device__ __forceinline__ unsigned long long wave_scan_u46(unsigned long long x) {
    const unsigned lo = (unsigned)wave_scan_inclusive((int)(x & 0xfffffu)), hi = (unsigned)wave_scan_inclusive((int)(x >> 20));
    return ((unsigned long long)hi << 20) + lo;
}
__device__ __forceinline__ unsigned long long readlane64(unsigned long long x, int lane) {
    return (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// n / d for n < 2^20, where inv is 1 / d to a unit in its last place: n + 1/2 is at least 1 / (2 d) from a multiple of d
// away, and n inv at most 2^20 / d * 2^-22.4 off.
__device__ __forceinline__ unsigned quotient20(unsigned n, float inv) { return (unsigned)(((float)n + 0.5f) * inv); }
__device__ __forceinline__ float reciprocal(unsigned d) { return __builtin_amdgcn_rcpf((float)d); }
__device__ __forceinline__ unsigned long long divide64(unsigned long long n, unsigned d) {
    return n >> 32 ? n / d : n >> 20 ? (unsigned)n / d : quotient20((unsigned)n, reciprocal(d));
}

// An item (a block of a sequence's rows for one head of keys), and a place in it: step j is place
// kKv4ItemSteps + j.
struct Kv4Item {
    int seq, row0, rows, length, old, head, first_row;
    unsigned place, steps;
    __device__ __forceinline__ unsigned step_at(unsigned at) const {
        return at < kKv4ItemSteps ? 0 : at - kKv4ItemSteps < steps ? at - kKv4ItemSteps : steps;
    }
};
// All sequences' items lie one behind the other; 64 sequences at a time are looked at, one a lane.
template <int ROWS>
struct Kv4Line {
    Kv4Seq lanes;
    unsigned long long upto, before;     // of these sequences; of all before them
    int s0;
    unsigned long long each;             // places of a share, and how many shares of all have one more, spread evenly
    unsigned more, shares;               // (shares at most 768)
    float inv_shares;

    __device__ __forceinline__ void load(const Kv4AttnParams& p, int from, int lane) {
        s0 = from;
        lanes = kv4_sequence<ROWS>(p, from + lane);
        upto = wave_scan_u46(lanes.cost);
    }
    __device__ __forceinline__ void open(const Kv4AttnParams& p, int lane) {
        unsigned long long total = 0;
        for (int s = p.S > kWave ? kWave : p.S; s < p.S; s += kWave) {
            load(p, s, lane);
            total += readlane64(upto, kWave - 1);
        }
        load(p, 0, lane);
        before = 0;
        deal(p, total + readlane64(upto, kWave - 1));
    }
    __device__ __forceinline__ void deal(const Kv4AttnParams& p, unsigned long long total) {
        shares = total < (unsigned)p.workgroups ? (unsigned)total : (unsigned)p.workgroups;       // each has a place at least
        inv_shares = reciprocal(shares ? shares : 1);
        each = shares ? divide64(total, shares) : 0;
        more = shares ? (unsigned)(total - each * shares) : 0;
    }
    // which share has a place
    __device__ __forceinline__ unsigned share_of(unsigned long long place) const {
        unsigned w = (unsigned)((float)place * __builtin_amdgcn_rcpf((float)each + (float)more * inv_shares));     // nearly
        w = w < shares ? w : shares - 1;
        while (begin(w) > place) --w;
        while (w + 1 < shares && begin(w + 1) <= place) ++w;
        return w;
    }
    // where share w begins
    __device__ __forceinline__ unsigned long long begin(unsigned w) const { return each * w + quotient20(more * w, inv_shares); }
    // what lies at a place below the total; places do not go back
    __device__ __forceinline__ Kv4Item find(const Kv4AttnParams& p, unsigned long long place, int lane) {
        for (;;) {
            const uint64_t found = __builtin_amdgcn_ballot_w64(place - before < upto);
            if (found) {
                const int src = __builtin_ctzll(found);
                return at(p, src, place - before - (readlane64(upto, src) - readlane64(lanes.cost, src)));
            }
            before += readlane64(upto, kWave - 1);
            load(p, s0 + kWave, lane);
        }
    }
    __device__ __forceinline__ Kv4Item at(const Kv4AttnParams& p, int src, unsigned long long in) const {
        Kv4Item t;
        t.seq = s0 + src;
        t.row0 = __builtin_amdgcn_readlane(lanes.row0, src);
        t.rows = __builtin_amdgcn_readlane(lanes.rows, src);
        t.length = __builtin_amdgcn_readlane(lanes.length, src);
        t.old = __builtin_amdgcn_readlane(lanes.old, src);
        t.steps = (unsigned)__builtin_amdgcn_readlane((int)lanes.steps, src);
        const unsigned size = t.steps + kKv4ItemSteps, item = (unsigned)divide64(in, size), blocks = (unsigned)(t.rows * p.group + ROWS - 1) / ROWS;
        t.place = (unsigned)(in - (unsigned long long)item * size);
        t.head = (int)divide64(item, blocks);
        t.first_row = (int)(item - t.head * blocks) * ROWS;
        return t;
    }
};

// What products take for calls of storage type DT: fp16 as it is, bf16 as it is, and fp32 as three bf16 values (exactly).
constexpr int kv4_operand_type(int dt) { return dt == kF16 ? kF16 : kBF16; }
constexpr int kv4_terms(int dt) { return dt == kF32 ? 3 : 1; }
// N values of type OT whose sum is x (8 or 11 bits more each).
template <int OT, int N>
__device__ __forceinline__ void split_terms(float x, float (&part)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = OT == kF16 ? (float)(_Float16)x : (float)(__bf16)x;
        x -= part[i];
    }
}

// A dword of codes with its unit as eight values of type OT.
template <int OT>
__device__ __forceinline__ uint4 kv4_operand(unsigned codes, float unit) {
    uint4 r;
    if (OT == kF16) {
        r.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 0));
        r.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 1));
        r.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 2));
        r.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 3));
    } else {
        r.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
        r.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
        r.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
        r.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
    }
    return r;
}

// Sixteen tokens' codes of one kind as a lane holds them: dword c of lane (token, g) has the values
// kv4_column(c, g) .. + 7, its unit is scale[c / 4].
template <int D>
struct Kv4Tile {
    static constexpr int kDwords = D / 32, kScales = D == 256 ? 2 : 1;
    unsigned code[kDwords], scale[kScales];
};
template <int D>
__device__ __forceinline__ int kv4_column(int c, int g) {
    return D == 64 ? 16 * g + 8 * c : D == 128 ? 32 * g + 8 * c : 128 * (c >> 2) + 32 * g + 8 * (c & 3);
}
template <int D>
__device__ __forceinline__ void kv4_load(Kv4Tile<D>& t, const unsigned char* codes, const unsigned char* scales, unsigned token, unsigned g) {
    // (offsets without a sign: the instructions then take the bases from scalar registers)
    if (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2*>(codes + (token * 32u + g * 8u));
        t.code[0] = w.x;
        t.code[1] = w.y;
        t.scale[0] = scales[token * 2u + g / 2u];
    } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
            const uint4 w = load_stream(reinterpret_cast<const uint4*>(codes + (token * (D / 2u) + i * 64u + g * 16u)));
            t.code[4 * i % Kv4Tile<D>::kDwords] = w.x;
            t.code[(4 * i + 1) % Kv4Tile<D>::kDwords] = w.y;
            t.code[(4 * i + 2) % Kv4Tile<D>::kDwords] = w.z;
            t.code[(4 * i + 3) % Kv4Tile<D>::kDwords] = w.w;
            t.scale[i % Kv4Tile<D>::kScales] = scales[token * (D / 32u) + i * 4u + g];
        }
    }
}

// Where a token's values begin in a wave's part of LDS (bytes): eight banks further from token to token and four more for
// every second eight of them, so that neither 16 tokens' pieces of 16 bytes nor eight tokens' of 32 meet a bank twice.
template <int D>
__device__ __forceinline__ int kv4_place(int token) { return token * (D * 2 + 32) + (token >> 3 & 1) * 16; }
template <int D>
constexpr int kKv4Values = (kKv4WaveStep * (D * 2 + 32) + 16 + 255) / 256 * 256;
template <int D>
constexpr int kKv4SumRow = D + 4;                            // floats from row to row when the waves' sums meet

// What a workgroup has to know of an item behind its steps: which rows, in how many shares' parts it lies, in which of
// them its first step, and whether that share begins inside it.
struct Kv4Kept {
    int row0, head, first_row, n_rows, s0;
    unsigned w0, parts;
    bool opens;
    unsigned more, shares;
    unsigned long long before, place, share_end, each;
};
__device__ __forceinline__ Kv4Kept kv4_kept(const Kv4Kept& from) {
    auto one = [](int x) CORAL_INLINE { return __builtin_amdgcn_readfirstlane(x); };
    auto two = [&](unsigned long long x) CORAL_INLINE { return (unsigned long long)(unsigned)one((int)(x >> 32)) << 32 | (unsigned)one((int)x); };
    return {one(from.row0), one(from.head), one(from.first_row), one(from.n_rows), one(from.s0), (unsigned)one((int)from.w0), (unsigned)one((int)from.parts),
            one(from.opens) != 0, (unsigned)one((int)from.more), (unsigned)one((int)from.shares), two(from.before), two(from.place), two(from.share_end),
            two(from.each)};
}

// Two floats to and from memory that other dies read, past the L2.
__device__ __forceinline__ void publish2(float* to, float a, float b) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(to), (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 published2(const float* from) {
    const unsigned long long w = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32)));
}

// D / 16 values of a row, divided by the sum of its weights; a row that sees nothing is zero.
template <int DT, int D>
__device__ __forceinline__ void kv4_write(const Kv4AttnParams& p, const Kv4Kept& item, int r, float inv_group, int d0, const float (&o)[D / 16], float all) {
    constexpr int kBytes = DT == kF32 ? 4 : 2;
    const float inv = all > 0.f ? 1.f / all : all == 0.f ? 0.f : all;
    const int i = (int)quotient20(r, inv_group);
    char* to = p.out + (int64_t)(item.row0 + i) * p.out_stride + (int64_t)(item.head * p.group + r - i * p.group) * (D * kBytes) + d0 * kBytes;
#pragma unroll
    for (int j = 0; j < D / 16; j += 4) {
        if (DT == kF32) *reinterpret_cast<f32x4_t*>(to + j * 4) = f32x4_t{o[j] * inv, o[j + 1] * inv, o[j + 2] * inv, o[j + 3] * inv};
        else *reinterpret_cast<uint2*>(to + j * 2) = make_uint2(narrow2<DT>(o[j] * inv, o[j + 1] * inv), narrow2<DT>(o[j + 2] * inv, o[j + 3] * inv));
    }
}

// A wave joins the parts of a row, D / 64 values a lane: the parts' statistics first, one a lane, then eight parts' sums
// at a time.  Sums are relative to `ref` then, `all` is the sum of their weights.
template <int D, class RowOf>
__device__ __forceinline__ void kv4_join_row(const Kv4AttnParams& p, unsigned parts, int lane, RowOf row_of, float (&o)[D / kWave], float& ref, float& all) {
    constexpr int N = D / kWave;
    ref = -INFINITY;
    all = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] = 0.f;
    for (unsigned j0 = 0; j0 < parts; j0 += kWave) {
        float2 stat = make_float2(-INFINITY, 0.f);
        if (j0 + lane < parts) stat = published2(&p.part_stats[row_of(j0 + lane)].x);
        float top = lane_xor_max<16>(lane_xor_max<32>(lanes_reduce<16>(stat.x, [](float a, float b) { return fmaxf(a, b); })));
        top = fmaxf(top, ref);
        const float keep = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top), by = stat.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat.x - top);
        ref = top;
        all = fmaf(all, keep, by * stat.y);
#pragma unroll
        for (int n = 0; n < N; ++n) o[n] *= keep;
        const unsigned left = parts - j0 < kWave ? parts - j0 : kWave;
        for (unsigned i = 0; i < left; i += 8) {
            float x[8][N];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* from = p.part + row_of(j0 + (i + u < left ? i + u : left - 1)) * D + lane * N;
                if (N == 1) x[u][0] = __uint_as_float(__hip_atomic_load(reinterpret_cast<const unsigned*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
#pragma unroll
                for (int n = 0; n + 1 < N; n += 2) {
                    const float2 w = published2(from + n);
                    x[u][n] = w.x;
                    x[u][n + 1] = w.y;
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float f = i + u < left ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), (int)(i + u) & (kWave - 1))) : 0.f;
#pragma unroll
                for (int n = 0; n < N; ++n) o[n] = f == 0.f ? o[n] : fmaf(f, x[u][n], o[n]);
            }
        }
    }
    all = wave_sum(all);
}
template <int DT, int D>
__device__ __forceinline__ void kv4_write_row(const Kv4AttnParams& p, const Kv4Kept& item, int r, float inv_group, int lane, const float (&o)[D / kWave], float all) {
    constexpr int N = D / kWave, kBytes = DT == kF32 ? 4 : 2;
    const float inv = all > 0.f ? 1.f / all : all == 0.f ? 0.f : all;
    const int i = (int)quotient20(r, inv_group);
    char* to = p.out + (int64_t)(item.row0 + i) * p.out_stride + (int64_t)(item.head * p.group + r - i * p.group) * (D * kBytes) + lane * (N * kBytes);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (DT == kF32) reinterpret_cast<float*>(to)[n] = o[n] * inv;
        else reinterpret_cast<unsigned short*>(to)[n] = narrow16<DT>(o[n] * inv);
    }
}

typedef const __attribute__((address_space(4))) Kv4AttnParams* Kv4ArgsPtr;

// Four waves take the steps of an item in turn, 32 tokens each of a step, and add up at the end.  A workgroup's share of
// all steps is a run of them that may cross items: the first and the last may be parts of an item, which the item's last
// workgroup puts together, or, where parts and rows are many, k_kv4_join.
// Bound by memory where one row reads a long cache (64 sequences of up to 8192 tokens, 32 heads of 128 on 8: 61 to 66 us, 4.9 to 4.6 TB/s;
// 131072 tokens: 32); by a step's instructions for 32 rows (8 nodes over 131072 tokens: 43; 60 nodes of 28 heads on 4 over 4111: 21); for one token
// over 2000 by the chain of dependent trips (11).  Work is dealt by cost (kKv4ItemSteps), not by sequences,
// whose lengths differ.
template <int DT, int D, int NT, int TP>
__global__ __launch_bounds__(kKv4Threads, (kv4_occupancy(D, NT, kv4_terms(DT)))) void k_kv4_attention(Kv4AttnParams) {
    // The arguments are read where they are used: held in scalar registers all the way they would be spilled.
    const Kv4ArgsPtr args = (Kv4ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
    const Kv4AttnParams& p = *(const Kv4AttnParams*)args;
    constexpr int OT = kv4_operand_type(DT), TQ = kv4_terms(DT), C = D / 32, DTILES = D / 16, kBytes = DT == kF32 ? 4 : 2;
    static_assert(kKv4Values<D> >= 16 * kKv4SumRow<D> * 4, "a wave's sums of 16 rows fit where its values were");
    __shared__ __align__(256) char staged[kKv4Waves][kKv4Values<D>];
    __shared__ float wave_top[kKv4Waves][NT * 16], wave_sum_[kKv4Waves][NT * 16];
    __shared__ Kv4Kept kept;
    __shared__ bool is_last[2];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, g = lane >> 4;
    unsigned long long place, share_end;
    Kv4Line<NT * 16> line;
    if (p.apart) {
        line.load(p, (int)blockIdx.y, lane);
        line.before = line.each = line.more = line.shares = 0;
        const unsigned size = (unsigned)__builtin_amdgcn_readlane((int)line.lanes.steps, 0) + kKv4ItemSteps;
        place = (unsigned long long)blockIdx.x * size;
        if (place >= readlane64(line.lanes.cost, 0)) return;
        share_end = place + size;
    } else {
        line.open(p, lane);
        if (blockIdx.x >= line.shares) return;
        place = line.begin(blockIdx.x);
        share_end = line.begin(blockIdx.x + 1);
    }
    for (int slot = 0;; slot = 1) {                              // where the sums of a part of an item go: the share's first or its last
    Kv4ArgsPtr args_here = args;
    asm volatile("" : "+s"(args_here));
    const Kv4AttnParams& p = *(const Kv4AttnParams*)args_here;
    const Kv4 cache = p.cache;                                   // what the steps use
    const float scale_log2 = p.scale_log2;
    const int page_mask = (1 << cache.page_shift) - 1;
    const Kv4Item work = line.find(p, place, lane);
    const unsigned size = work.steps + kKv4ItemSteps, rest = share_end - place < size - work.place ? (unsigned)(share_end - place) : size - work.place;
    const unsigned first_step = work.step_at(work.place), n_steps = work.step_at(work.place + rest) - first_step;
    if (n_steps == 0) break;                                     // the share ends before the item's first step
    const int head = work.head, first_row = work.first_row, n_rows = work.rows * p.group, length = work.length, old = work.old;
    const unsigned begin = first_step * kKv4Step, stop = begin + n_steps * kKv4Step, end = stop < (unsigned)length ? stop : (unsigned)length;

    // Pages of the wave's next 32 steps, two tiles of 16 tokens each: one a lane.
    const int32_t* table = p.page_table + (int64_t)work.seq * p.max_pages;
    auto pages_from = [&](int step) CORAL_INLINE {
        const unsigned token = begin + (unsigned)(step + lane / 2) * kKv4Step + wave * kKv4WaveStep + (lane & 1) * 16;
        return token < end ? table[token >> cache.page_shift] : -1;
    };
    int pages = pages_from(0);
    Kv4Tile<D> k[2][2], v[2][2];
    unsigned now[2];
    bool held[2][2];
    // tiles of a step; a page that is none is read from the cache's first and not seen
    auto fetch = [&](int set, int step) CORAL_INLINE {
        now[set] = begin + (unsigned)step * kKv4Step + wave * kKv4WaveStep;
        if (now[set] >= end) return;                             // (uniform)
        if (step && (step & 31) == 0) pages = pages_from(step);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * (step & 31) + i);
            held[set][i] = page >= 0 && page < cache.pages;
            const int64_t row = (((int64_t)(held[set][i] ? page : 0) * cache.kv_heads + head) << cache.page_shift) + (((int)now[set] + i * 16) & page_mask);
            kv4_load<D>(k[set][i], cache.k_codes + row * (D / 2), cache.k_scales + row * (D / 32), col, g);
            kv4_load<D>(v[set][i], cache.v_codes + row * (D / 2), cache.v_scales + row * (D / 32), col, g);
        }
    };
    fetch(0, 0);
    fetch(1, 1);
    // what is wanted behind the steps goes through LDS: scalar registers are short
    if (threadIdx.x == 0) {
        kept.row0 = work.row0;
        kept.head = head;
        kept.first_row = first_row;
        kept.n_rows = n_rows;
        kept.s0 = line.s0;
        kept.before = line.before;
        kept.place = place + rest;
        kept.share_end = share_end;
        kept.each = line.each;
        kept.more = line.more;
        kept.shares = line.shares;
        kept.parts = 1;
        if (n_steps != work.steps) {
            const unsigned long long start = place - work.place;
            const unsigned w0 = line.share_of(start + kKv4ItemSteps);
            kept.parts = line.share_of(start + size - 1) - w0 + 1;
            kept.w0 = w0;
            kept.opens = line.begin(w0) >= start;
        }
    }

    // the query's operands (rows are below 2^16)
    const float inv_group = reciprocal(p.group);
    uint4 q[NT][TQ][C];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = first_row + n * 16 + col, i = (int)quotient20(r, inv_group);
        const char* from = p.q + (int64_t)(work.row0 + i) * p.q_stride + (int64_t)(head * p.group + r - i * p.group) * (D * kBytes);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (r < n_rows) {
                uint4 raw[DT == kF32 ? 2 : 1];
                load8<DT>(from + kv4_column<D>(c, g) * kBytes, raw);
#pragma unroll
                for (int k = 0; k < (DT == kF32 ? 2 : 1); ++k) {
                    raw[k].x ^= p.q_sign; raw[k].y ^= p.q_sign; raw[k].z ^= p.q_sign; raw[k].w ^= p.q_sign;
                }
                if (TQ == 1) {
                    q[n][0][c] = raw[0];
                } else {
                    float x[8], part[8][TQ];
                    widen8<DT>(raw, x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) split_terms<OT>(x[j], part[j]);
#pragma unroll
                    for (int k = 0; k < TQ; ++k)
                        q[n][k][c] = make_uint4(narrow2<OT>(part[0][k], part[1][k]), narrow2<OT>(part[2][k], part[3][k]),
                                                narrow2<OT>(part[4][k], part[5][k]), narrow2<OT>(part[6][k], part[7][k]));
                }
            } else {
#pragma unroll
                for (int k = 0; k < TQ; ++k) q[n][k][c] = make_uint4(0, 0, 0, 0);
            }
        }
    }
    // which tokens this lane's rows see
    int sees_to[NT];
    uint64_t sees[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = first_row + n * 16 + col, i = (int)quotient20(r < n_rows ? r : n_rows - 1, inv_group);
        sees_to[n] = p.tree ? old : old + i;
        sees[n] = p.tree ? p.tree[work.row0 + i] : 0;
    }

    f32x4_t sum[NT][DTILES];
    float ref[NT], total[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n] = -INFINITY;
        total[n] = 0.f;
#pragma unroll
        for (int d = 0; d < DTILES; ++d) sum[n][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    char* values = staged[wave];
    auto process = [&](int set, int step) CORAL_INLINE {
        // scores: tokens along the registers (4 g + i of each tile), rows along the lanes
        f32x4_t score[NT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) score[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 a = kv4_operand<OT>(k[set][i].code[c], kv4_unit<DT>(k[set][i].scale[c / 4]));
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < TQ; ++t) score[n][i] = mfma_tile<OT>(a, q[n][t][c], score[n][i]);
            }
        }
        // values into LDS, token by token
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c)
                store_vec(reinterpret_cast<uint4*>(values + kv4_place<D>(col) + i * (16 * (D * 2 + 32)) + kv4_column<D>(c, g) * 2),
                          kv4_operand<OT>(v[set][i].code[c], kv4_unit<DT>(v[set][i].scale[c / 4])));
        const int at = (int)now[set];
        const bool held0 = held[set][0], held1 = held[set][1];
        const bool all_seen = at + kKv4WaveStep <= old && held0 && held1;
        fetch(set, step + 2);
        uint4 weight[NT][TP];
        float s[NT][8], to[NT];
        bool any = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[n][j] = score[n][j / 4][j % 4];
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int token = at + (j / 4) * 16 + 4 * g + j % 4, bit = token - old;
                    const bool in = token < sees_to[n] || (bit >= 0 && bit < 64 && (sees[n] >> (bit & 63) & 1));
                    s[n][j] = in && token < length && (j < 4 ? held0 : held1) ? s[n][j] : -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])), fmaxf(fmaxf(s[n][4], s[n][5]), fmaxf(s[n][6], s[n][7])));
            top = lane_xor_max<16>(lane_xor_max<32>(top)) * scale_log2;
            const bool move = top > ref[n] + (kWeightsAt<OT> + kWeightsUpTo) || (ref[n] == -INFINITY && top > -INFINITY);
            to[n] = move ? top - kWeightsAt<OT> : ref[n];
            any |= move;
        }
        if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float keep = to[n] == ref[n] ? 1.f : ref[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[n] - to[n]);
                ref[n] = to[n];
                total[n] *= keep;
#pragma unroll
                for (int d = 0; d < DTILES; ++d) sum[n][d] *= keep;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float base = ref[n] == -INFINITY ? 0.f : ref[n];
            float w[8], part[8][TP];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = __builtin_amdgcn_exp2f(fmaf(s[n][j], scale_log2, -base));
                split_terms<OT>(w[j], part[j]);
            }
            total[n] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
            for (int t = 0; t < TP; ++t)
                weight[n][t] = make_uint4(narrow2<OT>(part[0][t], part[1][t]), narrow2<OT>(part[2][t], part[3][t]),
                                          narrow2<OT>(part[4][t], part[5][t]), narrow2<OT>(part[6][t], part[7][t]));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < DTILES; ++d) {
            const char* from = values + kv4_place<D>(4 * g + col / 4) + d * 32 + (col & 3) * 8;
            const uint2 lo = lds_transposed(from), hi = lds_transposed(from + 16 * (D * 2 + 32));
            const uint4 a = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < TP; ++t) sum[n][d] = mfma_tile<OT>(a, weight[n][t], sum[n][d]);
        }
        __builtin_amdgcn_wave_barrier();
    };
    for (int step = 0; now[0] < end; step += 2) {
        process(0, step);
        if (now[1] >= end) break;
        process(1, step + 1);
    }

    // the waves' sums relative to the largest reference, in the order of the waves
    Kv4ArgsPtr args_again = args;
    asm volatile("" : "+s"(args_again));
    {
    const Kv4AttnParams& p = *(const Kv4AttnParams*)args_again;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float all = lane_xor_sum<16>(lane_xor_sum<32>(total[n]));
        if (g == 0) {
            wave_top[wave][n * 16 + col] = ref[n];
            wave_sum_[wave][n * 16 + col] = all;
        }
    }
    const int row = threadIdx.x / 16, d0 = (threadIdx.x & 15) * (D / 16);
    __syncthreads();
    const Kv4Kept end_of = kv4_kept(kept);
    const float inv_group_ = reciprocal(p.group);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* mine = reinterpret_cast<float*>(staged[wave]);
        if (n) __syncthreads();
#pragma unroll
        for (int d = 0; d < DTILES; ++d)
            *reinterpret_cast<f32x4_t*>(mine + col * kKv4SumRow<D> + d * 16 + 4 * g) = sum[n][d];
        __syncthreads();
        float top = -INFINITY, by[kKv4Waves], all = 0.f;
#pragma unroll
        for (int w = 0; w < kKv4Waves; ++w) top = fmaxf(top, wave_top[w][n * 16 + row]);
#pragma unroll
        for (int w = 0; w < kKv4Waves; ++w) {
            const float t = wave_top[w][n * 16 + row];
            by[w] = t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t - top);
            all = fmaf(by[w], wave_sum_[w][n * 16 + row], all);
        }
        const int r = end_of.first_row + n * 16 + row;
        if (r >= end_of.n_rows) continue;
        float o[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kKv4Waves; ++w) {
            const float* from = reinterpret_cast<const float*>(staged[w]);
#pragma unroll
            for (int j = 0; j < D / 16; j += 4) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(from + row * kKv4SumRow<D> + d0 + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j + i] = by[w] == 0.f ? o[j + i] : fmaf(by[w], x[i], o[j + i]);
            }
        }
        if (end_of.parts > 1) {
            const int64_t at_row = ((int64_t)blockIdx.x * 2 + slot) * (NT * 16) + n * 16 + row;
#pragma unroll
            for (int j = 0; j < D / 16; j += 2) publish2(p.part + at_row * D + d0 + j, o[j], o[j + 1]);
            if (d0 == 0) publish2(&p.part_stats[at_row].x, top, all);
        } else {
            kv4_write<DT, D>(p, end_of, r, inv_group_, d0, o, all);
        }
    }
    if (end_of.parts > 1 && p.join_inside) {
        // The last workgroup of kEach neighbouring parts joins them, into the first one's place, and the last of these joins what has
        // come together so (131072 tokens among 15 short sequences, 14 heads of 64 on 2: 67 us with one workgroup for all
        // parts, 26 so).  Arrivals are counted in the words of the share that the neighbours begin with: word 0 of the item's
        // first share, word 1 of others, which may be another item's first; word 2 of the first for the second step.
        constexpr unsigned kEach = D == 256 ? kKv4JoinParts / 2 : kKv4JoinParts;
        int at_lane = lane, at_wave = wave;
        asm volatile("" : "+v"(at_lane), "+s"(at_wave));         // (what follows from them would be held from the beginning on, and spilled)
        const unsigned mine = blockIdx.x - end_of.w0, first = mine - mine % kEach, groups = (end_of.parts + kEach - 1) / kEach;
        const unsigned in_group = end_of.parts - first < kEach ? end_of.parts - first : kEach;
        auto place_of = [&](unsigned j) CORAL_INLINE { return ((int64_t)(end_of.w0 + j) * 2 + (j == 0 && !end_of.opens ? 1 : 0)) * (NT * 16); };
        auto arrive = [&](unsigned* word, unsigned of, bool& last) CORAL_INLINE {
            __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wave's stores are out
            __syncthreads();
            if (threadIdx.x == 0) {
                const unsigned old = __hip_atomic_fetch_add(word, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last = old + 1 == of;
                if (last) __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            return last;
        };
        unsigned from = first, n = in_group, step = 1;
        bool whole = groups == 1;
        unsigned* word = p.arrived + (end_of.w0 + first) * kKv4ArrivalStride + (first ? 1 : 0);
        while (arrive(word, n, is_last[whole])) {                // (uniform)
            for (int r = at_wave; r < NT * 16 && end_of.first_row + r < end_of.n_rows; r += kKv4Waves) {
                float o[D / kWave], top, all;
                kv4_join_row<D>(p, n, at_lane, [&](unsigned j) CORAL_INLINE { return place_of(from + j * step) + r; }, o, top, all);
                if (whole) {
                    kv4_write_row<DT, D>(p, end_of, end_of.first_row + r, inv_group_, at_lane, o, all);
                    continue;
                }
                const int64_t at_row = place_of(from) + r;
                if (D == kWave) __hip_atomic_store(reinterpret_cast<unsigned*>(p.part + at_row * D + at_lane), __float_as_uint(o[0]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int i = 0; i + 1 < D / kWave; i += 2) publish2(p.part + at_row * D + at_lane * (D / kWave) + i, o[i], o[i + 1]);
                if (at_lane == 0) publish2(&p.part_stats[at_row].x, top, all);
            }
            if (whole) break;
            whole = true;
            from = 0;
            n = groups;
            step = kEach;
            word = p.arrived + end_of.w0 * kKv4ArrivalStride + 2;
        }
    }
    asm volatile("" ::: "memory");                               // (read again: held over the join they would be spilled)
    const Kv4Kept next = kv4_kept(kept);
    place = next.place;
    share_end = next.share_end;
    if (place >= share_end) return;
    __syncthreads();                                             // the sums have been read: the next item's values may come
    line.load(p, next.s0, lane);
    line.before = next.before;
    line.each = next.each;
    line.more = next.more;
    line.shares = next.shares;
    line.inv_shares = reciprocal(line.shares ? line.shares : 1);
    }
    }
}

// Joins the parts of an item that several workgroups have taken: WAVES waves a row, which take parts in turn.  Bound by its chain (arguments,
// shares, parts): 4 to 5 us, 8 for 7784 rows.
template <int DT, int D, int NT, int WAVES>
__global__ __launch_bounds__(kKv4Threads) void k_kv4_join(Kv4AttnParams p) {
    constexpr int N = D / kWave, kBytes = DT == kF32 ? 4 : 2, kRows = NT * 16;
    static_assert(WAVES == 1 || WAVES == kKv4Waves, "");
    __shared__ float sums[kKv4Waves][D];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int t = blockIdx.x, of_row = wave % WAVES;
    Kv4Line<kRows> line;
    unsigned long long total = 0, base = 0;
    unsigned steps = 0, blocks = 0;
    int row = 0;
    for (int s = 0; s < p.S; s += kWave) {
        line.load(p, s, lane);
        const uint64_t found = __builtin_amdgcn_ballot_w64(t >= line.lanes.row0 && t < line.lanes.row0 + line.lanes.rows);
        if (found) {
            const int src = __builtin_ctzll(found);
            const Kv4Item first = line.at(p, src, 0);
            steps = first.steps;
            if (steps == 1) return;                              // one workgroup's, which has written it
            row = (t - first.row0) * p.group;
            blocks = (unsigned)(first.rows * p.group + kRows - 1) / kRows;
            base = total + readlane64(line.upto, src) - readlane64(line.lanes.cost, src);
        }
        total += readlane64(line.upto, kWave - 1);
    }
    if (!steps) return;                                          // a row of no sequence
    line.deal(p, total);
    for (int h = 0; h < p.join_heads; ++h) {                     // (four waves a row: one)
        const int q_head = (blockIdx.y * p.join_heads + h) * (kKv4Waves / WAVES) + wave / WAVES;
        if (q_head >= p.group * p.kv_heads) return;
        const int of_kv = q_head / p.group, r = row + q_head - of_kv * p.group;
        const unsigned long long start = base + (unsigned long long)(of_kv * blocks + r / kRows) * (steps + kKv4ItemSteps);
        const unsigned long long end = start + kKv4ItemSteps + steps;
        const unsigned w0 = line.share_of(start + kKv4ItemSteps), last = line.share_of(end - 1);
        if (w0 == last) continue;
        // part j: share w0 + j; the first lies behind what else its share holds, unless it begins with the item
        const int64_t first = ((int64_t)w0 * 2 + (line.begin(w0) >= start ? 0 : 1)) * kRows + r % kRows, others = (int64_t)(w0 + 1) * 2 * kRows + r % kRows;
        const int parts = (int)(last - w0) + 1;
        auto row_of = [&](int j) CORAL_INLINE { return j == 0 ? first : others + (int64_t)(j - 1) * 2 * kRows; };
        float ref = -INFINITY, all = 0.f, o[N];
#pragma unroll
        for (int n = 0; n < N; ++n) o[n] = 0.f;
        for (int j0 = 0; j0 < parts; j0 += kWave) {
            float2 stat = make_float2(-INFINITY, 0.f);
            if (j0 + lane < parts) stat = p.part_stats[row_of(j0 + lane)];
            const int left = parts - j0 < kWave ? parts - j0 : kWave;
            float x[8][N];
            auto load = [&](int i) CORAL_INLINE {                    // eight parts of the wave's
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int j = i + u * WAVES + of_row;
                    const float* from = p.part + row_of(j0 + (j < left ? j : left - 1)) * D + lane * N;
#pragma unroll
                    for (int n = 0; n < N; ++n) x[u][n] = from[n];
                }
            };
            load(0);
            float top = lane_xor_max<16>(lane_xor_max<32>(lanes_reduce<16>(stat.x, [](float a, float b) { return fmaxf(a, b); })));
            top = fmaxf(top, ref);
            const float keep = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top), by = stat.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat.x - top);
            ref = top;
            all = fmaf(all, keep, by * stat.y);
#pragma unroll
            for (int n = 0; n < N; ++n) o[n] *= keep;
            for (int i = 0;;) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int j = i + u * WAVES + of_row;
                    const float f = j < left ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), j & (kWave - 1))) : 0.f;
#pragma unroll
                    for (int n = 0; n < N; ++n) o[n] = f == 0.f ? o[n] : fmaf(f, x[u][n], o[n]);
                }
                i += 8 * WAVES;
                if (i >= left) break;
                load(i);
            }
        }
        all = wave_sum(all);
        char* to = p.out + (int64_t)t * p.out_stride + (int64_t)q_head * (D * kBytes);
        auto put = [&](int d, float v) CORAL_INLINE {
            const float y = all > 0.f ? v / all : all == 0.f ? 0.f : all;
            if (DT == kF32) reinterpret_cast<float*>(to)[d] = y;
            else reinterpret_cast<unsigned short*>(to)[d] = narrow16<DT>(y);
        };
        if (WAVES == 1) {
#pragma unroll
            for (int n = 0; n < N; ++n) put(lane * N + n, o[n]);
            continue;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) sums[wave][lane * N + n] = o[n];
        __syncthreads();
        if (threadIdx.x >= D) return;
        const int d = threadIdx.x;
        put(d, (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]));
    }
}

using kv4_attn_fn = void (*)(Kv4AttnParams);
using kv4_join_fn = void (*)(Kv4AttnParams);
// The weights p of bf16 and fp16 calls are two values of that type where a wave has one tile (which memory bounds: no cost;
// the result's only rounding is then its own) and one where it has more (the products bound it: a second would take half
// as long again; with the roundings of single weights, 2^-9 and 2^-12 each, the error against 64 bits is 1.2 (16 nodes, 4000 tokens) to
// 1.4 (131072 tokens) times that of the result's rounding alone).
template <int DT, int D>
kv4_attn_fn kv4_kernel(int tiles) {
    constexpr int most = kv4_most_tiles(D, kv4_terms(DT)), many = kv4_terms(DT);
    if (tiles == 2) return k_kv4_attention<DT, D, most >= 2 ? 2 : 1, most >= 2 ? many : DT == kF32 ? 3 : 2>;
    return k_kv4_attention<DT, D, 1, DT == kF32 ? 3 : 2>;
}
template <int DT, int D>
kv4_join_fn kv4_join(int tiles, bool wave_a_row) {
    constexpr int many = kv4_most_tiles(D, kv4_terms(DT)) >= 2 ? 2 : 1;
    if (tiles == 2) return wave_a_row ? k_kv4_join<DT, D, many, 1> : k_kv4_join<DT, D, many, kKv4Waves>;
    return wave_a_row ? k_kv4_join<DT, D, 1, 1> : k_kv4_join<DT, D, 1, kKv4Waves>;
}

}  // namespace
