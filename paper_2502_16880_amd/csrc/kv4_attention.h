// Attention over a cache of 4-bit floats.
//
//   out[t,h] = sum_j p_j v_j,  p = softmax_j(scale * q[t,h] . k_j)  over the cached tokens j that row t sees
//
// Codes become bf16 operands of the matrix cores exactly (one conversion instruction for two values, the
// unit of their 32 included), so scores and sums have exact products and fp32 sums.  A wave takes 32
// tokens a step: 16 bytes of a token's key a lane, in the order of memory (D = 128: the whole KB of 16 keys
// in one load); which of the lane's values goes with which column of a product is free as long as the
// query's operand has the same order.  Scores come out with the token along a lane's registers, which is
// how the second product wants the weights; the values' operand needs eight tokens of one column in a
// lane, so converted values pass through the wave's part of LDS and come back transposed
// (ds_read_b64_tr_b16).  Softmax is taken in one pass: sums are kept relative to a reference of each
// row that is moved up only when a score passes it by 2^8, so most steps do not touch the sums.
// fp16 queries are two bf16 values and fp32 ones three (exactly); so are the weights p.
#pragma once
#include "attention_common.h"
#include "kv4_plan.h"

namespace {

constexpr int kKv4Threads = 256;
constexpr int kKv4Waves = kKv4Threads / kWave;
constexpr int kKv4WaveStep = kKv4Step / kKv4Waves;          // 32 tokens
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kMoveAt = 8.f;                               // weights stay below 2^8

struct Kv4AttnParams {
    const char* q;
    char* out;
    int64_t q_stride, out_stride;       // bytes from token to token
    Kv4 cache;
    const int32_t *page_table, *lengths, *q_offsets, *history;
    const uint64_t* tree;
    float* part;                        // [item][split][row][D] sums, then [item][split][row] (largest, sum) pairs
    float2* part_stats;
    int max_pages, T, max_rows, group, kv_heads, row_blocks, splits, q_heads;
    float scale_log2;                   // scores are kept in powers of two
};

// What the arguments say about a sequence, cut to the arrays.
struct Kv4Seq {
    int row0, rows, length, seen_by_all, history;
    bool tree;
};
__device__ __forceinline__ Kv4Seq kv4_sequence(const Kv4AttnParams& p, int s) {
    Kv4Seq q;
    const int a = p.q_offsets[s], b = p.q_offsets[s + 1];
    q.row0 = a < 0 ? 0 : a > p.T ? p.T : a;
    const int end = b > p.T ? p.T : b;
    q.rows = end - q.row0 < p.max_rows ? end - q.row0 : p.max_rows;
    const int64_t room = (int64_t)p.max_pages << p.cache.page_shift;
    int length = p.lengths[s];
    length = length < 0 ? 0 : length > room ? (int)room : length;
    q.tree = p.tree != nullptr;
    if (q.tree) {
        const int h = p.history[s];
        q.history = h < 0 ? 0 : h > length ? length : h;
        q.length = length - q.history > 64 ? q.history + 64 : length;
        q.seen_by_all = q.history;
    } else {
        q.history = 0;
        q.length = length;
        q.seen_by_all = length - (q.rows - 1);                  // row i of n sees tokens up to length - n + i
    }
    return q;
}
// Tokens of one split: a multiple of the workgroup's step.
__device__ __forceinline__ int kv4_chunk(int length, int splits) {
    const int steps = (length + kKv4Step - 1) / kKv4Step;
    return (steps + splits - 1) / splits * kKv4Step;
}

// N bf16 values whose sum is x (8 bits more each).
template <int N>
__device__ __forceinline__ void split_bf16(float x, float (&part)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = (float)(__bf16)x;
        x -= part[i];
    }
}

// A dword of codes with its unit as eight bf16 values.
__device__ __forceinline__ uint4 kv4_operand(unsigned codes, float unit) {
    uint4 r;
    r.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
    r.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
    r.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
    r.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
    return r;
}
__device__ __forceinline__ float kv4_unit(unsigned byte) {
    return __uint_as_float((byte < kKv4LargestScale ? byte : kKv4LargestScale) << 23);
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
__device__ __forceinline__ void kv4_load(Kv4Tile<D>& t, const unsigned char* codes, const unsigned char* scales, int token, int g) {
    if (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2*>(codes + token * 32 + g * 8);
        t.code[0] = w.x;
        t.code[1] = w.y;
        t.scale[0] = scales[token * 2 + g / 2];
    } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
            const uint4 w = load_stream(reinterpret_cast<const uint4*>(codes + token * (D / 2) + i * 64 + g * 16));
            t.code[4 * i % Kv4Tile<D>::kDwords] = w.x;
            t.code[(4 * i + 1) % Kv4Tile<D>::kDwords] = w.y;
            t.code[(4 * i + 2) % Kv4Tile<D>::kDwords] = w.z;
            t.code[(4 * i + 3) % Kv4Tile<D>::kDwords] = w.w;
            t.scale[i % Kv4Tile<D>::kScales] = scales[token * (D / 32) + i * 4 + g];
        }
    }
}

__device__ __forceinline__ f32x4_t mfma_bf16(uint4 a, uint4 b, f32x4_t acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
// Four rows of LDS, 16 columns: lane l of sixteen gets column l of the rows whose pieces the lanes point at
// (lane l: row l / 4, columns 4 (l % 4) on).
__device__ __forceinline__ uint2 lds_transposed(const unsigned short* at) {
    const s16x4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4_t*)const_cast<unsigned short*>(at));
    return __builtin_bit_cast(uint2, r);
}

template <int D>
constexpr int kKv4LdsRow = D + 16;                           // values from token to token: 16 rows in different banks
template <int D>
constexpr int kKv4SumRow = D + 4;                            // floats from row to row when the waves' sums meet

// One workgroup: NT tiles of 16 rows of one sequence and one head of keys, one split of its tokens; its four
// waves take steps of 32 tokens in turn and add up at the end.
template <int DT, int D, int NT, int TP>
__global__ __launch_bounds__(kKv4Threads) void k_kv4_attention(Kv4AttnParams p) {
    constexpr int TQ = DT == kBF16 ? 1 : DT == kF16 ? 2 : 3, C = D / 32, DTILES = D / 16, kBytes = DT == kF32 ? 4 : 2;
    constexpr int kWaveValues = kKv4WaveStep * kKv4LdsRow<D>;
    static_assert(kWaveValues * 2 >= 16 * kKv4SumRow<D> * 4, "a wave's sums fit where its values were");
    __shared__ __align__(16) unsigned short staged[kKv4Waves][kWaveValues];
    __shared__ float wave_top[kKv4Waves][NT * 16], wave_sum_[kKv4Waves][NT * 16];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, head = blockIdx.y / p.row_blocks, block = blockIdx.y % p.row_blocks;
    const Kv4Seq seq = kv4_sequence(p, blockIdx.z);
    const int n_rows = seq.rows * p.group, first_row = block * NT * 16;
    if (first_row >= n_rows) return;
    const int chunk = kv4_chunk(seq.length, p.splits);
    const int used = seq.length > 0 ? (seq.length + chunk - 1) / chunk : 1;
    if (split >= used) return;
    const int begin = split * chunk, end = begin + chunk < seq.length ? begin + chunk : seq.length;

    // the query's operands
    uint4 q[NT][TQ][C];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = first_row + n * 16 + col, i = r / p.group;
        const char* from = p.q + (int64_t)(seq.row0 + i) * p.q_stride + (int64_t)(head * p.group + r % p.group) * (D * kBytes);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (r < n_rows) {
                uint4 raw[DT == kF32 ? 2 : 1];
                load8<DT>(from + kv4_column<D>(c, g) * kBytes, raw);
                if (DT == kBF16) {
                    q[n][0][c] = raw[0];
                } else {
                    float x[8], part[8][TQ];
                    widen8<DT>(raw, x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) split_bf16<TQ>(x[j], part[j]);
#pragma unroll
                    for (int k = 0; k < TQ; ++k)
                        q[n][k][c] = make_uint4(narrow2<kBF16>(part[0][k], part[1][k]), narrow2<kBF16>(part[2][k], part[3][k]),
                                                narrow2<kBF16>(part[4][k], part[5][k]), narrow2<kBF16>(part[6][k], part[7][k]));
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
        const int r = first_row + n * 16 + col, i = (r < n_rows ? r : n_rows - 1) / p.group;
        sees_to[n] = seq.tree ? seq.history : seq.length - seq.rows + i + 1;
        sees[n] = seq.tree ? p.tree[seq.row0 + i] : 0;
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
    unsigned short* values = staged[wave];
    const int32_t* table = p.page_table + (int64_t)blockIdx.z * p.max_pages;
    const int page_mask = (1 << p.cache.page_shift) - 1;
    // the pages of the wave's next 32 steps, two tiles of 16 tokens each: one a lane
    int pages = 0, step = 0;
    auto fetch_pages = [&]() CORAL_INLINE {
        const int token = begin + ((step + lane / 2) * kKv4Waves + wave) * kKv4WaveStep + (lane & 1) * 16;
        pages = token < end ? table[token >> p.cache.page_shift] : -1;
    };
    Kv4Tile<D> k[2], v[2];
    bool held[2];
    // tiles of a step; a page that is none (or behind the end) is read from the cache's first and not seen
    auto fetch = [&](int at) CORAL_INLINE {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * (step & 31) + i);
            held[i] = page >= 0 && page < p.cache.pages;
            const int64_t row = (((int64_t)(held[i] ? page : 0) * p.kv_heads + head) << p.cache.page_shift) + ((at + i * 16) & page_mask);
            kv4_load<D>(k[i], p.cache.k_codes + row * (D / 2), p.cache.k_scales + row * (D / 32), col, g);
            kv4_load<D>(v[i], p.cache.v_codes + row * (D / 2), p.cache.v_scales + row * (D / 32), col, g);
        }
    };
    int at = begin + wave * kKv4WaveStep;
    if (at < end) {
        fetch_pages();
        fetch(at);
    }
    while (at < end) {
        // scores: tokens along the registers (4 g + i of each tile), rows along the lanes
        f32x4_t score[NT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) score[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 a = kv4_operand(k[i].code[c], kv4_unit(k[i].scale[c / 4]));
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < TQ; ++t) score[n][i] = mfma_bf16(a, q[n][t][c], score[n][i]);
            }
        }
        // values into LDS, token by token
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c)
                store_vec(reinterpret_cast<uint4*>(values + (i * 16 + col) * kKv4LdsRow<D> + kv4_column<D>(c, g)),
                          kv4_operand(v[i].code[c], kv4_unit(v[i].scale[c / 4])));
        const bool all_seen = at + kKv4WaveStep <= seq.seen_by_all && at + kKv4WaveStep <= end && held[0] && held[1];
        const bool held0 = held[0], held1 = held[1];
        const int now = at;
        at += kKv4Step;
        ++step;
        if (at < end) {
            if ((step & 31) == 0) fetch_pages();
            fetch(at);
        }
        uint4 weight[NT][TP];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = score[n][j / 4][j % 4] * p.scale_log2;
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int token = now + (j / 4) * 16 + 4 * g + j % 4, bit = token - seq.history;
                    const bool in = token < sees_to[n] || (bit >= 0 && bit < 64 && (sees[n] >> (bit & 63) & 1));
                    s[j] = in && token < seq.length && (j < 4 ? held0 : held1) ? s[j] : -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
            top = lane_xor_max<16>(lane_xor_max<32>(top));
            const bool move = top > ref[n] + kMoveAt || (ref[n] == -INFINITY && top > -INFINITY);
            if (__builtin_amdgcn_ballot_w64(move)) {
                const float to = move ? top : ref[n];
                const float by = ref[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[n] - to);
                const float keep = move ? by : 1.f;
                ref[n] = to;
                total[n] *= keep;
#pragma unroll
                for (int d = 0; d < DTILES; ++d) sum[n][d] *= keep;
            }
            const float base = ref[n] == -INFINITY ? 0.f : ref[n];
            float w[8], part[8][TP];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = __builtin_amdgcn_exp2f(s[j] - base);
                split_bf16<TP>(w[j], part[j]);
            }
            total[n] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
            for (int t = 0; t < TP; ++t)
                weight[n][t] = make_uint4(narrow2<kBF16>(part[0][t], part[1][t]), narrow2<kBF16>(part[2][t], part[3][t]),
                                          narrow2<kBF16>(part[4][t], part[5][t]), narrow2<kBF16>(part[6][t], part[7][t]));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < DTILES; ++d) {
            const unsigned short* from = values + (4 * g + col / 4) * kKv4LdsRow<D> + d * 16 + (col & 3) * 4;
            const uint2 lo = lds_transposed(from), hi = lds_transposed(from + 16 * kKv4LdsRow<D>);
            const uint4 a = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < TP; ++t) sum[n][d] = mfma_bf16(a, weight[n][t], sum[n][d]);
        }
        __builtin_amdgcn_wave_barrier();
    }

    // the waves' sums relative to the largest reference, in the order of the waves
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float all = lane_xor_sum<16>(lane_xor_sum<32>(total[n]));
        if (g == 0) {
            wave_top[wave][n * 16 + col] = ref[n];
            wave_sum_[wave][n * 16 + col] = all;
        }
    }
    const int row = threadIdx.x / 16, d0 = (threadIdx.x & 15) * (D / 16);
    const int64_t item = ((int64_t)blockIdx.z * p.kv_heads + head) * p.row_blocks + block;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* mine = reinterpret_cast<float*>(staged[wave]);
        __syncthreads();
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
        const int r = first_row + n * 16 + row;
        if (r >= n_rows) continue;
        float o[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kKv4Waves; ++w) {
            const float* from = reinterpret_cast<const float*>(staged[w]) + row * kKv4SumRow<D> + d0;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] = by[w] == 0.f ? o[j] : fmaf(by[w], from[j], o[j]);
        }
        if (used > 1) {
            const int64_t at_row = (item * p.splits + split) * (NT * 16) + n * 16 + row;
#pragma unroll
            for (int j = 0; j < D / 16; j += 4)
                *reinterpret_cast<f32x4_t*>(p.part + at_row * D + d0 + j) = f32x4_t{o[j], o[j + 1], o[j + 2], o[j + 3]};
            if (d0 == 0) p.part_stats[at_row] = make_float2(top, all);
        } else {
            const float inv = all > 0.f ? 1.f / all : all == 0.f ? 0.f : all;      // a row that sees nothing: zeros
            char* to = p.out + (int64_t)(seq.row0 + r / p.group) * p.out_stride + (int64_t)(head * p.group + r % p.group) * (D * kBytes) + d0 * kBytes;
#pragma unroll
            for (int j = 0; j < D / 16; j += 4) {
                if (DT == kF32) {
                    *reinterpret_cast<f32x4_t*>(to + j * 4) = f32x4_t{o[j] * inv, o[j + 1] * inv, o[j + 2] * inv, o[j + 3] * inv};
                } else {
                    *reinterpret_cast<uint2*>(to + j * 2) = make_uint2(narrow2<DT>(o[j] * inv, o[j + 1] * inv), narrow2<DT>(o[j + 2] * inv, o[j + 3] * inv));
                }
            }
        }
    }
}

// Joins the splits of a row: one workgroup a row, its waves take splits in turn.
template <int DT, int D>
__global__ __launch_bounds__(kKv4Threads) void k_kv4_join(Kv4AttnParams p, int tiles) {
    constexpr int N = D / kWave, kBytes = DT == kF32 ? 4 : 2;
    __shared__ float sums[kKv4Waves][D];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int q_head = blockIdx.x, i = blockIdx.y;
    const Kv4Seq seq = kv4_sequence(p, blockIdx.z);
    if (i >= seq.rows || seq.length <= 0) return;
    const int chunk = kv4_chunk(seq.length, p.splits), used = (seq.length + chunk - 1) / chunk;
    if (used < 2) return;                                     // written already
    const int head = q_head / p.group, r = i * p.group + q_head % p.group, rows = tiles * 16;
    const int64_t item = ((int64_t)blockIdx.z * p.kv_heads + head) * p.row_blocks + r / rows;
    const int64_t first = item * p.splits * rows + r % rows;  // the row in split s: first + s * rows
    // each wave looks at all splits' statistics, at most four a lane
    float top = -INFINITY;
    float2 stat[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int s = j * kWave + lane;
        stat[j] = s < used ? p.part_stats[first + (int64_t)s * rows] : make_float2(-INFINITY, 0.f);
        top = fmaxf(top, stat[j].x);
    }
    top = lane_xor_max<16>(lane_xor_max<32>(lanes_reduce<16>(top, [](float a, float b) { return fmaxf(a, b); })));
    float all = 0.f, by[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        by[j] = stat[j].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[j].x - top);
        all = fmaf(by[j], stat[j].y, all);
    }
    all = wave_sum(all);
    float o[N];
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll 4
        for (int s = j * kWave + wave; s < (j + 1) * kWave && s < used; s += kKv4Waves) {
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by[j]), s & (kWave - 1)));
            const float* from = p.part + (first + (int64_t)s * rows) * D + lane * N;
#pragma unroll
            for (int n = 0; n < N; ++n) o[n] = f == 0.f ? o[n] : fmaf(f, from[n], o[n]);
        }
#pragma unroll
    for (int n = 0; n < N; ++n) sums[wave][lane * N + n] = o[n];
    __syncthreads();
    if (threadIdx.x >= D) return;
    const int d = threadIdx.x;
    const float v = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
    const float y = all > 0.f ? v / all : all == 0.f ? 0.f : all;
    char* to = p.out + (int64_t)(seq.row0 + i) * p.out_stride + ((int64_t)q_head * D + d) * kBytes;
    if (DT == kF32) *reinterpret_cast<float*>(to) = y;
    else *reinterpret_cast<unsigned short*>(to) = narrow16<DT>(y);
}

using kv4_attn_fn = void (*)(Kv4AttnParams);
using kv4_join_fn = void (*)(Kv4AttnParams, int);
// The weights p of bf16 calls are two bf16 values where a wave has one tile (which memory bounds: no cost; the result's
// only rounding is then its own) and one where it has more (the products bound it: a second term would
// take a third longer; the roundings of single weights, 2^-9 each, average out to about the result's own).
template <int DT, int D>
kv4_attn_fn kv4_kernel(int tiles) {
    constexpr int terms = DT == kBF16 ? 1 : DT == kF16 ? 2 : 3, most = 512 / (D * terms), many = DT == kBF16 ? 1 : terms;
    if (tiles == 4) return k_kv4_attention<DT, D, most >= 4 ? 4 : 1, most >= 4 ? many : DT == kF32 ? 3 : 2>;
    if (tiles == 2) return k_kv4_attention<DT, D, most >= 2 ? 2 : 1, most >= 2 ? many : DT == kF32 ? 3 : 2>;
    return k_kv4_attention<DT, D, 1, DT == kF32 ? 3 : 2>;
}

}  // namespace
