// Causal attention over whole prompts, packed one behind the other.
//
//   out[t,h] = sum_j p_j v_j,  p = softmax_j(scale * q[t,h] . k_j)  over j <= m - n + i for row i of a sequence
//   of n rows and m keys
//
// A workgroup takes 128 rows (fp32: 64) of one sequence and head and passes over the keys once, 64 at a time
// (D = 256: 32), with the running largest score and sum of each row; a wave's rows, their sums and
// weights never leave its registers.  Scores are taken as K Q^T, so that keys lie along a lane's registers
// and rows along the lanes: that is how the second product, V^T P^T, wants its weights, and a row's maximum
// is one exchange between halves of the wave.  Keys and values go through LDS once for all waves, in 16-byte
// pieces whose place in a row is exchanged by the row's number, so that neither the reading of keys (16 rows, one
// piece each) nor the transposing one of values (four rows, four pieces each) meets a bank twice.
#pragma once
#include "attention_tiles.h"

#include <type_traits>

namespace {

constexpr float kNoReference = -3.402823466e38f;             // of a row before its first score: finite, so that a weight of -inf is zero
constexpr int kXcds = 8;
constexpr int kPromptLevelled = kWave;                      // sequences beyond which tiles come in the sequences' order

struct PromptParams {
    const char *q, *k, *v;
    char* out;
    int64_t q_stride, k_stride, v_stride, out_stride;        // bytes from token to token
    const int32_t *q_offsets, *k_offsets;
    int T, keys, S, q_heads, group, tiles, parts;            // tiles: of rows, at most, over all sequences; parts: of a head's tiles
    float scale_log2;                                        // above zero; the sign is taken by q
    unsigned q_sign;                                         // bit to flip in every value of q
};

// Which rows a workgroup takes.
struct PromptTile {
    int head, row0, rows, first, k0, keys;                   // the sequence's rows and keys, and the tile's first row in it
    bool any;
};
// A sequence a lane: its rows, its tiles, and a tile's level: how many blocks of ROWS keys its last row sees (the levels of a
// sequence's tiles are base + 1 .. base + tiles).
struct PromptSeq {
    int row0, rows, tiles, base;
};
template <int ROWS>
__device__ __forceinline__ PromptSeq prompt_sequence(const PromptParams& p, int s) {
    PromptSeq q = {0, 0, 0, 0};
    if (s >= p.S) return q;
    q.row0 = cut_offset(p.q_offsets[s], p.T);
    q.rows = cut_offset(p.q_offsets[s + 1], p.T) - q.row0;
    q.rows = q.rows < 0 ? 0 : q.rows;
    q.tiles = (q.rows + ROWS - 1) / ROWS;
    if (p.k_offsets) {
        const int64_t before = (int64_t)p.k_offsets[s + 1] - p.k_offsets[s] - q.rows;       // (where the offsets are wrong any number: the order only)
        q.base = before <= 0 ? 0 : before > (1 << 30) ? (1 << 30) / ROWS : (int)before / ROWS;
    }
    return q;
}
__device__ __forceinline__ int wave_sum_int(int x) { return __builtin_amdgcn_readlane(wave_scan_inclusive(x), kWave - 1); }

// Workgroups are dealt to the eight dies in turn, and a die takes neighbouring heads, whose keys are then read through one
// L2: of `parts` as few as make the heads' parts a multiple of eight, a part being every parts-th tile.  Tiles of all of a
// die's heads come by their levels, the longest first (each pair on one card): twelve prompts of 8191 tokens whose tiles came in order took 148 us,
// the last of them alone, against 118; one of 8192 whose tiles came head after head 527 us against 508, of 2115 64 against 55.
// More than 64 sequences come in their own order, found by a search (levels of 256 prompts of 300 tokens: 994 us, order 664).
template <int ROWS>
__device__ __forceinline__ PromptTile prompt_tile(const PromptParams& p, int x, int lane) {
    PromptTile r = {};
    const int die = x % kXcds, local = x / kXcds, mine = p.q_heads * p.parts / kXcds;        // heads' parts of a die
    const int per = (p.tiles + p.parts - 1) / p.parts;
    const int of = local % mine, at = local / mine;
    if (at >= per) return r;
    const int part = die * mine + of;
    r.head = part / p.parts;
    const int rank = at * p.parts + part % p.parts;
    PromptSeq q = prompt_sequence<ROWS>(p, p.S == 1 ? 0 : lane);
    int seq = 0, src = 0;
    if (p.S == 1) {
        r.first = (__builtin_amdgcn_readfirstlane(q.tiles) - 1 - rank) * ROWS;
        r.any = r.first >= 0;
    } else if (p.S > kPromptLevelled) {
        // sequence s has the places from before(s) on: at least as many as it has tiles
        auto before = [&](int s) CORAL_INLINE { return cut_offset(p.q_offsets[s], p.T) / ROWS + s; };
        for (int n = p.S; n > 1;) {                          // among the n from seq on, 64 at once
            const int step = (n + kWave - 1) / kWave;
            const bool reached = lane * step < n && before(seq + (lane * step < n ? lane * step : 0)) <= rank;
            const uint64_t behind = ~__builtin_amdgcn_ballot_w64(reached);
            const int last = behind ? __builtin_ctzll(behind) - 1 : kWave - 1;
            if (last < 0) return r;
            seq += last * step;
            n = n - last * step < step ? n - last * step : step;
        }
        q = prompt_sequence<ROWS>(p, seq);
        const int i = rank - __builtin_amdgcn_readfirstlane(before(seq)), tiles = __builtin_amdgcn_readfirstlane(q.tiles);
        r.first = (tiles - 1 - i) * ROWS;
        r.any = i >= 0 && i < tiles;
    } else {
        // the largest level l that, with all above it, has more than `rank` tiles
        auto from_level = [&](int l) CORAL_INLINE {
            const int k = q.tiles + q.base - l + 1;
            return wave_sum_int(k < 0 ? 0 : k > q.tiles ? q.tiles : k);
        };
        if (from_level(1) <= rank) return r;
        const float top = q.tiles ? (float)(q.tiles + q.base) : 0.f;       // (to 24 bits: a few levels too many at most)
        int low = 1, high = __builtin_amdgcn_readfirstlane((int)(lane_xor_max<16>(lane_xor_max<32>(lanes_reduce<16>(top, [](float x, float y) { return fmaxf(x, y); }))) * 1.000001f)) + 2;
        while (high - low > 1) {                             // from_level(low) > rank >= from_level(high)
            const int mid = low + (high - low) / 2;
            if (from_level(mid) > rank) low = mid;
            else high = mid;
        }
        const int left = rank - from_level(high);            // so many sequences of the level come before
        const int i = low - 1 - q.base;
        const bool has = i >= 0 && i < q.tiles;
        const uint64_t all = __builtin_amdgcn_ballot_w64(has);
        seq = src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(has && __builtin_popcountll(all & ((1ull << lane) - 1ull)) == left));
        r.any = true;
        r.first = __builtin_amdgcn_readlane(i, src) * ROWS;
    }
    if (!r.any) return r;
    r.row0 = __builtin_amdgcn_readlane(q.row0, src);
    r.rows = __builtin_amdgcn_readlane(q.rows, src);
    r.k0 = r.row0;
    r.keys = r.rows;
    if (p.k_offsets) {
        r.k0 = cut_offset(p.k_offsets[seq], p.keys);
        r.keys = cut_offset(p.k_offsets[seq + 1], p.keys) - r.k0;
        r.keys = r.keys < 0 ? 0 : r.keys;
    }
    return r;
}

// Two 16-bit values, those that are infinite or NaN made zero; `odd` tells whether there were any.
template <int DT>
__device__ __forceinline__ unsigned only_finite2(unsigned w, bool& odd) {
    const unsigned e = DT == kF16 ? 0x7c00u : 0x7f80u;
    const bool lo = (w & e) == e, hi = (w >> 16 & e) == e;
    odd |= lo | hi;
    return (lo ? 0u : w & 0xffffu) | (hi ? 0u : w & 0xffff0000u);
}
__device__ __forceinline__ unsigned only_finite(unsigned w, bool& odd) {
    const bool bad = (w & 0x7f800000u) == 0x7f800000u;
    odd |= bad;
    return bad ? 0u : w;
}
// Keys 0 .. most of a tile, one bit each.
__device__ __forceinline__ unsigned long long keys_to(int most) { return most < 0 ? 0ull : most > 62 ? ~0ull : (2ull << most) - 1ull; }

// A wave's 64 pieces of 16 bytes from memory into 1 KB of LDS, past the registers; what lies behind the view's end comes as
// zero.  Nothing waits for it but dma_arrived.  (m0 is the compiler's own to write, and these kernels give it no other use:
// neither dynamic register indexes nor messages.)
__device__ __forceinline__ void dma_piece(Buffer from, unsigned at, unsigned lds_place) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(at), "s"(from), "s"(lds_place) : "memory");
}
__device__ __forceinline__ void dma_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Bound by the matrix cores and the clock they leave (8192 tokens, 32 heads of 128: 515 to 557 us by card, 635 in calls one behind the
// other; 1.07 to 0.87 PFLOP/s), where tiles of rows are few by a row's chain: 1.0 us for a tile of keys, 0.43 of it products, and 5 before
// and behind (300 tokens: 11.8; twelve prompts of 8191: 111 to 125, 136).
// 128 rows a workgroup, as two of them fill a compute unit's registers and LDS and share their keys' reading.
// A tile's weights are summed by themselves before they are added to the row's total: of tens of thousands of weights below 2^-25 of it
// that are added two at a time none would arrive.
// 16-bit types.  Weights p are rounded to the storage type, as the products' operand: errors of 2^-9
// (2^-12) each with random signs.  With the result's own rounding the error against 64 bits is 1.15 (300 tokens) to 1.3 (8192) times
// that of the rounding alone.
// RW waves take 32 rows each; with KS = 2 two such groups take every second tile of keys and add up at the end, so that a
// row's way along its keys is half as long (the entry point takes that where the card has few rows).
template <int DT, int D, int RW, int KS>
__global__ __launch_bounds__(RW * KS * kWave, D == 256 ? 1 : 2) void k_prompt(PromptParams p) {
    constexpr int kGroup = RW * kWave;
    constexpr int BN = D == 256 ? 32 : 64, ROWS = RW * 32, PIECES = D / 8, LOADS = BN * PIECES / kGroup;
    constexpr int QC = D / 16, KT = BN / 32, DT32 = D / 32, KC = BN / 16, kTile = BN * D * 2;
    static_assert(KS == 1 || KS * 4 * kTile >= ROWS * D * 4, "a group's sums fit where the tiles were");
    __shared__ struct {
        __align__(256) char tile[KS][2][2][kTile];               // [group][buffer][keys, values]
        unsigned long long odd[KS][4];                           // of a tile that rows see a part of: keys whose values are not finite
        float2 stats[KS == 1 ? 1 : ROWS];
    } lds;
    const int lane = threadIdx.x & (kWave - 1), all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = KS == 1 ? 0 : all_wave / RW, wave = KS == 1 ? all_wave : all_wave % RW, thread = wave * kWave + lane;
    const int col = lane & 31, h = lane >> 5;
    const PromptTile t = prompt_tile<ROWS>(p, blockIdx.x, lane);
    if (!t.any) return;
    const int head = t.head;
    const int reach = t.keys - t.rows;                           // row i sees keys up to reach + i
    const int last = t.first + ROWS < t.rows ? t.first + ROWS : t.rows;
    const int n_keys = reach + last < 0 ? 0 : reach + last;      // keys that some row of the tile sees
    const int n_tiles = (n_keys + BN - 1) / BN;
    const int my_first = t.first + wave * 32, row = my_first + col;

    const int64_t kv_head = head / p.group;
    const char* k_base = p.k + (int64_t)t.k0 * p.k_stride + kv_head * (D * 2);
    const char* v_base = p.v + (int64_t)t.k0 * p.v_stride + kv_head * (D * 2);
    const size_t k_bytes = t.keys ? (size_t)(t.keys - 1) * p.k_stride + D * 2 : 0, v_bytes = t.keys ? (size_t)(t.keys - 1) * p.v_stride + D * 2 : 0;
    // the group's piece i * kGroup + thread of a tile goes to that place of LDS; which piece of the row that is, is exchanged by
    // the row's number
    unsigned k_at[LOADS], v_at[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int at = i * kGroup + thread, r = at / PIECES, c = tile_place<PIECES>(r, at % PIECES) / 16 % PIECES;
        k_at[i] = (unsigned)(r * (int)p.k_stride + c * 16);
        v_at[i] = (unsigned)(r * (int)p.v_stride + c * 16);
    }
    char* const tiles = &lds.tile[group][0][0][0];
    const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)tiles;
    auto fetch = [&](int j) CORAL_INLINE {                       // the group's j-th tile
        const int tile = j * KS + group;
        if (tile >= n_tiles) return;                             // (uniform over the wave)
        const Buffer kb = buffer_view(k_base, (size_t)tile * BN * p.k_stride, k_bytes), vb = buffer_view(v_base, (size_t)tile * BN * p.v_stride, v_bytes);
        const unsigned to = __builtin_amdgcn_readfirstlane(lds_base + (j & 1) * 2 * kTile + wave * 1024);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) dma_piece(kb, k_at[i], to + i * (kGroup * 16));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) dma_piece(vb, v_at[i], to + kTile + i * (kGroup * 16));
    };
    fetch(0);
    uint4 q[QC];
    {
        const char* from = p.q + (int64_t)(t.row0 + row) * p.q_stride + (int64_t)head * (D * 2) + h * 16;
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            q[c] = make_uint4(0, 0, 0, 0);
            if (row < t.rows) q[c] = load_vec(reinterpret_cast<const uint4*>(from + c * 32));
            q[c].x ^= p.q_sign; q[c].y ^= p.q_sign; q[c].z ^= p.q_sign; q[c].w ^= p.q_sign;
        }
    }
    // From this tile on some rows see a part of a tile.  A product of 0 and infinity must not reach the rows that do not
    // see the value: it is made zero, and the rows that see it become NaN by the key's bit.
    const int first_cut = (reach + t.first + 1 < 0 ? 0 : reach + t.first + 1) / BN;
    f32x16_t sum[DT32];
#pragma unroll
    for (int d = 0; d < DT32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[d][i] = 0.f;
    float ref = kNoReference, total = 0.f;
    const float scale_log2 = p.scale_log2;
    // operands' places in a buffer: keys (32 kt + col, piece 2 c + h), values (column 32 d + lane % 32; keys 16 c + 4 h + 0..3 and
    // 16 c + 8 + 4 h + 0..3: rows r = 4 h + lane % 16 / 4 and r + 8, lanes pointing at four pieces of eight bytes)
    const int k_place = tile_place<PIECES>(col, h), r = 4 * h + (lane & 15) / 4, quad = (lane >> 4 & 1) * 2 + (lane & 3) / 2;
    const int v_place = tile_place<PIECES>(r, quad) + (lane & 1) * 8, v_place8 = tile_place<PIECES>(r + 8, quad) + (lane & 1) * 8;
    if (thread < 4) lds.odd[group][thread] = 0;
    dma_arrived();
    __syncthreads();
    // one tile: CUT where some row may see a part of it only
    auto step = [&](int j, auto parity, auto may_cut) CORAL_INLINE {
        constexpr bool CUT = decltype(may_cut)::value;
        const char *keys = tiles + parity * (2 * kTile), *values = keys + kTile;
        fetch(j + 1);
        const int tile = j * KS + group, k0 = tile * BN;
        if (CUT) {
            if (tile < n_tiles) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    uint4* at = reinterpret_cast<uint4*>(const_cast<char*>(values) + (i * kGroup + thread) * 16);
                    const uint4 raw = load_vec(at);
                    bool bad = false;
                    const uint4 fine = make_uint4(only_finite2<DT>(raw.x, bad), only_finite2<DT>(raw.y, bad), only_finite2<DT>(raw.z, bad), only_finite2<DT>(raw.w, bad));
                    if (bad) {
                        store_vec(at, fine);
                        atomicOr(&lds.odd[group][j & 3], 1ull << ((i * kGroup + thread) / PIECES));
                    }
                }
            }
            if (thread == 0) lds.odd[group][(j + 2) & 3] = 0;    // the group's tile before the last
            __syncthreads();
        }
        // some row of the wave sees some key (uniform)
        if (!CUT || (tile < n_tiles && k0 <= reach + my_first + 31 && my_first < t.rows)) {
            f32x16_t s[KT];
            constexpr int N = KT * QC, AHEAD = 8;                // products, and operands on their way
            uint4 a[AHEAD];
            auto key_operand = [&](int i) CORAL_INLINE {
                return load_vec(reinterpret_cast<const uint4*>(keys + (k_place ^ (i % QC * 32)) + i / QC * (32 * PIECES * 16)));
            };
#pragma unroll
            for (int i = 0; i < AHEAD && i < N; ++i) a[i] = key_operand(i);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s[i / QC] = mfma_32<DT>(a[i % AHEAD], q[i % QC], s[i / QC]);
                if (i + AHEAD < N) a[i % AHEAD] = key_operand(i + AHEAD);
                __builtin_amdgcn_sched_barrier(0);               // (left alone, the compiler reads each operand right before its product)
            }
            __builtin_amdgcn_s_setprio(0);
            const int most = reach + row - k0;                   // newest key of the tile that the row sees
            if (CUT) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (kt * 32 + 8 * (i / 4) + 4 * h + i % 4 > most) s[kt][i] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kt][i]);
            top = lane_xor_max<32>(top) * scale_log2;
            const bool move = top > ref + (kWeightsAt<DT> + kWeightsUpTo);
            if (__builtin_amdgcn_ballot_w64(move)) {
                const float to = move ? top - kWeightsAt<DT> : ref, keep = move ? __builtin_amdgcn_exp2f(ref - to) : 1.f;
                ref = to;
                total *= keep;
#pragma unroll
                for (int d = 0; d < DT32; ++d) sum[d] *= keep;
            }
            // values' operand i: columns of tile i % DT32, keys of chunk i / DT32
            constexpr int M = DT32 * KC, VAHEAD = 4;
            uint4 b[VAHEAD];
            auto value_operand = [&](int i) CORAL_INLINE {
                const uint2 lo = lds_transposed(values + (v_place ^ (i % DT32 * 64)) + i / DT32 * (16 * PIECES * 16));
                const uint2 hi = lds_transposed(values + (v_place8 ^ (i % DT32 * 64)) + i / DT32 * (16 * PIECES * 16));
                return make_uint4(lo.x, lo.y, hi.x, hi.y);
            };
#pragma unroll
            for (int i = 0; i < VAHEAD && i < M; ++i) b[i] = value_operand(i);
            // Weights of keys 16 c + 8 (g / 2) + 4 h + 2 (g % 2) and the next, g = 0..3: the products of chunk c wait for these four
            // only, so the others' vector instructions run beside products.
            unsigned w[KC][4];
            float part = 0.f;                                    // of the total: this tile's weights first (see above)
            auto weigh = [&](int c, int g) CORAL_INLINE {
                const float x = s[c / 2][8 * (c % 2) + 2 * g], y = s[c / 2][8 * (c % 2) + 2 * g + 1];
                w[c][g] = narrow2<DT>(__builtin_amdgcn_exp2f(fmaf(x, scale_log2, -ref)), __builtin_amdgcn_exp2f(fmaf(y, scale_log2, -ref)));
                part = add_pair<DT>(w[c][g], part);              // of the weights as rounded: half the additions
            };
#pragma unroll
            for (int g = 0; g < 4; ++g) weigh(0, g);
            if (CUT && (lds.odd[group][j & 3] & keys_to(most))) part = NAN;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const int c = i / DT32, d = i % DT32;
                sum[d] = mfma_32<DT>(b[i % VAHEAD], make_uint4(w[c][0], w[c][1], w[c][2], w[c][3]), sum[d]);
                if (i + VAHEAD < M) b[i % VAHEAD] = value_operand(i + VAHEAD);
                if (c + 1 < KC) {
#pragma unroll
                    for (int g = d * 4 / DT32; g < (d + 1) * 4 / DT32; ++g) weigh(c + 1, g);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            total += part;
        }
        dma_arrived();
        __syncthreads();
    };
    int j = 0;
    const int whole = (first_cut < n_tiles ? first_cut : n_tiles) / KS, rounds = (n_tiles + KS - 1) / KS;
    for (; j + 1 < whole; j += 2) {
        step(j, std::integral_constant<int, 0>(), std::false_type());
        step(j + 1, std::integral_constant<int, 1>(), std::false_type());
    }
    for (; j < whole; ++j) step(j, j & 1, std::false_type());
    for (; j < rounds; ++j) step(j, j & 1, std::true_type());
    if (KS == 2) {                                               // the second group hands its sums over, lane to lane
        f32x4_t* to = reinterpret_cast<f32x4_t*>(&lds.tile[0][0][0][0]) + wave * (DT32 * 4 * kWave) + lane;
        total = lane_xor_sum<32>(total);
        if (group == 1) {
#pragma unroll
            for (int d = 0; d < DT32; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) to[(d * 4 + i) * kWave] = f32x4_t{sum[d][4 * i], sum[d][4 * i + 1], sum[d][4 * i + 2], sum[d][4 * i + 3]};
            if (h == 0) lds.stats[wave * 32 + col] = make_float2(ref, total);
        }
        __syncthreads();
        if (group == 1) return;
        const float2 other = lds.stats[wave * 32 + col];
        const float top = fmaxf(ref, other.x), mine = __builtin_amdgcn_exp2f(ref - top), its = __builtin_amdgcn_exp2f(other.x - top);
        total = total * mine + other.y * its;
#pragma unroll
        for (int d = 0; d < DT32; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4_t x = to[(d * 4 + i) * kWave];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[d][4 * i + e] = fmaf(x[e], its, sum[d][4 * i + e] * mine);
            }
    } else {
        total = lane_xor_sum<32>(total);
    }
    if (row >= t.rows) return;
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;          // a row that sees nothing: zeros
    char* to = p.out + (int64_t)(t.row0 + row) * p.out_stride + (int64_t)head * (D * 2) + h * 8;
#pragma unroll
    for (int d = 0; d < DT32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint2*>(to + (d * 32 + 2 * i) * 2) =
                make_uint2(narrow2<DT>(sum[d][i] * inv, sum[d][i + 1] * inv), narrow2<DT>(sum[d][i + 2] * inv, sum[d][i + 3] * inv));
}

// fp32 on the matrix cores' fp32 products (a sixteenth of the 16-bit rate): 16 rows a wave, 32 keys at a time, no
// rounding of the weights.  One value a lane and product: lane (key or column, g) has the g-th of four.  KS groups of RW waves
// take every KS-th tile of keys, as in k_prompt.  Bound by the products (4096 tokens, 8 heads of 256: 720 to 771 us, 95 to
// 89 TFLOP/s).
template <int D, int RW, int KS>
__global__ __launch_bounds__(RW * KS * kWave) void k_prompt_f32(PromptParams p) {
    constexpr int kGroup = RW * kWave;
    constexpr int BN = 32, ROWS = RW * 16, PIECES = D / 4, LOADS = BN * PIECES / kGroup, QC = D / 16, DTILES = D / 16, kRow = D + 4;
    static_assert(BN * kRow >= ROWS * D || KS == 1, "a group's sums fit where the keys were");
    __shared__ struct {
        __align__(16) float k[KS][BN][kRow], v[KS][BN][kRow];
        unsigned long long odd[KS][2];
        float2 stats[KS][ROWS];
    } lds;
    const int lane = threadIdx.x & (kWave - 1), all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = KS == 1 ? 0 : all_wave / RW, wave = KS == 1 ? all_wave : all_wave % RW, thread = wave * kWave + lane;
    float (*const k_lds)[kRow] = lds.k[group], (*const v_lds)[kRow] = lds.v[group];
    unsigned long long* const odd = lds.odd[group];
    const int col = lane & 15, g = lane >> 4;
    const PromptTile t = prompt_tile<ROWS>(p, blockIdx.x, lane);
    if (!t.any) return;
    const int head = t.head;
    const int reach = t.keys - t.rows, last = t.first + ROWS < t.rows ? t.first + ROWS : t.rows;
    const int n_keys = reach + last < 0 ? 0 : reach + last, n_tiles = (n_keys + BN - 1) / BN;
    const int my_first = t.first + wave * 16, row = my_first + col;
    uint4 q[QC];
    {
        const char* from = p.q + (int64_t)(t.row0 + row) * p.q_stride + (int64_t)head * (D * 4) + g * 16;
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            q[c] = make_uint4(0, 0, 0, 0);
            if (row < t.rows) q[c] = load_vec(reinterpret_cast<const uint4*>(from + c * 64));
            q[c].x ^= p.q_sign; q[c].y ^= p.q_sign; q[c].z ^= p.q_sign; q[c].w ^= p.q_sign;
        }
    }
    const int64_t kv_head = head / p.group;
    const char* k_base = p.k + (int64_t)t.k0 * p.k_stride + kv_head * (D * 4);
    const char* v_base = p.v + (int64_t)t.k0 * p.v_stride + kv_head * (D * 4);
    const size_t k_bytes = t.keys ? (size_t)(t.keys - 1) * p.k_stride + D * 4 : 0, v_bytes = t.keys ? (size_t)(t.keys - 1) * p.v_stride + D * 4 : 0;
    f32x4_t sum[DTILES];
#pragma unroll
    for (int d = 0; d < DTILES; ++d) sum[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY, total = 0.f;
    const int first_cut = (reach + t.first + 1 < 0 ? 0 : reach + t.first + 1) / BN;       // as in k_prompt
    if (thread < 2) odd[thread] = 0;
    const int rounds = (n_tiles + KS - 1) / KS;
    for (int j = 0; j < rounds; ++j) {
        const int k0 = (j * KS + group) * BN;                    // (no row sees a tile behind the last)
        const Buffer kb = buffer_view(k_base, (size_t)k0 * p.k_stride, k_bytes), vb = buffer_view(v_base, (size_t)k0 * p.v_stride, v_bytes);
        uint4 nk[LOADS], nv[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * kGroup + thread, r = at / PIECES, c = at % PIECES;
            nk[i] = buffer_read16(kb, (unsigned)(r * (int)p.k_stride + c * 16));
            nv[i] = buffer_read16(vb, (unsigned)(r * (int)p.v_stride + c * 16));
        }
        __syncthreads();                                         // the tile before has been read
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * kGroup + thread, r = at / PIECES, c = at % PIECES;
            if (j * KS + group >= first_cut) {
                bool bad = false;
                nv[i].x = only_finite(nv[i].x, bad);
                nv[i].y = only_finite(nv[i].y, bad);
                nv[i].z = only_finite(nv[i].z, bad);
                nv[i].w = only_finite(nv[i].w, bad);
                if (bad) atomicOr(&odd[j & 1], 1ull << r);
            }
            store_vec(reinterpret_cast<uint4*>(&k_lds[r][c * 4]), nk[i]);
            store_vec(reinterpret_cast<uint4*>(&v_lds[r][c * 4]), nv[i]);
        }
        __syncthreads();
        if (thread == 0) odd[(j + 1) & 1] = 0;              // read before the barrier above, written behind the next one
        if (k0 > reach + my_first + 15 || my_first >= t.rows) continue;      // uniform over the wave
        f32x4_t s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < QC; ++c)
                s[i] = mfma_tile<kF32>(load_vec(reinterpret_cast<const uint4*>(&k_lds[i * 16 + col][c * 16 + 4 * g])), q[c], s[i]);
        }
        const bool cut = k0 + BN - 1 > reach + my_first;
        const int most = reach + row - k0;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = s[i / 4][i % 4] * p.scale_log2;
            if (cut && (i / 4) * 16 + 4 * g + i % 4 > most) x[i] = -INFINITY;
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = lane_xor_max<16>(lane_xor_max<32>(top));
        const bool move = top > ref + kWeightsUpTo || (ref == -INFINITY && top > -INFINITY);
        if (__builtin_amdgcn_ballot_w64(move)) {
            const float to = move ? top : ref, by = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - to), keep = move ? by : 1.f;
            ref = to;
            total *= keep;
#pragma unroll
            for (int d = 0; d < DTILES; ++d) sum[d] *= keep;
        }
        const float base = ref == -INFINITY ? 0.f : ref;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = __builtin_amdgcn_exp2f(x[i] - base);
        }
        total += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        if (j * KS + group >= first_cut && (odd[j & 1] & keys_to(most))) total = NAN;
#pragma unroll
        for (int d = 0; d < DTILES; ++d)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v_lds[(i / 4) * 16 + 4 * g + i % 4][d * 16 + col], w[i], sum[d], 0, 0, 0);
    }
    total = lane_xor_sum<16>(lane_xor_sum<32>(total));
    if (KS > 1) {                                                // the other groups hand their sums over, lane to lane
        __syncthreads();
        f32x4_t* to = reinterpret_cast<f32x4_t*>(&k_lds[0][0]) + wave * (DTILES * kWave) + lane;
        if (group) {
#pragma unroll
            for (int d = 0; d < DTILES; ++d) to[d * kWave] = sum[d];
            if (g == 0) lds.stats[group][wave * 16 + col] = make_float2(ref, total);
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int o = 1; o < KS; ++o) {
            const f32x4_t* from = reinterpret_cast<const f32x4_t*>(&lds.k[o][0][0]) + wave * (DTILES * kWave) + lane;
            const float2 other = lds.stats[o][wave * 16 + col];
            const float top = fmaxf(ref, other.x), mine = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top);
            const float its = other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other.x - top);
            ref = top;
            total = total * mine + other.y * its;
#pragma unroll
            for (int d = 0; d < DTILES; ++d) {
                const f32x4_t x = from[d * kWave];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[d][e] = fmaf(x[e], its, sum[d][e] * mine);
            }
        }
    }
    if (row >= t.rows) return;
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
    char* to = p.out + (int64_t)(t.row0 + row) * p.out_stride + (int64_t)head * (D * 4) + g * 16;
#pragma unroll
    for (int d = 0; d < DTILES; ++d) *reinterpret_cast<f32x4_t*>(to + d * 64) = sum[d] * inv;
}

}  // namespace
