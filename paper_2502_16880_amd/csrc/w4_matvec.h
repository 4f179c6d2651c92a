// Products with 4-bit weights: y[m,n] = act(sum_j x[m,j] w[n,j] + bias[n]) + residual[m,n] for up to
// 64 tokens, w[n,j] = scale[n,j/group] * (code[n,j] - zero[n,j/group]), or scale * e2m1(code).
//
// All products go through v_mfma_f32_16x16x32, tokens as its rows and weight rows as its columns, so
// that a lane holds the sums of one weight row and the row's scales and zero points are one value a
// lane.  Codes become 16-bit operands exactly: an integer code n is put into the mantissa of 16.0
// (16 + n, two operations for two codes) and the sum of (16 + zero) x is taken off per group in fp32,
// or is where the accumulator starts; an e2m1 code has an instruction.  (So sums of (16 + code) |x| and of
// (16 + zero) |x|, 31 and 271 at most, have to stay in fp32's range.)  Scales multiply the group's
// fp32 sum, never a 16-bit weight.  fp32 activations are split into three bf16 values whose sum they
// are, and every product is taken three times: the sums are fp32 sums of exact products in all types.
#pragma once
#include "buffer_loads.h"
#include "w4_plan.h"

namespace {

enum W4Kind { kW4Sym = 0, kW4Zero = 1, kW4E2M1 = 2 };

struct W4Params {
    const void* x;              // [M,K] storage type
    const unsigned char* codes; // [N,K/2], column 2 j in the low half of byte j
    const void* scales;         // [N,n_groups] storage type
    const unsigned char* zeros; // [N,n_groups] or null
    const float* bias;          // [N] or null
    const void* residual;       // [M,N] storage type or null
    void* y;                    // [M,N] fp32 or storage type
    int M, N, K, group, n_groups, act, out_f32;
    unsigned per_group, per_group_inv;           // units of a group (at least one), 2^32 / that, rounded up
};

// A slot is the columns of a unit that share a scale: SLOTS of them, of 32 or 64 columns, where groups are
// finer than a unit, else one.

template <int DT>
constexpr int kW4Op = DT == kF16 ? kF16 : kBF16; // operand type of the products

// (w & mask) | bits.  Of two constants the compiler makes two instructions; with values that it does not know
// it takes v_and_or_b32.  The instruction itself is not written in asm: the compiler does not see there that
// what it writes is a product's operand, or was the last one's, and leaves out the waits between them.
__device__ __forceinline__ unsigned w4_and_or(unsigned w, unsigned mask, unsigned bits) {
    asm("" : "+s"(mask));
    asm("" : "+v"(bits));
    return (w & mask) | bits;
}

// Eight codes of a dword as 16-bit operands.  Integers: 16 + code, in the order 0 4 1 5 2 6 3 7.
template <int OP, int KIND>
__device__ __forceinline__ uint4 w4_operand(unsigned w) {
    uint4 o;
    if constexpr (KIND == kW4E2M1) {
        if constexpr (OP == kF16) {
            o.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
            o.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
            o.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
            o.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
        } else {
            o.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
            o.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
            o.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
            o.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
        }
    } else if constexpr (OP == kF16) {           // four bits at the top of a ten-bit mantissa
        constexpr unsigned kMask = 0x03C003C0u, kSixteen = 0x4C004C00u;
        o.x = w4_and_or(w << 6, kMask, kSixteen);
        o.y = w4_and_or(w << 2, kMask, kSixteen);
        o.z = w4_and_or(w >> 2, kMask, kSixteen);
        o.w = w4_and_or(w >> 6, kMask, kSixteen);
    } else {                                     // ... of a seven-bit mantissa
        constexpr unsigned kMask = 0x00780078u, kSixteen = 0x41804180u;
        o.x = w4_and_or(w << 3, kMask, kSixteen);
        o.y = w4_and_or(w >> 1, kMask, kSixteen);
        o.z = w4_and_or(w >> 5, kMask, kSixteen);
        o.w = w4_and_or(w >> 9, kMask, kSixteen);
    }
    return o;
}

// Eight activations in the order of the codes' operands.
template <int KIND>
__device__ __forceinline__ uint4 w4_order(uint4 v) {
    if constexpr (KIND == kW4E2M1) return v;
    uint4 o;                                     // (low, high) halves of values j and j + 4
    o.x = __builtin_amdgcn_perm(v.z, v.x, 0x05040100u);
    o.y = __builtin_amdgcn_perm(v.z, v.x, 0x07060302u);
    o.z = __builtin_amdgcn_perm(v.w, v.y, 0x05040100u);
    o.w = __builtin_amdgcn_perm(v.w, v.y, 0x07060302u);
    return o;
}

// Part c of eight fp32 values, x = hi + mid + lo exactly in bf16: the significand's 24 bits are cut off in
// eights.  (Below 2^-133, the smallest step of a bf16, there is nothing: that affects |x| < 2^-110 only.)
__device__ __forceinline__ uint4 w4_part(uint4 x, uint4 y, int c) {
    const unsigned f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    unsigned b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float v = __uint_as_float(f[j]), hi = __uint_as_float(f[j] & 0xffff0000u), rest = v - hi;
        const float mid = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
        b[j] = c == 0 ? f[j] : __float_as_uint(c == 1 ? rest : rest - mid);      // (their upper halves)
    }
    return make_uint4(__builtin_amdgcn_perm(b[1], b[0], 0x07060302u), __builtin_amdgcn_perm(b[3], b[2], 0x07060302u),
                      __builtin_amdgcn_perm(b[5], b[4], 0x07060302u), __builtin_amdgcn_perm(b[7], b[6], 0x07060302u));
}

template <int DT>
__device__ __forceinline__ float w4_load(const void* p, size_t i) {
    if constexpr (DT == kF32) return static_cast<const float*>(p)[i];
    else return widen16<DT>(static_cast<const unsigned short*>(p)[i]);
}

__device__ __forceinline__ float w4_act(float y, int act) {
    if (act == CORAL_ACT_SILU) return y / (1.0f + expf(-y));
    if (act == CORAL_ACT_RELU) return y > 0.f ? y : 0.f;
    return y;
}

// y[m,n] from its sum: bias, activation and residual in fp32, one rounding at the end.
template <int DT>
__device__ __forceinline__ void w4_store(const W4Params& p, int m, int n, float sum) {
    const size_t at = (size_t)m * p.N + n;
    float y = sum;
    if (p.bias) y += p.bias[n];
    y = w4_act(y, p.act);
    if (p.residual) y += w4_load<DT>(p.residual, at);
    if constexpr (DT == kF32) {
        static_cast<float*>(p.y)[at] = y;
    } else {
        if (p.out_f32) static_cast<float*>(p.y)[at] = y;
        else static_cast<unsigned short*>(p.y)[at] = narrow16<DT>(y);
    }
}

// ---------------------------------------------------------------- activations held in registers
// A workgroup of eight waves streams tiles of 16 weight rows; the waves share the columns in units of
// 128 (wave w: NB units from w NB on), so a wave's activations are the same for every tile and stay in
// its registers.  The codes are loaded in the order of memory, several rows a load, and exchanged
// through a slice of LDS of the wave's own: loaded in the layout of the products, 16 bytes of 16 rows
// each, a load kept the address unit busy for 130 cycles and the kernel at 4.9 TB/s.  A load's registers
// are loaded again, with the next tile's codes, as soon as they are in LDS: the wave always has about
// NB KB on the way.  The tile's scales and zero points, which lie scattered for a lane, are loaded row
// by row by the whole workgroup one tile ahead and kept in LDS as fp32.  The waves' sums meet in LDS
// once a tile.  More tokens than T tiles hold are other workgroups' (the grid's second dimension).
//
// Measured (copy 4.9 TB/s, reading alone 6.5 TB/s): bf16, one token, 128256 x 4096, groups of 128: 45 us, 6.0
// TB/s, bound by memory (48 to 53 where calls follow each other in a graph without a pause); e2m1 in groups of 32: 50 to 52 us
// there, 5.7 TB/s.  fp16, 16 tokens, 152064 x 3584, groups of 64
// with zero points: 63 us, 4.9 TB/s (69 to 73): a product of 32 columns takes a dozen vector instructions beside
// it (codes to operands, zero point, scale), which are about as long as the reading.  fp32, one token, 128256 x
// 4096: 51 us (54 to 57); 7 tokens, 50257 x 2568, groups of 32: 33 us, 2.6 TB/s: three products for one, and one workgroup
// a compute unit for its registers.  4096 x 4096, one token: 6.1 us, of which the launch is 2.5 and one trip to memory 2.
//
// Lane 16 q + r takes the 16 bytes of row r that hold columns 32 q to 32 q + 31 of a unit, and product
// s their dword s: columns 32 q + 8 s ... + 7 of the four chunks q, which is a group or part of one
// where a group has 128 columns or more.  With finer groups it takes dword q of the four chunks, and
// product s columns 32 s to 32 s + 31.
//
// The operands are read through buffer descriptors, which drop what lies behind their end: rows behind
// the last one, and tokens and columns behind the activations, read as zero without a comparison.
// Codes behind a row's last column are another row's and meet activations of zero.
constexpr int kW4Block = kW4Held * kWave;

// The value is wanted in registers here: what makes it is neither moved behind this point nor, with a
// value that a loop does not change, in front of the loop.
__device__ __forceinline__ void w4_settle(uint4& v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

// Group of a unit where groups are whole units: unit / (group / 128) by the host's reciprocal.
__device__ __forceinline__ unsigned w4_group_of(const W4Params& p, unsigned unit) {
    return p.per_group == 1 ? unit : __umulhi(unit, p.per_group_inv);
}

// T tiles of 16 rows of activations, NB units a wave.  PASSES: the columns are more than the waves hold and are taken
// in passes; the workgroup goes through a block of tiles once a pass, adding the tiles' sums up in
// LDS, before the next block.  Codes are still read once, activations once a block.
template <int DT, int KIND, int SLOTS, int T, int NB, bool PASSES = false, bool SPREAD = false>
__global__ __launch_bounds__(kW4Block, w4_held_regs(DT == kF32 && !SPREAD, T, NB) <= 4 ? 4 : 2) void k_w4_held(W4Params p) {
    static_assert(DT == kF32 || !SPREAD, "");
    constexpr bool CHAIN = DT == kF32 && !SPREAD;
    constexpr int OP = kW4Op<DT>, PARTS = CHAIN ? 3 : 1, ROWS = SPREAD ? 3 : 1, TOKENS = w4_held_tokens(SPREAD, T);
    constexpr bool PAIR = KIND == kW4Zero && DT != kF32;     // scale and zero as two 16-bit values of one word
    constexpr int PER = KIND == kW4Zero && DT == kF32 ? 2 : 1;
    // SL: slots of a row that a thread brings for a tile (the last ones may lie behind the row).
    constexpr bool FINE = SLOTS > 1;
    constexpr int EACH = 4 / SLOTS, SL = (NB * kW4Held * SLOTS + 31) / 32, STRIDE = (SL * 32 + 1) * PER;
    __shared__ float sums[2][kW4Held][T * 256];
    __shared__ float scales[2][16][STRIDE];                  // (scale, 1 + zero / 16); rows start on different banks
    // a wave's own: rows of codes that start on different banks, and before that the exchange of activations
    constexpr int CHUNKS = NB * 4, CODE_ROW = CHUNKS + 1, X_ROW = 17;
    constexpr int SLICE = 16 * CODE_ROW > 8 * X_ROW ? 16 * CODE_ROW : 8 * X_ROW;
    __shared__ uint4 slices[kW4Held][SLICE];
    __shared__ f32x4_t x_sums[KIND != kW4E2M1 ? kW4Held : 1][NB][SLOTS][T][4];     // of a slot's x, 16 tokens
    // sums of the passes so far, a block of tiles (as many as fit beside the rest)
    constexpr int kUsed = sizeof(sums) + sizeof(scales) + sizeof(slices) + sizeof(x_sums);
    constexpr int BLOCK = !PASSES ? 1 : (160 * 1024 - kUsed) / (T * 1024) < 24 ? (160 * 1024 - kUsed) / (T * 1024) : 24;
    __shared__ float so_far[PASSES ? BLOCK : 1][PASSES ? T * 256 : 1];
    constexpr int PASS_COLS = kW4Held * NB * kW4UnitCols;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane & 15, q = lane >> 4;
    const int token0 = blockIdx.y * TOKENS, tokens = p.M - token0 < TOKENS ? p.M - token0 : TOKENS;
    const int row_bytes = p.K / 2, tiles = (p.N - 1) / 16 + 1, passes = PASSES ? (p.K + PASS_COLS - 1) / PASS_COLS : 1;
    const int each = tiles / gridDim.x, more_of = tiles % gridDim.x, wg = blockIdx.x;
    const int first = wg * each + (wg < more_of ? wg : more_of), end = first + each + (wg < more_of ? 1 : 0);

    // scales: thread (row tid / 32, slots tid % 32 + 32 i)
    const int s_row = threadIdx.x / 32, s_slot = threadIdx.x % 32;
    unsigned s_raw[SL], z_raw[SL];
    // (of a slot behind the row's columns one behind the operand's end: zero, whatever the last scale is)
    auto s_at = [&](unsigned tid, int pass, int i, unsigned size) CORAL_INLINE {
        const unsigned slot = pass * (kW4Held * NB * SLOTS) + tid % 32 + 32 * i;
        const unsigned at = tid / 32 * p.n_groups + (FINE ? slot : w4_group_of(p, slot));
        const unsigned behind = slot * (kW4UnitCols / SLOTS) < (unsigned)p.K ? 0u : kBufferBehind;
        return at * size | behind;
    };
    constexpr unsigned W = DT == kF32 ? 4u : 2u;
    auto load_scales = [&](int tile, int pass, bool any) CORAL_INLINE {
        const size_t first_group = (size_t)tile * 16 * p.n_groups, all = (size_t)p.N * p.n_groups;
        const Buffer view = buffer_view(p.scales, first_group * W, all * W, any);
        const Buffer z_view = buffer_view(p.zeros, first_group, all, any);
        unsigned tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                        // (what follows from it is not kept through the products)
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            if constexpr (DT == kF32) s_raw[i] = buffer_read4(view, s_at(tid, pass, i, W));
            else s_raw[i] = buffer_read2(view, s_at(tid, pass, i, W));
            if constexpr (KIND == kW4Zero) z_raw[i] = buffer_read1(z_view, s_at(tid, pass, i, 1u));
        }
    };
    auto put_scales = [&](int parity) CORAL_INLINE {
        float* dst = scales[parity][s_row] + s_slot * PER;
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const float zero = KIND == kW4Zero ? fmaf((float)z_raw[i], 0.0625f, 1.0f) : 0.f;       // (exact in fp16 too)
            if constexpr (PAIR) dst[i * 32] = __uint_as_float(s_raw[i] << 16 | __builtin_bit_cast(unsigned short, (_Float16)zero));
            else dst[i * 32 * PER] = DT == kF32 ? __uint_as_float(s_raw[i]) : widen16<DT>((unsigned short)s_raw[i]);
            if constexpr (PER == 2) dst[i * 32 * PER + 1] = zero;
        }
    };
    // codes: the wave's 4 NB chunks of 16 rows, dealt to the lanes of its NB loads in the order of memory
    constexpr bool EVEN = kWave % CHUNKS == 0;               // a load takes whole rows: the next one's are so many rows on
    uint4 w[NB];
    unsigned at[EVEN ? 1 : NB];
#pragma unroll
    for (int j = 0; j < (EVEN ? 1 : NB); ++j) {
        const int e = j * kWave + lane;
        at[j] = (unsigned)(e / CHUNKS) * (unsigned)row_bytes + (unsigned)(wave * CHUNKS + e % CHUNKS) * 16u;
    }
    auto read_codes = [&](const Buffer& view, int j) CORAL_INLINE {
        if constexpr (EVEN) return buffer_read16<kBufferStream>(view, at[0] + (unsigned)(j * (kWave / CHUNKS)) * (unsigned)row_bytes);
        else return buffer_read16<kBufferStream>(view, at[EVEN ? 0 : j]);
    };
    auto code_view = [&](int tile, int pass, bool any) CORAL_INLINE {
        return buffer_view(p.codes, (size_t)tile * 16 * row_bytes + pass * (PASS_COLS / 2), (size_t)p.N * row_bytes, any);
    };
    auto put = [&](int j) CORAL_INLINE {
        const int e = j * kWave + lane;
        store_vec(&slices[wave][e / CHUNKS * CODE_ROW + e % CHUNKS], w[j]);
    };
    uint4 x[T][NB][4][PARTS];
    const Buffer x_view = buffer_view(p.x, (size_t)token0 * p.K * W, (size_t)p.M * p.K * W);
    // In the order of memory first, lane 16 a + c the eight columns c of a unit of row 4 i + a in register
    // i (the products' own layout, 64 bytes of 16 rows a load, made the first tile of 32 tokens wait for
    // several us; three products one after the other keep it).  Spread: row 3 m + c is part c of token m.
    auto load_x = [&](int pass) CORAL_INLINE {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int unit = pass * PASS_COLS + (wave * NB + j) * kW4UnitCols;
                    const int col = unit + (!CHAIN ? r * 8 : FINE ? s * 32 + q * 8 : q * 32 + s * 8);
                    const int row = t * 16 + (!CHAIN ? 4 * s + q : r), token = row / ROWS;
                    // (behind the end; the last row of spread ones may be no token's)
                    const unsigned off = col < p.K && (!SPREAD || token < TOKENS) ? ((unsigned)token * (unsigned)p.K + col) * W : kBufferEnd;
                    const uint4 a = buffer_read16(x_view, off);
                    if constexpr (DT == kF32) {
                        const uint4 b = buffer_read16(x_view, off + 16u);
                        if constexpr (SPREAD) {
                            x[t][j][s][0] = w4_part(a, b, row - token * 3);
                            if (s == 3) __builtin_amdgcn_sched_barrier(0);       // (a unit at a time: it takes twice the registers until then)
                        } else {
                            x[t][j][s][0] = a;
                            x[t][j][s][1] = b;
                        }
                    } else {
                        x[t][j][s][0] = a;
                    }
                }
    };
    // ... then lane 16 q + r row r, chunk q and eight columns s in register s (fine groups: chunk s,
    // eight columns q), through the wave's slice: as many rows at a time as it holds
    constexpr int HALVES = SLICE >= 16 * X_ROW ? 1 : 2, X_MASK = 16 / HALVES - 1;
    auto exchange = [&](uint4 (&v)[4][PARTS]) CORAL_INLINE {
        u32x4_t o[4] = {};
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
#pragma unroll
            for (int i = 0; i < 4 / HALVES; ++i) store_vec(&slices[wave][(4 * i + q) * X_ROW + r], v[4 / HALVES * h + i][0]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint4 got = load_vec(&slices[wave][(r & X_MASK) * X_ROW + (FINE ? 4 * s + q : 4 * q + s)]);
                const bool take = h == 0 || r >= 8;
                o[s].x = take ? got.x : o[s].x;
                o[s].y = take ? got.y : o[s].y;
                o[s].z = take ? got.z : o[s].z;
                o[s].w = take ? got.w : o[s].w;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s][0] = make_uint4(o[s].x, o[s].y, o[s].z, o[s].w);
    };
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    // the offset's part of the sums: of -24 x where every zero point is 8, else of -16 x, times 1 + zero / 16
    constexpr unsigned kMinus = KIND == kW4Sym ? (OP == kF16 ? 0xCE00CE00u : 0xC1C0C1C0u) : OP == kF16 ? 0xCC00CC00u : 0xC180C180u;
    const uint4 minus = make_uint4(kMinus, kMinus, kMinus, kMinus);
    auto arrange_x = [&]() CORAL_INLINE {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int t = 0; t < T; ++t) {
                if constexpr (!CHAIN) exchange(x[t][j]);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if constexpr (CHAIN) {
                        const uint4 a = x[t][j][s][0], b = x[t][j][s][1];
#pragma unroll
                        for (int c = 0; c < PARTS; ++c) x[t][j][s][c] = w4_part(a, b, c);
                    }
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) x[t][j][s][c] = w4_order<KIND>(x[t][j][s][c]);
                }
                if constexpr (CHAIN) __builtin_amdgcn_sched_barrier(0);
            }
        // (arranged here, not at every use)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int v = 0; v < PARTS; ++v) w4_settle(x[t][j][s][v]);
        if constexpr (KIND != kW4E2M1) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    f32x4_t sum = zero4;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        if (s % EACH == 0) sum = zero4;
#pragma unroll
                        for (int c = PARTS - 1; c >= 0; --c) sum = mfma_tile<OP>(x[t][j][s][c], minus, sum);
                        if (r == 0 && s % EACH == EACH - 1) x_sums[wave][j][s / EACH][t][q] = sum;      // (read by this wave only)
                    }
                    if constexpr (DT == kF32) __builtin_amdgcn_sched_barrier(0);
                }
        }
    };
    load_scales(first, 0, true);
    if constexpr (!PASSES) load_x(0);
    {
        const Buffer view = code_view(first, 0, true);
#pragma unroll
        for (int j = 0; j < NB; ++j) w[j] = read_codes(view, j);
    }
    put_scales(0);
    if constexpr (!PASSES) arrange_x();
    __syncthreads();                                         // the first tile's scales are there
    // one tile of a pass, which requests the scales and codes of the next one; more: there is one (else the
    // requests find nothing: a branch around them would wait for them where it ends)
    auto step = [&](int tile, int pass, int in_block, int parity, bool more, int next_tile, int next_pass) CORAL_INLINE {
        load_scales(next_tile, next_pass, more);
        const Buffer next_codes = code_view(next_tile, next_pass, more);
        const float* my_scales = scales[parity][r] + wave * (NB * SLOTS * PER);
        f32x4_t y[T];
#pragma unroll
        for (int t = 0; t < T; ++t) y[t] = zero4;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            put(j);
            w[j] = read_codes(next_codes, j);                // the registers are free again
        }
        // A wave's LDS accesses complete in order; the compiler has to keep the order too, though no
        // lane reads what it wrote itself.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            uint4 v;
            if constexpr (FINE) {                            // dword q of the four chunks: their transposition
                const unsigned* d = reinterpret_cast<const unsigned*>(&slices[wave][r * CODE_ROW + j * 4]) + q;
                v = make_uint4(d[0], d[4], d[8], d[12]);
            } else {
                v = load_vec(&slices[wave][r * CODE_ROW + j * 4 + q]);
            }
            f32x4_t acc[T];
            float scale = 0.f;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s % EACH == 0) {                         // the sums start at the offset's part
                    const int slot = j * SLOTS + s / EACH;
                    scale = my_scales[slot * PER];
                    float zero = 0.f;
                    if constexpr (PER == 2) zero = my_scales[slot * PER + 1];
                    if constexpr (PAIR) {
                        const unsigned pair = __float_as_uint(scale);
                        scale = widen16<DT>((unsigned short)(pair >> 16));
                        zero = (float)__builtin_bit_cast(_Float16, (unsigned short)pair);
                    }
#pragma unroll
                    for (int t = 0; t < T; ++t) {
                        acc[t] = zero4;
                        if constexpr (KIND != kW4E2M1) acc[t] = x_sums[wave][j][s / EACH][t][q];
                        if constexpr (KIND == kW4Zero) {
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[t][v] *= zero;
                        }
                    }
                }
                const uint4 op = w4_operand<OP, KIND>(s == 0 ? v.x : s == 1 ? v.y : s == 2 ? v.z : v.w);
#pragma unroll
                for (int t = 0; t < T; ++t) {
#pragma unroll
                    for (int c = PARTS - 1; c >= 0; --c) acc[t] = mfma_tile<OP>(x[t][j][s][c], op, acc[t]);        // the small parts first
                }
                if (s % EACH != EACH - 1) continue;
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v) y[t][v] = fmaf(scale, acc[t][v], y[t][v]);
                if constexpr (FINE && T > 1) __builtin_amdgcn_sched_barrier(0);
            }
            // (summed here: left to itself the compiler keeps every product's result until the sums are stored)
#pragma unroll
            for (int t = 0; t < T; ++t) asm volatile("" : "+v"(y[t]));
            __builtin_amdgcn_sched_barrier(0);               // units one after the other: side by side they take too many registers
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // (before the next tile's codes)
        put_scales(parity ^ 1);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[parity][wave][(t * 16 + 4 * q + v) * 16 + r] = y[t][v];
        // (the other buffers are written next: who still reads them is past that at the next barrier)
        __syncthreads();
        int o = threadIdx.x;
        asm volatile("" : "+v"(o));                       // (what follows from it is not kept through the products)
        for (; o < tokens * 16; o += kW4Block) {
            float sum = 0.f;
#pragma unroll
            for (int c = ROWS - 1; c >= 0; --c)
#pragma unroll
                for (int v = 0; v < kW4Held; ++v) sum += sums[parity][v][o / 16 * (ROWS * 16) + c * 16 + o % 16];
            if constexpr (PASSES) {                          // (a place of so_far is one thread's own)
                if (pass > 0) sum += so_far[in_block][o];
                if (pass + 1 < passes) {
                    so_far[in_block][o] = sum;
                    continue;
                }
            }
            const int n = tile * 16 + o % 16;
            if (n < p.N) w4_store<DT>(p, token0 + o / 16, n, sum);
        }
    };
    int parity = 0;
    if constexpr (!PASSES) {
        for (int tile = first; tile < end; ++tile, parity ^= 1) step(tile, 0, 0, parity, tile + 1 < end, tile + 1, 0);
    } else {
        for (int from = first; from < end; from += BLOCK) {
            const int to = from + BLOCK < end ? from + BLOCK : end;
            for (int pass = 0; pass < passes; ++pass) {
                load_x(pass);
                arrange_x();
                for (int tile = from; tile < to; ++tile, parity ^= 1) {
                    const bool last = tile + 1 == to, last_pass = last && pass + 1 == passes;
                    const int next_tile = !last ? tile + 1 : !last_pass ? from : to, next_pass = !last ? pass : !last_pass ? pass + 1 : 0;
                    step(tile, pass, tile - from, parity, next_tile < end, next_tile, next_pass);
                }
            }
        }
    }
}

// ---------------------------------------------------------------- activations shared in LDS
// Many tokens and many rows, 16-bit activations: a wave takes four tiles of 16 weight rows for itself, the
// columns from first to last, and all tokens.  The activations of a unit of 128 columns lie in LDS, in the layout
// of the products, for all eight waves; the next unit's are on their way to the other buffer.  So a
// unit's activations are read from LDS once for four tiles of rows, the sums stay in registers, and no
// wave waits for another's.  The codes come two units at a time, 128 bytes of eight rows a load, and are
// exchanged through a slice of LDS of the wave's own, as are the scales.  With slots finer than a unit a
// stage's loads are spread over its products (all at once they keep the waves waiting: 64 tokens, e2m1, groups
// of 32, 126 against 118 us); with one slot the registers do not allow it.
// Measured: bf16, 64 tokens, 128256 x 4096: 105 us with integers in groups of 128, 112 to 120 us with e2m1 in groups
// of 32, 640 and 560 TFLOP/s.  The products alone take 33 us.  Of a stage's 11800 cycles 5100 are products, 3000
// the issue of its loads, 1200 the barrier, the rest reads of LDS and vector instructions that the two waves
// of a SIMD, which its registers allow, do not hide from each other.
template <int DT, int KIND, int SLOTS>
__global__ __launch_bounds__(kW4Block, 2) void k_w4_rows(W4Params p) {
    static_assert(DT != kF32, "");
    constexpr bool INT = KIND != kW4E2M1, ZERO = KIND == kW4Zero, LATE = !INT;
    constexpr bool FINE = SLOTS > 1;
    constexpr int T = kMaxM / 16, R = kW4RowTiles, ROWS = 16 * R, EACH = 4 / SLOTS;
    constexpr int STAGE_SLOTS = 2 * SLOTS, ENTRIES = ROWS * STAGE_SLOTS, SL = ENTRIES / kWave, STRIDE = STAGE_SLOTS + 1;
    constexpr int CODE_ROW = 9, XL = T * 256 / kW4Block;
    static_assert(SL * kWave == ENTRIES && XL * kW4Block == T * 256, "");
    __shared__ uint4 xs[2][2][T][4][kWave];                  // two stages of two units
    __shared__ uint4 slices[kW4Held][ROWS * CODE_ROW];
    __shared__ unsigned scales[kW4Held][ROWS * STRIDE];      // fp32 scale, or the 16-bit scale and 1 + zero / 16 in fp16
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane & 15, q = lane >> 4;
    const int row_bytes = p.K / 2, units = (p.K + kW4UnitCols - 1) / kW4UnitCols;
    const size_t row0 = ((size_t)blockIdx.x * kW4Held + wave) * ROWS;

    // (a lane's number anew: addresses are worked out where they are used, not kept through the products)
    auto fresh_lane = [&]() CORAL_INLINE {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    const size_t code_bytes = (size_t)p.N * row_bytes;
    uint4 w[2 * R];
    auto load_codes = [&](int stage, int i) CORAL_INLINE {
        const int l = fresh_lane();
        const Buffer view = buffer_view(p.codes, row0 * row_bytes + (size_t)stage * kW4UnitCols, code_bytes, 2 * stage < units);
        w[i] = buffer_read16<kBufferStream>(view, (unsigned)(i * 8 + l / 8) * (unsigned)row_bytes + (unsigned)(l % 8) * 16u);
    };
    auto put_codes = [&]() CORAL_INLINE {
        const int l = fresh_lane();
#pragma unroll
        for (int i = 0; i < 2 * R; ++i) store_vec(&slices[wave][(i * 8 + l / 8) * CODE_ROW + l % 8], w[i]);
    };
    const size_t scale_first = row0 * p.n_groups, scale_all = (size_t)p.N * p.n_groups;
    unsigned s_raw[SL], z_raw[SL];
    auto load_scales = [&](int stage, int i) CORAL_INLINE {
        const Buffer view = buffer_view(p.scales, scale_first * 2, scale_all * 2, 2 * stage < units);
        const Buffer z_view = buffer_view(p.zeros, scale_first, scale_all, 2 * stage < units);
        const int e = i * kWave + fresh_lane();
        const unsigned slot = stage * STAGE_SLOTS + e % STAGE_SLOTS, g = FINE ? slot : w4_group_of(p, slot);
        const unsigned at = (unsigned)(e / STAGE_SLOTS) * (unsigned)p.n_groups + g;
        const unsigned behind = slot * (kW4UnitCols / SLOTS) < (unsigned)p.K ? 0u : kBufferBehind;         // (as in k_w4_held)
        s_raw[i] = buffer_read2(view, at * 2u | behind);
        if constexpr (ZERO) z_raw[i] = buffer_read1(z_view, at | behind);
    };
    // one of a stage's loads
    constexpr int LOADS = 2 * R + SL;
    static_assert(LOADS <= 4 * R, "one for every product of a unit");
    auto load_part = [&](int stage, int i) CORAL_INLINE {
        if (i < 2 * R) load_codes(stage, i);
        else if (i < LOADS) load_scales(stage, i - 2 * R);
    };
    auto put_scales = [&]() CORAL_INLINE {
        const int l = fresh_lane();
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const int e = i * kWave + l;
            const unsigned zero = ZERO ? __builtin_bit_cast(unsigned short, (_Float16)fmaf((float)z_raw[i], 0.0625f, 1.0f)) : 0u;
            const unsigned word = ZERO ? s_raw[i] << 16 | zero : __float_as_uint(widen16<DT>((unsigned short)s_raw[i]));
            scales[wave][e / STAGE_SLOTS * STRIDE + e % STAGE_SLOTS] = word;
        }
    };
    const Buffer x_view = buffer_view(p.x, 0, (size_t)p.M * p.K * 2);
    uint4 x_next[XL];
    // a wave's load is of eight tokens, 128 bytes each; eight neighbouring lanes write to different banks
    auto x_token = [&](int i, int l) CORAL_INLINE { return (i * kW4Held + wave) / 2 * 8 + l % 8; };
    auto x_chunk = [&](int i, int l) CORAL_INLINE { return (i * kW4Held + wave) % 2 * 8 + l / 8; };
    auto load_x = [&](int unit) CORAL_INLINE {
        const int l = fresh_lane();
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int col = unit * kW4UnitCols + x_chunk(i, l) * 8;
            x_next[i] = buffer_read16(x_view, col < p.K ? ((unsigned)x_token(i, l) * (unsigned)p.K + (unsigned)col) * 2u : kBufferEnd);
        }
    };
    auto put_x = [&](int buffer, int j) CORAL_INLINE {
        const int l = fresh_lane();
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int token = x_token(i, l), c = x_chunk(i, l);
            const int s = FINE ? c / 4 : c % 4, chunk = FINE ? c % 4 : c / 4;
            store_vec(&xs[buffer][j][token / 16][s][chunk * 16 + token % 16], w4_order<KIND>(x_next[i]));
        }
    };
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    constexpr unsigned kMinus = KIND == kW4Sym ? (DT == kF16 ? 0xCE00CE00u : 0xC1C0C1C0u) : DT == kF16 ? 0xCC00CC00u : 0xC180C180u;
    const uint4 minus = make_uint4(kMinus, kMinus, kMinus, kMinus);
    f32x4_t y[R][T];
#pragma unroll
    for (int a = 0; a < R; ++a)
#pragma unroll
        for (int t = 0; t < T; ++t) y[a][t] = zero4;
    auto scale_word = [&](int a, int slot) CORAL_INLINE { return scales[wave][(a * 16 + r) * STRIDE + slot]; };
    auto scale_of = [&](unsigned word) CORAL_INLINE { return ZERO ? widen16<DT>((unsigned short)(word >> 16)) : __uint_as_float(word); };
    // where the sums of a group start: at the offset's part
    auto start = [&](unsigned word, const f32x4_t (&offset)[T], f32x4_t (&acc)[T]) CORAL_INLINE {
        const float zero = ZERO ? (float)__builtin_bit_cast(_Float16, (unsigned short)word) : 0.f;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            acc[t] = offset[t];
            if constexpr (ZERO) {
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[t][v] *= zero;
            }
        }
    };
    auto add = [&](int a, int t, float scale, const f32x4_t& acc) CORAL_INLINE {
#pragma unroll
        for (int v = 0; v < 4; ++v) y[a][t][v] = fmaf(scale, acc[v], y[a][t][v]);
    };
    // Unit j of a stage.  The products of T token tiles go off together, and while they run the last ones' sums
    // are scaled and added and the next ones' operand is made: the fences keep it so, or the compiler waits
    // for each product by itself.
    auto unit = [&](int buffer, int j, auto meanwhile) CORAL_INLINE {
        if constexpr (FINE) {
            // a slot's EACH products one after the other, and the next slot's operands on their way where the
            // registers allow it
            constexpr bool AHEAD = EACH == 1;
            uint4 x[EACH][T];
            unsigned code[EACH][R], word[R];
            auto fetch = [&](int slot, uint4 (&to)[EACH][T], unsigned (&c)[EACH][R], unsigned (&w)[R]) CORAL_INLINE {
#pragma unroll
                for (int a = 0; a < R; ++a) {
#pragma unroll
                    for (int e = 0; e < EACH; ++e)
                        c[e][a] = reinterpret_cast<const unsigned*>(&slices[wave][(a * 16 + r) * CODE_ROW + j * 4 + slot * EACH + e])[q];
                    w[a] = scale_word(a, j * SLOTS + slot);
                }
#pragma unroll
                for (int e = 0; e < EACH; ++e)
#pragma unroll
                    for (int t = 0; t < T; ++t) to[e][t] = load_vec(&xs[buffer][j][t][slot * EACH + e][lane]);
            };
            f32x4_t acc[LATE ? 2 : 1][T];
            float scale[LATE ? 2 : 1] = {};
            fetch(0, x, code, word);
#pragma unroll
            for (int slot = 0; slot < SLOTS; ++slot) {
                uint4 x_then[EACH][T];
                unsigned code_then[EACH][R], word_then[R];
                if (AHEAD && slot + 1 < SLOTS) fetch(slot + 1, x_then, code_then, word_then);
                f32x4_t offset[T];
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    offset[t] = zero4;
#pragma unroll
                    for (int e = 0; e < EACH; ++e)
                        if constexpr (INT) offset[t] = mfma_tile<DT>(x[e][t], minus, offset[t]);
                }
                uint4 op = w4_operand<DT, KIND>(code[0][0]);
#pragma unroll
                for (int a = 0; a < R; ++a) {
                    const int now = LATE ? (slot * R + a) & 1 : 0;
                    start(word[a], offset, acc[now]);
                    scale[now] = scale_of(word[a]);
#pragma unroll
                    for (int e = 0; e < EACH; ++e) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int t = 0; t < T; ++t) acc[now][t] = mfma_tile<DT>(x[e][t], op, acc[now][t]);
                        __builtin_amdgcn_sched_barrier(0);
                        if (LATE && e == 0 && slot + a > 0) {
#pragma unroll
                            for (int t = 0; t < T; ++t) add(a > 0 ? a - 1 : R - 1, t, scale[LATE ? now ^ 1 : 0], acc[LATE ? now ^ 1 : 0][t]);
                        }
                        if (e + 1 < EACH) op = w4_operand<DT, KIND>(code[e + 1 < EACH ? e + 1 : 0][a]);
                        else if (a + 1 < R) op = w4_operand<DT, KIND>(code[0][a + 1]);
                        meanwhile((slot * R + a) * EACH + e);
                    }
                    if constexpr (!LATE) {
#pragma unroll
                        for (int t = 0; t < T; ++t) add(a, t, scale[now], acc[now][t]);
                    }
                }
                if (!AHEAD && slot + 1 < SLOTS) fetch(slot + 1, x, code, word);
                if (AHEAD && slot + 1 < SLOTS) {
#pragma unroll
                    for (int t = 0; t < T; ++t) x[0][t] = x_then[0][t];
#pragma unroll
                    for (int a = 0; a < R; ++a) {
                        code[0][a] = code_then[0][a];
                        word[a] = word_then[a];
                    }
                }
            }
            if constexpr (LATE) {
#pragma unroll
                for (int t = 0; t < T; ++t) add(R - 1, t, scale[(SLOTS * R - 1) & 1], acc[(SLOTS * R - 1) & 1][t]);
            }
        } else {
            uint4 x[T][4];
            f32x4_t offset[T];
            uint4 code = load_vec(&slices[wave][r * CODE_ROW + j * 4 + q]);
            unsigned word = scale_word(0, j);
#pragma unroll
            for (int t = 0; t < T; ++t) offset[t] = zero4;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < T; ++t) x[t][s] = load_vec(&xs[buffer][j][t][s][lane]);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < T; ++t)
                    if constexpr (INT) offset[t] = mfma_tile<DT>(x[t][s], minus, offset[t]);
            uint4 op = w4_operand<DT, KIND>(code.x);
#pragma unroll
            for (int a = 0; a < R; ++a) {
                f32x4_t acc[T];
                start(word, offset, acc);
                const float scale = scale_of(word);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int t = 0; t < T; ++t) acc[t] = mfma_tile<DT>(x[t][s], op, acc[t]);
                    __builtin_amdgcn_sched_barrier(0);
                    op = w4_operand<DT, KIND>(s == 0 ? code.y : s == 1 ? code.z : s == 2 ? code.w : code.x);
                    if (s == 2 && a + 1 < R) {               // the next tile's
                        code = load_vec(&slices[wave][((a + 1) * 16 + r) * CODE_ROW + j * 4 + q]);
                        word = scale_word(a + 1, j);
                    }
                }
#pragma unroll
                for (int t = 0; t < T; ++t) add(a, t, scale, acc[t]);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_part(0, i);
    load_x(0);
    put_x(0, 0);
    load_x(1);                                               // (behind the last column there is none)
    put_x(0, 1);
    __syncthreads();
    for (int stage = 0; 2 * stage < units; ++stage) {        // uniform, as all here
        const int buffer = stage & 1;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        put_codes();
        put_scales();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        load_x(2 * stage + 2);                               // (in front of the codes, which take longer)
        if constexpr (!FINE) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_part(stage + 1, i);
        }
        unit(buffer, 0, [&](int i) CORAL_INLINE { load_part(stage + 1, i); });
        put_x(buffer ^ 1, 0);
        load_x(2 * stage + 3);
        if (2 * stage + 1 < units) unit(buffer, 1, [](int) {});
        put_x(buffer ^ 1, 1);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
        const size_t n = row0 + a * 16 + r;
        if (n >= (size_t)p.N) continue;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int m = t * 16 + 4 * q + v;
                if (m < p.M) w4_store<DT>(p, m, (int)n, y[a][t][v]);
            }
    }
}

}  // namespace
