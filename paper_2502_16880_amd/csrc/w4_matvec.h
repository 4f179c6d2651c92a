// Products with 4-bit weights: y[m,n] = act(sum_j x[m,j] w[n,j] + bias[n]) + residual[m,n] for up to
// 64 tokens, w[n,j] = scale[n,j/group] * (code[n,j] - zero[n,j/group]), or scale * e2m1(code).
//
// All products go through v_mfma_f32_16x16x32, tokens as its rows and weight rows as its columns, so
// that a lane holds the sums of one weight row and the row's scales and zero points are one value a
// lane.  Codes become 16-bit operands exactly: an integer code n is put into the mantissa of 16.0
// (16 + n, two operations for two codes) and the sum of (16 + zero) x is taken off per group in fp32,
// or is where the accumulator starts; an e2m1 code has an instruction.  Scales multiply the group's
// fp32 sum, never a 16-bit weight.  fp32 activations are split into three bf16 values whose sum they
// are, and every product is taken three times: the sums are fp32 sums of exact products in all types.
#pragma once
#include "device_utils.h"

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
};

constexpr int kW4Waves = 4;
constexpr int kW4UnitCols = 128;                 // columns of a unit: four products of 32

template <int DT>
constexpr int kW4Op = DT == kF16 ? kF16 : kBF16; // operand type of the products
template <int DT>
constexpr int kW4Parts = DT == kF32 ? 3 : 1;     // operands that an activation is split into

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
        o.x = ((w << 6) & kMask) | kSixteen;
        o.y = ((w << 2) & kMask) | kSixteen;
        o.z = ((w >> 2) & kMask) | kSixteen;
        o.w = ((w >> 6) & kMask) | kSixteen;
    } else {                                     // ... of a seven-bit mantissa
        constexpr unsigned kMask = 0x00780078u, kSixteen = 0x41804180u;
        o.x = ((w << 3) & kMask) | kSixteen;
        o.y = ((w >> 1) & kMask) | kSixteen;
        o.z = ((w >> 5) & kMask) | kSixteen;
        o.w = ((w >> 9) & kMask) | kSixteen;
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

// Eight fp32 values as three bf16 values each, x = hi + mid + lo exactly: the significand's 24 bits
// are cut off in eights.
__device__ __forceinline__ void w4_split(const float (&f)[8], uint4 (&part)[3]) {
    unsigned b[3][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float r = f[j];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            b[c][j] = __float_as_uint(r) & 0xffff0000u;
            r -= __uint_as_float(b[c][j]);
        }
    }
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        part[c].x = __builtin_amdgcn_perm(b[c][1], b[c][0], 0x07060302u);
        part[c].y = __builtin_amdgcn_perm(b[c][3], b[c][2], 0x07060302u);
        part[c].z = __builtin_amdgcn_perm(b[c][5], b[c][4], 0x07060302u);
        part[c].w = __builtin_amdgcn_perm(b[c][7], b[c][6], 0x07060302u);
    }
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

// 16 weight rows and 16 tokens a workgroup; its waves share the columns in units of 128 and their
// sums meet in LDS.
template <int DT, int KIND>
__global__ __launch_bounds__(kW4Waves * kWave) void k_w4(W4Params p) {
    constexpr int OP = kW4Op<DT>, PARTS = kW4Parts<DT>;
    __shared__ float sums[kW4Waves][256];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
    const int n = n0 + r < p.N ? n0 + r : p.N - 1;           // what is read twice is not stored
    const int m = m0 + r < p.M ? m0 + r : p.M - 1;
    const unsigned char* codes = p.codes + (size_t)n * (p.K / 2);
    const size_t scales = (size_t)n * p.n_groups;
    const uint4* x = static_cast<const uint4*>(p.x) + (size_t)m * p.K / (DT == kF32 ? 4 : 8);
    uint4 minus;                                             // sums of (16 + zero) x: the zero comes later
    minus.x = minus.y = minus.z = minus.w = OP == kF16 ? 0xCC00CC00u : 0xC180C180u;        // -16.0
    if (KIND == kW4Sym) minus.x = minus.y = minus.z = minus.w = OP == kF16 ? 0xCE00CE00u : 0xC1C0C1C0u;   // -24.0
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = wave * kW4UnitCols; c0 < p.K; c0 += kW4Waves * kW4UnitCols) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int col = c0 + s * 32 + q * 8;
            if (c0 + s * 32 >= p.K) break;                   // wave-uniform
            const bool in = col < p.K;                       // (K is a multiple of 8)
            unsigned w = 0u;
            uint4 part[PARTS];
            if constexpr (DT == kF32) {
                float f[8];
                uint4 a = make_uint4(0, 0, 0, 0), b = a;
                if (in) {
                    a = load_vec(x + col / 4);
                    b = load_vec(x + col / 4 + 1);
                }
                f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y);
                f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
                f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y);
                f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
                w4_split(f, part);
            } else {
                part[0] = in ? load_vec(x + col / 8) : make_uint4(0, 0, 0, 0);
            }
            if (in) w = *reinterpret_cast<const unsigned*>(codes + col / 2);
            const uint4 op = w4_operand<OP, KIND>(w);
            const int g = (c0 + s * 32) / p.group;
            const float scale = w4_load<DT>(p.scales, scales + g);
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f}, ones = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = PARTS - 1; c >= 0; --c) {           // the small parts first
                const uint4 a = w4_order<KIND>(part[c]);
                if constexpr (KIND == kW4Sym) acc = mfma_tile<OP>(a, minus, acc);
                if constexpr (KIND == kW4Zero) ones = mfma_tile<OP>(a, minus, ones);
                acc = mfma_tile<OP>(a, op, acc);
            }
            if constexpr (KIND == kW4Zero) {
                const float zero = 1.0f + (float)p.zeros[scales + g] * 0.0625f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = fmaf(zero, ones[i], acc[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fmaf(scale, acc[i], y[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][(4 * q + i) * 16 + r] = y[i];
    __syncthreads();
    const int at = threadIdx.x;                              // token at / 16, weight row at % 16
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kW4Waves; ++w) sum += sums[w][at];
    if (m0 + at / 16 < p.M && n0 + at % 16 < p.N) w4_store<DT>(p, m0 + at / 16, n0 + at % 16, sum);
}

}  // namespace
