// What the kernels and entry points of a drafter's attention share: eight values of a head in a lane,
// the cache of 4-bit floats, and the host's checks.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <cmath>

#include "buffer_loads.h"
#include "coral_lmhead.h"
#include "device_utils.h"

namespace {

// The cache as a kernel sees it: a token's values of a head lie side by side, two codes a byte, with one
// scale byte (2^(byte - 127)) for 32 of them; a head's tokens of a page lie side by side too, so that the
// tokens which a wave reads together are whole lines.
struct Kv4 {
    unsigned char *k_codes, *k_scales, *v_codes, *v_scales;
    int pages, page_shift, kv_heads;
};
constexpr unsigned kKv4LargestScale = 252;       // 6 * 2^125 is finite in bf16 and fp32; larger bytes count as this one
constexpr unsigned kKv4LargestScaleF16 = 140;    // and 6 * 2^13 in fp16
// A unit as calls of storage type DT read it: no value that they make of it is infinite, whatever the byte.
template <int DT>
__device__ __forceinline__ float kv4_unit(unsigned byte) {
    const unsigned most = DT == kF16 ? kKv4LargestScaleF16 : kKv4LargestScale;
    return __uint_as_float((byte < most ? byte : most) << 23);
}

// An offset cut to an array of `most` rows: differences of two such never pass 32 bits, whatever the offsets are.
__device__ __forceinline__ int cut_offset(int at, int most) { return at < 0 ? 0 : at > most ? most : at; }

// Eight values of storage type DT as fp32, and back with one rounding to nearest even.
template <int DT>
__device__ __forceinline__ void widen8(const uint4 (&raw)[DT == kF32 ? 2 : 1], float (&x)[8]) {
    const unsigned w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, DT == kF32 ? raw[DT == kF32].x : 0, DT == kF32 ? raw[DT == kF32].y : 0,
                           DT == kF32 ? raw[DT == kF32].z : 0, DT == kF32 ? raw[DT == kF32].w : 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (DT == kF32) x[j] = __uint_as_float(w[j]);
        else x[j] = widen16<DT>((unsigned short)(j & 1 ? w[j / 2] >> 16 : w[j / 2]));
    }
}
// Two values rounded to nearest even (one instruction each for bf16 and fp16; NaN stays NaN).
template <int DT>
__device__ __forceinline__ unsigned narrow2(float a, float b) {
    if (DT == kF16) {
        const f16x2_t h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(unsigned, h);
    }
    const bf16x2_t h = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, h);
}
template <int DT>
__device__ __forceinline__ void narrow8(const float (&x)[8], uint4 (&raw)[DT == kF32 ? 2 : 1]) {
    if (DT == kF32) {
        raw[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        raw[DT == kF32] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
    } else {
        raw[0] = make_uint4(narrow2<DT>(x[0], x[1]), narrow2<DT>(x[2], x[3]), narrow2<DT>(x[4], x[5]), narrow2<DT>(x[6], x[7]));
    }
}
template <int DT>
__device__ __forceinline__ void load8(const void* at, uint4 (&raw)[DT == kF32 ? 2 : 1]) {
    raw[0] = load_vec(static_cast<const uint4*>(at));
    if (DT == kF32) raw[DT == kF32] = load_vec(static_cast<const uint4*>(at) + 1);
}
template <int DT>
__device__ __forceinline__ void store8(void* at, const uint4 (&raw)[DT == kF32 ? 2 : 1]) {
    store_vec(static_cast<uint4*>(at), raw[0]);
    if (DT == kF32) store_vec(static_cast<uint4*>(at) + 1, raw[DT == kF32]);
}

// x combined with the other lanes of a group of N = 4, 8, 16 or 32, by data movement inside the vector unit.
template <int N, class Op>
__device__ __forceinline__ float lanes_reduce(float x, Op op) {
    x = op(x, dpp_move<0xB1>(x));                // quad_perm 1,0,3,2
    x = op(x, dpp_move<0x4E>(x));                // quad_perm 2,3,0,1
    if (N >= 8) x = op(x, dpp_move<0x141>(x));   // row_half_mirror
    if (N >= 16) x = op(x, dpp_move<0x140>(x));  // row_mirror
    if (N >= 32) {
        float y = x;
        swap_rows(x, y);
        x = op(x, y);
    }
    return x;
}

// Eight values of a lane as 4-bit floats; four lanes hold a block of 32 and share its scale: the power of
// two that puts the largest of them at 3.5 to 7 units (above 7 a unit twice as large is nearer), as a
// biased exponent.  The division by it is exact, the rounding to nearest with ties to even codes is the
// conversion instruction's, which also cuts at 6.
template <int DT>
__device__ __forceinline__ unsigned kv4_codes(const float (&x)[8], unsigned* scale) {
    float top = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
    top = lanes_reduce<4>(top, [](float a, float b) { return fmaxf(a, b); });
    const unsigned bits = __float_as_uint(top);
    const int e = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    const int most = DT == kF16 ? (int)kKv4LargestScaleF16 : (int)kKv4LargestScale;
    *scale = (unsigned)(e < 1 ? 1 : e > most ? most : e);
    const float unit = __uint_as_float(*scale << 23);
    unsigned c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
}

// ---------------------------------------------------------------- host checks
inline size_t storage_bytes(coral_dtype dt) { return dt == CORAL_F32 ? 4 : 2; }
inline bool storage_known(coral_dtype dt) { return dt == CORAL_F32 || dt == CORAL_BF16 || dt == CORAL_F16; }
inline bool head_dim_known(int d) { return d == 64 || d == 128 || d == 256; }
constexpr int kMostHeads = 1024;
constexpr int kMostSequences = 65535;
constexpr int kMostTokens = (1 << 24) - 1;                   // a grid's threads are counted in 32 bits

// Scores are multiplied by a number above zero, to powers of two: the sign goes to q (exactly), and a scale of nothing (all
// weights equal) is little enough.
inline float score_scale(float scale) { return fmaxf(fabsf(scale) * 1.44269504088896340736f, 1e-37f); }
inline unsigned score_sign(float scale, coral_dtype dt) { return !std::signbit(scale) ? 0u : dt == CORAL_F32 ? 0x80000000u : 0x80008000u; }

// Rows of `width` bytes, `stride` bytes apart.
struct Rows {
    const void* base;
    int64_t stride, width;
    int n;
    int64_t extent() const { return n < 1 || !base ? 0 : (n - 1) * stride + width; }
    bool same(const Rows& o) const { return base == o.base && stride == o.stride; }
};
inline bool ranges_overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && a_bytes > 0 && b_bytes > 0 && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}
// Whether rows share memory; columns of one wider matrix do not.
inline bool rows_overlap(const Rows& a, const Rows& b) {
    if (!ranges_overlap(a.base, a.extent(), b.base, b.extent())) return false;
    if (a.stride != b.stride) return true;
    const int64_t d = (int64_t)((uintptr_t)b.base - (uintptr_t)a.base);
    const int64_t gap = ((d % a.stride) + a.stride) % a.stride;
    return gap < a.width || gap + b.width > a.stride;
}
// Rows of `heads` heads that kernels read or write in 16-byte pieces.
inline coral_status check_rows(const void* base, int64_t stride, int heads, int head_dim, coral_dtype dt, int n, Rows* out) {
    const int64_t w = (int64_t)storage_bytes(dt), width = (int64_t)heads * head_dim;
    if (!base) return CORAL_ERR_NULL;
    if (stride < width) return CORAL_ERR_SHAPE;
    if (((uintptr_t)base & 15u) || (stride * w) % 16 != 0 || stride > ((int64_t)1 << 40) || n > kMostTokens) return CORAL_ERR_UNSUPPORTED;
    *out = {base, stride * w, width * w, n};
    return CORAL_OK;
}

inline coral_status check_kv4(const coral_kv4_cache* c, Kv4* out) {
    if (!c) return CORAL_ERR_NULL;
    if (c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return CORAL_ERR_SHAPE;
    if (!head_dim_known(c->head_dim) || c->kv_heads > kMostHeads) return CORAL_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1))) return CORAL_ERR_UNSUPPORTED;
    if ((int64_t)c->pages * c->page_size > INT32_MAX) return CORAL_ERR_UNSUPPORTED;
    if (!c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return CORAL_ERR_NULL;
    if (((uintptr_t)c->k_codes | (uintptr_t)c->k_scales | (uintptr_t)c->v_codes | (uintptr_t)c->v_scales) & 15u)
        return CORAL_ERR_UNSUPPORTED;
    *out = {c->k_codes, c->k_scales, c->v_codes, c->v_scales, c->pages, __builtin_ctz((unsigned)c->page_size), c->kv_heads};
    return CORAL_OK;
}
// The cache's four arrays, each as one row.
inline void kv4_parts(const coral_kv4_cache* c, Rows (&out)[4]) {
    const int64_t heads = (int64_t)c->pages * c->page_size * c->kv_heads, codes = heads * (c->head_dim / 2), scales = heads * (c->head_dim / 32);
    out[0] = {c->k_codes, codes, codes, 1};
    out[1] = {c->k_scales, scales, scales, 1};
    out[2] = {c->v_codes, codes, codes, 1};
    out[3] = {c->v_scales, scales, scales, 1};
}

}  // namespace
