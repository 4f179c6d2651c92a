// Norms and rotation of queries and keys, and the cache of 4-bit floats: append and read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_common.h"

namespace {

constexpr int kHeadThreads = 256;
constexpr int kHeadWaves = kHeadThreads / kWave;

struct HeadsParams {
    const char *q, *k, *v;
    char *q_out, *k_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;   // bytes from token to token
    const char *q_weight, *k_weight;
    const int32_t* positions;
    const float* inv_freq;
    const int32_t* slots;
    Kv4 cache;
    int q_heads, kv_heads, rot, passes;
    float eps;
};

enum RotationForm { kRotNone = 0, kRotPairs = 1, kRotLanes = 2, kRotAny = 3 };

// y = x / sqrt(mean x^2 + eps) * weight, pairs of y turned by position * inv_freq, one rounding at the end.
// A lane holds eight neighbouring values, D / 8 lanes a head; a workgroup takes the heads of one token,
// so that its angles are computed once: in turns, by a product in 64 bits of which only the fraction is
// kept (a position of 10^6 times a frequency of 1 in 32 bits would be off by 0.03 radians), and handed
// over in LDS.  The partner of a value is in the same lane (kRotPairs: neighbours turn), in the lane
// rot / 16 further (kRotLanes) or, where rot is no multiple of 16, anywhere (kRotAny: through LDS).
// With CACHE the keys so made (rounded to DT first, as two calls would) and the values go into the cache.
// Bound by memory: each value is read and written once (8192 tokens of 40 heads of 128, bf16: 33 us, 5.0 TB/s; one token: 3.1, the launch).  With the
// cache, whose pieces are 64 bytes, 49 us (the same tokens and 8 heads of values, 3.6 TB/s) and 3.4.
template <int DT, int D, int FORM, bool CACHE>
__global__ __launch_bounds__(kHeadThreads) void k_heads(HeadsParams p) {
    constexpr int kRaw = DT == kF32 ? 2 : 1, kLanes = D / 8, kPer = kWave / kLanes, kBytes = DT == kF32 ? 4 : 2;
    __shared__ float2 turn[FORM == kRotNone ? 1 : D / 2];
    __shared__ float staged[FORM == kRotAny ? kHeadWaves : 1][FORM == kRotAny ? kWave * 8 : 1];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, l = lane % kLanes;
    const int64_t t = blockIdx.x;
    const int n_turned = p.q_heads + p.kv_heads, n = CACHE ? n_turned + p.kv_heads : n_turned;
    const int per_pass = kHeadWaves * kPer;
    int head = (int)blockIdx.y * p.passes * per_pass + wave * kPer + lane / kLanes;
    auto place = [&](int h) CORAL_INLINE {
        h = h < n ? h : n - 1;
        const char* row = h < p.q_heads ? p.q + t * p.q_stride : h < n_turned ? p.k + t * p.k_stride : p.v + t * p.v_stride;
        const int at = h < p.q_heads ? h : h < n_turned ? h - p.q_heads : h - n_turned;
        return row + ((int64_t)at * D + l * 8) * kBytes;
    };
    uint4 raw[kRaw];
    load8<DT>(place(head), raw);
    const bool q_norm = p.q_weight != nullptr, k_norm = p.k_weight != nullptr;
    float q_w[8], k_w[8];
    if (q_norm) {
        uint4 w[kRaw];
        load8<DT>(p.q_weight + l * 8 * kBytes, w);
        widen8<DT>(w, q_w);
    }
    if (k_norm) {
        uint4 w[kRaw];
        load8<DT>(p.k_weight + l * 8 * kBytes, w);
        widen8<DT>(w, k_w);
    }
    const int half = p.rot / 2;
    float c[8], s[8];
    if (FORM != kRotNone) {
        if ((int)threadIdx.x < half) {
            const double turns = (double)p.positions[t] * (double)p.inv_freq[threadIdx.x] * 0.15915494309189533577;
            float sn, cs;
            sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
            turn[threadIdx.x] = make_float2(cs, sn);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int d = l * 8 + j;
            const bool first = FORM == kRotPairs ? (j & 1) == 0 : d < half;
            const int i = FORM == kRotPairs ? d / 2 : first ? d : d - half;
            const bool in = d < p.rot;
            const float2 a = turn[in ? i : 0];
            c[j] = in ? a.x : 1.f;
            s[j] = in ? (first ? -a.y : a.y) : 0.f;
        }
    }
    // where the partners of this lane's values are (kRotLanes: a lane, kRotAny: places of the wave's part of LDS)
    const int d0 = l * 8;
    const int partner = FORM == kRotLanes ? (d0 >= p.rot ? lane : d0 < half ? lane + half / 8 : lane - half / 8) : 0;
    for (int pass = 0; pass < p.passes; ++pass, head += per_pass) {
        if (head - lane / kLanes >= n) break;                    // the wave's first head (uniform)
        uint4 next[kRaw] = {};
        if (pass + 1 < p.passes) load8<DT>(place(head + per_pass), next);
        float x[8];
        widen8<DT>(raw, x);
        const bool is_q = head < p.q_heads, is_v = CACHE && head >= n_turned, real = head < n;
        if (q_norm || k_norm) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
            sum = lanes_reduce<kLanes>(sum, [](float a, float b) { return a + b; });
            const float inv = 1.f / sqrtf(fmaf(sum, 1.f / D, p.eps));
            const bool norm = is_q ? q_norm : k_norm && !is_v;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = norm ? x[j] * inv * (is_q ? q_w[j] : k_w[j]) : x[j];
        }
        if (FORM != kRotNone) {
            float y[8];
            if (FORM == kRotPairs) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j ^ 1];
            } else if (FORM == kRotLanes) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = __shfl(x[j], partner, kWave);
            } else {
                float* mine = staged[FORM == kRotAny ? wave : 0];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int j = 0; j < 8; ++j) mine[lane * 8 + j] = x[j];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int d = d0 + j;
                    y[j] = mine[lane * 8 + j + (d >= p.rot ? 0 : d < half ? half : -half)];
                }
                __builtin_amdgcn_wave_barrier();
            }
            if (!is_v) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf(x[j], c[j], y[j] * s[j]);
            }
        }
        // (the rounding is of the fp32 value in every form of the kernel: not joined with the product before it)
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(x[j]));
        uint4 done[kRaw];
        narrow8<DT>(x, done);
        if (real && is_q) store8<DT>(p.q_out + t * p.q_out_stride + ((int64_t)head * D + d0) * kBytes, done);
        if (real && !is_q && !is_v && (!CACHE || p.k_out))
            store8<DT>(p.k_out + t * p.k_out_stride + ((int64_t)(head - p.q_heads) * D + d0) * kBytes, done);
        if (CACHE) {
            widen8<DT>(done, x);
            unsigned scale;
            const unsigned codes = kv4_codes<DT>(x, &scale);
            const int slot = p.slots[t];
            const bool held = real && !is_q && slot >= 0 && (slot >> p.cache.page_shift) < p.cache.pages;
            if (held) {
                const int h = is_v ? head - n_turned : head - p.q_heads;
                const int64_t page = slot >> p.cache.page_shift, at = slot & ((1 << p.cache.page_shift) - 1);
                const int64_t row = ((page * p.cache.kv_heads + h) << p.cache.page_shift) + at;
                *reinterpret_cast<unsigned*>((is_v ? p.cache.v_codes : p.cache.k_codes) + row * (D / 2) + l * 4) = codes;
                if ((l & 3) == 0) (is_v ? p.cache.v_scales : p.cache.k_scales)[row * (D / 32) + l / 4] = (unsigned char)scale;
            }
        }
#pragma unroll
        for (int j = 0; j < kRaw; ++j) raw[j] = next[j];
    }
}

struct Kv4Params {
    const char *k, *v;
    char *k_out, *v_out;
    int64_t k_stride, v_stride;
    const int32_t* slots;
    Kv4 cache;
    int64_t items;
};

// A token's keys and values into the cache, or out of it: eight values a lane, D / 8 lanes a head, first all
// keys of a token, then its values.  Bound by the launch (8192 tokens of 4 heads of 128: 7 us; 64 of 8: 2.9), by pieces of
// 64 bytes and a thread's two 64-bit divisions (16384 of 32, bf16: 88 us in, 98 out, 3.9 and 3.5 TB/s; fp32, 8192 of 8: 16 and 18).
template <int DT, int D, bool READ>
__global__ __launch_bounds__(kHeadThreads) void k_kv4_move(Kv4Params p) {
    constexpr int kRaw = DT == kF32 ? 2 : 1, kLanes = D / 8, kBytes = DT == kF32 ? 4 : 2;
    const int64_t item = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kHeadThreads + threadIdx.x;
    if (item >= p.items) return;                                 // whole heads: groups of lanes leave together
    const int l = (int)(item % kLanes);
    const int64_t head = item / kLanes;
    const int at_head = (int)(head % (2 * p.cache.kv_heads));
    const int64_t t = head / (2 * p.cache.kv_heads);
    const bool is_v = at_head >= p.cache.kv_heads;
    const int h = is_v ? at_head - p.cache.kv_heads : at_head;
    const int slot = p.slots[t];
    if (slot < 0 || (slot >> p.cache.page_shift) >= p.cache.pages) return;
    const int64_t page = slot >> p.cache.page_shift, at = slot & ((1 << p.cache.page_shift) - 1);
    const int64_t row = ((page * p.cache.kv_heads + h) << p.cache.page_shift) + at;
    unsigned* codes = reinterpret_cast<unsigned*>((is_v ? p.cache.v_codes : p.cache.k_codes) + row * (D / 2) + l * 4);
    unsigned char* scale = (is_v ? p.cache.v_scales : p.cache.k_scales) + row * (D / 32) + l / 4;
    uint4 raw[kRaw];
    float x[8];
    if (READ) {
        const unsigned w = *codes;
        const float unit = kv4_unit<DT>(*scale);
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
        const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
        narrow8<DT>(x, raw);
        store8<DT>((is_v ? p.v_out : p.k_out) + (t * p.cache.kv_heads + h) * (int64_t)(D * kBytes) + l * 8 * kBytes, raw);
    } else {
        const char* from = is_v ? p.v + t * p.v_stride : p.k + t * p.k_stride;
        load8<DT>(from + ((int64_t)h * D + l * 8) * kBytes, raw);
        widen8<DT>(raw, x);
        unsigned byte;
        *codes = kv4_codes<DT>(x, &byte);
        if ((l & 3) == 0) *scale = (unsigned char)byte;
    }
}

using heads_fn = void (*)(HeadsParams);
template <int DT, int D, bool CACHE>
heads_fn heads_kernel(int form) {
    switch (form) {
        case kRotNone: return k_heads<DT, D, kRotNone, CACHE>;
        case kRotPairs: return k_heads<DT, D, kRotPairs, CACHE>;
        case kRotLanes: return k_heads<DT, D, kRotLanes, CACHE>;
        default: return k_heads<DT, D, kRotAny, CACHE>;
    }
}
template <int DT>
heads_fn heads_kernel(int head_dim, int form, bool cache) {
    if (head_dim == 64) return cache ? heads_kernel<DT, 64, true>(form) : heads_kernel<DT, 64, false>(form);
    if (head_dim == 128) return cache ? heads_kernel<DT, 128, true>(form) : heads_kernel<DT, 128, false>(form);
    return cache ? heads_kernel<DT, 256, true>(form) : heads_kernel<DT, 256, false>(form);
}
using kv4_fn = void (*)(Kv4Params);
template <bool READ, int DT>
kv4_fn move_kernel(int head_dim) {
    return head_dim == 64 ? k_kv4_move<DT, 64, READ> : head_dim == 128 ? k_kv4_move<DT, 128, READ> : k_kv4_move<DT, 256, READ>;
}
template <bool READ>
kv4_fn move_kernel(int head_dim, coral_dtype dt) {
    return dt == CORAL_F32 ? move_kernel<READ, kF32>(head_dim) : dt == CORAL_BF16 ? move_kernel<READ, kBF16>(head_dim) : move_kernel<READ, kF16>(head_dim);
}

coral_status move_launch(kv4_fn fn, Kv4Params& p, int T, int head_dim, void* hip_stream) {
    p.items = (int64_t)T * 2 * p.cache.kv_heads * (head_dim / 8);
    const int64_t blocks = (p.items + kHeadThreads - 1) / kHeadThreads;
    const int64_t down = (blocks + kMostTokens - 1) / kMostTokens;
    hipLaunchKernelGGL(fn, dim3((unsigned)((blocks + down - 1) / down), (unsigned)down), dim3(kHeadThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}

}  // namespace

extern "C" coral_status coral_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const coral_rope* rope, int T,
                                           int q_heads, int kv_heads, int head_dim, coral_dtype dt, void* q_out, int64_t q_out_stride,
                                           void* k_out, int64_t k_out_stride, const coral_kv4_cache* cache, const void* v,
                                           int64_t v_stride, const int32_t* slots, void* hip_stream) {
    if (!rope) return CORAL_ERR_NULL;
    if (!storage_known(dt) || T < 0 || q_heads < 0 || kv_heads < 0 || q_heads + kv_heads < 1 || head_dim < 1) return CORAL_ERR_SHAPE;
    if (rope->rot_dim < 0 || rope->rot_dim > head_dim || rope->rot_dim % 2) return CORAL_ERR_SHAPE;
    if (!(rope->eps >= 0.f)) return CORAL_ERR_SHAPE;
    if (!head_dim_known(head_dim) || q_heads > kMostHeads || kv_heads > kMostHeads) return CORAL_ERR_UNSUPPORTED;
    HeadsParams p = {};
    if (cache) {
        const coral_status st = check_kv4(cache, &p.cache);
        if (st != CORAL_OK) return st;
        if (cache->kv_heads != kv_heads || cache->head_dim != head_dim) return CORAL_ERR_SHAPE;
    } else if (v || slots) {
        return CORAL_ERR_NULL;
    }
    if (T == 0) return CORAL_OK;
    Rows in_q = {}, in_k = {}, in_v = {}, out_q = {}, out_k = {};
    coral_status st = CORAL_OK;
    if (q_heads) {
        if ((st = check_rows(q, q_stride, q_heads, head_dim, dt, T, &in_q)) != CORAL_OK) return st;
        if ((st = check_rows(q_out, q_out_stride, q_heads, head_dim, dt, T, &out_q)) != CORAL_OK) return st;
    }
    if (kv_heads) {
        if ((st = check_rows(k, k_stride, kv_heads, head_dim, dt, T, &in_k)) != CORAL_OK) return st;
        if (k_out || !cache) {
            if ((st = check_rows(k_out, k_out_stride, kv_heads, head_dim, dt, T, &out_k)) != CORAL_OK) return st;
        }
    }
    if (cache) {
        if ((st = check_rows(v, v_stride, kv_heads, head_dim, dt, T, &in_v)) != CORAL_OK) return st;
        if (!slots) return CORAL_ERR_NULL;
    }
    if (rope->rot_dim && (!rope->positions || !rope->inv_freq)) return CORAL_ERR_NULL;
    if (((uintptr_t)rope->positions | (uintptr_t)rope->inv_freq | (uintptr_t)slots) & 3u) return CORAL_ERR_UNSUPPORTED;
    if (((uintptr_t)rope->q_weight | (uintptr_t)rope->k_weight) & 15u) return CORAL_ERR_UNSUPPORTED;
    // an output may be its own input; it shares memory with nothing else
    const int64_t w = (int64_t)storage_bytes(dt), weight = head_dim * w;
    const Rows small[5] = {{rope->q_weight, weight, weight, 1}, {rope->k_weight, weight, weight, 1}, {rope->positions, T * 4ll, T * 4ll, 1},
                           {rope->inv_freq, rope->rot_dim * 2, rope->rot_dim * 2, 1}, {slots, T * 4ll, T * 4ll, 1}};
    Rows parts[4] = {};
    if (cache) kv4_parts(cache, parts);
    auto clash = [&](const Rows& out, const Rows& own, const Rows& other) {
        if (!out.base) return false;
        if ((rows_overlap(out, own) && !out.same(own)) || rows_overlap(out, other) || rows_overlap(out, in_v)) return true;
        for (const Rows& r : small)
            if (rows_overlap(out, r)) return true;
        for (const Rows& r : parts)
            if (rows_overlap(out, r)) return true;
        return false;
    };
    if (clash(out_q, in_q, in_k) || clash(out_k, in_k, in_q) || rows_overlap(out_q, out_k)) return CORAL_ERR_UNSUPPORTED;
    for (const Rows& r : parts) {
        if (rows_overlap(r, in_q) || rows_overlap(r, in_k) || rows_overlap(r, in_v)) return CORAL_ERR_UNSUPPORTED;
        for (const Rows& o : small)
            if (rows_overlap(r, o)) return CORAL_ERR_UNSUPPORTED;
    }
    p.q = static_cast<const char*>(q); p.k = static_cast<const char*>(k); p.v = static_cast<const char*>(v);
    p.q_out = static_cast<char*>(q_out); p.k_out = static_cast<char*>(k_out);
    p.q_stride = in_q.stride; p.k_stride = in_k.stride; p.v_stride = in_v.stride;
    p.q_out_stride = out_q.stride; p.k_out_stride = out_k.stride;
    p.q_weight = q_heads ? static_cast<const char*>(rope->q_weight) : nullptr;
    p.k_weight = kv_heads ? static_cast<const char*>(rope->k_weight) : nullptr;
    p.positions = rope->positions; p.inv_freq = rope->inv_freq; p.slots = slots;
    p.q_heads = q_heads; p.kv_heads = kv_heads; p.rot = rope->rot_dim; p.eps = rope->eps;
    const int heads = q_heads + (cache ? 2 : 1) * kv_heads, per_pass = kHeadWaves * (kWave / (head_dim / 8));
    const int all = (heads + per_pass - 1) / per_pass;
    // A token's heads are one workgroup's where tokens fill the chip; of few tokens each pass is its own workgroup's.
    p.passes = T >= 1024 ? all : 1;
    const int form = rope->rot_dim == 0 ? kRotNone : rope->interleaved ? kRotPairs : rope->rot_dim % 16 == 0 ? kRotLanes : kRotAny;
    const heads_fn fn = dt == CORAL_F32 ? heads_kernel<kF32>(head_dim, form, cache != nullptr) : dt == CORAL_BF16 ? heads_kernel<kBF16>(head_dim, form, cache != nullptr)
                                                                                              : heads_kernel<kF16>(head_dim, form, cache != nullptr);
    hipLaunchKernelGGL(fn, dim3(T, (all + p.passes - 1) / p.passes), dim3(kHeadThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return hipGetLastError() == hipSuccess ? CORAL_OK : CORAL_ERR_HIP;
}

extern "C" coral_status coral_kv4_append(const coral_kv4_cache* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                         const int32_t* slots, int T, coral_dtype dt, void* hip_stream) {
    Kv4Params p = {};
    coral_status st = check_kv4(cache, &p.cache);
    if (st != CORAL_OK) return st;
    if (!storage_known(dt) || T < 0) return CORAL_ERR_SHAPE;
    if (T == 0) return CORAL_OK;
    Rows in_k, in_v, parts[4];
    if ((st = check_rows(k, k_stride, cache->kv_heads, cache->head_dim, dt, T, &in_k)) != CORAL_OK) return st;
    if ((st = check_rows(v, v_stride, cache->kv_heads, cache->head_dim, dt, T, &in_v)) != CORAL_OK) return st;
    if (!slots) return CORAL_ERR_NULL;
    if ((uintptr_t)slots & 3u) return CORAL_ERR_UNSUPPORTED;
    kv4_parts(cache, parts);
    for (const Rows& r : parts)
        if (rows_overlap(r, in_k) || rows_overlap(r, in_v) || rows_overlap(r, {slots, T * 4ll, T * 4ll, 1})) return CORAL_ERR_UNSUPPORTED;
    p.k = static_cast<const char*>(k); p.v = static_cast<const char*>(v);
    p.k_stride = in_k.stride; p.v_stride = in_v.stride; p.slots = slots;
    return move_launch(move_kernel<false>(cache->head_dim, dt), p, T, cache->head_dim, hip_stream);
}

extern "C" coral_status coral_kv4_read(const coral_kv4_cache* cache, const int32_t* slots, int T, coral_dtype dt, void* k_out, void* v_out,
                                       void* hip_stream) {
    Kv4Params p = {};
    coral_status st = check_kv4(cache, &p.cache);
    if (st != CORAL_OK) return st;
    if (!storage_known(dt) || T < 0) return CORAL_ERR_SHAPE;
    if (T == 0) return CORAL_OK;
    Rows out_k, out_v, parts[4];
    const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
    if ((st = check_rows(k_out, width, cache->kv_heads, cache->head_dim, dt, T, &out_k)) != CORAL_OK) return st;
    if ((st = check_rows(v_out, width, cache->kv_heads, cache->head_dim, dt, T, &out_v)) != CORAL_OK) return st;
    if (!slots) return CORAL_ERR_NULL;
    if ((uintptr_t)slots & 3u) return CORAL_ERR_UNSUPPORTED;
    kv4_parts(cache, parts);
    const Rows in_slots = {slots, T * 4ll, T * 4ll, 1};
    for (const Rows& r : parts)
        if (rows_overlap(r, out_k) || rows_overlap(r, out_v)) return CORAL_ERR_UNSUPPORTED;
    if (rows_overlap(out_k, out_v) || rows_overlap(in_slots, out_k) || rows_overlap(in_slots, out_v)) return CORAL_ERR_UNSUPPORTED;
    p.k_out = static_cast<char*>(k_out); p.v_out = static_cast<char*>(v_out); p.slots = slots;
    return move_launch(move_kernel<true>(cache->head_dim, dt), p, T, cache->head_dim, hip_stream);
}
