// Reads through buffer descriptors: what lies behind an operand's end is dropped and reads as zero, so
// that loads need no branch (which would wait for them where it ends) and no address cut to size.
#pragma once
#include "device_utils.h"

// A lambda that works on registers it captures (they are in memory where it is not inlined).
#define CORAL_INLINE __attribute__((always_inline))

namespace {

typedef __amdgpu_buffer_rsrc_t Buffer;
// The bytes from `first` on of an operand of `bytes`, or none: of more than kBufferEnd those before it, so that
// an offset from kBufferEnd on lies behind every view's end.
constexpr unsigned kBufferEnd = 0xffffffe0u;
constexpr unsigned kBufferBehind = 0xfffffffcu;  // such an offset, to be or'ed to any (the instructions hold a small negative number)
__device__ __forceinline__ Buffer buffer_view(const void* base, size_t first, size_t bytes, bool any = true) {
    const size_t left = any && first < bytes ? bytes - first : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + first, 0,
                                             left < kBufferEnd ? (unsigned)left : kBufferEnd, 0x00020000);
}
// An offset is a lane's own: a part in a scalar register of its own is not compared with the view's end.
constexpr int kBufferStream = 2;                 // non-temporal: what is read once
template <int AUX = 0>
__device__ __forceinline__ uint4 buffer_read16(Buffer b, unsigned at) {
    const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, AUX);
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ unsigned buffer_read4(Buffer b, unsigned at) { return (unsigned)__builtin_amdgcn_raw_buffer_load_b32(b, (int)at, 0, 0); }
__device__ __forceinline__ unsigned buffer_read2(Buffer b, unsigned at) { return (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(b, (int)at, 0, 0); }
__device__ __forceinline__ unsigned buffer_read1(Buffer b, unsigned at) { return (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(b, (int)at, 0, 0); }

}  // namespace
