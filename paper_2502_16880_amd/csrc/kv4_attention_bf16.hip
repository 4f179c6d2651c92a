// Kernels of attention over the 4-bit cache for bf16 queries.
#include "kv4_attention.h"
#include "kv4_kernels.h"

const void* coral_kv4_kernel_bf16(int head_dim, int tiles) {
    return reinterpret_cast<const void*>(head_dim == 64 ? kv4_kernel<kBF16, 64>(tiles) : head_dim == 128 ? kv4_kernel<kBF16, 128>(tiles) : kv4_kernel<kBF16, 256>(tiles));
}
const void* coral_kv4_join_bf16(int head_dim, int tiles, bool wave_a_row) {
    return reinterpret_cast<const void*>(head_dim == 64 ? kv4_join<kBF16, 64>(tiles, wave_a_row) : head_dim == 128 ? kv4_join<kBF16, 128>(tiles, wave_a_row) : kv4_join<kBF16, 256>(tiles, wave_a_row));
}
