// Kernels of attention over the 4-bit cache for f16 queries.
#include "kv4_attention.h"
#include "kv4_kernels.h"

const void* coral_kv4_kernel_f16(int head_dim, int tiles) {
    return reinterpret_cast<const void*>(head_dim == 64 ? kv4_kernel<kF16, 64>(tiles) : head_dim == 128 ? kv4_kernel<kF16, 128>(tiles) : kv4_kernel<kF16, 256>(tiles));
}
const void* coral_kv4_join_f16(int head_dim, int tiles, bool wave_a_row) {
    return reinterpret_cast<const void*>(head_dim == 64 ? kv4_join<kF16, 64>(tiles, wave_a_row) : head_dim == 128 ? kv4_join<kF16, 128>(tiles, wave_a_row) : kv4_join<kF16, 256>(tiles, wave_a_row));
}
