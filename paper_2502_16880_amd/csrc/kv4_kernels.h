// Kernels of attention over the 4-bit cache by storage type: one translation unit each, so that they compile
// side by side.
#pragma once

__attribute__((visibility("hidden"))) const void* coral_kv4_kernel_bf16(int head_dim, int tiles);
__attribute__((visibility("hidden"))) const void* coral_kv4_kernel_f16(int head_dim, int tiles);
__attribute__((visibility("hidden"))) const void* coral_kv4_kernel_f32(int head_dim, int tiles);
__attribute__((visibility("hidden"))) const void* coral_kv4_join_bf16(int head_dim, int tiles, bool wave_a_row);
__attribute__((visibility("hidden"))) const void* coral_kv4_join_f16(int head_dim, int tiles, bool wave_a_row);
__attribute__((visibility("hidden"))) const void* coral_kv4_join_f32(int head_dim, int tiles, bool wave_a_row);
