// How a call of attention over the 4-bit cache is cut into workgroups, in plain C++.
#pragma once
#include <stddef.h>
#include <stdint.h>

struct Kv4Plan {
    int tiles;         // tiles of 16 rows (a row: one token, one query head) that a workgroup takes
    int row_blocks;    // workgroups beside each other for one sequence's rows of one head of keys
    int splits;        // workgroups along a sequence's tokens, at most
};

constexpr int kKv4Step = 128;           // tokens that a workgroup's four waves take together: 32 each
constexpr int kKv4MostRows = 64;        // rows (tokens) of a sequence in one call

// Query operands and sums of a wave's tiles stay in registers: with `terms` bf16 values for a query value
// (1 for bf16, 2 for fp16, 3 for fp32) this many tiles fit.
inline int kv4_most_tiles(int head_dim, int terms) {
    const int n = 512 / (head_dim * terms);
    return n >= 4 ? 4 : n >= 2 ? 2 : 1;
}

inline Kv4Plan kv4_plan(int S, int max_rows, int max_length, int q_heads, int kv_heads, int head_dim, int terms) {
    Kv4Plan p;
    const int tiles = (max_rows * (q_heads / kv_heads) + 15) / 16, most = kv4_most_tiles(head_dim, terms);
    p.tiles = 1;
    while (p.tiles < tiles && p.tiles < most) p.tiles *= 2;
    p.row_blocks = (tiles + p.tiles - 1) / p.tiles;
    const int64_t steps = ((int64_t)max_length + kKv4Step - 1) / kKv4Step, items = (int64_t)S * kv_heads * p.row_blocks;
    int64_t n = (2048 + items - 1) / items;
    if (n > steps) n = steps;
    if (n > 256) n = 256;
    p.splits = n < 1 ? 1 : (int)n;
    return p;
}

// One split's share of a row: head_dim sums, the largest score and the sum of exponentials, in fp32.
inline size_t kv4_workspace(const Kv4Plan& p, int S, int kv_heads, int head_dim) {
    if (p.splits < 2) return 0;
    return (size_t)S * kv_heads * p.row_blocks * p.splits * (16 * p.tiles) * ((size_t)head_dim + 2) * sizeof(float);
}
