// How a call of attention over the 4-bit cache is cut into workgroups, in plain C++.
#pragma once
#include <stddef.h>
#include <stdint.h>

struct Kv4Plan {
    int tiles;         // tiles of 16 rows (a row: one token, one query head) that a workgroup takes together: 1 or 2
    int row_blocks;    // so many times that, at most, for one sequence's rows of one head of keys
    int workgroups;    // among which all sequences' steps are shared equally, or
    bool apart;        // one workgroup for each sequence, head of keys and block of rows
    bool join_inside;  // an item's last workgroup joins its parts; or a kernel of its own does, many workgroups at once,
    bool wave_a_row;   // with a wave a row, or four
};

constexpr size_t kKv4Control = 16896;   // bytes of the workspace's control words and the words behind them
constexpr int kKv4Step = 128;           // tokens that a workgroup's four waves take together: 32 each
constexpr int kKv4MostRows = 64;        // rows (tokens) of a sequence in one call
constexpr int kKv4Units = 256;          // compute units of the card
constexpr int kKv4Apart = 256;          // sequences beyond which they are not shared out (each workgroup sums them all up)
constexpr int kKv4JoinRows = 8;         // rows and parts of an item, at most, that one workgroup joins as fast as another
constexpr int kKv4JoinParts = 40;       // kernel begins: two rows a wave (D = 256: half as many; eight tokens' 34 parts 34 us, apart 22).  An
                                        // item that has more than sequences have on average is joined in two steps
// Parts of an item, at most, that a wave joins by itself: 60 nodes over 4111 tokens (11 parts) 27.8 us with four waves a row, 25.9 with
// one; 32 sequences' 16 rows (2 parts) 58.6 and 45.2; one token of 32768 (98 parts) 20.5 and 24.6, eight of 131072 (66) 48.8 and 51.2.
constexpr int kKv4JoinWave = 16;

// Query operands and sums of a wave's tiles stay in registers: with `terms` 16-bit values for a query value
// (3 for fp32, else 1) this many tiles fit.
constexpr int kv4_most_tiles(int head_dim, int terms) { return head_dim * terms <= 128 ? 2 : 1; }
// Workgroups that a compute unit holds: waves on a SIMD that registers are kept for (sums and query operands of the
// tiles, two steps' codes).
constexpr int kv4_occupancy(int head_dim, int tiles, int terms) {
    return head_dim == 256 ? 1 : tiles == 2 || head_dim * (terms + 2) > 384 ? 2 : 3;
}

inline Kv4Plan kv4_plan(int S, int max_rows, int max_length, int q_heads, int kv_heads, int head_dim, int terms) {
    Kv4Plan p;
    const int tiles = (max_rows * (q_heads / kv_heads) + 15) / 16, most = kv4_most_tiles(head_dim, terms);
    p.tiles = tiles < most ? tiles : most;
    p.row_blocks = (tiles + p.tiles - 1) / p.tiles;
    const int64_t steps = max_length > kKv4Step ? ((int64_t)max_length + kKv4Step - 1) / kKv4Step : 1;
    const int64_t all = (int64_t)S * kv_heads * p.row_blocks * steps, places = kKv4Units * kv4_occupancy(head_dim, p.tiles, terms);
    p.workgroups = (int)(all < places ? all : places);
    p.apart = S > kKv4Apart;
    const int64_t parts = p.workgroups / ((int64_t)S * kv_heads * p.row_blocks) + 2, rows = max_rows * (q_heads / kv_heads);
    p.join_inside = rows <= kKv4JoinRows && parts <= kKv4JoinParts && parts * head_dim <= kKv4JoinParts * 128;
    p.wave_a_row = parts <= kKv4JoinWave;
    return p;
}

// A workgroup's share begins and ends inside an item (a sequence's block of rows for a head of keys) in two places at
// most: two blocks of sums of head_dim values, the largest score and the sum of exponentials for each row, in fp32,
// behind the control words.
inline size_t kv4_workspace(const Kv4Plan& p, int head_dim) {
    if (p.apart || p.workgroups < 2) return 0;
    return kKv4Control + (size_t)p.workgroups * 2 * (16 * p.tiles) * ((size_t)head_dim + 2) * sizeof(float);
}
