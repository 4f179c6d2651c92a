// Which kernel of the products with 4-bit weights a call takes (kernels: w4_matvec.h).  Plain C++, so that a
// host compiler can include it too: a test lists the forms that calls of any size take from it.
#pragma once
#include <stdint.h>

namespace {

constexpr int kW4UnitCols = 128;                 // columns of a unit: four products of 32
constexpr int kW4Held = 8;                       // waves of a workgroup
constexpr int kW4RowTiles = 4, kW4RowsRows = kW4Held * kW4RowTiles * 16;      // k_w4_rows: tiles of a wave; rows of a workgroup

// What decides how many workgroups fit a compute unit: the registers that the activations take, in 16s
// (chain: fp32 ones as three products one after the other).
constexpr int w4_held_regs(bool chain, int t, int nb) { return !chain ? t * nb : nb > 1 ? 8 : 4; }
// fp32 activations are three rows of the products a token (spread), or, up to three units a wave, three
// products one after the other.
constexpr int w4_held_tokens(bool spread, int t) { return spread ? t * 16 / 3 : t * 16; }

struct W4Plan {
    int t, nb;                  // k_w4_held's parameters
    bool passes, spread;
};

// More than 16 tokens are taken 32 at a time (a workgroup for each 32): all 64 at once need fewer reads of the
// codes and four times the activations a workgroup.  Measured with 64 tokens, bf16 (us), 64, 32 and 16 at a
// time: 4096 x 4096 18, 11, 11; 16384 x 4096 30, 22, 29; 50257 x 4096 62, 58, 73; 4096 x 14336 48, 35, 32.  (What takes
// 64 at a time, and chains four units a wave, was measured before it left.)
// fp32 activations are spread over three rows of the products, five or ten tokens at a time, or taken as
// three products one after the other, 16 tokens at a time, where their parts fit the registers (up to 24
// units of columns) and more than five tokens share them.  Measured (us), chained and spread: one token, 128256 x 2048
// 44, 40; x 4096 144, 55; 4096 x 4096 12, 8; 5 tokens, 32000 x 2048 14, 18; 8 tokens, 32000 x 2048 15, 25; x 4096 46, 27;
// 7 tokens, 50257 x 2568 33, 49; 64 tokens, 32000 x 2048 45, 103.
// Registers hold eight units of 128 columns a wave for 16 rows of activations, four for 32; four of fp32
// ones (LDS for their scales).  More columns are taken in passes.
inline W4Plan w4_plan_held(int M, int K, bool f32) {
    const int units = (K + kW4UnitCols - 1) / kW4UnitCols;
    int nb = (units + kW4Held - 1) / kW4Held;
    if (f32) {
        const bool spread = M <= w4_held_tokens(true, 1) || nb > 3;
        const int t = !spread || M <= w4_held_tokens(true, 1) ? 1 : 2;
        return {t, nb > 4 || t == 2 ? 4 : nb, nb > 4, spread};
    }
    const int t = M <= 16 ? 1 : 2, most = 8 / t;
    if (nb > most) return {t, most, true, false};
    nb = nb == 5 ? 6 : nb == 7 ? 8 : nb;
    return {t, nb, false, false};
}

// k_w4_held's grid: four, two or one workgroup a compute unit, by the registers that the activations take (one token,
// 128256 rows, one, two and four (us): 1024 columns 33, 22, 20; 4096 57, 52, 54; 8192 94, 98, 105).  That is what stays
// resident but for some forms, where LDS or other registers allow fewer, and the rest loads the activations in
// a second round.  Measured (us), as it is and with as many as fit: 16 bits, two units a wave (three fit): one
// token, 128256 x 2048 29, 26; 8 tokens, 32000 x 2048, zero points 12.7, 11.0; 16 bits, 17 tokens and more, up to 1024 columns (two):
// 20 tokens, 128256 x 1024 28, 27; 32000 x 1024, e2m1 12.2, 10.1; 64 tokens, 32000 x 1024 21, 19; fp32 spread, two units (two):
// one token, 128256 x 2048 36, 32; 4 tokens, 32000 x 2048 18, 15; fp32 in passes, up to five tokens (one): 128256 x 8192
// 119, 117; 32000 x 8192, zero points, groups of 32 55, 48; fp32, four units, zero points, groups of 32 (one): 128256 x
// 4096 77, 74; 5 tokens, 32000 x 4096 29, 25.
struct W4Grid {
    int x, y;
};
inline W4Grid w4_held_grid(const W4Plan& plan, int M, int N, bool f32) {
    const int regs = w4_held_regs(f32 && !plan.spread, plan.t, plan.nb);
    const int tiles = (N - 1) / 16 + 1, groups = (M - 1) / w4_held_tokens(plan.spread, plan.t) + 1, most = 256 * (regs <= 2 ? 4 : regs <= 4 ? 2 : 1) / groups;
    return {tiles < most ? tiles : most, groups};
}

// Whether k_w4_rows is taken: for more than 32 tokens, where the rows fill its rounds of workgroups (one of 512
// rows for each of 256 compute units), which take as long as 6000 tiles of k_w4_held.  Measured with 64
// tokens, bf16 (us), held and shared: 128256 rows of 1024 columns 60, 40; 2048 78, 60; 4096 121, 106 (48 tokens 123,
// 104; e2m1, groups of 32: 133, 120); 8192 241, 205.  100000 x 2048 62, 56; x 4096 99, 95; x 14336 371, 303;
// 65536 x 2048 44, 52; x 4096 67, 90; 152064 x 1024 66, 64; x 3584 138, 166.  32 tokens, 128256 x 4096 74, 99.
inline bool w4_plan_rows(int M, int N, bool f32) {
    const int tiles = (N - 1) / 16 + 1, rounds = (N - 1) / (256 * kW4RowsRows) + 1;
    return !f32 && M > 32 && (int64_t)rounds * 6000 < tiles;
}

}  // namespace
