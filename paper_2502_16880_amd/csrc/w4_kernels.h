// Host side of the products with 4-bit weights: which kernel a call takes (w4_matvec.hip), and the
// kernels' instantiations by storage type (w4_held_{bf16,f16,f32}.hip, w4_rows_{bf16,f16}.hip, compiled side
// by side).
#pragma once
#include "w4_matvec.h"

namespace {
typedef void (*w4_fn)(W4Params);
}

// k_w4_held for t tiles of 16 tokens and nb units a wave (in passes: the most there are).
__attribute__((visibility("hidden"))) const void* coral_w4_held_bf16(int kind, bool fine, int t, int nb, bool passes);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f16(int kind, bool fine, int t, int nb, bool passes);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f32(int kind, bool fine, int t, int nb, bool passes);

// k_w4_rows for r tiles of 16 rows a wave.
__attribute__((visibility("hidden"))) const void* coral_w4_rows_bf16(int kind, bool fine, int r);
__attribute__((visibility("hidden"))) const void* coral_w4_rows_f16(int kind, bool fine, int r);

namespace {

template <int DT, int KIND, bool FINE>
w4_fn w4_pick_rows(int r) {
    return r == 2 ? k_w4_rows<DT, KIND, FINE, 2> : r == 3 ? k_w4_rows<DT, KIND, FINE, 3> : k_w4_rows<DT, KIND, FINE, 4>;
}
template <int DT>
const void* w4_rows(int kind, bool fine, int r) {
    w4_fn fn = nullptr;
    if (fine) fn = kind == kW4E2M1 ? w4_pick_rows<DT, kW4E2M1, true>(r) : kind == kW4Sym ? w4_pick_rows<DT, kW4Sym, true>(r) : w4_pick_rows<DT, kW4Zero, true>(r);
    else fn = kind == kW4E2M1 ? w4_pick_rows<DT, kW4E2M1, false>(r) : kind == kW4Sym ? w4_pick_rows<DT, kW4Sym, false>(r) : w4_pick_rows<DT, kW4Zero, false>(r);
    return reinterpret_cast<const void*>(fn);
}

template <int DT, int KIND, bool FINE>
w4_fn w4_pick_held(int t, int nb, bool passes) {
    constexpr bool k16 = DT != kF32;             // fp32 activations take twice the registers
    if (passes) {                                // as many units as the registers hold
        constexpr int NB = k16 ? 8 : 4;
        return t == 1 ? k_w4_held<DT, KIND, FINE, 1, NB, true> : t == 2 ? k_w4_held<DT, KIND, FINE, 2, NB / 2, true> : k_w4_held<DT, KIND, FINE, 4, NB / 4, true>;
    }
    switch (t * 16 + nb) {
        case 17: return k_w4_held<DT, KIND, FINE, 1, 1>;
        case 18: return k_w4_held<DT, KIND, FINE, 1, 2>;
        case 19: return k_w4_held<DT, KIND, FINE, 1, 3>;
        case 20: return k_w4_held<DT, KIND, FINE, 1, 4>;
        case 33: return k_w4_held<DT, KIND, FINE, 2, 1>;
        case 34: return k_w4_held<DT, KIND, FINE, 2, 2>;
        case 65: return k_w4_held<DT, KIND, FINE, 4, 1>;
    }
    if constexpr (k16) {
        switch (t * 16 + nb) {
            case 22: return k_w4_held<DT, KIND, FINE, 1, 6>;
            case 24: return k_w4_held<DT, KIND, FINE, 1, 8>;
            case 36: return k_w4_held<DT, KIND, FINE, 2, 4>;
            case 66: return k_w4_held<DT, KIND, FINE, 4, 2>;
        }
    }
    return nullptr;
}

template <int DT>
const void* w4_held(int kind, bool fine, int t, int nb, bool passes) {
    w4_fn fn = nullptr;
    if (fine) fn = kind == kW4E2M1 ? w4_pick_held<DT, kW4E2M1, true>(t, nb, passes) : kind == kW4Sym ? w4_pick_held<DT, kW4Sym, true>(t, nb, passes) : w4_pick_held<DT, kW4Zero, true>(t, nb, passes);
    else fn = kind == kW4E2M1 ? w4_pick_held<DT, kW4E2M1, false>(t, nb, passes) : kind == kW4Sym ? w4_pick_held<DT, kW4Sym, false>(t, nb, passes) : w4_pick_held<DT, kW4Zero, false>(t, nb, passes);
    return reinterpret_cast<const void*>(fn);
}

}  // namespace
