// Host side of the products with 4-bit weights: which kernel a call takes (w4_matvec.hip), and the
// kernels' instantiations by storage type (w4_held_{bf16,f16,f32}.hip, w4_rows_{bf16,f16}.hip, compiled side
// by side).
#pragma once
#include "w4_matvec.h"
#include <type_traits>

namespace {
typedef void (*w4_fn)(W4Params);
}

// k_w4_held for a unit of so many slots, t tiles of 16 tokens and nb units a wave (in passes: the most there are).
__attribute__((visibility("hidden"))) const void* coral_w4_held_bf16(int kind, int slots, int t, int nb, bool passes);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f16(int kind, int slots, int t, int nb, bool passes);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f32(int kind, int slots, int t, int nb, bool passes);

// k_w4_rows for r tiles of 16 rows a wave.
__attribute__((visibility("hidden"))) const void* coral_w4_rows_bf16(int kind, int slots, int r);
__attribute__((visibility("hidden"))) const void* coral_w4_rows_f16(int kind, int slots, int r);

namespace {

template <int DT, int KIND, int SLOTS>
w4_fn w4_pick_rows(int r) {
    return r == 2 ? k_w4_rows<DT, KIND, SLOTS, 2> : r == 3 ? k_w4_rows<DT, KIND, SLOTS, 3> : k_w4_rows<DT, KIND, SLOTS, 4>;
}
template <int DT>
const void* w4_rows(int kind, int slots, int r) {
    const auto pick = [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        return slots == 4 ? w4_pick_rows<DT, KIND, 4>(r) : slots == 2 ? w4_pick_rows<DT, KIND, 2>(r) : w4_pick_rows<DT, KIND, 1>(r);
    };
    return reinterpret_cast<const void*>(kind == kW4E2M1 ? pick(std::integral_constant<int, kW4E2M1>())
                                         : kind == kW4Sym ? pick(std::integral_constant<int, kW4Sym>()) : pick(std::integral_constant<int, kW4Zero>()));
}

template <int DT, int KIND, int SLOTS>
w4_fn w4_pick_held(int t, int nb, bool passes) {
    constexpr bool k16 = DT != kF32;             // fp32 activations take twice the registers
    if (passes) {                                // as many units as the registers hold
        constexpr int NB = k16 ? 8 : 4;
        return t == 1 ? k_w4_held<DT, KIND, SLOTS, 1, NB, true> : t == 2 ? k_w4_held<DT, KIND, SLOTS, 2, NB / 2, true> : k_w4_held<DT, KIND, SLOTS, 4, NB / 4, true>;
    }
    switch (t * 16 + nb) {
        case 17: return k_w4_held<DT, KIND, SLOTS, 1, 1>;
        case 18: return k_w4_held<DT, KIND, SLOTS, 1, 2>;
        case 19: return k_w4_held<DT, KIND, SLOTS, 1, 3>;
        case 20: return k_w4_held<DT, KIND, SLOTS, 1, 4>;
        case 33: return k_w4_held<DT, KIND, SLOTS, 2, 1>;
        case 34: return k_w4_held<DT, KIND, SLOTS, 2, 2>;
        case 65: return k_w4_held<DT, KIND, SLOTS, 4, 1>;
    }
    if constexpr (k16) {
        switch (t * 16 + nb) {
            case 22: return k_w4_held<DT, KIND, SLOTS, 1, 6>;
            case 24: return k_w4_held<DT, KIND, SLOTS, 1, 8>;
            case 36: return k_w4_held<DT, KIND, SLOTS, 2, 4>;
            case 66: return k_w4_held<DT, KIND, SLOTS, 4, 2>;
        }
    }
    return nullptr;
}

template <int DT>
const void* w4_held(int kind, int slots, int t, int nb, bool passes) {
    const auto pick = [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        return slots == 4 ? w4_pick_held<DT, KIND, 4>(t, nb, passes) : slots == 2 ? w4_pick_held<DT, KIND, 2>(t, nb, passes) : w4_pick_held<DT, KIND, 1>(t, nb, passes);
    };
    return reinterpret_cast<const void*>(kind == kW4E2M1 ? pick(std::integral_constant<int, kW4E2M1>())
                                         : kind == kW4Sym ? pick(std::integral_constant<int, kW4Sym>()) : pick(std::integral_constant<int, kW4Zero>()));
}

}  // namespace
