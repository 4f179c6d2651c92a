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
__attribute__((visibility("hidden"))) const void* coral_w4_held_bf16(int kind, int slots, int t, int nb, bool passes, bool spread);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f16(int kind, int slots, int t, int nb, bool passes, bool spread);
__attribute__((visibility("hidden"))) const void* coral_w4_held_f32(int kind, int slots, int t, int nb, bool passes, bool spread);

// k_w4_rows.
__attribute__((visibility("hidden"))) const void* coral_w4_rows_bf16(int kind, int slots);
__attribute__((visibility("hidden"))) const void* coral_w4_rows_f16(int kind, int slots);

namespace {

template <int DT>
const void* w4_rows(int kind, int slots) {
    const auto pick = [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        return slots == 4 ? k_w4_rows<DT, KIND, 4> : slots == 2 ? k_w4_rows<DT, KIND, 2> : k_w4_rows<DT, KIND, 1>;
    };
    return reinterpret_cast<const void*>(kind == kW4E2M1 ? pick(std::integral_constant<int, kW4E2M1>())
                                         : kind == kW4Sym ? pick(std::integral_constant<int, kW4Sym>()) : pick(std::integral_constant<int, kW4Zero>()));
}

template <int DT, int KIND, int SLOTS>
w4_fn w4_pick_held(int t, int nb, bool passes, bool spread) {
    if constexpr (DT == kF32) {
        if (!spread) return nb == 1 ? k_w4_held<DT, KIND, SLOTS, 1, 1> : nb == 2 ? k_w4_held<DT, KIND, SLOTS, 1, 2> : k_w4_held<DT, KIND, SLOTS, 1, 3>;
        if (passes) return t == 1 ? k_w4_held<DT, KIND, SLOTS, 1, 4, true, true> : k_w4_held<DT, KIND, SLOTS, 2, 4, true, true>;
        if (t == 2) return k_w4_held<DT, KIND, SLOTS, 2, 4, false, true>;
        return nb == 1 ? k_w4_held<DT, KIND, SLOTS, 1, 1, false, true> : nb == 2 ? k_w4_held<DT, KIND, SLOTS, 1, 2, false, true>
               : nb == 3 ? k_w4_held<DT, KIND, SLOTS, 1, 3, false, true> : k_w4_held<DT, KIND, SLOTS, 1, 4, false, true>;
    } else {
        if (passes) return t == 1 ? k_w4_held<DT, KIND, SLOTS, 1, 8, true> : k_w4_held<DT, KIND, SLOTS, 2, 4, true>;
        if (t == 2) return nb == 1 ? k_w4_held<DT, KIND, SLOTS, 2, 1> : nb == 2 ? k_w4_held<DT, KIND, SLOTS, 2, 2> : nb == 3 ? k_w4_held<DT, KIND, SLOTS, 2, 3> : k_w4_held<DT, KIND, SLOTS, 2, 4>;
        switch (nb) {
            case 1: return k_w4_held<DT, KIND, SLOTS, 1, 1>;
            case 2: return k_w4_held<DT, KIND, SLOTS, 1, 2>;
            case 3: return k_w4_held<DT, KIND, SLOTS, 1, 3>;
            case 4: return k_w4_held<DT, KIND, SLOTS, 1, 4>;
            case 6: return k_w4_held<DT, KIND, SLOTS, 1, 6>;
            default: return k_w4_held<DT, KIND, SLOTS, 1, 8>;
        }
    }
}

template <int DT>
const void* w4_held(int kind, int slots, int t, int nb, bool passes, bool spread) {
    const auto pick = [&](auto k) {
        constexpr int KIND = decltype(k)::value;
        return slots == 4 ? w4_pick_held<DT, KIND, 4>(t, nb, passes, spread) : slots == 2 ? w4_pick_held<DT, KIND, 2>(t, nb, passes, spread) : w4_pick_held<DT, KIND, 1>(t, nb, passes, spread);
    };
    return reinterpret_cast<const void*>(kind == kW4E2M1 ? pick(std::integral_constant<int, kW4E2M1>())
                                         : kind == kW4Sym ? pick(std::integral_constant<int, kW4Sym>()) : pick(std::integral_constant<int, kW4Zero>()));
}

}  // namespace
