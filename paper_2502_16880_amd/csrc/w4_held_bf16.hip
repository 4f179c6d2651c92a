// k_w4_held for bf16 activations.
#include "coral_lmhead.h"
#include "w4_kernels.h"

const void* coral_w4_held_bf16(int kind, int slots, int t, int nb, bool passes, bool spread) { return w4_held<kBF16>(kind, slots, t, nb, passes, spread); }
