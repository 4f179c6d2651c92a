// k_w4_held for fp16 activations.
#include "coral_lmhead.h"
#include "w4_kernels.h"

const void* coral_w4_held_f16(int kind, int slots, int t, int nb, bool passes, bool spread) { return w4_held<kF16>(kind, slots, t, nb, passes, spread); }
