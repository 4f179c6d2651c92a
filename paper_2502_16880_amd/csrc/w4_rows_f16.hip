// k_w4_rows for fp16 activations.
#include "coral_lmhead.h"
#include "w4_kernels.h"

const void* coral_w4_rows_f16(int kind, int slots) { return w4_rows<kF16>(kind, slots); }
