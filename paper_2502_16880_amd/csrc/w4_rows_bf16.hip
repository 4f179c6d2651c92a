// k_w4_rows for bf16 activations.
#include "coral_lmhead.h"
#include "w4_kernels.h"

const void* coral_w4_rows_bf16(int kind, int slots) { return w4_rows<kBF16>(kind, slots); }
