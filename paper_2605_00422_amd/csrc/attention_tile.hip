// att_tile_kernel for bf16, and the choice by type and columns.  (fp32: attention_tile_f32.hip)
#include "attention_tile.h"

hipError_t bwla_launch_attention_tile(const AttArgs& a, int dtype, hipStream_t st) {
    if (dtype == BWLA_X_F32) return bwla_launch_attention_tile_f32(a, st);
    if (a.d <= 64) return at_launch<true, 64>(a, st);
    if (a.d <= 128) return at_launch<true, 128>(a, st);
    return at_launch<true, 256>(a, st);
}
