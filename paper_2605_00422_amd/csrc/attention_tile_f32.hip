// att_tile_kernel for fp32
#include "attention_tile.h"

hipError_t bwla_launch_attention_tile_f32(const AttArgs& a, hipStream_t st) {
    if (a.d <= 64) return at_launch<false, 64>(a, st);
    if (a.d <= 128) return at_launch<false, 128>(a, st);
    return at_launch<false, 256>(a, st);
}
