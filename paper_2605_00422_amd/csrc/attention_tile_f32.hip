// att_tile_kernel for fp32
#include "attention_tile.h"

hipError_t bwla_launch_attention_tile_f32(const AttArgs& a, const AttSplit& s, void* ws, hipStream_t st) {
    if (a.d <= 64) return at_launch<false, 64>(a, s, ws, st);
    if (a.d <= 128) return at_launch<false, 128>(a, s, ws, st);
    return at_launch<false, 256>(a, s, ws, st);
}
