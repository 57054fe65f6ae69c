// att8_tile_kernel for fp32 queries and outputs, two fp16 terms of each query and weight, and integers.
#include "attention8_tile.h"

hipError_t bwla_launch_attention8_tile_f32(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st) {
    return at8_launch_columns<2, true>(a, e, s, ws, st);
}
