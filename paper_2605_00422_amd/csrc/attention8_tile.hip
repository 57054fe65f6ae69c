// att8_tile_kernel for bf16 queries and outputs, and the choice by type.  (fp32: attention8_tile_f32.hip)
#include "attention8_tile.h"

hipError_t bwla_launch_attention8_tile(const AttArgs& a, const Att8& e, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    const hipError_t r = dtype == BWLA_X_F32 ? bwla_launch_attention8_tile_f32(a, e, s, ws, st) : at8_launch_columns<1>(a, e, s, ws, st);
    return r != hipSuccess || s.splits == 1 ? r : bwla_launch_attention_join(a, s, dtype, ws, st);
}
