// att8_tile_kernel for bf16 queries and outputs and integers, and the choice by types.  (The others: attention8_tile_e4m3.hip, _f32.hip, _f32_e4m3.hip)
#include "attention8_tile.h"

hipError_t bwla_launch_attention8_tile(const AttArgs& a, const Att8& e, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    const bool ints = e.code == BWLA_CODE_I8;
    hipError_t r;
    if (dtype == BWLA_X_F32) r = ints ? bwla_launch_attention8_tile_f32(a, e, s, ws, st) : bwla_launch_attention8_tile_f32_e4m3(a, e, s, ws, st);
    else r = ints ? at8_launch_columns<1, true>(a, e, s, ws, st) : bwla_launch_attention8_tile_e4m3(a, e, s, ws, st);
    return r != hipSuccess || s.splits == 1 ? r : bwla_launch_attention_join(a, s, dtype, ws, st);
}
