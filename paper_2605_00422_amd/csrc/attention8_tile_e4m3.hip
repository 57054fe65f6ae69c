// att8_tile_kernel for bf16 queries and outputs and e4m3 codes.
#include "attention8_tile.h"

hipError_t bwla_launch_attention8_tile_e4m3(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st) {
    return at8_launch_columns<1, false>(a, e, s, ws, st);
}
