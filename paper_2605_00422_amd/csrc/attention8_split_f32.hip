// att8_split_kernel for fp32 queries and outputs: two fp16 terms of each query and weight.
#include "attention8_split.h"

hipError_t bwla_launch_attention8_split_f32(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st) {
    return launch8_columns<false>(a, e, s, ws, st);
}
