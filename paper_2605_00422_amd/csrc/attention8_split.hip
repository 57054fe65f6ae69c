// att8_split_kernel for bf16 queries and outputs.  (fp32: attention8_split_f32.hip)
#include "attention8_split.h"

hipError_t bwla_launch_attention8_split(const AttArgs& a, const Att8& e, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    return dtype == BWLA_X_F32 ? bwla_launch_attention8_split_f32(a, e, s, ws, st) : launch8_columns<true>(a, e, s, ws, st);
}
