// att_tile_kernel for bf16, and the choice by type and columns.  (fp32: attention_tile_f32.hip)
#include <algorithm>
#include "attention_tile.h"

// Whether the cached tokens are dealt out over several workgroups, whose parts are then added up, and how many go to each:
// so many that there are workgroups for the whole GPU, where the rows alone make fewer than a third of them (128 tokens behind 8192,
// 8 key-value heads: 229 -> 45 us; a prompt of 1024 of 16 heads 36 -> 29 us), or half of them and the cache is long (256 workgroups:
// 67 -> 62 us of 2048 tokens, but 55 -> 56 us of 1500).  Of more workgroups the parts cost as much as they bring (384 workgroups: 401
// against 399 us of 8192 tokens, 58 against 60 of 1500), but for chunks of several sequences, whose lengths differ: the longest one's
// would be the last for long (four of 900 to 7001 tokens, 448 workgroups: 275 -> 235 us, though 366 -> 399 us if all have 8192).
AttSplit bwla_att_tile_split(const AttArgs& a) {
    AttSplit s = {};
    s.rows = a.max_new * a.group;
    s.row_tiles = (s.rows + 15) / 16;
    s.chunk = INT32_MAX;
    const int64_t room = (int64_t)bwla_device_cus() * (a.d > 128 ? 1 : 2);
    const int64_t groups = (int64_t)((s.rows + AT_ROWS - 1) / AT_ROWS) * a.seqs * a.hkv;
    int64_t chunk = 0;
    if (groups * 3 <= room || (groups * 2 <= room && a.max_len >= 2048)) chunk = std::max(groups * a.max_len / room, (int64_t)256);
    else if (groups <= room && a.seqs > 1 && a.max_new <= a.max_len / 2) chunk = std::max(a.max_len / 4, 2048);
    chunk = (chunk + 63) / 64 * 64;
    if (chunk > 0 && chunk < a.max_len) s.chunk = (int)chunk;
    s.splits = s.chunk == INT32_MAX ? 1 : (a.max_len + s.chunk - 1) / s.chunk;
    const int dp = a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256;
    const int64_t parts = s.splits > 1 ? (int64_t)a.seqs * a.hkv * s.row_tiles * s.splits * 16 : 0;
    s.part_bytes = (size_t)parts * dp * 4;
    s.stat_bytes = (size_t)bwla_align256((uint64_t)parts * 16);
    return s;
}

hipError_t bwla_launch_attention_tile(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    hipError_t e;
    if (dtype == BWLA_X_F32) e = bwla_launch_attention_tile_f32(a, s, ws, st);
    else if (a.d <= 64) e = at_launch<true, 64>(a, s, ws, st);
    else if (a.d <= 128) e = at_launch<true, 128>(a, s, ws, st);
    else e = at_launch<true, 256>(a, s, ws, st);
    return e != hipSuccess || s.splits == 1 ? e : bwla_launch_attention_join(a, s, dtype, ws, st);
}
