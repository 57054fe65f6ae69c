// att_tile_kernel for bf16, and the choice by type and columns.  (fp32: attention_tile_f32.hip)
#include <algorithm>
#include "attention_tile.h"

// Whether the cached tokens are dealt out over several workgroups, whose parts are then added up, and how many go to each.  The GPU has
// places for 512 workgroups (of up to 128 columns); "->": without parts, with them.
// - Rows that make up to a third of these: so many parts that all places are taken.  128 tokens behind 8192, 8 key-value heads: 229 -> 45
//   us; prompts of 768, 1024, 1536 and 2048 tokens with 8 heads 27 -> 24, 34 -> 23, 47 -> 33, 61 -> 40.  (Prompts of 512 get two
//   parts: 20 -> 20 us with 8 and 16 heads, 20 -> 24 with 32.)
// - Up to half, and the cache is long: 192 workgroups of 3000 tokens 88 -> 58 us, 256 of 4096 118 -> 96, 256 of 2048 62 -> 58.  Shorter
//   ones can lose: 256 of 1024 35 -> 40, 192 of 768 27 -> 32 (though 192 of 1536 48 -> 40).
// - More: of one prompt the parts cost as much as they bring (384 workgroups: 401 against 399 us of 8192 tokens, 58 against 60 of 1500).
//   Chunks of several sequences may differ in length, and the longest one's workgroups would be the last for long, so caches are cut in
//   four, in parts of 2048 at least.  2 to 8 chunks, 320 to 448 workgroups: caches of an eighth to the whole of 16384 tokens 595 -> 358 to
//   460 us, of a half on 559 to 599 -> 453 to 518, all alike 595 to 633 -> 501 to 619; of 8192 271 to 300 -> 186 to 245, 282 to 303
//   -> 241 to 272, 302 to 311 -> 259 to 323.  The lengths are not known here, and it does not pay for all: of 4000 alike 147 to 153 -> 149
//   to 170, and of 512 workgroups with caches of 8192 280 -> 275 from an eighth on, but 341 -> 390 alike.
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
