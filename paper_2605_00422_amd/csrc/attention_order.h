// What the kernels of many rows share: their workgroups' rows and order, and exchanges between the halves of a wavefront.
#pragma once
#include "attention.h"

namespace {

constexpr int AT_WAVES = 4;
constexpr int AT_ROWS = 32 * AT_WAVES;
constexpr int AT_MAP = 4096;                           // blocks of keys that the map of active ones covers; those behind count as active

__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Workgroups are dealt round-robin to the 8 XCDs, and units (sequence, key-value head) to workgroups, so that the rows of one unit mostly
// lie on one XCD, whose L2 then has their keys and values.  (A few units at a time instead of all: 795 -> 810 us for a prompt of 8192
// with 32 heads.)  The parts of a divided cache come one after the other, the first, which all sequences have, in front (all units
// and parts at once: 296 -> 391 us for four chunks behind caches of 900 to 7001 tokens).  With each tile the units are turned by one
// an XCD, whose shader engines are dealt workgroups in turn as well: else each of the four has a sequence for itself, and where the
// shortest is done the next workgroup still waits for its own (297 -> 358 us there).  Later tiles of rows see more keys: the longest
// first, which evens out where there are many workgroups, or, where all run at once, the first half of them from the longest down
// and the second from the shortest up, so that a compute unit gets a long one and a short one.
struct AtOrder {
    int tiles, units, fold;
};
inline AtOrder at_order_of(int tiles, int units, int splits, int per_cu) {
    return AtOrder{tiles, units, (int64_t)tiles * units * splits <= (int64_t)per_cu * bwla_device_cus()};
}
__device__ __forceinline__ void at_place(int id, const AtOrder& o, int& split, int& unit, int& tile) {
    const int size = o.units * o.tiles;
    split = id / size;
    const int at = id - split * size, k = at / o.units, half = o.tiles / 2;
    unit = (int)((unsigned)(at - k * o.units + 8 * k) % (unsigned)o.units);
    tile = o.fold && k >= o.tiles - half ? k - (o.tiles - half) : o.tiles - 1 - k;
}

}  // namespace
