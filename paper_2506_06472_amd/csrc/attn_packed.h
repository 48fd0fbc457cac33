// Where the workgroups of attention over a packed batch find their rows.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "packing.h"

namespace tio {
namespace k {

// The sequences' rows and how their items and heads are dealt to workgroups.  `heads` heads (of keys, or of queries) are taken by every item.
// Workgroups go to the eight XCDs in turn, each of which has an L2 of its own: with g the greatest common divisor of heads and 8, an XCD
// has the heads of one remainder by g and every 8/g-th item, so that the blocks of a head's sequence meet in as few L2s as the heads allow.
// An XCD's workgroups are in the order of their items, the longest first, all its heads of an item one behind the other.
struct PackedPlaces {
    const int32_t *items;
    int32_t n, words, rows, heads, g;
    // head and item of workgroup `block`; false: none.  The item's first words are checked against the batch: nothing is read or
    // written outside it, whatever the list holds.
    __device__ __forceinline__ bool find(unsigned block, int &head, const int32_t *&item) const {
        const unsigned xcd = block & 7, slot = block >> 3, of_xcd = (unsigned)(heads / g);
        const unsigned i = slot / of_xcd * (8 / g) + xcd / g;
        if (i >= (unsigned)n) return false;
        head = (int)(slot % of_xcd * g + xcd % g);
        item = items + (int64_t)i * words;
        const int first = item[0], len = item[1];
        return first >= 0 && len > 0 && first <= rows - len;
    }
    unsigned grid() const { return (unsigned)((n + 8 / g - 1) / (8 / g) * (heads / g) * 8); }
};
inline PackedPlaces packed_places(const Packing &p, const void *device, const ItemList &list, int words, int heads) {
    int g = 1;
    while (g < 8 && heads % (2 * g) == 0) g *= 2;
    return PackedPlaces{(const int32_t *)device + list.at, list.n, words, p.rows, heads, g};
}

}  // namespace k
}  // namespace tio
