// Random bits from a counter: Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), and
// the masks of dropout made from them.
//
// Element (row, col) of a matrix with `groups` = ceil(cols / 8) groups of eight neighbours to a row has half-word col % 8 (the low half of a word
// first) of the four words at counter (row groups + col / 8, offset), two words each, under the key `seed`.  It is dropped where its 16 bits are
// below `limit`, and multiplied by 65536 / (65536 - limit) elsewhere.  The mask depends on nothing else, so that the backward pass draws it again.
#pragma once
#include "device_common.h"
#include "kernels.h"

namespace tio {
namespace k {

// The ten rounds; each is two 32 x 32 -> 64 bit products.
__device__ __forceinline__ uint4 philox(uint64_t index, const Dropout &d) {
    uint32_t c0 = (uint32_t)index, c1 = (uint32_t)(index >> 32), c2 = d.offset0, c3 = d.offset1, k0 = d.key0, k1 = d.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96);         // exclusive or of three
        c1 = (uint32_t)b;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// the random bits of eight neighbours, sixteen each
struct Mask8 {
    uint4 w;
    __device__ __forceinline__ void draw(uint64_t row, uint32_t groups, uint32_t group, const Dropout &d) { w = philox(row * groups + group, d); }
    // what the compiler has found from it it finds again, rather than keep it in registers
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w)); }
    __device__ __forceinline__ bool kept(int j, const Dropout &d) const {
        const uint32_t v = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
        return (j & 1 ? v >> 16 : v & 0xffffu) >= d.limit;
    }
};

}  // namespace k
}  // namespace tio
