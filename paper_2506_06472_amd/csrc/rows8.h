// Eight neighbours of a row: 16 bytes of bf16, or 32 of fp32.
#pragma once
#include "device_common.h"

namespace tio {
namespace k {

template <typename T> struct Row8;
template <> struct Row8<bf16_t> {
    Vec16<bf16_t> v;
    __device__ __forceinline__ void load(const bf16_t *p) { v.load(p); }
    __device__ __forceinline__ void store(bf16_t *p) const { v.store(p); }
    __device__ __forceinline__ void put(bf16_t *p) const { __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, v.raw), reinterpret_cast<tio_u32x4 *>(p)); }
    __device__ __forceinline__ void get(float *f) const { v.get(f); }
    __device__ __forceinline__ void set(const float *f) { v.set(f); }
    // what the compiler has found from them it finds again, rather than keep it in registers
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(v.raw.x), "+v"(v.raw.y), "+v"(v.raw.z), "+v"(v.raw.w)); }
};
template <> struct Row8<float> {
    Vec16<float> lo, hi;
    __device__ __forceinline__ void load(const float *p) { lo.load(p); hi.load(p + 4); }
    __device__ __forceinline__ void store(float *p) const { lo.store(p); hi.store(p + 4); }
    __device__ __forceinline__ void put(float *p) const {                    // past the caches
        __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, lo.raw), reinterpret_cast<tio_u32x4 *>(p));
        __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, hi.raw), reinterpret_cast<tio_u32x4 *>(p + 4));
    }
    __device__ __forceinline__ void get(float *f) const { lo.get(f); hi.get(f + 4); }
    __device__ __forceinline__ void set(const float *f) { lo.set(f); hi.set(f + 4); }
    __device__ __forceinline__ void forget() {}
};
// through a buffer descriptor over a row: columns past its end read as zeros, and are not written; stores go past the caches
__device__ __forceinline__ void row_load(Row8<bf16_t> &v, __amdgpu_buffer_rsrc_t row, uint32_t col) { buffer_load16(v.v, row, col * 2); }
__device__ __forceinline__ void row_load(Row8<float> &v, __amdgpu_buffer_rsrc_t row, uint32_t col) {
    buffer_load16(v.lo, row, col * 4);
    buffer_load16(v.hi, row, col * 4 + 16);
}
constexpr int BUFFER_NT = 2;
__device__ __forceinline__ void row_put(const Row8<bf16_t> &v, __amdgpu_buffer_rsrc_t row, uint32_t col) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(tio_u32x4, v.v.raw), row, (int)(col * 2), 0, BUFFER_NT);
}
__device__ __forceinline__ void row_put(const Row8<float> &v, __amdgpu_buffer_rsrc_t row, uint32_t col) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(tio_u32x4, v.lo.raw), row, (int)(col * 4), 0, BUFFER_NT);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(tio_u32x4, v.hi.raw), row, (int)(col * 4 + 16), 0, BUFFER_NT);
}
// columns from n on become zero
__device__ __forceinline__ void cut8(float *f, int n) {
    if (n >= 8) return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j >= n) f[j] = 0.f;
}

}  // namespace k
}  // namespace tio
