// Rotary positions with several axes on the heads of packed rows: pair i of a head, elements 2i and 2i + 1, turns by
// position[row][axis(i)] * frequency(i); elements behind the last pair are copied.
//
// Angles are in 64 bits up to the reduction by 2 pi: at position 2^20 an angle in 32 bits is off by 2^-4.
// Bound: HBM (8192 rows of 40 heads of 128 in bf16: 32 us, 5.2 TB/s).  A workgroup takes rows one after the other; the angles of a row are found once for all of its heads.
#include <cmath>

#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"
#include "rows8.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;

struct Angles {
    double frequency[ROPE_PAIRS];
    uint8_t axis[ROPE_PAIRS];
};

template <typename T>
__global__ void __launch_bounds__(TPB) rope_axes_k(const T *x, int64_t ldx, T *y, int64_t ldy, const int32_t *__restrict__ pos, int64_t rows, int heads, int dh,
                                                   int axes, int pairs, float sign, Angles a) {
    __shared__ float turn[2][ROPE_PAIRS];
    const int tid = threadIdx.x, per = dh / 8, chunks = heads * per;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        __syncthreads();
        if (tid < dh / 2) {
            float s = 0.f, c = 1.f;
            if (tid < pairs) {
                constexpr double TURN = 6.283185307179586476925, REST = 2.449293598294706e-16;      // 2 pi as a sum of two
                const double angle = (double)pos[row * axes + a.axis[tid]] * a.frequency[tid], n = rint(angle * (1.0 / TURN));
                sincosf((float)fma(-n, REST, fma(-n, TURN, angle)), &s, &c);
            }
            turn[0][tid] = c;
            turn[1][tid] = s * sign;
        }
        __syncthreads();
        for (int i = tid; i < chunks; i += TPB) {
            Row8<T> v;
            v.load(x + row * ldx + i * 8);
            float f[8];
            v.get(f);
            const int p = i % per * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float c = turn[0][p + j], s = turn[1][p + j], u = f[2 * j], w = f[2 * j + 1];
                if (p + j >= pairs) continue;
                f[2 * j] = u * c - w * s;
                f[2 * j + 1] = u * s + w * c;
            }
            v.set(f);
            v.put(y + row * ldy + i * 8);
        }
    }
}

}  // namespace

void rope_axes(hipStream_t s, int dtype, int64_t rows, int heads, int dh, const void *x, int64_t ldx, void *y, int64_t ldy, const int32_t *pos, int axes,
               const int32_t *sections, float theta, bool own_ladder, bool inverse) {
    Angles a = {};
    int pairs = 0;
    for (int ax = 0; ax < axes; ++ax)
        for (int j = 0; j < sections[ax]; ++j, ++pairs) {
            a.frequency[pairs] = std::pow((double)theta, own_ladder ? -(double)j / sections[ax] : -2.0 * pairs / dh);
            a.axis[pairs] = (uint8_t)ax;
        }
    const unsigned grid = (unsigned)(rows < 2048 ? rows : 2048);
    const float sign = inverse ? -1.f : 1.f;
    if (dtype == TIO_PREC_BF16) rope_axes_k<bf16_t><<<grid, TPB, 0, s>>>((const bf16_t *)x, ldx, (bf16_t *)y, ldy, pos, rows, heads, dh, axes, pairs, sign, a);
    else rope_axes_k<float><<<grid, TPB, 0, s>>>((const float *)x, ldx, (float *)y, ldy, pos, rows, heads, dh, axes, pairs, sign, a);
}

}  // namespace k
}  // namespace tio
