// Dropout from a counter (philox.h), with or without the residual that it is added to; the mask is not stored anywhere.
//
// Bound: HBM, with the generator's products close behind (8192 x 4096 in bf16: 20 us, 6.6 TB/s, partly from the memory-side cache).  Eight elements, whose
// bits are one call of the generator, to a thread.
#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"
#include "philox.h"
#include "rows8.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;

template <typename T, bool RESID>
__global__ void __launch_bounds__(TPB) dropout_k(const T *x, int64_t ldx, const T *resid, int64_t ldr, T *y, int64_t ldy, uint32_t rows, uint32_t cols,
                                                 uint32_t groups, Dropout d) {
    const uint32_t idx = blockIdx.x * TPB + threadIdx.x, row = idx / groups, c = idx - row * groups;      // below 2^31 + TPB
    if (row >= rows) return;
    Row8<T> v, r;
    v.load(x + (int64_t)row * ldx + c * 8);
    if (RESID) r.load(resid + (int64_t)row * ldr + c * 8);
    Mask8 m;
    m.draw(row, groups, c, d);
    float f[8], g[8];
    v.get(f);
    if (RESID) r.get(g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f[j] = m.kept(j, d) ? f[j] * d.scale : 0.f;
        if (RESID) f[j] += g[j];
    }
    cut8(f, (int)(cols - c * 8));
    v.set(f);
    v.put(y + (int64_t)row * ldy + c * 8);
}

}  // namespace

bool dropout_fits(int64_t rows, int64_t cols) {
    const int64_t most = (int64_t)1 << 31;
    return rows < most && cols < most && rows * ((cols + 7) / 8) < most;
}
void dropout(hipStream_t s, int dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, const void *resid, int64_t ldr, void *y, int64_t ldy,
             const Dropout &d) {
    const uint32_t groups = (uint32_t)((cols + 7) / 8);
    const unsigned grid = (unsigned)((rows * groups + TPB - 1) / TPB);
#define TIO_DROPOUT(T, RESID) \
    dropout_k<T, RESID><<<grid, TPB, 0, s>>>((const T *)x, ldx, (const T *)resid, ldr, (T *)y, ldy, (uint32_t)rows, (uint32_t)cols, groups, d)
    if (dtype == TIO_PREC_BF16 && resid) TIO_DROPOUT(bf16_t, true);
    else if (dtype == TIO_PREC_BF16) TIO_DROPOUT(bf16_t, false);
    else if (resid) TIO_DROPOUT(float, true);
    else TIO_DROPOUT(float, false);
#undef TIO_DROPOUT
}

}  // namespace k
}  // namespace tio
