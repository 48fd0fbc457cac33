// What the C entries of the single operators share: checks of arguments, the stream's device, errors of a launch.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <stdexcept>
#include <string>

#include "../../include/teraio.h"
#include "handles.h"

namespace tio {
namespace {

bool aligned(const void *p, int to = 16) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }
bool known_type(int32_t dtype) { return dtype == TIO_PREC_FP32 || dtype == TIO_PREC_BF16; }
// elements of a 16-byte chunk
int64_t chunk_of(int32_t dtype) { return dtype == TIO_PREC_BF16 ? 8 : 4; }

// The stream's device is the current one while this lives: a kernel goes to a stream of the current device.
class OnDeviceOf {
    int before_ = -1;
public:
    explicit OnDeviceOf(hipStream_t s) {
        hipDevice_t of = 0;
        int now = 0;
        if (!s || hipStreamGetDevice(s, &of) != hipSuccess || hipGetDevice(&now) != hipSuccess || now == (int)of) return;
        if (hipSetDevice((int)of) == hipSuccess) before_ = now;
    }
    ~OnDeviceOf() { if (before_ >= 0) (void)hipSetDevice(before_); }
    OnDeviceOf(const OnDeviceOf &) = delete;
    OnDeviceOf &operator=(const OnDeviceOf &) = delete;
};

int launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TIO_OK : fail(TIO_ERR_HIP, std::string("launch: ") + hipGetErrorString(e));
}

#define TIO_OP_BEGIN try {
#define TIO_OP_END                                                                                \
    } catch (const std::bad_alloc &) { return fail(TIO_ERR_OOM_HOST, "out of host memory");       \
    } catch (const std::exception &e) { return fail(TIO_ERR_INVALID_ARG, e.what()); }

bool stride_ok(int64_t ld, int64_t cols) { return ld % 8 == 0 && ld >= (cols + 7) / 8 * 8; }
const char *const BAD_STRIDE = "row strides must be multiples of 8 elements and at least the columns rounded up to 8";
const char *const BAD_POINTER = "pointers must be 16-byte aligned";

}  // namespace
}  // namespace tio
