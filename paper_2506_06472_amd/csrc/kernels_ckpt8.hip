// Activations kept in eight bits from the forward to the backward pass, and the activations whose gradients are computed from them.
//
// Blocks of 32 neighbours of a row share a power of two.  With a the largest magnitude of a block, e = max(floor(log2 a), -120) and
// q = clamp(round(x 2^(6 - e)), -127, 127), ties to even; a block stands for the values q 2^(e - 6).  Products with powers of two are
// exact, so q does not depend on the precision of the arithmetic, and the values are exact bf16 numbers (seven bits and a sign).  A
// block with an infinity or a NaN stands for NaNs.  The rounding is at most half a step, 2^(e - 7), which is 2^-7 of the block's
// largest magnitude at worst; the clamp makes it a whole step for magnitudes from 127.5 steps on.
//
// A checkpoint of [rows, cols] holds [rows][32 blocks] bytes q + 128, where blocks = ceil(cols / 32), then [rows][blocks] bytes
// e + 127 (255: not finite).  Columns past the end of a row's last block hold zeros.
//
// Bound: HBM (8192 x 4096, bf16: stored 16.5 us, 6.1 TB/s, read back 15.6, 6.5; SwiGLU of 8192 x 11008 119 us forward and 148 back, 6.1 TB/s of what
// they have to move).  A thread takes eight neighbours (16 bytes of bf16, two loads of fp32): a block is four lanes, which exchange their
// largest magnitude through two data-parallel-primitive moves; magnitudes are compared as integers, so that a NaN is the largest.
#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;
constexpr int MIN_CODE = 127 - 120;          // exponent byte of the smallest block
constexpr float L2E = 1.4426950408889634f;

// eight neighbours of a row.  Results go past the caches (put): read again they are by the next product, long after, and kept they push out what this
// pass still reads, or the checkpoint (8192 x 4096, bf16, stored and read back: 40.9 -> 36.1 us; SwiGLU of 2048 x 4096 31.3 -> 25.4).
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    Vec16<bf16_t> v;
    __device__ __forceinline__ void load(const bf16_t *p) { v.load(p); }
    __device__ __forceinline__ void put(bf16_t *p) const { __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, v.raw), reinterpret_cast<tio_u32x4 *>(p)); }
    __device__ __forceinline__ void get(float *f) const { v.get(f); }
    __device__ __forceinline__ void set(const float *f) { v.set(f); }
};
template <> struct Eight<float> {
    Vec16<float> lo, hi;
    __device__ __forceinline__ void load(const float *p) { lo.load(p); hi.load(p + 4); }
    __device__ __forceinline__ void put(float *p) const {
        __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, lo.raw), reinterpret_cast<tio_u32x4 *>(p));
        __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, hi.raw), reinterpret_cast<tio_u32x4 *>(p + 4));
    }
    __device__ __forceinline__ void get(float *f) const { lo.get(f); hi.get(f + 4); }
    __device__ __forceinline__ void set(const float *f) { lo.set(f); hi.set(f + 4); }
};

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    const uint32_t a = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);         // lanes 1 0 3 2
    x = x > a ? x : a;
    const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);         // lanes 2 3 0 1
    return x > b ? x : b;
}
// A block's exponent byte from its lanes' values, which all four lanes of the block take part in.
__device__ __forceinline__ uint32_t block_code(const float *f) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(f[j]) & 0x7fffffffu;
        top = b > top ? b : top;
    }
    const uint32_t code = quad_max(top) >> 23;
    return code < (uint32_t)MIN_CODE ? (uint32_t)MIN_CODE : code;
}
// q + 128 of eight values as bytes.  Adding 1.5 2^23 + 128 rounds to the nearest integer, ties to even, and leaves it in the low byte.
__device__ __forceinline__ uint2 quantise(const float *f, uint32_t code) {
    const float up = __uint_as_float((260u - code) << 23);               // 2^(6 - e); of a block that is not finite: whatever
    uint32_t b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = __float_as_uint(__builtin_amdgcn_fmed3f(f[j] * up, -127.0f, 127.0f) + 12583040.0f);
    auto four = [](uint32_t a, uint32_t c, uint32_t d, uint32_t e) __attribute__((always_inline)) {
        const uint32_t lo = __builtin_amdgcn_perm(c, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(e, d, 0x04000c0cu);
        return lo | hi;
    };
    return make_uint2(four(b[0], b[1], b[2], b[3]), four(b[4], b[5], b[6], b[7]));
}
__device__ __forceinline__ void dequantise(uint2 q, uint32_t code, float *f) {
    const float down = code == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((code - 6u) << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = ((float)(((j < 4 ? q.x : q.y) >> (8 * (j & 3))) & 255u) - 128.0f) * down;
}

// A thread's place: chunk c of eight columns in a row, of `chunks` (a multiple of four: whole blocks) to a row.  32-bit division; the
// launchers keep rows * chunks below 2^31.
struct Place {
    uint32_t row, c;
    __device__ __forceinline__ Place(uint32_t idx, uint32_t chunks) : row(idx / chunks), c(idx - row * chunks) {}
};
// a checkpoint of [rows, 8 chunks]
struct Kept {
    uint8_t *q, *e;
    __device__ __forceinline__ Kept(uint8_t *p, uint32_t rows, uint32_t chunks) : q(p), e(p + (int64_t)rows * chunks * 8) {}
    // idx: row * chunks + c.  STREAM: past the caches
    template <bool STREAM> __device__ __forceinline__ void store(uint32_t idx, const float *f) const {
        const uint32_t code = block_code(f);
        const uint2 v = quantise(f, code);
        if (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, v), reinterpret_cast<uint64_t *>(q + (int64_t)idx * 8));
        else *reinterpret_cast<uint2 *>(q + (int64_t)idx * 8) = v;
        if ((idx & 3) == 0) e[idx >> 2] = (uint8_t)code;
    }
};
// columns from n on become zero
__device__ __forceinline__ void cut(float *f, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j >= n) f[j] = 0.f;
}

// A thread stores or loads U chunks, a workgroup's width apart, all loads first (8192 x 4096, bf16, stored and read back: 35.7 us with one chunk, 33.7 with
// two and with four).  The activations' threads take one, whose loads are several (SwiGLU of 8192 x 11008: 267 us, two chunks 279, four 284).
constexpr int U = 2;
template <typename T, bool STREAM>
__global__ void __launch_bounds__(TPB) ckpt8_store_k(const T *__restrict__ x, int64_t ld, uint8_t *__restrict__ kept, uint32_t rows, uint32_t cols,
                                                     uint32_t chunks) {
    const uint32_t first = blockIdx.x * (TPB * U) + threadIdx.x, n = rows * chunks;
    Eight<T> v[U];
    int left[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place p(first + u * TPB, chunks);
        left[u] = (int)cols - (int)p.c * 8;
        if (first + u * TPB < n && left[u] > 0) v[u].load(x + p.row * ld + p.c * 8);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (first + u * TPB >= n) return;                  // whole blocks: their lanes leave together
        float f[8];
        v[u].get(f);
        cut(f, left[u]);
        Kept(kept, rows, chunks).store<STREAM>(first + u * TPB, f);
    }
}

template <typename T>
__global__ void __launch_bounds__(TPB) ckpt8_load_k(const uint8_t *__restrict__ kept, T *__restrict__ x, int64_t ld, uint32_t rows, uint32_t cols,
                                                    uint32_t chunks) {
    const uint32_t first = blockIdx.x * (TPB * U) + threadIdx.x, n = rows * chunks;
    const uint8_t *e = kept + (int64_t)n * 8;
    uint2 q[U];
    uint32_t code[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t idx = first + u * TPB;
        if (idx < n) {
            q[u] = *reinterpret_cast<const uint2 *>(kept + (int64_t)idx * 8);
            code[u] = e[idx >> 2];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t idx = first + u * TPB;
        if (idx >= n) return;
        const Place p(idx, chunks);
        const int left = (int)cols - (int)p.c * 8;
        if (left <= 0) continue;
        float f[8];
        dequantise(q[u], code[u], f);
        cut(f, left);
        Eight<T> v;
        v.set(f);
        v.put(x + p.row * ld + p.c * 8);
    }
}

// 1 / (1 + exp(-x)): in bf16 the hardware's exponential and reciprocal (relative error about 1e-6 against the 2e-3 of the output's
// rounding), in fp32 the library's.
template <typename T> __device__ __forceinline__ float logistic(float x) {
    if (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-L2E * x));
    return 1.0f / (1.0f + expf(-x));
}
// GELU's tanh form: (1 + tanh u) / 2 is the logistic function of 2 u, without the cancellation of 1 + tanh u for negative u
constexpr float GELU_A = 1.5957691216057308f, GELU_B = 0.044715f;       // 2 sqrt(2 / pi)
template <typename T> __device__ __forceinline__ float gelu(float x) { return x * logistic<T>(GELU_A * (x + GELU_B * x * x * x)); }
template <typename T> __device__ __forceinline__ void gelu_both(float x, float &y, float &dy) {
    const float s = logistic<T>(GELU_A * (x + GELU_B * x * x * x));
    y = x * s;
    dy = s + y * (1.0f - s) * GELU_A * (1.0f + 3.0f * GELU_B * fminf(x * x, 1e4f));      // beyond |x| = 100 y (1 - s) is zero, and must not meet infinity
}

// y = act(gate[, up]) of the values as they come; the checkpoint keeps the inputs (SwiGLU: the gate half's checkpoint, then the up half's).
template <typename T, bool SWIGLU, bool STREAM>
__global__ void __launch_bounds__(TPB) act_ckpt8_k(const T *__restrict__ gate, const T *__restrict__ up, int64_t ldu, T *__restrict__ y, int64_t ldy,
                                                   uint8_t *__restrict__ kept, int64_t half_bytes, uint32_t rows, uint32_t cols, uint32_t chunks) {
    const uint32_t idx = blockIdx.x * TPB + threadIdx.x;
    if (idx >= rows * chunks) return;                      // whole blocks: their lanes leave together
    const Place p(idx, chunks);
    const int left = (int)cols - (int)p.c * 8;
    Eight<T> a, b;
    if (left > 0) {
        a.load(gate + p.row * ldu + p.c * 8);
        if (SWIGLU) b.load(up + p.row * ldu + p.c * 8);
    }
    float g[8], u[8];
    a.get(g);
    cut(g, left);
    Kept(kept, rows, chunks).store<STREAM>(idx, g);
    if (SWIGLU) {
        b.get(u);
        cut(u, left);
        Kept(kept + half_bytes, rows, chunks).store<STREAM>(idx, u);
    }
    if (left > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = SWIGLU ? g[j] * logistic<T>(g[j]) * u[j] : gelu<T>(g[j]);
        cut(g, left);
        Eight<T> v;
        v.set(g);
        v.put(y + p.row * ldy + p.c * 8);
    }
}

// The gradient of the activation's inputs, and its output again (y: nullptr, or where it goes), from the checkpoint.
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(TPB) act_ckpt8_bwd_k(const uint8_t *__restrict__ kept, int64_t half_bytes, const T *__restrict__ dy, int64_t lddy,
                                                       T *__restrict__ dgate, T *__restrict__ dup, int64_t ldu, T *__restrict__ y, int64_t ldy,
                                                       uint32_t rows, uint32_t cols, uint32_t chunks) {
    const uint32_t idx = blockIdx.x * TPB + threadIdx.x, n = rows * chunks;
    if (idx >= n) return;
    const Place p(idx, chunks);
    const int left = (int)cols - (int)p.c * 8;
    if (left <= 0) return;
    float g[8], u[8], d[8], out[8];
    Eight<T> v;
    v.load(dy + p.row * lddy + p.c * 8);
    const uint8_t *const q = kept + (int64_t)idx * 8, *const e = kept + (int64_t)n * 8 + (idx >> 2);
    dequantise(*reinterpret_cast<const uint2 *>(q), *e, g);
    if (SWIGLU) dequantise(*reinterpret_cast<const uint2 *>(q + half_bytes), e[half_bytes], u);
    v.get(d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (SWIGLU) {
            const float s = logistic<T>(g[j]), gs = g[j] * s;
            out[j] = gs * u[j];
            const float dg = d[j] * u[j] * (s + gs * (1.0f - s));
            u[j] = d[j] * gs;
            g[j] = dg;
        } else {
            float grad;
            gelu_both<T>(g[j], out[j], grad);
            g[j] = d[j] * grad;
        }
    }
    cut(g, left);
    v.set(g);
    v.put(dgate + p.row * ldu + p.c * 8);
    if (SWIGLU) {
        cut(u, left);
        v.set(u);
        v.put(dup + p.row * ldu + p.c * 8);
    }
    if (y) {
        cut(out, left);
        v.set(out);
        v.put(y + p.row * ldy + p.c * 8);
    }
}

uint32_t chunks_of(int64_t cols) { return (uint32_t)((cols + 31) / 32 * 4); }
unsigned grid_of(int64_t rows, int64_t cols, int of_thread) { return (unsigned)((rows * chunks_of(cols) + TPB * of_thread - 1) / (TPB * of_thread)); }
// a checkpoint this large goes past the caches: the memory-side cache (256 MiB) would not hold it until it is read
bool large(int64_t bytes) { return bytes > (int64_t)128 << 20; }

}  // namespace

bool ckpt8_fits(int64_t rows, int64_t cols) {
    const int64_t most = ((int64_t)1 << 31) - 4 * TPB;       // a thread's chunk past the last one is counted too
    return cols <= most && rows <= most && rows * (int64_t)chunks_of(cols) <= most;
}
int64_t ckpt8_bytes(int64_t rows, int64_t cols) {
    const int64_t blocks = rows * (chunks_of(cols) / 4);
    return (blocks * 33 + 15) / 16 * 16;
}

#define TIO_BY_TYPE(dtype, ...)                                       \
    do {                                                              \
        if ((dtype) == TIO_PREC_BF16) { using T = bf16_t; __VA_ARGS__; } \
        else { using T = float; __VA_ARGS__; }                        \
    } while (0)

void ckpt8_store(hipStream_t s, int dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *kept) {
#define TIO_STORE(STREAM)                                                                                                                       \
    TIO_BY_TYPE(dtype, (ckpt8_store_k<T, STREAM><<<grid_of(rows, cols, U), TPB, 0, s>>>((const T *)x, ldx, (uint8_t *)kept, (uint32_t)rows, \
                                                                                           (uint32_t)cols, chunks_of(cols))))
    if (large(ckpt8_bytes(rows, cols))) TIO_STORE(true);
    else TIO_STORE(false);
#undef TIO_STORE
}
void ckpt8_load(hipStream_t s, int dtype, int64_t rows, int64_t cols, const void *kept, void *x, int64_t ldx) {
    TIO_BY_TYPE(dtype, (ckpt8_load_k<T><<<grid_of(rows, cols, U), TPB, 0, s>>>((const uint8_t *)kept, (T *)x, ldx, (uint32_t)rows, (uint32_t)cols,
                                                                                  chunks_of(cols))));
}
void act_ckpt8(hipStream_t s, int dtype, bool swiglu, int64_t rows, int64_t f, const void *gate, const void *up, int64_t ldu, void *y, int64_t ldy,
               void *kept) {
    const bool past = large(ckpt8_bytes(rows, f) * (swiglu ? 2 : 1));
#define TIO_ACT(SWIGLU, STREAM)                                                                                                                    \
    TIO_BY_TYPE(dtype, (act_ckpt8_k<T, SWIGLU, STREAM><<<grid_of(rows, f, 1), TPB, 0, s>>>((const T *)gate, (const T *)up, ldu, (T *)y, ldy,  \
                                                                                              (uint8_t *)kept, ckpt8_bytes(rows, f),              \
                                                                                              (uint32_t)rows, (uint32_t)f, chunks_of(f))))
    if (swiglu && past) TIO_ACT(true, true);
    else if (swiglu) TIO_ACT(true, false);
    else if (past) TIO_ACT(false, true);
    else TIO_ACT(false, false);
#undef TIO_ACT
}
void act_ckpt8_bwd(hipStream_t s, int dtype, bool swiglu, int64_t rows, int64_t f, const void *kept, const void *dy, int64_t lddy, void *dgate,
                   void *dup, int64_t ldu, void *y, int64_t ldy) {
#define TIO_ACT(SWIGLU)                                                                                                                          \
    TIO_BY_TYPE(dtype, (act_ckpt8_bwd_k<T, SWIGLU><<<grid_of(rows, f, 1), TPB, 0, s>>>((const uint8_t *)kept, ckpt8_bytes(rows, f),         \
                                                                                          (const T *)dy, lddy, (T *)dgate, (T *)dup, ldu,       \
                                                                                          (T *)y, ldy, (uint32_t)rows, (uint32_t)f, chunks_of(f))))
    if (swiglu) TIO_ACT(true);
    else TIO_ACT(false);
#undef TIO_ACT
}

}  // namespace k
}  // namespace tio
