// A matrix stored in 8-bit floating point with a power of two for each block of 128 (fp8_blocks.h), as it is and transposed in one pass, and
// read back.
//
// Bound: HBM (8192 x 11008 from bf16 in both forms 61 us, 5.9 TB/s; 6656 x 6656 in 128 x 128 blocks 36 us and read back 20 us a form, 4.9 and 6.5 TB/s).
// A workgroup takes 128 x 128 elements, a thread 8 x 8 of them, so that eight neighbours of a row and eight of a column are one
// thread's: both forms' codes go to LDS as 8-byte words, from which fragments leave in whole 1 KiB stores.
#include <type_traits>

#include "../../include/teraio.h"
#include "device_common.h"
#include "fp8_blocks.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;

// Eight neighbours of a row.  Magnitudes are compared as integers, so that infinities and NaN are the largest; two bf16 at a time.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    uint32_t w[4];
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void load(const bf16_t *p) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ void cut(int n) {               // n < 8 of them are there
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = n >= 2 * j + 2 ? w[j] : n == 2 * j + 1 ? w[j] & 0xffffu : 0u;
    }
    template <int FORM> __device__ __forceinline__ uint2 codes(float scale) const {
        return make_uint2(f8_codes<FORM>(w[0], w[1], scale), f8_codes<FORM>(w[2], w[3], scale));
    }
};
template <> struct Eight<float> {
    float f[8];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.f;
    }
    __device__ __forceinline__ void load(const float *p) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void cut(int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = j < n ? f[j] : 0.f;
    }
    template <int FORM> __device__ __forceinline__ uint2 codes(float scale) const {
        return make_uint2(f8_codes<FORM>(f[0], f[1], f[2], f[3], scale), f8_codes<FORM>(f[4], f[5], f[6], f[7], scale));
    }
};

// The largest magnitudes of eight columns: bits of an fp32 each, or of two bf16 to a word.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {        // of both halves
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t max1(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <typename T> struct Tops;
template <> struct Tops<bf16_t> {
    static constexpr int N = 4;
    uint32_t m[N];
    __device__ __forceinline__ void start() { m[0] = m[1] = m[2] = m[3] = 0; }
    __device__ __forceinline__ void take(const Eight<bf16_t> &v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = max2(m[j], v.w[j] & 0x7fff7fffu);
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max2(a, b); }
    static __device__ __forceinline__ uint32_t of_row(const Eight<bf16_t> &v) {
        const uint32_t a = max2(v.w[0] & 0x7fff7fffu, v.w[1] & 0x7fff7fffu), b = max2(v.w[2] & 0x7fff7fffu, v.w[3] & 0x7fff7fffu), c = max2(a, b);
        return max1(c << 16, c & 0xffff0000u);
    }
    __device__ __forceinline__ uint32_t column(int j) const { return j & 1 ? m[j >> 1] & 0xffff0000u : m[j >> 1] << 16; }
};
template <> struct Tops<float> {
    static constexpr int N = 8;
    uint32_t m[N];
    __device__ __forceinline__ void start() {
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = 0;
    }
    __device__ __forceinline__ void take(const Eight<float> &v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = max1(m[j], __float_as_uint(v.f[j]) & 0x7fffffffu);
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max1(a, b); }
    static __device__ __forceinline__ uint32_t of_row(const Eight<float> &v) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) t = max1(t, __float_as_uint(v.f[j]) & 0x7fffffffu);
        return t;
    }
    __device__ __forceinline__ uint32_t column(int j) const { return m[j]; }
};

// the largest of 16 neighbouring lanes, in all of them
__device__ __forceinline__ uint32_t row16_max(uint32_t x) {
    x = max1(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));          // lanes 1 0 3 2
    x = max1(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));          // lanes 2 3 0 1
    x = max1(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true));         // eight lanes mirrored
    return max1(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, true));      // sixteen lanes mirrored
}

// column J of rows 2 P and 2 P + 1 and the two behind them, as codes
template <int FORM, int J> __device__ __forceinline__ uint32_t column_codes(const Eight<bf16_t> (&v)[8], int half, float scale) {
    constexpr uint32_t PICK = J & 1 ? 0x07060302u : 0x05040100u;
    const int i = half * 4;
    const uint32_t ab = __builtin_amdgcn_perm(v[i + 1].w[J / 2], v[i].w[J / 2], PICK), cd = __builtin_amdgcn_perm(v[i + 3].w[J / 2], v[i + 2].w[J / 2], PICK);
    return f8_codes<FORM>(ab, cd, scale);
}
template <int FORM, int J> __device__ __forceinline__ uint32_t column_codes(const Eight<float> (&v)[8], int half, float scale) {
    const int i = half * 4;
    return f8_codes<FORM>(v[i].f[J], v[i + 1].f[J], v[i + 2].f[J], v[i + 3].f[J], scale);
}

// A 128 x 128 tile of codes in LDS: fragments of 16 rows, the 16-byte piece q of row r (q = k / 16) at 256 q + 16 (r ^ q), so that the words of
// one store instruction, eight pieces of two rows, fall into different banks.
struct Codes {
    unsigned char b[8 * F8_FRAG];
    // where a thread's eight rows from 8 rows8 on have their neighbours 8 k8 .. + 7; row i of them is at ((k8 / 2) ^ i) 16 from there
    static __device__ __forceinline__ int place(int rows8, int k8) { return (rows8 >> 1) * F8_FRAG + (rows8 & 1) * 128 + (k8 >> 1) * 256 + (k8 & 1) * 8; }
    __device__ __forceinline__ void put(int place, int k8, int i, uint2 v) { *reinterpret_cast<uint2 *>(b + place + (((k8 >> 1) ^ i) << 4)) = v; }
    // to the fragments of block kb of the `groups` row groups from `group` on
    template <bool FULL> __device__ __forceinline__ void write(uint8_t *out, const Fp8Shape &s, int64_t group, int64_t kb, int tid) const {
        const int64_t KB = s.kb(), groups = s.groups();
        const int p = tid & 127, q = p >> 4, r = p & 15, f0 = tid >> 7;
        uint8_t *to = out + ((group + f0) * KB + kb) * F8_FRAG + p * 16;
        const unsigned char *from = b + f0 * F8_FRAG + q * 256 + ((r ^ q) << 4);
#pragma unroll
        for (int i = 0; i < 4; ++i, to += 2 * KB * F8_FRAG, from += 2 * F8_FRAG)
            if (FULL || group + f0 + 2 * i < groups) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
    }
};
// the exponents of 128 rows, as two words of 64 rows
struct Exponents {
    uint8_t e[128];
    __device__ __forceinline__ void put(int row, uint32_t code) { e[(row >> 6) * 64 + (row & 15) * 4 + ((row >> 4) & 3)] = (uint8_t)code; }
    __device__ __forceinline__ void write(uint8_t *out, const Fp8Shape &s, int64_t row0, int64_t kb, int tid) const {
        if (tid >= 32) return;
        const int64_t g = row0 / 64 + (tid >> 4);
        if (g * 64 < s.rows) *reinterpret_cast<uint32_t *>(out + s.code_bytes() + (g * s.kb() + kb) * 64 + (tid & 15) * 4) = reinterpret_cast<const uint32_t *>(e)[tid];
    }
};

__device__ __forceinline__ float scale_of(uint32_t code) { return __uint_as_float(code << 23); }
// the larger of the two halves of a wavefront's rows of 16 lanes, and of those, in all lanes
template <typename T> __device__ __forceinline__ uint32_t over_rows(uint32_t x) {
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = Tops<T>::larger(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return Tops<T>::larger(b[0], b[1]);
}

// A wavefront's vector operations on 64 elements a lane cost about as much as its memory traffic does: whole tiles are loaded and written without tests, and
// blocks that are not finite are looked after only where a wavefront has any (8192 x 11008 from bf16, both forms, 361 MB: 79 us with tests and selections
// everywhere, about 800 operations, 61 with 520).
template <typename T, int FORM, bool TILES, bool TRANS, bool FULL>
__device__ __forceinline__ void store_tile8(Codes *codes, Exponents *exps, uint32_t (*tops)[16][Tops<T>::N], const T *__restrict__ x, int64_t ld, uint8_t *__restrict__ out,
                                            uint8_t *__restrict__ outt, int64_t rows, int64_t cols, int64_t tr, int64_t tc) {
    const int tid = threadIdx.x, wave = tid >> 6, c = tid & 15, rb = tid >> 4;
    const int64_t row0 = tr * 128, col0 = tc * 128;
    Eight<T> v[8];
    if (FULL) {
        const T *from = x + (row0 + rb * 8) * ld + col0 + c * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i, from += ld) v[i].load(from);
    } else {
        const int rows_here = rows - row0 < 128 ? (int)(rows - row0) : 128, left = (int)(cols - col0 < 128 ? cols - col0 : 128) - c * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i].clear();
            if (rb * 8 + i < rows_here && left > 0) v[i].load(x + (row0 + rb * 8 + i) * ld + col0 + c * 8);
        }
        if (left < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i].cut(left);
        }
    }

    Tops<T> top;
    uint32_t whole = 0;                                        // of the tile
    if (TILES || TRANS) {
        top.start();
#pragma unroll
        for (int i = 0; i < 8; ++i) top.take(v[i]);
#pragma unroll
        for (int j = 0; j < Tops<T>::N; ++j) top.m[j] = over_rows<T>(top.m[j]);          // over the wavefront's 32 rows
        if ((tid & 48) == 0) {
#pragma unroll
            for (int j = 0; j < Tops<T>::N; ++j) tops[wave][c][j] = top.m[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < Tops<T>::N; ++j) {
            top.m[j] = tops[0][c][j];
#pragma unroll
            for (int w = 1; w < 4; ++w) top.m[j] = Tops<T>::larger(top.m[j], tops[w][c][j]);
        }
        if (TILES) {
#pragma unroll
            for (int j = 0; j < 8; ++j) whole = max1(whole, top.column(j));
            whole = row16_max(whole);
        }
    }

    uint32_t by_row[8], most = TILES ? whole : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        by_row[i] = TILES ? whole : row16_max(Tops<T>::of_row(v[i]));
        most = max1(most, by_row[i]);
    }
    auto encode = [&](auto ALL_FINITE) __attribute__((always_inline)) {
        constexpr uint32_t NONE = 0x7f7f7f7fu;                 // NaN in both forms
        auto codes_or_none = [&](uint2 w, uint32_t t) __attribute__((always_inline)) { return ALL_FINITE() || f8_finite(t) ? w : make_uint2(NONE, NONE); };
        auto exponent = [&](uint32_t power, uint32_t t) __attribute__((always_inline)) { return ALL_FINITE() || f8_finite(t) ? power >> 23 : 127u; };
        const int by_rows = Codes::place(rb, c);
        uint32_t e = 0;                                        // of row c of the eight, which are the same to sixteen lanes
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t power = f8_power<FORM>(by_row[i]);
            codes[0].put(by_rows, c, i, codes_or_none(v[i].template codes<FORM>(__uint_as_float(power)), by_row[i]));
            e = c == i ? exponent(power, by_row[i]) : e;
        }
        if (c < 8) exps[0].put(rb * 8 + c, e);
        if constexpr (TRANS) {
            const int by_columns = Codes::place(c, rb);
            auto column = [&](auto J) __attribute__((always_inline)) {
                constexpr int j = decltype(J)::value;
                const uint32_t t = TILES ? whole : top.column(j), power = f8_power<FORM>(t);
                const float scale = __uint_as_float(power);
                codes[1].put(by_columns, rb, j, codes_or_none(make_uint2(column_codes<FORM, j>(v, 0, scale), column_codes<FORM, j>(v, 1, scale)), t));
                e = rb == j ? exponent(power, t) : e;
            };
            column(std::integral_constant<int, 0>{}); column(std::integral_constant<int, 1>{}); column(std::integral_constant<int, 2>{});
            column(std::integral_constant<int, 3>{}); column(std::integral_constant<int, 4>{}); column(std::integral_constant<int, 5>{});
            column(std::integral_constant<int, 6>{}); column(std::integral_constant<int, 7>{});
            if (rb < 8) exps[1].put(c * 8 + rb, e);
        }
    };
    if (TRANS && !TILES) {
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max1(most, top.column(j));
    }
    if (__any(!f8_finite(most))) encode(std::false_type{});
    else encode(std::true_type{});
    __syncthreads();
    const Fp8Shape s{rows, cols};
    if (out) {
        codes[0].template write<FULL>(out, s, tr * 8, tc, tid);
        exps[0].write(out, s, row0, tc, tid);
    }
    if constexpr (TRANS) {
        const Fp8Shape st{cols, rows};
        codes[1].template write<FULL>(outt, st, tc * 8, tr, tid);
        exps[1].write(outt, st, col0, tr, tid);
    }
}

template <typename T, int FORM, bool TILES, bool TRANS>
__global__ void __launch_bounds__(TPB) fp8_store_k(const T *__restrict__ x, int64_t ld, uint8_t *__restrict__ out, uint8_t *__restrict__ outt, int64_t rows,
                                                   int64_t cols, uint32_t tiles_c) {
    __shared__ __attribute__((aligned(16))) Codes codes[TRANS ? 2 : 1];
    __shared__ __attribute__((aligned(16))) Exponents exps[TRANS ? 2 : 1];
    __shared__ uint32_t tops[4][16][Tops<T>::N];               // [wavefront][eight columns]
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    if ((int64_t)tr * 128 + 128 <= rows && (int64_t)tc * 128 + 128 <= cols) store_tile8<T, FORM, TILES, TRANS, true>(codes, exps, tops, x, ld, out, outt, rows, cols, tr, tc);
    else store_tile8<T, FORM, TILES, TRANS, false>(codes, exps, tops, x, ld, out, outt, rows, cols, tr, tc);
}

// A wavefront takes a fragment: 16 rows of 128 neighbours, four rows at a time so that it writes whole rows of them.
template <typename T, int FORM>
__global__ void __launch_bounds__(TPB) fp8_load_k(const uint8_t *__restrict__ in, T *__restrict__ x, int64_t ld, int64_t rows, int64_t cols) {
    const Fp8Shape s{rows, cols};
    const int64_t KB = s.kb(), frag = (int64_t)blockIdx.x * (TPB / 64) + (threadIdx.x >> 6);
    if (frag >= s.groups() * KB) return;
    const int64_t g = frag / KB, kb = frag - g * KB;
    const int lane = threadIdx.x & 63, c = lane & 15;
    const int left = (int)(cols - kb * 128 < 128 ? cols - kb * 128 : 128) - c * 8;
    const uint8_t *const codes = in + frag * F8_FRAG + (c >> 1) * 256 + (c & 1) * 8;
    const uint8_t *const exps = in + s.code_bytes() + ((g >> 2) * KB + kb) * 64 + (g & 3);
    uint2 w[4];
    uint32_t e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 4 + (lane >> 4);
        w[i] = *reinterpret_cast<const uint2 *>(codes + r * 16);
        e[i] = exps[r * 4];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = g * 16 + i * 4 + (lane >> 4);
        if (row >= rows || left <= 0) continue;
        const float scale = scale_of(e[i]);
        if constexpr (sizeof(T) == 2) {
            Eight<bf16_t> v;
            v.w[0] = f8_pair_bf16<FORM, 0>(w[i].x, scale); v.w[1] = f8_pair_bf16<FORM, 1>(w[i].x, scale);
            v.w[2] = f8_pair_bf16<FORM, 0>(w[i].y, scale); v.w[3] = f8_pair_bf16<FORM, 1>(w[i].y, scale);
            if (left < 8) v.cut(left);
            __builtin_nontemporal_store((tio_u32x4){v.w[0], v.w[1], v.w[2], v.w[3]}, reinterpret_cast<tio_u32x4 *>(x + row * ld + kb * 128 + c * 8));
        } else {
            Eight<float> v;
            const f8_f32x2 p[4] = {f8_pair_f32<FORM, 0>(w[i].x, scale), f8_pair_f32<FORM, 1>(w[i].x, scale), f8_pair_f32<FORM, 0>(w[i].y, scale),
                                   f8_pair_f32<FORM, 1>(w[i].y, scale)};
#pragma unroll
            for (int j = 0; j < 8; ++j) v.f[j] = p[j >> 1][j & 1];
            if (left < 8) v.cut(left);
            float *const to = x + row * ld + kb * 128 + c * 8;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __builtin_nontemporal_store((tio_u32x4){__float_as_uint(v.f[4 * h]), __float_as_uint(v.f[4 * h + 1]), __float_as_uint(v.f[4 * h + 2]),
                                                        __float_as_uint(v.f[4 * h + 3])}, reinterpret_cast<tio_u32x4 *>(to + 4 * h));
        }
    }
}

}  // namespace

// a tile's fragments in a product are within 32-bit offsets, and the launches here within a grid
bool fp8_fits(int64_t rows, int64_t cols) {
    return rows <= (int64_t)1 << 22 && cols <= (int64_t)1 << 22 && Fp8Shape{rows, cols}.groups() * Fp8Shape{rows, cols}.kb() <= (int64_t)1 << 25;
}
int64_t fp8_bytes(int64_t rows, int64_t cols) { return Fp8Shape{rows, cols}.bytes(); }

void fp8_store(hipStream_t s, int dtype, int form, bool tiles, int64_t rows, int64_t cols, const void *x, int64_t ld, void *out, void *outt) {
    const int64_t tiles_r = (rows + 127) / 128, tiles_c = (cols + 127) / 128;
#define TIO_STORE(T, FORM, TILES, TRANS)                                                                                                            \
    fp8_store_k<T, FORM, TILES, TRANS><<<(unsigned)(tiles_r * tiles_c), TPB, 0, s>>>((const T *)x, ld, (uint8_t *)out, (uint8_t *)outt, rows, cols, \
                                                                                    (uint32_t)tiles_c)
#define TIO_STORE_OF(T, FORM)                       \
    do {                                            \
        if (tiles && outt) TIO_STORE(T, FORM, true, true);    \
        else if (tiles) TIO_STORE(T, FORM, true, false);      \
        else if (outt) TIO_STORE(T, FORM, false, true);       \
        else TIO_STORE(T, FORM, false, false);                \
    } while (0)
    if (dtype == TIO_PREC_BF16 && form) TIO_STORE_OF(bf16_t, 1);
    else if (dtype == TIO_PREC_BF16) TIO_STORE_OF(bf16_t, 0);
    else if (form) TIO_STORE_OF(float, 1);
    else TIO_STORE_OF(float, 0);
#undef TIO_STORE_OF
#undef TIO_STORE
}

void fp8_load(hipStream_t s, int dtype, int form, int64_t rows, int64_t cols, const void *in, void *x, int64_t ld) {
    const Fp8Shape shape{rows, cols};
    const unsigned grid = (unsigned)((shape.groups() * shape.kb() + TPB / 64 - 1) / (TPB / 64));
#define TIO_LOAD(T, FORM) fp8_load_k<T, FORM><<<grid, TPB, 0, s>>>((const uint8_t *)in, (T *)x, ld, rows, cols)
    if (dtype == TIO_PREC_BF16 && form) TIO_LOAD(bf16_t, 1);
    else if (dtype == TIO_PREC_BF16) TIO_LOAD(bf16_t, 0);
    else if (form) TIO_LOAD(float, 1);
    else TIO_LOAD(float, 0);
#undef TIO_LOAD
}

}  // namespace k
}  // namespace tio
