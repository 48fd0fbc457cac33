// Products of matrices stored in 8-bit floating point with a power of two for each block of 128 (fp8_blocks.h):
// C[M,N] = A[M,K] . B[N,K]^T (+ bias[N]) (+ resid[M,N]).
#include <type_traits>

#include "../../include/teraio.h"
#include "device_common.h"
#include "fp8_blocks.h"
#include "kernels.h"
#include "mfma_tiles.h"

namespace tio {
namespace k {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// What a lane hands to a product of 16 rows over a block of 128: its 32 codes, and its row's exponent byte.
struct Piece8 {
    uint4 h[2];
    uint32_t e;
    __device__ __forceinline__ void load(const uint8_t *frag, const uint8_t *exps, int lane) {
        h[0] = *reinterpret_cast<const uint4 *>(frag + lane * 16);
        h[1] = *reinterpret_cast<const uint4 *>(frag + 1024 + lane * 16);
        e = exps[(lane & 15) * 4];
    }
    __device__ __forceinline__ i32x8 codes() const {
        return (i32x8){(int)h[0].x, (int)h[0].y, (int)h[0].z, (int)h[0].w, (int)h[1].x, (int)h[1].y, (int)h[1].z, (int)h[1].w};
    }
    // a quarter of the codes as what they stand for
    template <int FORM> __device__ __forceinline__ bf16x8 values(int quarter) const {
        const float scale = __uint_as_float(e << 23);
        const uint32_t a = quarter & 1 ? h[quarter >> 1].z : h[quarter >> 1].x, b = quarter & 1 ? h[quarter >> 1].w : h[quarter >> 1].y;
        Frag f;
        f.u = make_uint4(f8_pair_bf16<FORM, 0>(a, scale), f8_pair_bf16<FORM, 1>(a, scale), f8_pair_bf16<FORM, 0>(b, scale), f8_pair_bf16<FORM, 1>(b, scale));
        return f.v;
    }
};

// a's rows and b's rows in one product; lane l of c holds row l % 16 of a's and rows 4 (l / 16) .. + 3 of b's
template <int FA, int FB> __device__ __forceinline__ floatx4 product8(const Piece8 &a, const Piece8 &b, floatx4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.codes(), a.codes(), c, FB, FA, 0, (int)b.e, 0, (int)a.e);
}
template <int FA, int FB> __device__ __forceinline__ floatx4 product16(const Piece8 &a, const Piece8 &b, floatx4 c) {
#pragma unroll
    for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.template values<FB>(q), a.template values<FA>(q), c, 0, 0, 0);
    return c;
}

template <typename T> __device__ __forceinline__ float element(const T *p) { return to_f32(*p); }

// A workgroup's tile of 16 TM x 16 TN results: its four wavefronts share the contraction, their sums are added in order.
template <int FA, int FB, typename T, int TM, int TN>
__global__ void __launch_bounds__(256) gemm_fp8_direct_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const T *__restrict__ bias,
                                                         const T *__restrict__ resid, int64_t ldr, T *__restrict__ C, int64_t ldc, int64_t M, int64_t N,
                                                         int64_t K, int tiles_n) {
    __shared__ float sums[4][TM * TN][256];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
    const Fp8Shape sa{M, K}, sb{N, K};
    const int64_t KB = sa.kb(), ga = sa.groups(), gb = sb.groups();
    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    for (int64_t kb = wave; kb < KB; kb += 4) {
        Piece8 a[TM], b[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t g = tm * TM + i < ga ? tm * TM + i : ga - 1;
            a[i].load(A + (g * KB + kb) * F8_FRAG, A + sa.code_bytes() + ((g >> 2) * KB + kb) * 64 + (g & 3), lane);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t g = tn * TN + j < gb ? tn * TN + j : gb - 1;
            b[j].load(B + (g * KB + kb) * F8_FRAG, B + sb.code_bytes() + ((g >> 2) * KB + kb) * 64 + (g & 3), lane);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = sizeof(T) == 2 ? product8<FA, FB>(a[i], b[j], acc[i][j]) : product16<FA, FB>(a[i], b[j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
            *reinterpret_cast<floatx4 *>(&sums[wave][i * TN + j][lane * 4]) = acc[i][j];
    __syncthreads();
    const int row = tid >> 4, col = tid & 15, at = ((col >> 2) * 16 + row) * 4 + (col & 3);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t m = (tm * TM + i) * 16 + row, n = (tn * TN + j) * 16 + col;
            if (m >= M || n >= (N + 7) / 8 * 8) continue;
            float v = sums[0][i * TN + j][at];
#pragma unroll
            for (int w = 1; w < 4; ++w) v += sums[w][i * TN + j][at];
            if (bias && n < N) v += element(bias + n);
            if (resid && n < N) v += element(resid + m * ldr + n);
            C[m * ldc + n] = from_f32<T>(n < N ? v : 0.f);
        }
}

template <int FA, int FB, typename T> void launch(hipStream_t s, const Fp8Product &p) {
#define TIO_DIRECT(TM, TN)                                                                                                                              \
    do {                                                                                                                                                \
        const int64_t tiles_m = (p.M + 16 * TM - 1) / (16 * TM), tiles_n = (p.N + 16 * TN - 1) / (16 * TN);                                             \
        gemm_fp8_direct_k<FA, FB, T, TM, TN><<<(unsigned)(tiles_m * tiles_n), 256, 0, s>>>(                                                             \
            (const uint8_t *)p.A, (const uint8_t *)p.B, (const T *)p.bias, (const T *)p.resid, p.ldr, (T *)p.C, p.ldc, p.M, p.N, p.K, (int)tiles_n); \
    } while (0)
    if (p.M <= 16) TIO_DIRECT(1, 1);
    else TIO_DIRECT(2, 2);
#undef TIO_DIRECT
}

}  // namespace

int64_t gemm_fp8_work(int64_t, int64_t, int64_t) { return 0; }

void gemm_fp8(hipStream_t s, int dtype, const Fp8Product &p) {
#define TIO_FORMS(T)                                                  \
    do {                                                              \
        if (p.form_a && p.form_b) launch<1, 1, T>(s, p);              \
        else if (p.form_a) launch<1, 0, T>(s, p);                     \
        else if (p.form_b) launch<0, 1, T>(s, p);                     \
        else launch<0, 0, T>(s, p);                                   \
    } while (0)
    if (dtype == TIO_PREC_BF16) TIO_FORMS(bf16_t);
    else TIO_FORMS(float);
#undef TIO_FORMS
}

}  // namespace k
}  // namespace tio
