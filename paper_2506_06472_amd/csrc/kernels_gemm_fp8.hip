// Products of matrices stored in 8-bit floating point with a power of two for each block of 128 (fp8_blocks.h):
// C[M,N] = A[M,K] . B[N,K]^T (+ bias[N]) (+ resid[M,N]).
#include <type_traits>
#include <utility>

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

// ---- large products in bf16
// c += b's rows . a's rows over a block of 128, the accumulator held in an accumulation register (left to itself the compiler moves accumulators between
// the register files around the products); SB, SA: which byte of the lane's exponent words.
template <int FA, int FB, int SA, int SB> __device__ __forceinline__ void mfma8(floatx4 &c, const i32x8 &b, const i32x8 &a, uint32_t eb, uint32_t ea) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:%9 blgp:%10"
                 : "+a"(c)
                 : "v"(b), "v"(a), "v"(eb), "v"(ea), "n"(SB & 1), "n"(SA & 1), "n"(SB >> 1), "n"(SA >> 1), "n"(FB), "n"(FA));
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// the same with a load to LDS (see load_to_lds_b128) behind it: the product fills the wait state that M0 needs
template <int FA, int FB, int SA, int SB>
__device__ __forceinline__ void mfma8_load(floatx4 &c, const i32x8 &b, const i32x8 &a, uint32_t eb, uint32_t ea, i32x4 rsrc, uint32_t lds_addr, uint32_t voff,
                                           uint32_t soff) {
    asm volatile("s_mov_b32 m0, %11\n\t"
                 "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:%9 blgp:%10\n\t"
                 "buffer_load_dwordx4 %12, %13, %14 offen lds"
                 : "+a"(c)
                 : "v"(b), "v"(a), "v"(eb), "v"(ea), "n"(SB & 1), "n"(SA & 1), "n"(SB >> 1), "n"(SA >> 1), "n"(FB), "n"(FA), "s"(lds_addr), "v"(voff), "s"(rsrc),
                   "s"(soff)
                 : "memory", "m0");
}
// four bytes a lane from the lane's own address to LDS
__device__ __forceinline__ void load_to_lds_b32(const uint8_t *from, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_addr), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// f of each number as a constant
template <typename F, int... I> __device__ __forceinline__ void each(const F &f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }

// A tile of 32 TM x 32 TN results: four wavefronts, 16 TM x 16 TN each.  A step of the contraction is one block of 128: TM TN products of 32 clocks.
//  * Both operands' fragments go from memory straight into LDS, two steps deep; they are stored as the products take them, so that LDS is written and
//    read in consecutive KiB.  The exponents of a wavefront's rows and columns are one 4-byte load to LDS a step (lanes 0 .. 31 A's, the others B's).
//  * While the products of a step run, all fragments of the next one are read into registers: B's into a second set, A's into the registers of the row
//    group whose products are done, but for the last two groups, which have a second set too.  So a step's LDS is free when its products begin, and
//    the loads for the step after the next go there in their first half; they have the other half, at least, to land.
//  * One wavefront per SIMD (256 x 256) hides nothing by switching, so the order of all of it is pinned.
template <int FA, int FB, int TM, int TN>
__global__ void __launch_bounds__(256, TM == 8 ? 1 : 2)
    gemm_fp8_tile_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const uint16_t *__restrict__ bias, const uint16_t *resid, int64_t ldr, uint16_t *C,
                    int64_t ldc, int64_t M, int64_t N, int64_t K, int tiles_m, int tiles_n) {
    constexpr int BM = 32 * TM, BN = 32 * TN, TILE_A = BM * 128, TILE_B = BN * 128, NQ = TM * TN, NR = TM + TN, NL = TM + TN;
    constexpr uint32_t EXPS = 2 * (TILE_A + TILE_B);
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem8[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
    int split, nsplit, tm, tn;
    if (!place(tiles_m, tiles_n, 0, split, nsplit, tm, tn)) return;
    const Fp8Shape sa{M, K}, sb{N, K};
    const int64_t KB = sa.kb(), ga0 = (int64_t)tm * (2 * TM), gb0 = (int64_t)tn * (2 * TN);
    const int nk = (int)KB;

    // 1 KiB pieces of a step: half h of group g is piece 2 g + h, and wavefront p % 4's; groups past the last one repeat it
    const uint8_t *const baseA = A + ga0 * KB * F8_FRAG, *const baseB = B + gb0 * KB * F8_FRAG;
    const int64_t roomA = sa.code_bytes() - ga0 * KB * F8_FRAG, roomB = sb.code_bytes() - gb0 * KB * F8_FRAG;
    i32x4 rsA = make_rsrc(baseA, roomA < 0xfffffff0 ? (uint32_t)roomA : 0xfffffff0u), rsB = make_rsrc(baseB, roomB < 0xfffffff0 ? (uint32_t)roomB : 0xfffffff0u);
    const int lastA = (int)(sa.groups() - 1 - ga0), lastB = (int)(sb.groups() - 1 - gb0);
    uint32_t soA[TM], soB[TN];
#pragma unroll
    for (int l = 0; l < TM; ++l) {
        const int p = l * 4 + wave, g = p >> 1;
        soA[l] = __builtin_amdgcn_readfirstlane((uint32_t)((g < lastA ? g : lastA) * (int)KB * F8_FRAG + (p & 1) * 1024));
    }
#pragma unroll
    for (int l = 0; l < TN; ++l) {
        const int p = l * 4 + wave, g = p >> 1;
        soB[l] = __builtin_amdgcn_readfirstlane((uint32_t)((g < lastB ? g : lastB) * (int)KB * F8_FRAG + (p & 1) * 1024));
    }
    // lanes' exponents: words of 64 rows; TM, TN = 4: one of A's and one of B's, 8: two
    constexpr int WA = TM / 4, WB = TN / 4;
    const uint8_t *exps;
    {
        const bool isB = lane >= 32;
        const int64_t most = isB ? (N - 1) / 64 : (M - 1) / 64, g = (isB ? (int64_t)tn * (2 * WB) + wn * WB : (int64_t)tm * (2 * WA) + wm * WA) + (lane >> 4 & 1);
        exps = (isB ? B + sb.code_bytes() : A + sa.code_bytes()) + (g < most ? g : most) * KB * 64 + (lane & 15) * 4;
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem8));
    uint32_t ahead = 0, voff = lane * 16;                      // the step whose loads are next (the last one again when there is none), and where its codes are

    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};

    // where piece l of a step goes, in half S of LDS
    auto to_a = [&](auto S, int l) __attribute__((always_inline)) { return lds0 + S() * TILE_A + (l * 4 + wave) * 1024; };
    auto to_b = [&](auto S, int l) __attribute__((always_inline)) { return lds0 + 2 * TILE_A + S() * TILE_B + (l * 4 + wave) * 1024; };
    auto load_exps = [&](auto S) __attribute__((always_inline)) {
        load_to_lds_b32(exps + ahead * 64, lds0 + EXPS + wave * 512 + S() * 256);
    };
    auto go_on = [&]() __attribute__((always_inline)) {
        ahead = ahead + 1 < (uint32_t)nk ? ahead + 1 : (uint32_t)nk - 1;
        voff = lane * 16 + ahead * F8_FRAG;
    };
    auto load_step = [&](auto S) __attribute__((always_inline)) {
#pragma unroll
        for (int l = 0; l < TM; ++l) load_to_lds_b128(rsA, to_a(S, l), voff, soA[l]);
#pragma unroll
        for (int l = 0; l < TN; ++l) load_to_lds_b128(rsB, to_b(S, l), voff, soB[l]);
        load_exps(S);
        go_on();
    };
    i32x8 fa[TM], fa2[2], fb[2][TN];                           // fa2: of the last two row groups in odd steps
    uint32_t ea[2][WA], eb[2][WB];
    auto read_frag = [&](uint32_t at) __attribute__((always_inline)) {
        const uint4 u = *reinterpret_cast<const uint4 *>(smem8 + at + lane * 16), v = *reinterpret_cast<const uint4 *>(smem8 + at + 1024 + lane * 16);
        return (i32x8){(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
    };
    auto read_a = [&](auto S, auto I) __attribute__((always_inline)) {
        const i32x8 f = read_frag(S() * TILE_A + (wm * TM + I()) * F8_FRAG);
        if constexpr (S() == 1 && I() >= TM - 2) fa2[I() - (TM - 2)] = f;
        else fa[I()] = f;
    };
    auto read_b = [&](auto S, int j) __attribute__((always_inline)) { fb[S()][j] = read_frag(2 * TILE_A + S() * TILE_B + (wn * TN + j) * F8_FRAG); };
    auto read_exps = [&](auto S) __attribute__((always_inline)) {
        const unsigned char *const at = smem8 + EXPS + wave * 512 + S() * 256 + (lane & 15) * 4;
#pragma unroll
        for (int w = 0; w < WA; ++w) ea[S()][w] = *reinterpret_cast<const uint32_t *>(at + w * 64);
#pragma unroll
        for (int w = 0; w < WB; ++w) eb[S()][w] = *reinterpret_cast<const uint32_t *>(at + 128 + w * 64);
    };
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};

    // The products of a step from the registers of parity S.  Reads of the next step (read p at product RSTEP p / 8): B's groups in turn with A's last
    // two, then A's from the first on, each after its row group's products.  Loads two steps ahead at every NQ / 2 / NL-th product.
    constexpr int RSTEP = NQ * 13 / (NR * 2);                  // in eighths of a product: 0.8 of the step
    auto step = [&](auto S) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, (S() ^ 1)> next{};
        load_exps(S);
        read_exps(next);
        auto product = [&](auto Q) __attribute__((always_inline)) {
            constexpr int q = decltype(Q)::value, i = q / TN, j = i % 2 ? TN - 1 - q % TN : q % TN, l = q * 2 * NL / NQ;
            constexpr bool loads = l < NL && q % (NQ / (2 * NL)) == 0;
            const i32x8 &a = S() == 1 && i >= TM - 2 ? fa2[i >= TM - 2 ? i - (TM - 2) : 0] : fa[i];
            if constexpr (loads && l < TM) mfma8_load<FA, FB, i % 4, j % 4>(acc[i][j], fb[S()][j], a, eb[S()][j / 4], ea[S()][i / 4], rsA, to_a(S, l), voff, soA[l]);
            else if constexpr (loads) mfma8_load<FA, FB, i % 4, j % 4>(acc[i][j], fb[S()][j], a, eb[S()][j / 4], ea[S()][i / 4], rsB, to_b(S, l - TM), voff, soB[l - TM]);
            else mfma8<FA, FB, i % 4, j % 4>(acc[i][j], fb[S()][j], a, eb[S()][j / 4], ea[S()][i / 4]);
            constexpr int p = (q * 8 + RSTEP - 1) / RSTEP;       // the read whose turn it is
            if constexpr (p < NR && p * RSTEP / 8 == q) {
                if constexpr (p % 2 == 0) read_b(next, p / 2);
                else {
                    constexpr int g = p == 1 ? TM - 2 : p == 3 ? TM - 1 : (p - 5) / 2;
                    static_assert(p < 4 || q + 1 >= TN * (g + 1), "a row group's products come before its registers are read into");
                    read_a(next, std::integral_constant<int, g>{});
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        each(product, std::make_integer_sequence<int, NQ>{});
        go_on();
        __builtin_amdgcn_s_waitcnt(0x0070);                    // vmcnt(0) lgkmcnt(0): the step after the next has landed, the next one is in registers
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    load_step(c0);
    if (nk > 1) load_step(c1);
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    each([&](auto I) __attribute__((always_inline)) { read_a(c0, I); }, std::make_integer_sequence<int, TM>{});
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(c0, j);
    read_exps(c0);
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
    };
    pin();
    settle();
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // One loop for all steps; behind the contraction's end the descriptors are empty, so that nothing is fetched
    auto end = [&](int kt) __attribute__((always_inline)) {
        if (kt + 2 >= nk) rsA[2] = rsB[2] = 0;
    };
    for (int kt = 0;; kt += 2) {
        end(kt);
        step(c0);
        if (kt + 1 >= nk) break;
        end(kt + 1);
        step(c1);
        if (kt + 2 >= nk) break;
    }
    settle();
    pin();

    // Rows of 16 x 32 results: the two halves of a wavefront's register pairs trade places so that a lane has eight neighbours of a row.
    const int64_t row0 = (int64_t)tm * BM + wm * 16 * TM + (lane & 15), col0 = (int64_t)tn * BN + wn * 16 * TN + (lane >> 4 & 1) * 16 + (lane >> 5) * 8;
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
        const int64_t col = col0 + j * 16;
        const int left = N - col < 0 ? 0 : N - col < 8 ? (int)(N - col) : 8;
        float add[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) add[e] = bias && e < left ? bf16_bits_to_f32(bias[col + e]) : 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][j][e]), __float_as_uint(acc[i][j + 1][e]), false, false);
                v[e] = __uint_as_float(t[0]);
                v[4 + e] = __uint_as_float(t[1]);
            }
            const int64_t row = row0 + i * 16;
            if (row >= M || col >= N) continue;                // after the exchange, in which all lanes take part
            if (bias) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += add[e];
            }
            if (resid) {
                const uint4 r = *reinterpret_cast<const uint4 *>(resid + row * ldr + col);
                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
            }
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0.f;
            }
            *reinterpret_cast<uint4 *>(C + row * ldc + col) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
    }
}

template <int FA, int FB, int TM, int TN> void launch_tile(hipStream_t s, const Fp8Product &p) {
    constexpr int BM = 32 * TM, BN = 32 * TN, LDS = 2 * (BM + BN) * 128 + 4 * 512;
    static const hipError_t set = hipFuncSetAttribute((const void *)gemm_fp8_tile_k<FA, FB, TM, TN>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    (void)set;
    const int64_t tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
    gemm_fp8_tile_k<FA, FB, TM, TN><<<(unsigned)((tiles_m * tiles_n + 7) / 8 * 8), 256, LDS, s>>>(
        (const uint8_t *)p.A, (const uint8_t *)p.B, (const uint16_t *)p.bias, (const uint16_t *)p.resid, p.ldr, (uint16_t *)p.C, p.ldc, p.M, p.N, p.K, (int)tiles_m,
        (int)tiles_n);
}

template <int FA, int FB, typename T> void launch(hipStream_t s, const Fp8Product &p) {
#define TIO_DIRECT(TM, TN)                                                                                                                              \
    do {                                                                                                                                                \
        const int64_t tiles_m = (p.M + 16 * TM - 1) / (16 * TM), tiles_n = (p.N + 16 * TN - 1) / (16 * TN);                                             \
        gemm_fp8_direct_k<FA, FB, T, TM, TN><<<(unsigned)(tiles_m * tiles_n), 256, 0, s>>>(                                                             \
            (const uint8_t *)p.A, (const uint8_t *)p.B, (const T *)p.bias, (const T *)p.resid, p.ldr, (T *)p.C, p.ldc, p.M, p.N, p.K, (int)tiles_n); \
    } while (0)
    if (sizeof(T) == 2 && p.M > 256 && p.N > 256) return launch_tile<FA, FB, 8, 8>(s, p);
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
