// Products of matrices stored in 8-bit floating point with a power of two for each block of 128 (fp8_blocks.h):
// C[M,N] = A[M,K] . B[N,K]^T (+ bias[N]) (+ resid[M,N]).
//
// bf16 results: v_mfma_scale_f32_16x16x128_f8f6f4, one instruction for a block of 128 of 16 rows and 16 columns, which applies both operands' powers of two
// itself.  Measured on it: the accumulator is exact to 24 bits, but of the products of eight neighbours the bits below 2^-13 of the largest are cut off:
// errors of 1.2e-5 of the result's norm on normal values, a hundredth of what the rounding to bf16 leaves.  fp32 results need more, so there the codes
// become bf16 numbers, exactly, whose products and sums are those of 32 bits (error 4e-8).
//
// Bound, large products: the power limit with operands in the caches (8192^3 350 us, 3.1 PFLOP/s at 2.0 GHz; zeros 3.4; the instruction alone 4.0; 8192 x 11008 x 4096
// 278 us), memory without (400 and 306 us, 2.7 and 2.4 PFLOP/s, of the latter some 40 us its stores, which nothing overlaps; a large library product of plain 8-bit matrices
// 2.1 to 2.7).  A bias or residual takes the way out in 32 bits (8192 x 4096 x 4096 109 us, with both 162, of which 13 are the residual's bytes).
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "../../include/teraio.h"
#include "device_common.h"
#include "fp8_blocks.h"
#include "kernels.h"
#include "mfma_tiles.h"
#include "rows8.h"

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

// A workgroup's tile of 16 TM x 16 TN results, for products of few rows or few tiles: its NW wavefronts share the contraction, their sums are added in order.
template <int FA, int FB, typename T, int TM, int TN, int NW>
__global__ void __launch_bounds__(NW * 64) gemm_fp8_direct_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const T *__restrict__ bias,
                                                         const T *resid, int64_t ldr, T *C, int64_t ldc, int64_t M, int64_t N,
                                                         int64_t K, int tiles_n) {
    __shared__ float sums[NW][TM * TN][256];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int64_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
    const Fp8Shape sa{M, K}, sb{N, K};
    const int64_t KB = sa.kb(), ga = sa.groups(), gb = sb.groups();
    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    const uint8_t *fa[TM], *ea[TM], *fb[TN], *eb[TN];          // block 0 of each group; past the last one: the last
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t g = tm * TM + i < ga ? tm * TM + i : ga - 1;
        fa[i] = A + g * KB * F8_FRAG;
        ea[i] = A + sa.code_bytes() + (g >> 2) * KB * 64 + (g & 3);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t g = tn * TN + j < gb ? tn * TN + j : gb - 1;
        fb[j] = B + g * KB * F8_FRAG;
        eb[j] = B + sb.code_bytes() + (g >> 2) * KB * 64 + (g & 3);
    }
    // U blocks' loads before the first one's products: one after the other a wavefront waits for each (16 x 4096 x 11008, operands in no cache: 16.6 us, with
    // eight wavefronts of four at once 11.2); larger tiles have as many bytes on their way for one block.  None are while a wavefront multiplies: others cover that,
    // or nothing does (64 x 4096 x 11008 16.4 us, of which the matrix from HBM is 8.8)
    constexpr int U = TM * TN > 2 ? 1 : TM * TN == 2 ? (sizeof(T) == 2 ? 4 : 2) : NW == 8 ? 4 : 2;
    for (int64_t kb = wave; kb < KB; kb += NW * U) {
        Piece8 a[U][TM], b[U][TN];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = kb + NW * u;
            if (at >= KB) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i) a[u][i].load(fa[i] + at * F8_FRAG, ea[i] + at * 64, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[u][j].load(fb[j] + at * F8_FRAG, eb[j] + at * 64, lane);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb + NW * u >= KB) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = sizeof(T) == 2 ? product8<FA, FB>(a[u][i], b[u][j], acc[i][j]) : product16<FA, FB>(a[u][i], b[u][j], acc[i][j]);
        }
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
            if (tid >= 256 || m >= M || n >= (N + 7) / 8 * 8) continue;
            float v = sums[0][i * TN + j][at];
#pragma unroll
            for (int w = 1; w < NW; ++w) v += sums[w][i * TN + j][at];
            if (bias && n < N) v += element(bias + n);
            if (resid && n < N) v += element(resid + m * ldr + n);
            C[m * ldc + n] = from_f32<T>(n < N ? v : 0.f);
        }
}

// Eight neighbours of a row of results on their way out: bias and residual added in 32 bits, zeros behind the last column, rounded once.
template <typename T> struct Out8 {
    float add[8];
    int left;                                                  // columns that are there
    __device__ __forceinline__ Out8(const T *bias, int64_t col, int64_t N) : left(N - col < 0 ? 0 : N - col < 8 ? (int)(N - col) : 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) add[e] = bias && e < left ? to_f32(bias[col + e]) : 0.f;
    }
    __device__ __forceinline__ void put(float (&v)[8], const T *resid, T *to) const {
        if (resid) {
            Row8<T> r;
            r.load(resid);
            float f[8];
            r.get(f);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += f[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += add[e];
        cut8(v, left);
        Row8<T> r;
        r.set(v);
        r.store(to);
    }
};
// The sums of a cut contraction, [range][M][N rounded up to 8] in 32 bits, added in the ranges' order
template <typename T>
__global__ void __launch_bounds__(256) gemm_fp8_sums_k(const float *__restrict__ ws, int nsplit, const T *__restrict__ bias, const T *resid, int64_t ldr, T *C,
                                                       int64_t ldc, int64_t M, int64_t N) {
    const int64_t per = (N + 7) / 8, idx = (int64_t)blockIdx.x * 256 + threadIdx.x, row = idx / per, col = (idx - row * per) * 8;
    if (row >= M) return;
    const float *from = ws + idx * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < nsplit; ++i, from += M * per * 8) {
        const float4 a = *reinterpret_cast<const float4 *>(from), b = *reinterpret_cast<const float4 *>(from + 4);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    Out8<T>(bias, col, N).put(v, resid ? resid + row * ldr + col : nullptr, C + row * ldc + col);
}

// A wavefront's 16 TM x 16 TN results, from row mw and column nw on, 16 rows at a time through LDS (`stage`: STAGE bytes of its own), since a store or load
// whose neighbouring lanes are neighbours in memory moves 64 bytes a clock, one whose neighbouring lanes are in different rows, as the products leave their
// results, 16 (with operands and outputs that are in no cache 11008 x 4096 x 8192 287 -> 277 us, 8192 x 22016 x 768 173 -> 169).  Rows are rotated in LDS by an exclusive or with the row number, so that sixteen lanes
// write to different banks.  Outputs of 64 MiB and more go past the caches, which they would push the operands out of (8192 x 11008 x 4096
// 330 -> 321 us).
template <int TN> constexpr int stage_bytes() { return 64 * 64 * TN; }
template <typename T, int TM, int TN>
__device__ __forceinline__ void store_part(floatx4 (&acc)[TM][TN], unsigned char *stage, int lane, int64_t mw, int64_t nw, int64_t M, int64_t N,
                                           const T *__restrict__ bias, const T *resid, int64_t ldr, T *C, int64_t ldc, float *ws, int split, int nsplit) {
    const int r16 = lane & 15, g4 = lane >> 4;
    if (sizeof(T) == 2 && nsplit == 1 && !bias && !resid && mw + 16 * TM <= M && nw + 16 * TN <= N) {
        // As bf16: the two halves of register pairs trade places so that a lane has eight neighbours of a row.
        constexpr int CHUNKS = 2 * TN;                         // of eight results, to a row
        auto turn = [](int row) __attribute__((always_inline)) { return CHUNKS == 16 ? row : CHUNKS == 8 ? row >> 1 & 7 : row >> 2 & 3; };
        auto whole = [&](auto STREAM) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                unsigned char *const at = stage + (i & 1) * 16 * CHUNKS * 16;
                int l = lane;
                asm volatile("" : "+v"(l));                    // addresses are found anew: all blocks' at once would take more registers than there are
#pragma unroll
                for (int j = 0; j < TN; j += 2) {
                    float v[8];
                    // not found before the choice of STREAM, in which both ways would have all results in registers
                    if constexpr (STREAM()) asm volatile("; past the caches" : "+v"(acc[i][j]), "+v"(acc[i][j + 1]));
                    else asm volatile("; kept" : "+v"(acc[i][j]), "+v"(acc[i][j + 1]));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][j][e]), __float_as_uint(acc[i][j + 1][e]), false, false);
                        v[e] = __uint_as_float(t[0]);
                        v[4 + e] = __uint_as_float(t[1]);
                    }
                    *reinterpret_cast<uint4 *>(at + (r16 * CHUNKS + ((j * 2 + (g4 & 1) * 2 + (g4 >> 1)) ^ turn(r16))) * 16) =
                        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int p = 0; p < CHUNKS / 4; ++p) {
                    const int row = (p * 64 + l) / CHUNKS, chunk = l % CHUNKS;
                    Row8<bf16_t> out;
                    out.v.raw = *reinterpret_cast<const uint4 *>(at + (row * CHUNKS + (chunk ^ turn(row))) * 16);
                    bf16_t *const to = (bf16_t *)C + (mw + i * 16 + row) * ldc + nw + chunk * 8;
                    if constexpr (STREAM()) out.put(to);
                    else out.store(to);
                }
                __builtin_amdgcn_wave_barrier();
            }
        };
        if (M * N * (int64_t)sizeof(T) >= (int64_t)64 << 20) whole(std::true_type{});
        else whole(std::false_type{});
        return;
    }
    // As fp32, for sums of ranges, bias, residual and edges, 64 rows at a time; a loop, since straight-line code for what few wavefronts run has to be
    // fetched by them alone.
    constexpr int QUADS = 4 * TN;                              // of four results, to a row
    auto quad = [&](int row, int q) __attribute__((always_inline)) { return reinterpret_cast<float4 *>(stage + (row * QUADS + (q ^ (QUADS == 8 ? row >> 1 & 7 : row & 15))) * 16); };
    auto rows64 = [&](auto FIRST) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const floatx4 &t = acc[FIRST() + i][j];
                *quad(i * 16 + r16, j * 4 + g4) = make_float4(t[0], t[1], t[2], t[3]);
            }
        __builtin_amdgcn_wave_barrier();
        const int64_t m0 = mw + FIRST() * 16, N8 = (N + 7) / 8 * 8;
        if (nsplit > 1) {
            const int q = lane % QUADS;
            const int64_t n = nw + q * 4;
#pragma unroll 4
            for (int row = lane / QUADS; row < 64; row += 64 / QUADS)
                if (m0 + row < M && n < N8) *reinterpret_cast<float4 *>(ws + ((int64_t)split * M + m0 + row) * N8 + n) = *quad(row, q);
        } else {
            const int q = lane % (QUADS / 2) * 2;
            const int64_t n = nw + q * 4;
            const Out8<T> out(bias, n, N);
#pragma unroll 2
            for (int row = lane / (QUADS / 2); row < 64; row += 128 / QUADS) {
                if (m0 + row >= M || n >= N) continue;
                const float4 a = *quad(row, q), b = *quad(row, q + 1);
                float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                out.put(v, resid ? resid + (m0 + row) * ldr + n : nullptr, C + (m0 + row) * ldc + n);
            }
        }
        __builtin_amdgcn_wave_barrier();
    };
    static_assert(TM == 4 || TM == 8, "64 rows, once or twice");
    rows64(std::integral_constant<int, 0>{});
    if constexpr (TM == 8) rows64(std::integral_constant<int, 4>{});
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

// The loads of a tile of 32 TM x 32 TN results by four wavefronts: both operands' fragments from memory straight into LDS, D steps (blocks of 128 of the
// contraction) deep, and the exponents of each wavefront's rows and columns, a 4-byte load to LDS a step (lanes 0 .. 31 A's, the others B's).  Wavefronts are two
// by two, or with STRIPS side by side in a tile of 64 rows.
template <int TM, int TN, int D, bool STRIPS = false> struct Loads {
    static constexpr int BM = 32 * TM, BN = 32 * TN, TILE_A = BM * 128, TILE_B = BN * 128;
    static constexpr int WA = TM / 4, WB = TN / 4;             // words of exponents a lane has (64 rows each)
    static constexpr uint32_t EXPS = D * (TILE_A + TILE_B), LDS = EXPS + 4 * D * 256;
    static constexpr int PER = TM + TN + 1;                    // loads of a wavefront for a step
    i32x4 rsA, rsB;
    // 1 KiB pieces of a step: half h of group g is piece 2 g + h, and wavefront p % 4's; groups past the last one repeat it
    uint32_t soA[TM], soB[TN], lds0, ahead, voff;              // ahead: the step whose loads are next (the last one again when there is none); voff: its codes
    const uint8_t *exps;
    int wave, lane, nk;
    __device__ __forceinline__ Loads(const uint8_t *A, const uint8_t *B, int64_t M, int64_t N, int64_t K, int tm, int tn, int kb0, int steps, int w, int l,
                                     const unsigned char *smem)
        : ahead(0), voff(l * 16), wave(w), lane(l), nk(steps) {
        const Fp8Shape sa{M, K}, sb{N, K};
        const int64_t KB = sa.kb(), ga0 = (int64_t)tm * (2 * TM), gb0 = (int64_t)tn * (2 * TN);
        const int64_t atA = (ga0 * KB + kb0) * F8_FRAG, atB = (gb0 * KB + kb0) * F8_FRAG, roomA = sa.code_bytes() - atA, roomB = sb.code_bytes() - atB;
        rsA = make_rsrc(A + atA, roomA < 0xfffffff0 ? (uint32_t)roomA : 0xfffffff0u);
        rsB = make_rsrc(B + atB, roomB < 0xfffffff0 ? (uint32_t)roomB : 0xfffffff0u);
        const int lastA = (int)(sa.groups() - 1 - ga0), lastB = (int)(sb.groups() - 1 - gb0);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int p = i * 4 + wave, g = p >> 1;
            soA[i] = __builtin_amdgcn_readfirstlane((uint32_t)((g < lastA ? g : lastA) * (int)KB * F8_FRAG + (p & 1) * 1024));
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int p = i * 4 + wave, g = p >> 1;
            soB[i] = __builtin_amdgcn_readfirstlane((uint32_t)((g < lastB ? g : lastB) * (int)KB * F8_FRAG + (p & 1) * 1024));
        }
        const bool isB = lane >= 32;
        const int64_t most = isB ? (N - 1) / 64 : (M - 1) / 64,
                      g = STRIPS ? (isB ? (int64_t)tn * 2 + (wave >> 1) : tm)
                               : (isB ? (int64_t)tn * (2 * WB) + (wave & 1) * WB : (int64_t)tm * (2 * WA) + (wave >> 1) * WA) + (lane >> 4 & 1);
        exps = (isB ? B + sb.code_bytes() : A + sa.code_bytes()) + ((g < most ? g : most) * KB + kb0) * 64 + (lane & 15) * 4;
        lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
    }
    // where piece i of a step goes, in part S of LDS
    __device__ __forceinline__ uint32_t to_a(int S, int i) const { return lds0 + S * TILE_A + (i * 4 + wave) * 1024; }
    __device__ __forceinline__ uint32_t to_b(int S, int i) const { return lds0 + D * TILE_A + S * TILE_B + (i * 4 + wave) * 1024; }
    __device__ __forceinline__ void load_exps(int S) const { load_to_lds_b32(exps + ahead * 64, lds0 + EXPS + (wave * D + S) * 256); }
    __device__ __forceinline__ void go_on() {
        ahead = ahead + 1 < (uint32_t)nk ? ahead + 1 : (uint32_t)nk - 1;
        voff = lane * 16 + ahead * F8_FRAG;
    }
    // there_is false: the counters' loads, but nothing is fetched
    __device__ __forceinline__ void load_step(int S, bool there_is = true) {
        i32x4 a = rsA, b = rsB;
        if (!there_is) a[2] = b[2] = 0;
#pragma unroll
        for (int i = 0; i < TM; ++i) load_to_lds_b128(a, to_a(S, i), voff, soA[i]);
#pragma unroll
        for (int i = 0; i < TN; ++i) load_to_lds_b128(b, to_b(S, i), voff, soB[i]);
        load_exps(S);
        go_on();
    }
};

// f of each number as a constant
template <typename F, int... I> __device__ __forceinline__ void each(const F &f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }

// Waits until no more than LOADS of the wavefront's loads are on their way and all that it has read from LDS is in registers, then for the workgroup's other
// wavefronts, whose loads may write from then on where it has read.  The compiler orders reads of LDS with neither the wait nor the barrier, and one whose value is used
// only behind them might move there: so no access to memory moves over either end.
template <int LOADS> __device__ __forceinline__ void meet() {
    static_assert(LOADS < 64, "loads in flight fit the counter");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (LOADS & 15) | ((LOADS >> 4) << 14));       // vmcnt(LOADS) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A tile of 32 TM x 32 TN results: four wavefronts, 16 TM x 16 TN each.  A step of the contraction is one block of 128: TM TN products of 32 clocks.
//  * Fragments are stored as the products take them, so that LDS is written and read in consecutive KiB.
//  * While the products of a step run, all fragments of the next one are read into registers: B's into a second set, A's into the registers of the row
//    group whose products are done, but for the last two groups, which have a second set too.  So a step's LDS is free when its products begin, and
//    the loads for the step D later go there in their first half; with D = 2 they have the other half, at least, to land.
//  * One wavefront per SIMD (256 x 256) hides nothing by switching, so the order of all of it is pinned.
template <int FA, int FB, int TM, int TN, int D>
__global__ void __launch_bounds__(256)
    gemm_fp8_tile_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const bf16_t *__restrict__ bias, const bf16_t *resid, int64_t ldr, bf16_t *C, int64_t ldc,
                    int64_t M, int64_t N, int64_t K, int tiles_m, int tiles_n, float *__restrict__ ws) {
    using L = Loads<TM, TN, D>;
    constexpr int BM = L::BM, BN = L::BN, TILE_A = L::TILE_A, TILE_B = L::TILE_B, NQ = TM * TN, NR = TM + TN, NL = TM + TN, WA = L::WA, WB = L::WB;
    constexpr uint32_t EXPS = L::EXPS;
    static_assert(D % 2 == 0, "a step's registers go by its parity");
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem8[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
    int split, nsplit, tm, tn;
    if (!place(tiles_m, tiles_n, 0, split, nsplit, tm, tn)) return;
    const int KB = (int)Fp8Shape{M, K}.kb(), kb0 = (int)((int64_t)KB * split / nsplit), nk = (int)((int64_t)KB * (split + 1) / nsplit) - kb0;
    L in(A, B, M, N, K, tm, tn, kb0, nk, wave, lane, smem8);

    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};

    i32x8 fa[TM], fa2[2], fb[2][TN];                           // fa2: of the last two row groups in odd steps
    uint32_t ea[2][WA], eb[2][WB];
    auto read_frag = [&](uint32_t at) __attribute__((always_inline)) {
        const uint4 u = *reinterpret_cast<const uint4 *>(smem8 + at + lane * 16), v = *reinterpret_cast<const uint4 *>(smem8 + at + 1024 + lane * 16);
        return (i32x8){(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
    };
    // S: the step modulo D, whose part of LDS it is in; its parity says which registers
    auto read_a = [&](auto S, auto I) __attribute__((always_inline)) {
        const i32x8 f = read_frag(S() * TILE_A + (wm * TM + I()) * F8_FRAG);
        if constexpr (S() % 2 == 1 && I() >= TM - 2) fa2[I() - (TM - 2)] = f;
        else fa[I()] = f;
    };
    auto read_b = [&](auto S, int j) __attribute__((always_inline)) { fb[S() % 2][j] = read_frag(D * TILE_A + S() * TILE_B + (wn * TN + j) * F8_FRAG); };
    auto read_exps = [&](auto S) __attribute__((always_inline)) {
        const unsigned char *const at = smem8 + EXPS + (wave * D + S()) * 256 + (lane & 15) * 4;
#pragma unroll
        for (int w = 0; w < WA; ++w) ea[S() % 2][w] = *reinterpret_cast<const uint32_t *>(at + w * 64);
#pragma unroll
        for (int w = 0; w < WB; ++w) eb[S() % 2][w] = *reinterpret_cast<const uint32_t *>(at + 128 + w * 64);
    };
    constexpr std::integral_constant<int, 0> c0{};

    // The products of a step from the registers of parity S.  Reads of the next step (read p at product RSTEP p / 8): B's groups in turn with A's last
    // two, then A's from the first on, each after its row group's products.  Loads D steps ahead at every NQ / 2 / NL-th product.
    constexpr int RSTEP = NQ * 13 / (NR * 2);                  // in eighths of a product: 0.8 of the step
    auto step = [&](auto S) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, (S() + 1) % D> next{};
        constexpr int P = S() % 2;
        in.load_exps(S());
        read_exps(next);
        auto product = [&](auto Q) __attribute__((always_inline)) {
            constexpr int q = decltype(Q)::value, i = q / TN, j = i % 2 ? TN - 1 - q % TN : q % TN, l = q * 2 * NL / NQ;
            constexpr bool loads = l < NL && q % (NQ / (2 * NL)) == 0;
            const i32x8 &a = P == 1 && i >= TM - 2 ? fa2[i >= TM - 2 ? i - (TM - 2) : 0] : fa[i];
            if constexpr (loads && l < TM) mfma8_load<FA, FB, i % 4, j % 4>(acc[i][j], fb[P][j], a, eb[P][j / 4], ea[P][i / 4], in.rsA, in.to_a(S(), l), in.voff, in.soA[l]);
            else if constexpr (loads) mfma8_load<FA, FB, i % 4, j % 4>(acc[i][j], fb[P][j], a, eb[P][j / 4], ea[P][i / 4], in.rsB, in.to_b(S(), l - TM), in.voff, in.soB[l - TM]);
            else mfma8<FA, FB, i % 4, j % 4>(acc[i][j], fb[P][j], a, eb[P][j / 4], ea[P][i / 4]);
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
        in.go_on();
        meet<(D - 2) * L::PER>();                              // the step after the next has landed, the next one is in registers
        __builtin_amdgcn_sched_barrier(0);
    };

#pragma unroll
    for (int t = 0; t < D; ++t) in.load_step(t);
    meet<(D - 2) * L::PER>();
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
    meet<(D - 2) * L::PER>();
    __builtin_amdgcn_sched_barrier(0);
    // One loop for all steps; behind the contraction's end the descriptors are empty, so that nothing is fetched
    int kt = 0;
    auto done = [&](auto S) __attribute__((always_inline)) {
        if (kt + D >= nk) in.rsA[2] = in.rsB[2] = 0;
        step(S);
        return ++kt >= nk;
    };
    if constexpr (D == 2) {
        while (!done(c0) && !done(std::integral_constant<int, 1>{})) {}
    } else {
        static_assert(D == 4, "steps of the loop");
        while (!done(c0) && !done(std::integral_constant<int, 1>{}) && !done(std::integral_constant<int, 2>{}) && !done(std::integral_constant<int, 3>{})) {}
    }
    meet<0>();                                                 // nothing is on its way to LDS any more, for any wavefront: it takes the results
    settle();
    pin();

    static_assert(4 * stage_bytes<TN>() <= (int)L::EXPS, "the results' places fit the fragments'");
    store_part<bf16_t, TM, TN>(acc, smem8 + wave * stage_bytes<TN>(), lane, (int64_t)tm * BM + wm * 16 * TM, (int64_t)tn * BN + wn * 16 * TN, M, N, bias, resid,
                               ldr, C, ldc, ws, split, nsplit);
}

using StripLoads = Loads<2, 4, 3, true>;

// Tiles of 64 x 128 for products of some hundred rows or columns, which have too few tiles of 128 x 128 for all compute units (512 x 4096 x 11008 50 -> 39 us,
// 128 x 11008 x 4096 23 -> 18.8): each wavefront has all rows and 32 columns.  A step's fragments have a second set of registers, but the compiler
// puts their reads behind most or all products of the step before: it is two workgroups to a compute unit that cover each other's waits (six steps deep and one to a
// unit: 40 and 20 us).
template <int FA, int FB>
__global__ void __launch_bounds__(256, 2)
    gemm_fp8_strip_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const bf16_t *__restrict__ bias, const bf16_t *resid, int64_t ldr, bf16_t *C, int64_t ldc,
                     int64_t M, int64_t N, int64_t K, int tiles_m, int tiles_n, float *__restrict__ ws) {
    constexpr int D = 3;
    constexpr int TM = 4, TN = 2;                              // a wavefront's
    using L = StripLoads;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem8[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    int split, nsplit, tm, tn;
    if (!place(tiles_m, tiles_n, 0, split, nsplit, tm, tn)) return;
    const int KB = (int)Fp8Shape{M, K}.kb(), kb0 = (int)((int64_t)KB * split / nsplit), nk = (int)((int64_t)KB * (split + 1) / nsplit) - kb0;
    L in(A, B, M, N, K, tm, tn, kb0, nk, wave, lane, smem8);
    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    struct Step {
        i32x8 a[TM], b[TN];
        uint32_t ea, eb;
    };
    auto read = [&](Step &f, int S) __attribute__((always_inline)) {
        auto frag = [&](uint32_t at) __attribute__((always_inline)) {
            const uint4 u = *reinterpret_cast<const uint4 *>(smem8 + at + lane * 16), v = *reinterpret_cast<const uint4 *>(smem8 + at + 1024 + lane * 16);
            return (i32x8){(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
        };
        const unsigned char *const e = smem8 + L::EXPS + (wave * D + S) * 256 + (lane & 15) * 4;
        f.ea = *reinterpret_cast<const uint32_t *>(e);
        f.eb = *reinterpret_cast<const uint32_t *>(e + 128) >> (wave & 1) * 16;
#pragma unroll
        for (int j = 0; j < TN; ++j) f.b[j] = frag(D * L::TILE_A + S * L::TILE_B + (wave * TN + j) * F8_FRAG);
#pragma unroll
        for (int i = 0; i < TM; ++i) f.a[i] = frag(S * L::TILE_A + i * F8_FRAG);
    };
    auto product = [&](const Step &f, auto I, auto J) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value, j = decltype(J)::value;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f.b[j], f.a[i], acc[i][j], FB, FA, j, (int)f.eb, i, (int)f.ea);
    };
    auto products = [&](const Step &f) __attribute__((always_inline)) {
        each([&](auto I) __attribute__((always_inline)) {
            each([&](auto J) __attribute__((always_inline)) { product(f, I, J); }, std::make_integer_sequence<int, TN>{});
        }, std::make_integer_sequence<int, TM>{});
    };
#pragma unroll
    for (int t = 0; t < D; ++t) in.load_step(t);
    meet<(D - 1) * L::PER>();
    Step even, odd;
    int S = 0, kt = 0;
    read(even, 0);
    // the products of step kt, whose fragments are `now`
    auto step = [&](const Step &now, Step &next) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        meet<(D - 2) * L::PER>();                              // the next step has landed, and this one is in registers
        in.load_step(S, kt + D < nk);
        S = S + 1 < D ? S + 1 : 0;
        read(next, S);
        products(now);
        return ++kt >= nk;
    };
    while (!step(even, odd) && !step(odd, even)) {}
    meet<0>();                                                 // nothing is on its way to LDS any more, for any wavefront: it takes the results
    static_assert(4 * stage_bytes<TN>() <= (int)L::EXPS, "the results' places fit the fragments'");
    store_part<bf16_t, TM, TN>(acc, smem8 + wave * stage_bytes<TN>(), lane, (int64_t)tm * 64, (int64_t)tn * 128 + wave * 32, M, N, bias, resid, ldr, C, ldc, ws, split,
                               nsplit);
}

// ---- in fp32: the values, which bf16 holds exactly, in 16-bit products, whose sums are those of 32-bit arithmetic.  A quarter to half of the 8-bit products' rate.
// 128 x 128 results; two workgroups to a compute unit cover each other's conversions and loads.
template <int FA, int FB>
__global__ void __launch_bounds__(256, 2)
    gemm_fp8_tile32_k(const uint8_t *__restrict__ A, const uint8_t *__restrict__ B, const float *__restrict__ bias, const float *resid, int64_t ldr, float *C, int64_t ldc,
                      int64_t M, int64_t N, int64_t K, int tiles_m, int tiles_n, float *__restrict__ ws) {
    constexpr int TM = 4, TN = 4;
    using L = Loads<TM, TN, 2>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem8[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
    int split, nsplit, tm, tn;
    if (!place(tiles_m, tiles_n, 0, split, nsplit, tm, tn)) return;
    const int KB = (int)Fp8Shape{M, K}.kb(), kb0 = (int)((int64_t)KB * split / nsplit), nk = (int)((int64_t)KB * (split + 1) / nsplit) - kb0;
    L in(A, B, M, N, K, tm, tn, kb0, nk, wave, lane, smem8);
    floatx4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    auto piece = [&](uint32_t at, uint32_t word, int byte) __attribute__((always_inline)) {
        Piece8 p;
        p.h[0] = *reinterpret_cast<const uint4 *>(smem8 + at + lane * 16);
        p.h[1] = *reinterpret_cast<const uint4 *>(smem8 + at + 1024 + lane * 16);
        p.e = word >> (8 * byte) & 255u;
        return p;
    };
    in.load_step(0);
    for (int kt = 0; kt < nk; ++kt) {
        const int S = kt & 1;
        meet<0>();                                             // this step has landed, and the one before is in registers
        if (kt + 1 < nk) in.load_step(S ^ 1);
        const unsigned char *const e = smem8 + L::EXPS + (wave * 2 + S) * 256 + (lane & 15) * 4;
        const uint32_t ea = *reinterpret_cast<const uint32_t *>(e), eb = *reinterpret_cast<const uint32_t *>(e + 128);
        bf16x8 b[TN][4];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const Piece8 p = piece(2 * L::TILE_A + S * L::TILE_B + (wn * TN + j) * F8_FRAG, eb, j);
#pragma unroll
            for (int q = 0; q < 4; ++q) b[j][q] = p.template values<FB>(q);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const Piece8 p = piece(S * L::TILE_A + (wm * TM + i) * F8_FRAG, ea, i);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bf16x8 a = p.template values<FA>(q);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][q], a, acc[i][j], 0, 0, 0);
            }
        }
    }
    meet<0>();                                                 // every wavefront is done with the fragments: LDS takes the results
    store_part<float, TM, TN>(acc, smem8 + wave * stage_bytes<TN>(), lane, (int64_t)tm * L::BM + wm * 16 * TM, (int64_t)tn * L::BN + wn * 16 * TN, M, N, bias, resid, ldr, C, ldc, ws, split, nsplit);
}

// How a product is taken: tiles of 64 x 128, 128 x 128 or 256 x 256 through LDS, `deep` steps at a time, the contraction cut into ranges, or (deep 1) smaller ones from the
// caches, the contraction cut into the shares of four or eight wavefronts (gemm_fp8_direct_k).
//
// The least of an estimate of the time.  The large tiles' constants were fitted to 39 products, each taken in all ways: a workgroup's steps and its beginning and
// end (us), times the rounds of workgroups, and the sums of the ranges.  A step of a 128 tile is mostly waiting for loads where a compute unit has one
// such tile: 0.32 us four steps deep (0.44 where all units work), two deep 0.6, but two tiles to a unit share 0.88.  us, 768 x 768 x 8192 in one range: 26.9 four
// deep, 41.4 two deep, 69.8 in 256 tiles, and 19.1 in three ranges; 8192 x 768 x 768: 13.3, 10.8, 15.5; 8192 x 11008 x 4096: 380, 330, 288 (all with operands in the caches; without 455, 379, 323).  The small ones' were
// fitted to 380 products with B in no cache, so that the choice is 1.6 % behind the best way on average (7 % with tiles of 16 x 16 and 32 x 32 by four wavefronts
// alone): the larger of a wavefront's chain of steps, in rounds of workgroups, and the bytes from the caches.  us, bf16: 32 x 4096 x 11008: 18.4 in 32 x 32 by
// four wavefronts, in 32 x 16 by eight 13.9, in 16 x 16 16.0; 64 x 4096 x 11008: 18.2 in 32 x 32 by four, by eight 16.4; 256 x 4096 x 4096: 21.7 in 128 x 128,
// in 64 x 32 15.2, in 32 x 32 by eight 17.0; 1024 x 1000 x 1000: 8.2 in 128 x 128, 6.6 in 32 x 32 by four, by eight 7.2.  64 x 128 tiles' were fitted to 140 more (1.7 % behind the best way on
// average, 4.6 % without them).
struct Route {
    int rows, cols, deep, splits;                              // splits: ranges, or wavefronts that share a contraction
};
Route route(bool bf16, int64_t M, int64_t N, int64_t K) {
    constexpr double UNITS = 256;                              // compute units
    const int64_t KB = (K + F8_BLOCK - 1) / F8_BLOCK;
    // eight wavefronts where each has two blocks or more: 4 x 32000 x 4096 27.6 -> 25.4 us, 1 x 50256 x 768 8.6 -> 13
    if (M <= 16) return {16, 16, 1, KB > 15 ? 8 : 4};
    Route best{};
    double least = 1e300;
    auto tiles = [&](int rows, int cols) { return (double)((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
    auto take = [&](double t, Route r) {
        if (t < least) least = t, best = r;
    };
    auto small = [&](int rows, int cols, int waves, double step, int per_unit, double per_us, double each) {
        const double groups = tiles(rows, cols), chain = step * (double)((KB + waves - 1) / waves) * std::ceil(groups / (UNITS * per_unit));
        if (groups * waves * 64 >= 4294967296.0) return;       // threads that a launch may have
        take(2.0 + std::max(chain, groups * KB * (rows + cols) * 128 / per_us + groups * each), {rows, cols, 1, waves});
    };
    small(16, 16, 4, 0.17, 4, 17e6, 0.00016);
    small(16, 16, 8, 0.30, 2, 22e6, 0.00093);
    small(32, 16, 8, 0.42, 1, 20.5e6, 0.0014);
    small(32, 32, 4, 0.58, 2, 18e6, 0.0006);
    small(32, 32, 8, 0.80, 1, 18.5e6, 0.00106);
    small(64, 32, 8, 1.2, 1, 18e6, 0.0046);
    auto large = [&](int rows, int cols, int deep, int most, int per_unit, double step, double busy, double ends) {
        for (int splits = 1; splits <= most && splits <= KB; ++splits) {
            const double groups = tiles(rows, cols) * splits, full = std::min(1.0, groups / UNITS);
            if (per_unit > 1 && groups <= UNITS) continue;
            double t = std::ceil(groups / (UNITS * per_unit)) * ((KB + splits - 1) / splits * (step + busy * full) + ends);
            if (splits > 1) t += 3.0 + (double)M * N * 8 * (splits + 0.5) / 3.5e6;
            take(t, {rows, cols, deep, splits});
        }
    };
    if (bf16) {
        large(256, 256, 2, 16, 1, 1.06, 0.28, 5.0);
        large(128, 128, 2, 16, 2, 0.88, 0.0, 4.0);
        large(128, 128, 2, 1, 1, 0.60, 0.0, 4.2);
        large(128, 128, 4, 32, 1, 0.32, 0.12, 5.0);
        large(64, 128, 3, 8, 1, 0.25, 0.08, 3.8);
        large(64, 128, 3, 1, 2, 0.50, 0.0, 4.4);
    } else {
        large(128, 128, 2, 16, 2, 1.8, 0.0, 4.0);
        large(128, 128, 2, 32, 1, 1.05, 0.0, 4.6);
    }
    return best;
}

// more LDS than a launch has without asking; asked for once for each kernel
template <auto KERNEL, uint32_t LDS> void allow_lds() {
    static const hipError_t allowed = hipFuncSetAttribute((const void *)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS);
    (void)allowed;
}

template <int FA, int FB, typename T> void launch(hipStream_t s, const Fp8Product &p) {
    const Route r = route(sizeof(T) == 2, p.M, p.N, p.K);
    const T *const bias = (const T *)p.bias, *const resid = (const T *)p.resid;
    const uint8_t *const A = (const uint8_t *)p.A, *const B = (const uint8_t *)p.B;
    const int tiles_m = (int)((p.M + r.rows - 1) / r.rows), tiles_n = (int)((p.N + r.cols - 1) / r.cols);
    if (r.deep == 1) {
        auto direct = [&](auto TM, auto TN, auto NW) {
            if (r.rows != 16 * TM() || r.cols != 16 * TN() || r.splits != NW()) return;
            gemm_fp8_direct_k<FA, FB, T, TM(), TN(), NW()><<<(unsigned)((int64_t)tiles_m * tiles_n), NW() * 64, 0, s>>>(A, B, bias, resid, p.ldr, (T *)p.C, p.ldc, p.M,
                                                                                                                    p.N, p.K, tiles_n);
        };
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        using Four = std::integral_constant<int, 4>;
        using Eight = std::integral_constant<int, 8>;
        direct(One{}, One{}, Four{});
        direct(One{}, One{}, Eight{});
        direct(Two{}, One{}, Eight{});
        direct(Two{}, Two{}, Four{});
        direct(Two{}, Two{}, Eight{});
        direct(Four{}, Two{}, Eight{});
        return;
    }
    const dim3 grid((unsigned)(((int64_t)tiles_m * tiles_n + 7) / 8 * 8), (unsigned)r.splits);
    auto go = [&](auto kernel, uint32_t lds) { kernel<<<grid, 256, lds, s>>>(A, B, bias, resid, p.ldr, (T *)p.C, p.ldc, p.M, p.N, p.K, tiles_m, tiles_n, (float *)p.work); };
    if constexpr (sizeof(T) == 2) {
        if (r.rows == 256) allow_lds<gemm_fp8_tile_k<FA, FB, 8, 8, 2>, Loads<8, 8, 2>::LDS>(), go(gemm_fp8_tile_k<FA, FB, 8, 8, 2>, Loads<8, 8, 2>::LDS);
        else if (r.rows == 64) allow_lds<gemm_fp8_strip_k<FA, FB>, StripLoads::LDS>(), go(gemm_fp8_strip_k<FA, FB>, StripLoads::LDS);
        else if (r.deep == 4) allow_lds<gemm_fp8_tile_k<FA, FB, 4, 4, 4>, Loads<4, 4, 4>::LDS>(), go(gemm_fp8_tile_k<FA, FB, 4, 4, 4>, Loads<4, 4, 4>::LDS);
        else allow_lds<gemm_fp8_tile_k<FA, FB, 4, 4, 2>, Loads<4, 4, 2>::LDS>(), go(gemm_fp8_tile_k<FA, FB, 4, 4, 2>, Loads<4, 4, 2>::LDS);
    } else allow_lds<gemm_fp8_tile32_k<FA, FB>, Loads<4, 4, 2>::LDS>(), go(gemm_fp8_tile32_k<FA, FB>, Loads<4, 4, 2>::LDS);
    if (r.splits > 1)
        gemm_fp8_sums_k<T><<<(unsigned)((p.M * ((p.N + 7) / 8) + 255) / 256), 256, 0, s>>>((const float *)p.work, r.splits, bias, resid, p.ldr, (T *)p.C, p.ldc, p.M, p.N);
}

}  // namespace

int64_t gemm_fp8_work(int64_t M, int64_t N, int64_t K) {
    const Route a = route(true, M, N, K), b = route(false, M, N, K);
    const int most = std::max(a.deep > 1 ? a.splits : 1, b.deep > 1 ? b.splits : 1);
    return most > 1 ? most * M * ((N + 7) / 8 * 8) * 4 : 0;
}

void gemm_fp8_route(int dtype, int64_t M, int64_t N, int64_t K, int *rows, int *cols, int *deep, int *ranges) {
    const Route r = route(dtype == TIO_PREC_BF16, M, N, K);
    *rows = r.rows;
    *cols = r.cols;
    *deep = r.deep;
    *ranges = r.splits;
}

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
