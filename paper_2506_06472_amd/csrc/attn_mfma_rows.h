// Rows of causal attention on the matrix cores: the tiles, and what a workgroup does with its block of query rows (forward, dQ) or of
// key rows (dK/dV), wherever its sequence lies.  The layouts and what bounds these loops: at the top of kernels_attn_mfma.hip.
#pragma once
#include <type_traits>

#include "device_common.h"
#include "mfma_tiles.h"

namespace tio {
namespace k {

namespace {

constexpr int NT = 256;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float FAR = 1048576.0f;       // forward pass, GROUPED: reference exponents beyond this one, of either sign, are taken apart

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// two floats -> packed bf16 pair, round to nearest even (one v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    union { bf16x2 h; uint32_t u; } c;
    c.h = __builtin_convertvector((f32x2){a, b}, bf16x2);
    return c.u;
}

// c += a . b, 16x16x32 (lane layouts: see the top of the file)
__device__ __forceinline__ void mma(floatx4 &c, const bf16x8 &a, const bf16x8 &b) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// B operand of a product over 32 rows from the accumulators of their two groups of 16 (slots 0..3 of lane group g: rows 4 g + 0..3, slots
// 4..7: rows 16 + 4 g + 0..3)
__device__ __forceinline__ bf16x8 pack8(const floatx4 &a, const floatx4 &b) {
    Frag f;
    f.u = make_uint4(pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]), pack2(b[2], b[3]));
    return f.v;
}
__device__ __forceinline__ floatx4 zero4() { return (floatx4){0.f, 0.f, 0.f, 0.f}; }
// a value combined over the four lane groups (lanes i, i + 16, i + 32, i + 48), the same in all of them: the swaps hand every lane the
// values of two groups without a trip through the LDS queue, behind which a cross-lane read would wait
__device__ __forceinline__ float sum_neighbours(float x) {         // lanes i and i ^ 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_halves(float x) {             // lanes i and i ^ 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_groups(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
// Accumulators of columns 16 i .. + 15 (a) and 16 i + 16 .. + 31 (b) of a row to bf16 at p = row start + 16 i: a lane holds four columns
// of either and ends up with eight consecutive ones, so that a row's 32 columns are four stores of 16 bytes.
__device__ __forceinline__ void store32(uint16_t *p, const floatx4 &a, const floatx4 &b, float f, int group) {
    const auto lo = __builtin_amdgcn_permlane32_swap(pack2(a[0] * f, a[1] * f), pack2(b[0] * f, b[1] * f), false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(pack2(a[2] * f, a[3] * f), pack2(b[2] * f, b[3] * f), false, false);
    const auto l2 = __builtin_amdgcn_permlane16_swap(lo[0], lo[1], false, false);
    const auto h2 = __builtin_amdgcn_permlane16_swap(hi[0], hi[1], false, false);
    *reinterpret_cast<uint4 *>(p + 8 * group) = make_uint4(l2[0], h2[0], l2[1], h2[1]);
}
// the lane index, computed where it stands: not kept in a register over a loop
__device__ __forceinline__ int lane_here() {
    int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(l));
    return l;
}
__device__ __forceinline__ u32x4 buf_load(__amdgpu_buffer_rsrc_t rsrc, uint32_t off) {
    return __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)off, 0, 0);
}
// an offset behind every descriptor here (fits() below keeps them under 2 GiB)
constexpr uint32_t PAST_ALL = 0x80000000u;
// descriptor over rows [0, Tn) of one head's slice: rows at or past Tn read as zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t head_rsrc(const uint16_t *base, int64_t Tn, int64_t ld, int dh) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)(((Tn - 1) * ld + dh) * 2), 0x00020000);
}
// byte offset of a block's row at its heads' first column
template <bool GROUPED, int DH> __device__ __forceinline__ uint32_t row_offset(int v, int G, uint32_t ldb) {
    if (!GROUPED) return (uint32_t)v * ldb;
    const int q = v / G;
    return (uint32_t)q * ldb + (uint32_t)(v - q * G) * (DH * 2);
}
__device__ __forceinline__ bf16x8 buf_frag(__amdgpu_buffer_rsrc_t rsrc, uint32_t off) {
    union { u32x4 u; bf16x8 v; } f;
    f.u = buf_load(rsrc, off);
    return f.v;
}

// Where the rows of a block are.  q, k, v: the first row of the sequence, at the first of the query heads that share k and v; ld: from row to row of
// q, k and v; row, ldg: of that row and head in o and dO, from row to row; stat: in lse and delta, heads_ld: from head to head.  Tn: rows of
// the sequence; v0: the first of the block's rows.  GROUPED: G query heads share k and v, and the query rows here are those of row r and head
// i, r * G + i.
struct QueryPlace {
    const uint16_t *q, *k, *v;
    int64_t ld, row, ldg, stat, heads_ld;
    int Tn, v0, G;
};
// the same for a block of key rows from kv0 on; GROUPED: tiles [t0, t1) of its query rows
struct KeyPlace {
    const uint16_t *q, *k, *v;
    int64_t ld, row, ldg, stat, heads_ld;
    int Tn, kv0, G, t0, t1;
};

// ------------------------------------------------------------------------------------------ tiles
// LDS tiles: [rows][DH] bf16 without padding, filled straight from global memory (no staging registers, no LDS store instructions); the
// 16-byte chunk c of row r sits at chunk c ^ swz(r).  A tile is read row-wise (lane group g takes chunk 4 ks + g of sixteen rows) and
// through transposing reads (two lane groups at a time take 32 bytes, an aligned pair of chunks, of each of eight consecutive rows); the
// permutation keeps both free of bank conflicts (the banks span 256 bytes).  Of a row-wise read sixteen lanes are served at a time, but
// not of one group: rows 0..3 and 12..15 of one with rows 4..11 of the next, whose chunk differs in its last bit.  So swz takes
// 16 different values over the sixteen rows (DH 64: eight, two rows per 256 bytes) and values that differ in the last bit stay within
// either set of rows ((r>>2) ^ (r>>3) beside r>>3), and the pairs of eight consecutive rows land on different pairs.  With the bits of
// r>>2 alone the row-wise reads took twice their time (SQ_LDS_BANK_CONFLICT; now 0).
template <int DH> __device__ __forceinline__ int swz(int r) {
    return (DH == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2) | ((((r >> 2) ^ (r >> 3)) & 1) << 1) | ((r >> 3) & 1);
}
// per-lane parts of the fragment addresses (element offsets into a tile), computed once per kernel: the XOR makes
// them non-additive in the contraction step, so each step has its own; with LEAN only the first step's is kept and a step's
// is one more XOR away (for the kernel that has no registers to spare)
template <int DH, bool LEAN = false> struct TileLanes {
    static constexpr int CPR = DH / 8, KS = DH / 32, DT = DH / 16;
    int roff[LEAN ? 1 : KS];          // row-wise fragment of contraction step ks: row lane%16, chunk 4 ks + lane/16
    int troff[LEAN ? 1 : DT];         // transposing fragment of column block i: rows 4 (lane/16) + (lane%16)/4 (and + 16), columns by lane
    __device__ __forceinline__ TileLanes(int lane) {
        const int l16 = lane & 15, g = lane >> 4, rl = 4 * g + (l16 >> 2);
#pragma unroll
        for (int ks = 0; ks < (LEAN ? 1 : KS); ++ks) roff[ks] = (l16 * CPR + ((ks * 4 + g) ^ swz<DH>(l16))) * 8;
#pragma unroll
        for (int i = 0; i < (LEAN ? 1 : DT); ++i) troff[i] = (rl * CPR + ((2 * i + ((lane & 3) >> 1)) ^ swz<DH>(rl))) * 8 + 4 * (lane & 1);
    }
    // rows row0 + lane%16 (row0 a multiple of 16), contraction step ks
    __device__ __forceinline__ bf16x8 row(const uint16_t *lds, int row0, int ks) const {
        Frag f;
        f.u = *reinterpret_cast<const uint4 *>(lds + row0 * DH + (LEAN ? roff[0] ^ (ks * 32) : roff[LEAN ? 0 : ks]));
        return f.v;
    }
    // "column 16 i + lane%16, contraction over rows r0 .. r0+31 in the slot order of pack8" (r0 a multiple of 16)
    __device__ __forceinline__ bf16x8 tr(const uint16_t *lds, int r0, int i) const {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        union { s16x4 h[2]; bf16x8 v; } f;
        const uint16_t *p = lds + r0 * DH + (LEAN ? troff[0] ^ (16 * i) : troff[LEAN ? 0 : i]);
        f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 16 * DH));
        return f.v;
    }
};
// A [ROWS][DH] tile on its way from global memory into LDS: a wavefront-wide load fills 1 KiB of consecutive LDS bytes
// (lane i writes bytes 16 i ..), so which chunk a lane fetches decides where it lands: lane i of block b fetches, for
// row b*RPB + i/CPR, the logical chunk (i%CPR) ^ swz(row).  Rows past the sequence lie outside the descriptor and
// arrive as zeros.
template <int DH, int NW, int ROWS> struct DmaTile {
    static constexpr int CPR = DH / 8, RPB = 64 / CPR, BLOCKS = ROWS * DH * 2 / 1024, PER = BLOCKS / NW;
    static_assert(BLOCKS % NW == 0, "blocks divide over the wavefronts");
    static_assert((NW * RPB) % 16 == 0, "the permutation repeats from one load of a wavefront to its next");
    uint32_t voff, step;           // byte offset of this lane's chunk in the wavefront's first block; bytes between its blocks (uniform)
    __device__ __forceinline__ DmaTile(uint32_t ld_bytes, int wave, int lane) {
        const int row = wave * RPB + lane / CPR;
        voff = (uint32_t)row * ld_bytes + (uint32_t)(((lane % CPR) ^ swz<DH>(row & 15)) * 16);
        step = __builtin_amdgcn_readfirstlane((uint32_t)(NW * RPB) * ld_bytes);
    }
    // tile row r * G + i: row r, head i of G, a divisor of the rows between a wavefront's blocks
    __device__ __forceinline__ DmaTile(uint32_t ld_bytes, int wave, int lane, int G) {
        const int row = wave * RPB + lane / CPR, r = row / G;
        voff = (uint32_t)r * ld_bytes + (uint32_t)(row - r * G) * (DH * 2) + (uint32_t)(((lane % CPR) ^ swz<DH>(row & 15)) * 16);
        step = __builtin_amdgcn_readfirstlane((uint32_t)(NW * RPB / G) * ld_bytes);
    }
    // load i of the PER that make up this wavefront's share of a tile (soff = row0 * ld_bytes, uniform): rows
    // i * NW * RPB further down, which only moves the uniform part of the address (the scalar offset takes part
    // in the descriptor's range check like the per-lane one: checked on the hardware)
    __device__ __forceinline__ void load_one(int i, i32x4 rsrc, uint32_t soff, uint32_t lds_addr, int wave) const {
        load_to_lds_b128(rsrc, lds_addr + (uint32_t)(i * NW + wave) * 1024u, voff, soff + (uint32_t)i * step);
    }
    // rows row0 .. row0+ROWS-1 of the head behind rsrc to the tile at LDS address lds_addr
    __device__ __forceinline__ void load(i32x4 rsrc, uint32_t row0, uint32_t ld_bytes, uint32_t lds_addr, int wave) const {
        const uint32_t soff = __builtin_amdgcn_readfirstlane(row0 * ld_bytes);
#pragma unroll
        for (int i = 0; i < PER; ++i) load_one(i, rsrc, soff, lds_addr, wave);
    }
};

// The same for a [64][DH] tile of all G heads of 64 / G rows (row r * G + i: row r, head i; what is left of 64: zeros), whatever G is.  The rows of a
// wavefront's blocks are no fixed distance apart, so each block has its own offsets.
template <int DH, int NW> struct GroupTile {
    static constexpr int CPR = DH / 8, RPB = 64 / CPR, PER = 64 * DH * 2 / 1024 / NW;
    uint32_t voff[PER];
    __device__ __forceinline__ GroupTile(uint32_t ld_bytes, int wave, int lane, int G) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = (i * NW + wave) * RPB + lane / CPR, r = v / G;
            voff[i] = r < 64 / G ? (uint32_t)r * ld_bytes + (uint32_t)(v - r * G) * (DH * 2) + (uint32_t)(((lane % CPR) ^ swz<DH>(v & 15)) * 16) : PAST_ALL;
        }
    }
    __device__ __forceinline__ void load(i32x4 rsrc, uint32_t row0, uint32_t ld_bytes, uint32_t lds_addr, int wave) const {
        const uint32_t soff = __builtin_amdgcn_readfirstlane(row0 * ld_bytes);
#pragma unroll
        for (int i = 0; i < PER; ++i) load_to_lds_b128(rsrc, lds_addr + (uint32_t)(i * NW + wave) * 1024u, voff[i], soff);
    }
};

// ------------------------------------------------------------------------------------------ forward
// Tiles of 32 keys in a ring of three: loads are issued two tiles ahead, and a workgroup's 48 KiB (head size 128) and its registers
// leave room for three wavefronts per SIMD, where two tiles of 64 keys and a second set of scores allowed two.  A wavefront runs its own
// number of tiles in front of the diagonal, without mask and branch, so that no branch around a tile keeps a second copy of its
// accumulators alive.  4 x 2048 tokens, 32 heads of 128: 158 -> 151 us, 2 x 4096, 52 heads 470 -> 440 (before the change of the product).
// NG: groups of 16 query rows of a wavefront.
// W: where a workgroup's rows are (its place() says so, or that there are none).  The loop stands in the kernel itself: as a function of its
// own, the same code took 12 registers more, and at head size 128 spilled.
// SPLIT: that many sets of four wavefronts share the workgroup's rows, each with every SPLIT-th tile of keys (a step of the ring is SPLIT tiles, which all
// of them load together), and join their sums at the end, in order: for batches whose longest chain of tiles counts.
template <int DH, int NG, int SPLIT, class W>
__global__ void __launch_bounds__(NT *SPLIT, SPLIT > 1 ? 2 : DH == 64 || NG == 1 ? 4 : 3)
    attn_fwd_mfma_k(const W where, uint16_t *__restrict__ o, float *__restrict__ lse, float scale) {
    constexpr bool GROUPED = W::GROUPED;
    constexpr int KS = DH / 32, DT = DH / 16, TE = 32 * DH, TS = TE * SPLIT, RING = 4, ROWS = NT / 64 * 16 * NG;
    extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];    // ring of three steps: 32 SPLIT rows of K | as many of V
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int set = SPLIT == 1 ? 0 : wave / (NT / 64);
    QueryPlace at;
    if (!where.template place<DH, ROWS>(blockIdx.x, at)) return;
    const int64_t ld = at.ld;
    const uint32_t ldb = (uint32_t)(ld * 2);
    const int Tn = at.Tn, q0 = at.v0, G = GROUPED ? at.G : 1;
    const int q0w = q0 + (SPLIT == 1 ? wave : wave % (NT / 64)) * 16 * NG;
    const __amdgpu_buffer_rsrc_t rsQ = head_rsrc(at.q, Tn, ld, DH * G);
    const uint32_t head_bytes = (uint32_t)(((Tn - 1) * ld + DH) * 2);
    const i32x4 rsK = make_rsrc(at.k, head_bytes), rsV = make_rsrc(at.v, head_bytes);
    const float c = scale * LOG2E;
    const TileLanes<DH> L(lane);
    using Dma = DmaTile<DH, NT / 64 * SPLIT, 32 * SPLIT>;
    const Dma dma(ldb, wave, lane);
    constexpr int PER = Dma::PER;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

    bf16x8 qf[NG][KS];                                  // of rows q0w + 16 u + lane%16
#pragma unroll
    for (int u = 0; u < NG; ++u)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[u][ks] = buf_frag(rsQ, row_offset<GROUPED, DH>(q0w + 16 * u + l16, G, ldb) + (ks * 32 + grp * 8) * 2);
    floatx4 oacc[DT][NG];
    float m[NG], l[NG];                                 // reference exponent (log2 domain, scaled) and sum
#pragma unroll
    for (int u = 0; u < NG; ++u) {
        m[u] = -INFINITY;
        l[u] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) oacc[i][u] = zero4();
    }
    const int past = GROUPED ? (q0 + ROWS - 1) / G + 1 : q0 + ROWS, kv_end = past < Tn ? past : Tn;
    const int steps = (kv_end + 32 * SPLIT - 1) / (32 * SPLIT);

    dma.load(rsK, 0, ldb, lds0, wave);
    dma.load(rsV, 0, ldb, lds0 + TS * 2, wave);
    dma.load(rsK, 32 * SPLIT, ldb, lds0 + 2 * TS * 2, wave);
    dma.load(rsV, 32 * SPLIT, ldb, lds0 + 3 * TS * 2, wave);
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0): this wavefront's part of tile 0 has landed (and Q, which the compiler knows of)
    __builtin_amdgcn_s_barrier();
    int slot = 0;                                       // of step t in the ring
    bool far = GROUPED;                                 // GROUPED: some row of the wavefront has a reference exponent beyond FAR (uniform)
    // Step t + 2 goes to the slot of step t - 1, free since the barrier that ended it; past the last step the loads lie outside the
    // descriptor and bring zeros that nobody reads.  They are issued one at a time between the score products: issued together
    // right after the barrier, the loads of all wavefronts of a compute unit queue up behind one another and every wavefront stalls.
    struct Next { uint32_t soff, to; };
    auto next_of = [&](int t) __attribute__((always_inline)) {
        return Next{(uint32_t)__builtin_amdgcn_readfirstlane(t + 2 < steps ? (uint32_t)(t + 2) * (32 * SPLIT) * ldb : PAST_ALL),
                    lds0 + (uint32_t)(slot == 0 ? 2 : slot - 1) * 2 * TS * 2};
    };
    auto next_load = [&](int i, const Next &n) __attribute__((always_inline)) {         // PER loads of K, then as many of V
        if (i < PER) dma.load_one(i, rsK, n.soff, n.to, wave);
        else dma.load_one(i - PER, rsV, n.soff, n.to + TS * 2, wave);
    };
    auto end_of_tile = [&]() __attribute__((always_inline)) {
        slot = slot == 2 ? 0 : slot + 1;
        __builtin_amdgcn_s_waitcnt(0x0070 | 2 * PER);   // step t+1 has landed, step t+2 may be on its way; lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
    };
    // Tile t * SPLIT + set.  DIAG: the tile on the diagonal, which has key q0w (GROUPED: the tiles that a row of the wavefront sees part of)
    auto tile = [&](int t, auto DIAG) __attribute__((always_inline)) {
        const uint16_t *Ks = smem + slot * 2 * TS + set * TE, *Vs = Ks + TS;
        const Next next = next_of(t);
        floatx4 s[2][NG];                               // [keys 16 k ..][queries 16 u ..]
        {
            constexpr int N = 2 * KS;
            bf16x8 ring[RING];
            auto frag = [&](int f) { return L.row(Ks, (f & 1) * 16, f / 2); };
#pragma unroll
            for (int f = 0; f < RING; ++f) ring[f] = frag(f);
#pragma unroll
            for (int u = 0; u < NG; ++u) s[0][u] = s[1][u] = zero4();
#pragma unroll
            for (int f = 0; f < N; ++f) {
#pragma unroll
                for (int v = 0; v < NG; ++v) mma(s[f & 1][(f + v) % NG], ring[f % RING], qf[(f + v) % NG][f / 2]);
                if (f + RING < N) ring[f % RING] = frag(f + RING);
#pragma unroll
                for (int i = f * 2 * PER / N; i < (f + 1) * 2 * PER / N; ++i) next_load(i, next);
            }
            // pin the order: RING reads, then the products of a fragment and one read in turn, then the last products
            __builtin_amdgcn_sched_group_barrier(0x100, RING, 0);
#pragma unroll
            for (int f = 0; f < N - RING; ++f) {
                __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, NG * RING, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (DIAG()) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int u = 0; u < NG; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (GROUPED ? 16 * k + r > (q0w + 16 * u + l16) / G - 32 * (t * SPLIT + set) - 4 * grp
                                    : 16 * (k - u) + r > (NG == 1 ? q0w % 32 : 0) + l16 - 4 * grp)
                            s[k][u][r] = -INFINITY;
                    }
        }
        // The reference exponent m only has to keep exp2(x - m) in range, it need not be the running maximum.  The
        // probabilities are first taken with the m at hand, and their sum tells whether that was good enough: only
        // when the sum of some lane of a group of 16 rows reaches 2^16 (or is not a number: m is still -inf in the first tile of a row,
        // where key 0 is visible to every row) is the row maximum of the tile computed, m raised to it, everything
        // accumulated so far rescaled and the tile redone.  After the first keys that is rare, and the common
        // path has no maximum, no exchange between the lane groups and no rescale in it.
        // GROUPED: a row's tiles may hold nothing but scores of -inf (keys that it does not see: a set's first tile), or scores so large that the product with
        // c, rounded into m, is off by more than exp2 tolerates.  Where m is beyond FAR the probabilities are taken of rounded products, of which the largest
        // is m itself, in every tile (a tile's question whether there is such a row: 0.5 to 0.8 % of the pass at head size 128).
        floatx4 p[2][NG];
        float psum[NG];
        auto probabilities = [&](int u, float by, float ref) __attribute__((always_inline)) {
            psum[u] = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[k][u][r] = __builtin_amdgcn_exp2f(fmaf(s[k][u][r], by, -ref));
                    psum[u] += p[k][u][r];
                }
        };
#pragma unroll
        for (int u = 0; u < NG; ++u) probabilities(u, c, m[u]);
        if (far || __any(!(psum[0] < 65536.0f) || !(psum[NG - 1] < 65536.0f))) {
#pragma unroll
            for (int u = 0; u < NG; ++u) {
                if (!__any(!(psum[u] < 65536.0f) || (GROUPED && fabsf(m[u]) > FAR))) continue;       // by itself: the bits do not depend on the rows of a wavefront
                float tmax = -INFINITY;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r) tmax = fmaxf(tmax, s[k][u][r]);
                const float mn = fmaxf(m[u], max_groups(tmax) * c), ref = GROUPED && mn == -INFINITY ? 0.f : mn, corr = __builtin_amdgcn_exp2f(m[u] - ref);
                l[u] *= corr;
                m[u] = mn;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) oacc[i][u][r] *= corr;
                float cc = c;
                if (GROUPED) {
                    const bool rounded = fabsf(mn) > FAR;
                    cc = rounded ? 1.f : c;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[k][u][r] = rounded ? s[k][u][r] * c : s[k][u][r];
                }
                probabilities(u, cc, ref);
            }
            if (GROUPED) far = __any(fmaxf(fabsf(m[0]), fabsf(m[NG - 1])) > FAR);
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pk[NG];
#pragma unroll
        for (int u = 0; u < NG; ++u) {
            l[u] += psum[u];
            pk[u] = pack8(p[0][u], p[1][u]);
        }
        // V fragment i: columns 16 i .. + 15 of the 32 keys; like the K fragments they run through a ring of register sets
        constexpr int VR = 4;
        bf16x8 vf[VR];
#pragma unroll
        for (int i = 0; i < VR; ++i) vf[i] = L.tr(Vs, 0, i);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
#pragma unroll
            for (int v = 0; v < NG; ++v) mma(oacc[i][(i + v) % NG], vf[i % VR], pk[(i + v) % NG]);
            if (i + VR < DT) vf[i % VR] = L.tr(Vs, 0, i + VR);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * VR, 0);
#pragma unroll
        for (int i = 0; i < DT - VR; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, NG * VR, 0);
        end_of_tile();
    };
    // A wavefront's tiles: those in front of its diagonal, without mask and branch, the one on it, and those that only later
    // wavefronts of the workgroup need, of which it loads its share.
    int t = 0;
    if constexpr (GROUPED) {
        if (q0w / G < Tn) {
            const int whole = (q0w / G + 1) / 32, last = (q0w + 16 * NG - 1) / G, some = (last < Tn ? last : Tn - 1) / 32;
            for (; t * SPLIT + set < whole; ++t) tile(t, std::false_type{});
            for (; t * SPLIT + set <= some; ++t) tile(t, std::true_type{});
        }
    } else if (q0w < Tn) {
        static_assert(GROUPED || SPLIT == 1, "tiles of one set");
        for (; t < q0w / 32; ++t) tile(t, std::false_type{});
        tile(t++, std::true_type{});
    }
    for (; t < steps; ++t) {
        const Next next = next_of(t);
#pragma unroll
        for (int i = 0; i < 2 * PER; ++i) next_load(i, next);
        end_of_tile();
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // no load may be on its way to LDS that this workgroup gives back
#pragma unroll
    for (int u = 0; u < NG; ++u) l[u] = sum_halves(sum_neighbours(l[u]));
    if constexpr (SPLIT > 1) {
        // the sets' exponents, sums and accumulators, in the ring's place
        constexpr int LANE = NG * (2 + 4 * DT);                             // floats of a lane
        static_assert((SPLIT - 1) * (NT / 64) * 64 * LANE * 4 <= 3 * 2 * TS * 2, "room in the ring");
        __builtin_amdgcn_s_barrier();                   // nobody reads tiles any more
        float *const part = reinterpret_cast<float *>(smem);
        auto at_lane = [&](int of, int i) __attribute__((always_inline)) { return ((of * (NT / 64) + wave % (NT / 64)) * LANE + i) * 64 + lane; };
        if (set) {
#pragma unroll
            for (int u = 0; u < NG; ++u) {
                part[at_lane(set - 1, 2 * u)] = m[u];
                part[at_lane(set - 1, 2 * u + 1)] = l[u];
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) part[at_lane(set - 1, 2 * NG + (u * DT + i) * 4 + r)] = oacc[i][u][r];
            }
        }
        __syncthreads();
        if (set) return;
#pragma unroll
        for (int of = 0; of < SPLIT - 1; ++of)
#pragma unroll
            for (int u = 0; u < NG; ++u) {
                const float mo = part[at_lane(of, 2 * u)], M = fmaxf(m[u], mo), ref = M == -INFINITY ? 0.f : M;
                const float fa = __builtin_amdgcn_exp2f(m[u] - ref), fb = __builtin_amdgcn_exp2f(mo - ref);
                l[u] = l[u] * fa + part[at_lane(of, 2 * u + 1)] * fb;
                m[u] = M;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) oacc[i][u][r] = oacc[i][u][r] * fa + part[at_lane(of, 2 * NG + (u * DT + i) * 4 + r)] * fb;
            }
    }
#pragma unroll
    for (int u = 0; u < NG; ++u) {
        const int v = q0w + 16 * u + l16, q = GROUPED ? v / G : v, head = GROUPED ? v - q * G : 0;
        const float inv = 1.0f / l[u];
        uint16_t *orow = o + (at.row + q * at.ldg) + head * DH;
        // the lane groups exchange columns of a row, so they take part or not together
        if (q < Tn) {
#pragma unroll
            for (int i = 0; i < DT; i += 2) store32(orow + 16 * i, oacc[i][u], oacc[i + 1][u], inv, grp);
            if (grp == 0) lse[at.stat + head * at.heads_ld + q] = (m[u] + log2f(l[u])) * LN2;
        }
    }
}

// ------------------------------------------------------------------------------------------ dQ
// Sum of the products of eight elements, in order.
__device__ __forceinline__ float chunk_dot(const bf16x8 &g, const bf16x8 &o) {
    Frag a, b;
    a.v = g;
    b.v = o;
    const uint32_t x[4] = {a.u.x, a.u.y, a.u.z, a.u.w}, y[4] = {b.u.x, b.u.y, b.u.z, b.u.w};
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum);
        sum = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), sum);
    }
    return sum;
}
// Sum over the head dimension of two rows of which the four lane groups have the fragments, the same in all of them: in the order of
// attn_bwd_pre_k, whose bits these are (chains of eight elements, then pairs).
template <int KS> __device__ __forceinline__ float row_dot(const bf16x8 (&g)[KS], const bf16x8 (&o)[KS]) {
    float p[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) p[ks] = sum_halves(sum_neighbours(chunk_dot(g[ks], o[ks])));
#pragma unroll
    for (int o2 = 1; o2 < KS; o2 *= 2)
#pragma unroll
        for (int ks = 0; ks < KS; ks += 2 * o2) p[ks] += p[ks + o2];
    return p[0];
}

// GROUPED: delta of a sequence's first rows, from the probabilities instead of the rounded output.  A row's dO . O misses sum(P dP) by the rounding of O, which,
// relative to the row's dS, falls with the square root of its number of keys; and the first rows have the largest gradients.  dQ of 4 heads
// of 64, relative to the norm, with the output's throughout and like this: sequences of 34 and 2 rows 3.3e-3 / 2.5e-3, one of 1713 2.5e-3 / 2.4e-3, of
// which the roundings of dS and of the result make 2.3e-3.  It costs what a few loads in a row take: 12 heads, sequences of up to 100 rows
// 12.6 -> 13.3 us, 32 heads of 128 in 4 groups, up to 60 rows 20.6 -> 23.6, large batches less than 1 %; for eight rows instead of 16 half a
// microsecond less where groups are large, and dQ up to 2.6e-3.  q, g: fragments of Q and dO of sixteen rows, a lane's row of the sequence `row`;
// k, v: of its first sixteen keys.  A row whose scores are so large that its log-sum-exp, rounded, leaves infinite probabilities keeps the output's delta: its own
// gradients are lost, but delta meets the keys that it does not see too, times a probability of zero.
constexpr int EARLY = 16;
template <int KS> __device__ __forceinline__ float early_delta(const bf16x8 (&q)[KS], const bf16x8 (&g)[KS], const bf16x8 (&k)[KS], const bf16x8 (&v)[KS],
                                                               float c, float lse2, int row, int grp) {
    floatx4 s = zero4(), dp = zero4();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        mma(s, k[ks], q[ks]);
        mma(dp, v[ks], g[ks]);
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += 4 * grp + r <= row ? __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * dp[r] : 0.f;
    return sum_halves(sum_neighbours(sum));
}

// Bound: the matrix cores and the vector ALU, which work for 57 and 48 % of the time at head size 128 (39 and 57 at 64) and for a fifth to a third
// of the products' time together, and power; the tiles in front of the diagonal run through a loop of their own, without mask and
// branch.  Three wavefronts per SIMD at head size 64, two at 128.  With fragments of the transposed K tile four ahead in registers, where
// the compiler read each right before its products, 4 x 2048 tokens, 32 heads of 128, forward and backward 634 -> 614 us (dK/dV too).
// O: nullptr, or the forward pass's output: delta is then computed here, from the rows of dO that are in registers anyway, and
// written for the dK/dV kernel, in place of a launch that reads both tensors (forward and backward 100.8 -> 97.2 us and 708 -> 687).
template <int DH, int NW, int NG, bool GROUPED>
__device__ __forceinline__ void dq_rows(const QueryPlace &at, const uint16_t *__restrict__ dO, const uint16_t *__restrict__ O, const float *__restrict__ lse,
                                        float *__restrict__ delta, uint16_t *__restrict__ dq_out, float scale) {
    constexpr int KS = DH / 32, DT = DH / 16, TE = 64 * DH, RING = 4, TR = 4, ROWS = NW * 16 * NG;
    extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];    // [2 buffers][K tile | V tile] of 64 rows
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int64_t ld = at.ld, ldg = at.ldg;
    const uint32_t ldb = (uint32_t)(ld * 2);
    const int Tn = at.Tn, q0 = at.v0, G = GROUPED ? at.G : 1;
    const int q0w = q0 + wave * 16 * NG;
    const __amdgpu_buffer_rsrc_t rsQ = head_rsrc(at.q, Tn, ld, DH * G);
    const uint32_t head_bytes = (uint32_t)(((Tn - 1) * ld + DH) * 2);
    const i32x4 rsK = make_rsrc(at.k, head_bytes), rsV = make_rsrc(at.v, head_bytes);
    const __amdgpu_buffer_rsrc_t rsG = head_rsrc(dO, Tn, ldg, DH * G);
    const float c = scale * LOG2E;
    const TileLanes<DH> L(lane);
    const DmaTile<DH, NW, 64> dma(ldb, wave, lane);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

    bf16x8 qf[NG][KS], gf[NG][KS];                       // of rows q0w + 16 u + lane%16
    float lse2[NG], dl[NG];
#pragma unroll
    for (int u = 0; u < NG; ++u) {
        const int v = q0w + 16 * u + l16, q = GROUPED ? v / G : v, head = GROUPED ? v - q * G : 0;
        const uint32_t atq = (uint32_t)q * ldb + (GROUPED ? head * DH * 2 : 0), atg = (uint32_t)q * (uint32_t)(ldg * 2) + (GROUPED ? head * DH * 2 : 0);
        const int64_t stat = (GROUPED ? head * at.heads_ld : 0) + q;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[u][ks] = buf_frag(rsQ, atq + (ks * 32 + grp * 8) * 2);
            gf[u][ks] = buf_frag(rsG, atg + (ks * 32 + grp * 8) * 2);
        }
        lse2[u] = q < Tn ? lse[stat] * LOG2E : 0.f;
        if (O) {
            const __amdgpu_buffer_rsrc_t rsO = head_rsrc(O, Tn, ldg, DH * G);
            bf16x8 of[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) of[ks] = buf_frag(rsO, atg + (ks * 32 + grp * 8) * 2);
            dl[u] = row_dot<KS>(gf[u], of);
            if (!GROUPED && q < Tn && grp == 0) delta[stat] = dl[u];
        } else {
            dl[u] = q < Tn ? delta[stat] : 0.f;
        }
    }
    if (GROUPED && q0w / G < EARLY) {
        const __amdgpu_buffer_rsrc_t rsK1 = head_rsrc(at.k, Tn, ld, DH), rsV1 = head_rsrc(at.v, Tn, ld, DH);
        bf16x8 k1[KS], v1[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            k1[ks] = buf_frag(rsK1, (uint32_t)l16 * ldb + (ks * 32 + grp * 8) * 2);
            v1[ks] = buf_frag(rsV1, (uint32_t)l16 * ldb + (ks * 32 + grp * 8) * 2);
        }
#pragma unroll
        for (int u = 0; u < NG; ++u) {
            const int q = (q0w + 16 * u + l16) / G;
            const float early = early_delta<KS>(qf[u], gf[u], k1, v1, c, lse2[u], q, grp);
            if (q < EARLY && fabsf(early) < INFINITY) dl[u] = early;
        }
    }
    floatx4 dq[DT][NG];
#pragma unroll
    for (int i = 0; i < DT; ++i) dq[i][0] = dq[i][NG - 1] = zero4();
    const int past = GROUPED ? (q0 + ROWS - 1) / G + 1 : q0 + ROWS, kv_end = past < Tn ? past : Tn;
    const int ntiles = (kv_end + 63) / 64;

    dma.load(rsK, 0, ldb, lds0, wave);
    dma.load(rsV, 0, ldb, lds0 + TE * 2, wave);
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0): this wavefront's part of tile 0 has landed
    __syncthreads();
    // DIAG: tiles that cross the diagonal of some row of this workgroup, the last ones; the others have no mask and no branch in them
    auto tile = [&](int t, auto DIAG) __attribute__((always_inline)) {
        const int j0 = t * 64;
        const uint16_t *Ks = smem + (t & 1) * 2 * TE, *Vs = Ks + TE;
        if (t + 1 < ntiles) {                           // the other buffer is free since the barrier that ended tile t-1
            const uint32_t nx = lds0 + (uint32_t)((t + 1) & 1) * 2 * TE * 2;
            dma.load(rsK, (uint32_t)j0 + 64, ldb, nx, wave);
            dma.load(rsV, (uint32_t)j0 + 64, ldb, nx + TE * 2, wave);
        }
        if (!DIAG() || j0 <= (GROUPED ? (q0w + 16 * NG - 1) / G : q0w + 16 * NG - 1)) {
            int seen[NG];                                   // last key of the tile that a row of the lane sees, less 4 grp
#pragma unroll
            for (int u = 0; u < NG; ++u) seen[u] = DIAG() ? (GROUPED ? (q0w + 16 * u + l16) / G - j0 - 4 * grp : q0w - j0 + 16 * u + l16 - 4 * grp) : 0;
#pragma unroll
            for (int kb = 0; kb < 64; kb += 32) {           // 32 keys at a time: a second set of scores would take the registers of a wavefront
                floatx4 s[2][NG], dp[2][NG];                // [keys kb + 16 k ..][queries 16 u ..]
                {
                    // S = K.Q^T and dP = V.dO^T; the K and V fragments run RING ahead of their products
                    constexpr int N = 4 * KS;
                    bf16x8 ring[RING];
                    auto frag = [&](int f) { return L.row((f & 1) ? Vs : Ks, kb + ((f >> 1) & 1) * 16, f >> 2); };
#pragma unroll
                    for (int f = 0; f < RING; ++f) ring[f] = frag(f);
#pragma unroll
                    for (int u = 0; u < NG; ++u) s[0][u] = s[1][u] = dp[0][u] = dp[1][u] = zero4();
#pragma unroll
                    for (int f = 0; f < N; ++f) {
                        const int k = (f >> 1) & 1, ks = f >> 2;
#pragma unroll
                        for (int v = 0; v < NG; ++v) {
                            const int u = ((f >> 1) + v) % NG;
                            if (f & 1) mma(dp[k][u], ring[f % RING], gf[u][ks]);
                            else mma(s[k][u], ring[f % RING], qf[u][ks]);
                        }
                        if (f + RING < N) ring[f % RING] = frag(f + RING);
                    }
                    __builtin_amdgcn_sched_group_barrier(0x100, RING, 0);
#pragma unroll
                    for (int f = 0; f < N - RING; ++f) {
                        __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    }
                    __builtin_amdgcn_sched_group_barrier(0x008, NG * RING, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int u = 0; u < NG; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float p = __builtin_amdgcn_exp2f(fmaf(s[k][u][r], c, -lse2[u]));
                            if (DIAG() && kb + 16 * k + r > seen[u]) p = 0.0f;
                            s[k][u][r] = p * (dp[k][u][r] - dl[u]);          // the 1/sqrt(dh) factor is applied once, to the sums
                        }
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 ds[NG], kf[TR];
#pragma unroll
                for (int u = 0; u < NG; ++u) ds[u] = pack8(s[0][u], s[1][u]);
                // the transposed K fragments run TR ahead of their products
#pragma unroll
                for (int i = 0; i < TR; ++i) kf[i] = L.tr(Ks, kb, i);
#pragma unroll
                for (int i = 0; i < DT; ++i) {
#pragma unroll
                    for (int v = 0; v < NG; ++v) mma(dq[i][(i + v) % NG], kf[i % TR], ds[(i + v) % NG]);
                    if (i + TR < DT) kf[i % TR] = L.tr(Ks, kb, i + TR);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * TR, 0);
#pragma unroll
                for (int i = 0; i < DT - TR; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, NG * TR, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): this wavefront's part of tile t+1 has landed
        __syncthreads();
    };
    int t = 0;
    for (; t < (GROUPED ? (q0 / G + 1) / 64 : q0 / 64); ++t) tile(t, std::false_type{});
    for (; t < ntiles; ++t) tile(t, std::true_type{});
#pragma unroll
    for (int u = 0; u < NG; ++u) {
        const int v = q0w + 16 * u + l16, q = GROUPED ? v / G : v;
        if (q < Tn) {                                   // lane groups together: they exchange columns
            uint16_t *orow = dq_out + q * ld + (GROUPED ? (v - q * G) * DH : 0);
#pragma unroll
            for (int i = 0; i < DT; i += 2) store32(orow + 16 * i, dq[i][u], dq[i + 1][u], scale, grp);
        }
    }
}

// ------------------------------------------------------------------------------------------ dK, dV
// Both gradients in one launch: S and dP are computed once for the two of them, and the Q and dO tiles are loaded once.  The
// accumulators and K fragments of 32 key rows take 160 of the 256 registers that two wavefronts per SIMD allow at head size 128,
// so the V fragments are not kept in registers there but read from LDS (the workgroup's V rows, loaded once); to have room for
// them, and half the tile loads per product, a workgroup is eight wavefronts with 256 key rows.  Bound: latency between the
// products of two wavefronts per SIMD (three at head size 64), a third of their cycles, and power.  Nothing may spill: a reload from
// scratch in the loop waits for the tile loads in flight, and the wavefront with it keeps the others at the barrier.  So the offsets of the reads are one register and an
// exclusive or each at head size 128, each of two wavefronts fetches one of the statistics, and the lane index is computed where it is used.
// The tiles behind the diagonal run through a loop of their own, without mask and branch; at head size 64 a second loop gains nothing
// over a mask of two instructions.
// The same sum with a row spread over four neighbouring lanes, CH chunks of eight elements each, the same in all of them.
template <int CH> __device__ __forceinline__ float quad_dot(const bf16x8 (&g)[CH], const bf16x8 (&o)[CH]) {
    float p[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) p[c] = chunk_dot(g[c], o[c]);
#pragma unroll
    for (int o2 = 1; o2 < CH; o2 *= 2)
#pragma unroll
        for (int c = 0; c < CH; c += 2 * o2) p[c] += p[c + o2];
    auto add_from = [](float x, auto LANES) {
        return x + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), LANES(), 0xf, 0xf, true));
    };
    const float pair = add_from(p[0], std::integral_constant<int, 0xB1>{});         // lanes 1 0 3 2
    return add_from(pair, std::integral_constant<int, 0x4E>{});                    // lanes 2 3 0 1
}
// V rows in LDS instead of registers (NG: groups of 16 key rows of a wavefront)
template <int DH, int NG> constexpr bool dkv_v_in_lds() { return DH == 128 && NG == 2; }
template <int DH> constexpr int dkv_waves() { return DH == 128 ? 8 : 4; }
template <int DH, int NW> constexpr int rows_between_loads() { return NW * DmaTile<DH, NW, 64>::RPB; }
// GROUPED: a tile of 64 rows holds all heads of 64 / G rows of the sequence (TAIL: for any G up to 64; whole rows, so that the tile's last rows may
// be none, and every tile is masked.  Otherwise G divides the rows between a wavefront's loads, rows_between_loads), tiles [t0, t1) of them.  Their sums go to dk and dv, or, where a block's tiles are shared by several workgroups,
// to `partial` as they are in the registers, to be added in order (key_sums).  dk, dv: rows of the sequence as k and v.
template <int DH, int NW, int NG, bool DELTA, bool GROUPED, bool TAIL>
__device__ __forceinline__ void dkv_rows(const KeyPlace &at, const uint16_t *__restrict__ dO, const uint16_t *__restrict__ O,
                                         const float *__restrict__ lse, const float *__restrict__ delta, uint16_t *__restrict__ dk_out,
                                         uint16_t *__restrict__ dv_out, float *__restrict__ partial, float scale) {
    constexpr int KS = DH / 32, DT = DH / 16, TE = 64 * DH, RING = 4, TR = 4, KEYS = NW * 16 * NG;
    constexpr bool VLDS = dkv_v_in_lds<DH, NG>(), ONE_LOOP = DH == 64;
    constexpr int BUF = 2 * TE;                                          // Q tile | dO tile, filled as in the forward kernel
    // [2 buffers][Q | dO], [KEYS][DH] V rows if VLDS, then [2][64 lse | 64 delta] floats; GROUPED: then delta of the first EARLY rows
    extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int64_t ld = at.ld;
    const uint32_t ldb = (uint32_t)(ld * 2), ldg = (uint32_t)(at.ldg * 2);
    const int Tn = at.Tn, kv0 = at.kv0, G = GROUPED ? at.G : 1, per_tile = GROUPED ? 64 / G : 64;      // rows of the sequence in a tile
    const int kv0w = kv0 + wave * 16 * NG;
    const uint32_t head_bytes = (uint32_t)(((Tn - 1) * ld + DH) * 2);
    const __amdgpu_buffer_rsrc_t rsK = head_rsrc(at.k, Tn, ld, DH), rsV = head_rsrc(at.v, Tn, ld, DH);
    const i32x4 rsQ = make_rsrc(at.q, (uint32_t)(((Tn - 1) * ld + DH * G) * 2));
    const i32x4 rsG = make_rsrc(dO, (uint32_t)(((Tn - 1) * at.ldg + DH * G) * 2));
    const float c = scale * LOG2E;
    const TileLanes<DH, VLDS> L(lane);
    const DmaTile<DH, NW, 64> dmaK(ldb, wave, lane);
    using TileOf = std::conditional_t<TAIL, GroupTile<DH, NW>, DmaTile<DH, NW, 64>>;
    const TileOf dmaQ(ldb, wave, lane, G), dmaG(ldg, wave, lane, G);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
    const uint16_t *Vs = smem + 2 * BUF;

    bf16x8 kf[NG][KS], vf[NG][VLDS ? 1 : KS];             // of keys kv0w + 16 k + lane%16
#pragma unroll
    for (int k = 0; k < NG; ++k)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const uint32_t at = (uint32_t)(kv0w + 16 * k + l16) * ldb + (ks * 32 + grp * 8) * 2;
            kf[k][ks] = buf_frag(rsK, at);
            if (!VLDS) vf[k][VLDS ? 0 : ks] = buf_frag(rsV, at);
        }
    if (VLDS) {
        const i32x4 rs = make_rsrc(at.v, head_bytes);
#pragma unroll
        for (int i = 0; i < KEYS / 64; ++i) dmaK.load(rs, (uint32_t)(kv0 + 64 * i), ldb, lds0 + (2 * BUF + i * TE) * 2, wave);
    }
    floatx4 dk[DT][NG], dv[DT][NG];
#pragma unroll
    for (int i = 0; i < DT; ++i) dk[i][0] = dk[i][NG - 1] = dv[i][0] = dv[i][NG - 1] = zero4();
    const int ntiles = GROUPED ? at.t1 : (Tn - kv0 + 63) / 64;

    // Statistics of row i0 + lane, one tile ahead, log-sum-exp in wavefront 0 and delta in wavefront 1: through descriptors of the head's
    // rows (rows past the sequence read zero; no addresses to keep in registers), used only where they go to LDS, a tile after their fetch.
    // DELTA: four lanes to a row fetch its dO and O instead and multiply them.
    const float *const stat_at = DELTA || wave == 0 ? lse : delta;
    const __amdgpu_buffer_rsrc_t rsS = buffer_over(stat_at, (uint32_t)Tn * 4);
    const float to_lds = DELTA || wave == 0 ? LOG2E : 1.f;
    constexpr int STATS = DELTA ? 1 : 2, CH = DH / 32;                    // wavefronts that fetch statistics; chunks of a row to a lane
    static_assert(!DELTA || NW == 4, "four lanes to each of 64 rows");
    float st = 0.f;
    bf16x8 go[DELTA ? CH : 1], oo[DELTA ? CH : 1];
    const __amdgpu_buffer_rsrc_t rsD = head_rsrc(dO, Tn, at.ldg, DH * G), rsO = head_rsrc(DELTA ? O : dO, Tn, at.ldg, DH * G);
    float *stats = reinterpret_cast<float *>(smem + 2 * BUF + (VLDS ? KEYS * DH : 0));
    auto load_stats = [&](int i0) {
        if (GROUPED) {
            if (wave < STATS) {                                          // rows past the sequence or the tile: zero, and masked
                const int ln = lane_here(), r = ln / G, row = i0 + r;
                st = r < per_tile && row < Tn ? stat_at[(ln - r * G) * at.heads_ld + row] : 0.f;
            }
        } else if (wave < STATS) st = buffer_load4(rsS, (uint32_t)(i0 + lane_here()) * 4);
        if (DELTA) {
            const int ln = lane_here();
            const int v = wave * 16 + (ln >> 2), r = GROUPED ? v / G : v;
            uint32_t at = (uint32_t)(i0 + r) * ldg + (GROUPED ? (v - r * G) * (DH * 2) : 0) + (ln & 3) * CH * 16;
            if (TAIL && r >= per_tile) at = PAST_ALL;
#pragma unroll
            for (int c = 0; c < (DELTA ? CH : 0); ++c) {
                go[c] = buf_frag(rsD, at + c * 16);
                oo[c] = buf_frag(rsO, at + c * 16);
            }
        }
    };
    // delta of row v of the tile at i0
    auto delta_of = [&](float x, int v, int i0) __attribute__((always_inline)) {
        const int e = i0 * G + v;
        return v < per_tile * G && e < EARLY * G && fabsf(stats[256 + e]) < INFINITY ? stats[256 + e] : x;
    };
    auto store_stats = [&](int buf, int i0) {
        if (wave < STATS) {
            const int ln = lane_here();
            float x = st * to_lds;
            if (GROUPED && !DELTA && i0 < EARLY && wave == 1) x = delta_of(x, ln, i0);
            stats[buf * 128 + wave * 64 + ln] = x;
        }
        if (DELTA) {
            float sum = quad_dot<DELTA ? CH : 1>(go, oo);
            const int ln = lane_here();
            if (GROUPED && i0 < EARLY) sum = delta_of(sum, wave * 16 + (ln >> 2), i0);
            if ((ln & 3) == 0) stats[buf * 128 + 64 + wave * 16 + (ln >> 2)] = sum;
        }
    };
    auto load_tile = [&](int i0, int buf) {
        const uint32_t at = lds0 + (uint32_t)buf * BUF * 2;
        dmaQ.load(rsQ, (uint32_t)i0, ldb, at, wave);
        dmaG.load(rsG, (uint32_t)i0, ldg, at + TE * 2, wave);
    };
    int t = GROUPED ? at.t0 : 0;
    if (GROUPED && kv0 + t * per_tile < EARLY) {
        const __amdgpu_buffer_rsrc_t rsQ1 = head_rsrc(at.q, Tn, ld, DH * G);
        bf16x8 k1[KS], v1[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            k1[ks] = buf_frag(rsK, (uint32_t)l16 * ldb + (ks * 32 + grp * 8) * 2);
            v1[ks] = buf_frag(rsV, (uint32_t)l16 * ldb + (ks * 32 + grp * 8) * 2);
        }
        const int to = (ntiles * per_tile < EARLY ? ntiles * per_tile : EARLY) * G;         // of this workgroup's tiles
        for (int v0 = t * per_tile * G + wave * 16; v0 < to; v0 += NW * 16) {
            const int v = v0 + l16, r = v / G;
            bf16x8 q1[KS], g1[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                q1[ks] = buf_frag(rsQ1, row_offset<GROUPED, DH>(v, G, ldb) + (ks * 32 + grp * 8) * 2);
                g1[ks] = buf_frag(rsD, row_offset<GROUPED, DH>(v, G, ldg) + (ks * 32 + grp * 8) * 2);
            }
            const float lse2 = r < Tn ? lse[(v - r * G) * at.heads_ld + r] * LOG2E : 0.f;
            const float early = early_delta<KS>(q1, g1, k1, v1, c, lse2, r, grp);
            // of a row past the sequence zero, like its Q, dO and statistics: with an infinite key its scores are not numbers, and p = 0 does not take that out
            if (grp == 0 && v < EARLY * G) stats[256 + v] = r < Tn ? early : 0.f;
        }
        __syncthreads();
    }
    load_tile(kv0 + t * per_tile, t & 1);
    load_stats(kv0 + t * per_tile);
    store_stats(t & 1, kv0 + t * per_tile);
    if (t + 1 < ntiles) load_stats(kv0 + (t + 1) * per_tile);
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0): this wavefront's part of tile 0 (and of V) has landed
    __syncthreads();
    // DIAG: tiles that cross the diagonal of some key of this workgroup, the first ones; the others have no mask and no branch in them
    // (ONE_LOOP: every tile is taken for one).  END: the last tile where the sequence ends inside it, in code of its own.  Its rows past the
    // sequence are masked too: their Q, dO and statistics are zero, which adds nothing while K is finite, but with an infinite component
    // of a key their scores are not numbers.
    using Plain = std::integral_constant<int, 0>;
    using Diag = std::integral_constant<int, 1>;
    using End = std::integral_constant<int, 2>;
    auto key_less_4group = []() __attribute__((always_inline)) { const int ln = lane_here(); return (ln & 15) - 4 * (ln >> 4); };
    // GROUPED: the first row of the tile that this lane's key kv0w + more + lane % 16 is visible to, less 4 grp
    auto first_row = [&](int ahead, int more) __attribute__((always_inline)) { const int ln = lane_here(); return (ahead + more + (ln & 15)) * G - 4 * (ln >> 4); };
    auto tile = [&](int t, auto KIND) __attribute__((always_inline)) {
        constexpr bool DIAG = KIND() == Diag(), END = KIND() == End();
        const int i0 = kv0 + t * per_tile;
        const uint16_t *Qs = smem + (t & 1) * BUF, *Gs = Qs + TE;
        const float *L2s = stats + (t & 1) * 128, *Ds = L2s + 64;
        if (!END && t + 1 < ntiles) {                           // the other buffer is free since the barrier that ended tile t-1
            // The statistics fetched a tile ago go to LDS before the tile loads are issued: the write waits for every
            // outstanding vector memory operation of the wavefront, and behind the tile loads that would be their
            // whole latency, at the start of every tile.
            store_stats((t + 1) & 1, i0 + per_tile);
            load_tile(i0 + per_tile, (t + 1) & 1);
            if (t + 2 < ntiles) load_stats(i0 + 2 * per_tile);
        }
        if (KIND() == Plain() || i0 + per_tile - 1 >= kv0w) {
            // rows of the tile before this lane's first key, less 4 grp
            const int masked = DIAG ? (GROUPED ? first_row(kv0w - i0, 0) : kv0w - i0 + key_less_4group()) : 0;
            const int masked2 = DIAG && GROUPED && NG == 2 ? first_row(kv0w - i0, 16) : 0;             // its second key
#pragma unroll
            for (int qt = 0; qt < 2; ++qt) {
                floatx4 s[2][NG], dp[2][NG];             // [rows 16 u ..][keys 16 k ..]
                {
                    // S^T = Q.K^T, then dP^T = dO.V^T; the Q and dO fragments run RING ahead of their products, V's two ahead
                    constexpr int N = 4 * KS;
                    bf16x8 ring[RING], vr[2];
                    auto frag = [&](int f) { return L.row(f < 2 * KS ? Qs : Gs, qt * 32 + (f & 1) * 16, (f >> 1) % KS); };
                    auto vfrag = [&](int f) { return L.row(Vs, wave * 16 * NG + (f & 1) * 16, (f >> 1) % KS); };
#pragma unroll
                    for (int f = 0; f < RING; ++f) ring[f] = frag(f);
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[u][0] = s[u][NG - 1] = dp[u][0] = dp[u][NG - 1] = zero4();
#pragma unroll
                    for (int f = 0; f < N; ++f) {
                        const int u = f & 1, ks = (f >> 1) % KS;
#pragma unroll
                        for (int v = 0; v < NG; ++v) {
                            const int k = (f + v) % NG;
                            if (f < 2 * KS) mma(s[u][k], ring[f % RING], kf[k][ks]);
                            else mma(dp[u][k], ring[f % RING], VLDS ? vr[k] : vf[k][VLDS ? 0 : ks]);
                        }
                        if (f + RING < N) ring[f % RING] = frag(f + RING);
                        // V's fragments of the next contraction step, each behind the product that used the last of its predecessor
                        if (VLDS && f + 2 >= 2 * KS && f + 2 < N) {
                            if (f < 2 * KS) vr[f & 1] = vfrag(f + 2);
                            else if (f & 1) { vr[0] = vfrag(f + 1); vr[1] = vfrag(f + 2); }
                        }
                    }
                    __builtin_amdgcn_sched_group_barrier(0x100, RING, 0);
#pragma unroll
                    for (int f = 0; f < N; ++f) {
                        __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
                        const int reads = (f + RING < N ? 1 : 0) + (VLDS && f + 2 >= 2 * KS && f + 2 < N ? f < 2 * KS ? 1 : 2 * (f & 1) : 0);
                        if (reads == 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
                        else if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                        else if (reads == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    // rows 16 u + 4 grp + 0..3 of this 32-row group: their statistics are 16 contiguous bytes
                    const int group4 = 4 * (END || TAIL ? lane_here() >> 4 : grp), ql = qt * 32 + 16 * u + group4;
                    const float4 l4 = *reinterpret_cast<const float4 *>(L2s + ql), d4 = *reinterpret_cast<const float4 *>(Ds + ql);
                    const int first = END ? (GROUPED ? first_row(kv0w - i0, 0) : kv0w - i0 + key_less_4group()) : 0;
                    const int first2 = END && GROUPED && NG == 2 ? first_row(kv0w - i0, 16) : 0;
                    const int rows = (Tn - i0) * G, whole = per_tile * G;
                    const int end = GROUPED ? (rows < whole ? rows : whole) - group4 : Tn - i0 - group4;
                    const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dvv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int k = 0; k < NG; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = qt * 32 + 16 * u + r;
                            float p = __builtin_amdgcn_exp2f(fmaf(s[u][k][r], c, -lv[r]));
                            if (GROUPED) {
                                if (DIAG && row < (k ? masked2 : masked)) p = 0.0f;
                                if (END && row < (k ? first2 : first)) p = 0.0f;
                                if ((END || TAIL) && row >= end) p = 0.0f;
                            } else {
                                if (DIAG && row - 16 * k < masked) p = 0.0f;
                                if (END && (row - 16 * k < first || row >= end)) p = 0.0f;
                            }
                            dp[u][k][r] = p * (dp[u][k][r] - dvv[r]);        // the 1/sqrt(dh) factor is applied once, to the sums
                            s[u][k][r] = p;
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
                const bf16x8 pf[2] = {pack8(s[0][0], s[1][0]), pack8(s[0][NG - 1], s[1][NG - 1])};
                const bf16x8 ds[2] = {pack8(dp[0][0], dp[1][0]), pack8(dp[0][NG - 1], dp[1][NG - 1])};
                // dV += dO^T.P, then dK += Q^T.dS; the transposed fragments run TR ahead of their products
                auto trf = [&](int f) { return L.tr(f < DT ? Gs : Qs, qt * 32, f % DT); };
                bf16x8 fr[TR];
#pragma unroll
                for (int f = 0; f < TR; ++f) fr[f] = trf(f);
#pragma unroll
                for (int f = 0; f < 2 * DT; ++f) {
#pragma unroll
                    for (int v = 0; v < NG; ++v) {
                        const int k = (f + v) % NG;
                        if (f < DT) mma(dv[f][k], fr[f % TR], pf[k]);
                        else mma(dk[f - DT][k], fr[f % TR], ds[k]);
                    }
                    if (f + TR < 2 * DT) fr[f % TR] = trf(f + TR);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * TR, 0);
#pragma unroll
                for (int f = 0; f < 2 * DT - TR; ++f) {
                    __builtin_amdgcn_sched_group_barrier(0x008, NG, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, NG * TR, 0);
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): this wavefront's part of tile t+1 has landed
        __syncthreads();
    };
    const int whole_all = (Tn - kv0) / per_tile, whole = GROUPED && at.t1 < whole_all ? at.t1 : whole_all;
    const int crossed = GROUPED ? (KEYS + per_tile - 1) / per_tile : KEYS / 64, diag = ONE_LOOP || whole < crossed ? whole : crossed;
    for (; t < diag; ++t) tile(t, Diag());
    if constexpr (!ONE_LOOP)
        for (; t < whole; ++t) tile(t, Plain());
    if (t < ntiles) tile(t, End());
    const int last = lane_here();
    if (GROUPED && partial) {
        float *mine = partial + (wave * 2 * DT * NG * 64 + last) * 4;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                *reinterpret_cast<floatx4 *>(mine + (i * NG + k) * 256) = dk[i][k];
                *reinterpret_cast<floatx4 *>(mine + ((DT + i) * NG + k) * 256) = dv[i][k];
            }
        return;
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        const int key = kv0w + 16 * k + (last & 15);
        if (key < Tn) {                                 // lane groups together: they exchange columns
#pragma unroll
            for (int i = 0; i < DT; i += 2) {
                store32(dk_out + key * ld + 16 * i, dk[i][k], dk[i + 1][k], scale, last >> 4);
                store32(dv_out + key * ld + 16 * i, dv[i][k], dv[i + 1][k], 1.0f, last >> 4);
            }
        }
    }
}
// floats of a workgroup's partial sums
template <int DH, int NW, int NG> constexpr int key_partial() { return NW * 2 * (DH / 16) * NG * 256; }
// The sums of `pieces` workgroups' partial ones of a block of keys, in order, to dk (which = 0) or dv (1); wavefronts as in dkv_rows, block i of 32
// columns.  Bound: HBM.
template <int DH, int NW, int NG>
__device__ __forceinline__ void key_sums(const KeyPlace &at, const float *__restrict__ partial, int pieces, int which, int i, uint16_t *__restrict__ out,
                                         float scale) {
    constexpr int DT = DH / 16;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const float *mine = partial + ((wave * 2 + which) * DT + 2 * i) * NG * 256 + lane * 4;
    auto load = [&](int p, int e, int k) __attribute__((always_inline)) {
        return *reinterpret_cast<const floatx4 *>(mine + (int64_t)p * key_partial<DH, NW, NG>() + (e * NG + k) * 256);
    };
    floatx4 sum[2][NG];                                   // [half of the columns][keys 16 k ..]
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int k = 0; k < NG; ++k) sum[e][k] = load(0, e, k);
    int p = 1;
    for (; p + 2 < pieces; p += 2) {                      // two pieces' loads on their way
        floatx4 a[2][NG], b[2][NG];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < NG; ++k) a[e][k] = load(p, e, k), b[e][k] = load(p + 1, e, k);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < NG; ++k) sum[e][k] = (sum[e][k] + a[e][k]) + b[e][k];
    }
    for (; p < pieces; ++p)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < NG; ++k) sum[e][k] += load(p, e, k);
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        const int key = at.kv0 + wave * 16 * NG + 16 * k + (lane & 15);
        if (key < at.Tn) store32(out + key * at.ld + 32 * i, sum[0][k], sum[1][k], which ? 1.0f : scale, lane >> 4);
    }
}

}  // namespace
}  // namespace k
}  // namespace tio
