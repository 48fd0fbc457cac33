// Causal self-attention on the matrix cores (bf16, head dimension 64 or 128), forward and backward,
// on the packed [S, 3d] q|k|v layout.
//
// Each wavefront owns 32 query rows (forward, dQ) or 32 key rows (dK/dV), or 16 where the chip has room for twice as many
// workgroups, and keeps their operand fragments in registers for the whole kernel; the other side streams through LDS in row-major
// tiles.  Scores are produced transposed (keys x queries in the forward and dQ kernels, queries x keys in the dK/dV kernel) so that in
// the accumulator layout the row owned by the wavefront is the lane index: the softmax statistics of a row live in one lane of each of
// the four groups of sixteen, and the probabilities can be fed to the second product straight from registers as its B operand.  The
// operand whose contraction index is the sequence position (V in P.V, K in dS.K, Q and dO in the dK/dV products) is read from the same
// row-major tile with the transposing LDS read (ds_read_b64_tr_b16), in the slot order the accumulator registers dictate: no
// transposed copies.
//
// All products are v_mfma_f32_16x16x32_bf16, D[16x16] += A[16x32] . B[32x16]: lane l supplies row (A) or column (B) l%16 and eight
// contraction slots of lane group l/16; of D it holds column l%16 and rows 4 (l/16) + 0..3.  At head size 128 these kernels run into
// the power limit (the clock stands at 1.5 to 1.8 GHz of 2.4 in the forward kernel, by card; on zeros, which draw less, it takes a fifth to a
// quarter less; at head size 64 2.2 GHz and 6 %), and at that limit a loop of nothing but products on normal values does 2000 to 2060 TFLOP/s with
// this instruction and 1750 to 1800 with v_mfma_f32_32x32x16_bf16, on zeros both 2440.  Of a SIMD's time the matrix cores work 51 to 57 % at head
// size 128 and 35 to 43 at 64, the vector ALU 37 to 60 and 57 to 68.  Consecutive products share one operand (the order of
// the second index turns round with every step of the first), 2 % of the same loop.  With 32x32x16 products, two wavefronts per SIMD
// in the forward kernel and no fragments of the transposed operand ahead, forward / forward and backward, us, before and now:
//   4 x 2048, 32 heads of 128 158 / 685 -> 143 / 600    2 x 4096, 52 of 128 457 / 1935 -> 412 / 1745    8 x 1024, 12 of 64 22.9 / 95 -> 21 / 86
// Tiles go from global memory straight into LDS (buffer loads with the LDS bit; rows past the end of the sequence arrive as zeros), so
// a tile costs one barrier and neither staging registers nor LDS store instructions.  The tiles are unpadded; a permutation of the
// 16-byte chunks of every row, applied through the choice of the chunk each lane fetches, keeps both kinds of fragment reads free of
// bank conflicts.  All fragments run through small rings of registers a few fragments ahead of the products that use them.
// Statistics are fp32, exp2 with the 1/sqrt(dh) scale folded into the exponent; the causal mask is
// applied only on tiles that cross the diagonal; the backward pass recomputes P from the saved
// log-sum-exp; dQ and dK/dV come from workgroups of their own, so every sum has a fixed order and no atomics; no result depends on
// how many rows a wavefront owns.
#include "../../include/teraio.h"
#include "attn_mfma_rows.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

// Workgroup -> (batch*head, block of rows).  Workgroups are dealt to the 8 XCDs round-robin and each XCD has its own L2, so all row
// blocks of one head are given to one XCD (head = 8*i + xcd): the K and V rows of a head are then fetched into one L2 only, and reused
// there by the head's other row blocks.  Under the causal mask a head's blocks differ in length by up to their number (block 0 is the
// longest), and consecutive workgroups of an XCD go to its 32 compute units in turn.  In the order (head, block) a unit therefore gets
// blocks of one length wherever the number of blocks divides 32: of 8 x 1024 tokens, 12 heads of 64, three of the longest (48 tiles; 27
// on average) or three of the shortest.  So an XCD's heads are taken `heads` at a time, and within them all blocks 0 come first, then
// all blocks 1: the longest first, the shorter ones where units become free.  Where all workgroups are resident from the start and none
// becomes free, every other row of 32 is turned round (`turn`), which pairs long with short.  Forward / backward us, order (head,
// block) / this: 8 x 1024, 12 heads of 64 31 / 23.5, 101 / 82; 4 x 2048, 32 of 128 181 / 170, 654 / 553; 1 x 4096, 32 of 64 125 / 82.5,
// 344 / 274; 2 x 4096, 52 of 128 484 / 473, 1649 / 1570.
struct Order {
    int heads;
    bool turn;
};
// Returns false for the padding workgroups when the head count is not a multiple of 8.
__device__ __forceinline__ bool head_and_block(unsigned block, int64_t n_heads, int n_blocks, Order order, int64_t &bh, int &blk) {
    const int xcd = (int)(block & 7), slot = (int)(block >> 3);
    const int of_xcd = (int)((n_heads + 7) / 8), first = slot / (order.heads * n_blocks) * order.heads;
    const int here = of_xcd - first < order.heads ? of_xcd - first : order.heads;
    int w = slot - first * n_blocks;
    if (order.turn && (w & 32) && (w | 31) < here * n_blocks) w ^= 31;
    bh = (int64_t)(first + w % here) * 8 + xcd;
    blk = w / here;
    return bh < n_heads;
}


// the place of batch and head bh in the packed [B T, 3 d] layout
template <typename P> __device__ __forceinline__ P place_of(const uint16_t *qkv, int64_t Tn, int64_t H, int64_t DH, int64_t bh) {
    const int64_t d = H * DH, ld = 3 * d, b = bh / H, h = bh % H;
    P p{};
    p.q = qkv + b * Tn * ld + h * DH;
    p.k = p.q + d;
    p.v = p.q + 2 * d;
    p.ld = ld;
    p.row = b * Tn * d + h * DH;
    p.ldg = d;
    p.stat = bh * Tn;
    p.Tn = (int)Tn;
    p.G = 1;
    return p;
}
struct BatchRows {
    static constexpr bool GROUPED = false;
    const uint16_t *qkv;
    int64_t Bn, Tn, H;
    Order order;
    template <int DH, int ROWS> __device__ __forceinline__ bool place(unsigned block, QueryPlace &at) const {
        const int nblk = (int)((Tn + ROWS - 1) / ROWS);
        int64_t bh;
        int blk;
        if (!head_and_block(block, Bn * H, nblk, order, bh, blk)) return false;
        at = place_of<QueryPlace>(qkv, Tn, H, DH, bh);
        at.v0 = (nblk - 1 - blk) * ROWS;                                  // longest rows first
        return true;
    }
    template <int DH, int KEYS> __device__ __forceinline__ bool place(unsigned block, KeyPlace &at) const {
        int64_t bh;
        int blk;
        if (!head_and_block(block, Bn * H, (int)((Tn + KEYS - 1) / KEYS), order, bh, blk)) return false;
        at = place_of<KeyPlace>(qkv, Tn, H, DH, bh);
        at.kv0 = blk * KEYS;                                              // earliest keys see the most queries: first
        return true;
    }
};

template <int DH, int NW, int NG>
__device__ __forceinline__ void dq_block(const uint16_t *__restrict__ dO, const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ O,
                                         const float *__restrict__ lse, float *__restrict__ delta, uint16_t *__restrict__ dqkv, int64_t Bn, int64_t Tn,
                                         int64_t H, float scale, Order order, unsigned block) {
    QueryPlace at;
    if (!BatchRows{qkv, Bn, Tn, H, order}.place<DH, NW * 16 * NG>(block, at)) return;
    dq_rows<DH, NW, NG, false>(at, dO + at.row, O ? O + at.row : nullptr, lse + at.stat, delta + at.stat, dqkv + (at.q - qkv), scale);
}

template <int DH, int NW, int NG, bool DELTA>
__device__ __forceinline__ void dkv_block(const uint16_t *__restrict__ dO, const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ O,
                                          const float *__restrict__ lse, const float *__restrict__ delta, uint16_t *__restrict__ dqkv, int64_t Bn,
                                          int64_t Tn, int64_t H, float scale, Order order, unsigned block) {
    KeyPlace at;
    if (!BatchRows{qkv, Bn, Tn, H, order}.place<DH, NW * 16 * NG>(block, at)) return;
    dkv_rows<DH, NW, NG, DELTA, false, false>(at, dO + at.row, DELTA ? O + at.row : nullptr, lse + at.stat, delta + at.stat, dqkv + (at.k - qkv),
                                              dqkv + (at.v - qkv), nullptr, scale);
}

template <int DH>
__global__ void __launch_bounds__(NT, DH == 64 ? 3 : 2) attn_bwd_dq_mfma_k(const uint16_t *__restrict__ dO, const uint16_t *__restrict__ qkv,
                                                         const uint16_t *__restrict__ O, const float *__restrict__ lse, float *__restrict__ delta,
                                                         uint16_t *__restrict__ dqkv, int64_t Bn, int64_t Tn, int64_t H, float scale, Order order) {
    dq_block<DH, NT / 64, 2>(dO, qkv, O, lse, delta, dqkv, Bn, Tn, H, scale, order, blockIdx.x);
}

template <int DH>
__global__ void __launch_bounds__(dkv_waves<DH>() * 64, DH == 64 ? 3 : 2)
    attn_bwd_dkv_mfma_k(const uint16_t *__restrict__ dO, const uint16_t *__restrict__ qkv, const float *__restrict__ lse,
                        const float *__restrict__ delta, uint16_t *__restrict__ dqkv, int64_t Bn, int64_t Tn, int64_t H, float scale, Order order) {
    dkv_block<DH, dkv_waves<DH>(), 2, false>(dO, qkv, nullptr, lse, delta, dqkv, Bn, Tn, H, scale, order, blockIdx.x);
}

// Both kernels' blocks in one launch, those of key rows first: for sequences whose blocks leave the chip room, where each of the two
// kernels lasts as long as its longest chain of tiles.  The same rows to a block on either side; every output has the bits of the two
// launches.  Delta comes from a launch of its own, or (DELTA) both kinds of blocks multiply dO and O themselves: the blocks of query rows
// theirs, which they write, and those of key rows all that they meet, a tile ahead.
template <int DH, int NW, int NG, bool DELTA>
__global__ void __launch_bounds__(NW * 64, NG == 1 ? 2 : DH == 64 ? 3 : 2)
    attn_bwd_both_mfma_k(const uint16_t *__restrict__ dO, const uint16_t *__restrict__ qkv, const uint16_t *__restrict__ O, const float *__restrict__ lse,
                         float *__restrict__ delta, uint16_t *__restrict__ dqkv, int64_t Bn, int64_t Tn, int64_t H, float scale, Order order,
                         unsigned blocks) {
    if (blockIdx.x < blocks) dkv_block<DH, NW, NG, DELTA>(dO, qkv, O, lse, delta, dqkv, Bn, Tn, H, scale, order, blockIdx.x);
    else dq_block<DH, NW, NG>(dO, qkv, DELTA ? O : nullptr, lse, delta, dqkv, Bn, Tn, H, scale, order, blockIdx.x - blocks);
}

template <int DH> constexpr size_t fwd_smem() { return (size_t)3 * 2 * 32 * DH * 2; }      // three pairs of tiles
template <int DH> constexpr size_t kv_smem() { return (size_t)2 * 2 * 64 * DH * 2; }       // two buffers of two tiles
template <int DH, int NW, int NG> constexpr size_t dkv_smem() {         // tiles, V rows, then statistics
    return (size_t)2 * 2 * 64 * DH * 2 + (dkv_v_in_lds<DH, NG>() ? (size_t)NW * 16 * NG * DH * 2 : 0) + 2 * 128 * 4;
}

// Unsigned 32-bit buffer offsets: one head's rows, and PAST more, span less than 2 GiB.  A block's rows past the sequence (up to
// its size less one) are addressed too and refused by the descriptor, so their offsets must not wrap around 4 GiB: as many rows as
// twice PAST keep Tn + rows below twice Tn + PAST.
constexpr int64_t PAST = 192;
static_assert(dkv_waves<64>() * 32 <= 2 * PAST && dkv_waves<128>() * 32 <= 2 * PAST && 128 <= 2 * PAST, "offsets past the sequence do not wrap");
bool fits(int64_t Tn, int64_t H, int64_t dh) { return (Tn + PAST) * 3 * H * dh * 2 < ((int64_t)1 << 31); }

// The order and the grid of a kernel whose workgroups take `rows` rows each and of which a compute unit holds per_cu.  Heads taken
// together: all of them where that leaves nothing to wait for a free unit, otherwise as many as have 16 MiB of K and V (or Q and dO), so
// that an XCD's 4 MiB L2 sees most of a tile's reuse by the other blocks (4 x 2048, 32 heads of 128, 2 / 4 / 8 / 16 heads, forward: 176 /
// 169 / 167 / 171 us; 2 x 4096, 52 heads 486 / 487 / 473 / 483).
struct Launch {
    dim3 grid;
    Order order;
    Launch(int64_t n_heads, int64_t Tn, int64_t dh, int rows, int per_cu) {
        const int64_t of_xcd = (n_heads + 7) / 8, blocks = (Tn + rows - 1) / rows, by_bytes = ((int64_t)16 << 20) / (Tn * dh * 4);
        grid = dim3((unsigned)(blocks * of_xcd * 8));
        order.turn = of_xcd * blocks <= 32 * per_cu;
        order.heads = (int)(order.turn || by_bytes >= of_xcd ? of_xcd : by_bytes > 1 ? by_bytes : 1);
    }
};

}  // namespace

bool attn_mfma_supported(int dtype, int64_t Tn, int64_t H, int64_t dh) {
    return dtype == TIO_PREC_BF16 && (dh == 64 || dh == 128) && fits(Tn, H, dh);
}

void attn_fwd_mfma(hipStream_t s, const void *qkv, void *o, float *lse, int64_t B, int64_t Tn, int64_t H, int64_t dh) {
    const float scale = 1.0f / sqrtf((float)dh);
#define TIO_ATTN_FWD(DH, NG)                                                                                                                   \
    {                                                                                                                                          \
        const Launch l(B * H, Tn, DH, NT / 64 * 16 * NG, DH == 64 ? 4 : 3);                                                                    \
        attn_fwd_mfma_k<DH, NG, 1><<<l.grid, NT, fwd_smem<DH>(), s>>>(BatchRows{(const uint16_t *)qkv, B, Tn, H, l.order}, (uint16_t *)o, lse, scale); \
    }
    // Sixteen rows to a wavefront while the chip holds about all workgroups of 64 rows at once: half the work in a tile, where the chain
    // of a wavefront's tiles is what counts; more of them would load K and V twice as often.  us, 32 / 16 rows (workgroups of 64, the heads
    // rounded up to the XCDs: one with a head more than the others decides).  At head size 128 the line is where all of them are resident, four to
    // a unit, for long sequences: with as many workgroups of fewer heads, the longest chain of tiles is more of the launch, and half the work in
    // its tiles counts for more than twice the loads; for short ones it is lower.
    //   heads of 64:  8 x  192,  7  5.6 /  5.0 (168)    1 x 4096,  9 54.5 / 44.1 (1024)   3 x 2000, 13 29.9 / 29.7 (1280)
    //                 2 x 2048, 20 34.4 / 33.0 (1280)   4 x 3904,  5 57.8 / 59.3 (1464)   8 x 1024, 12 21.2 / 22.2 (1536)
    //   of 128:       4 x  333,  6 10.3 /  7.8 (144)    1 x 2048,  8 39.8 / 28.5 (256)    7 x  868,  8 23.3 / 19.6 (784)
    //                 8 x  256, 26 13.5 / 15.1 (832)    4 x 1024, 16 27.2 / 29.0 (1024)   1 x 4000,  9 72.7 / 65.1 (1008)
    const bool one = Launch(B * H, Tn, dh, 64, 1).grid.x <= (dh == 64 ? 1280 : Tn < 2048 ? 800 : 1024);
    if (dh == 64) {
        if (one) TIO_ATTN_FWD(64, 1) else TIO_ATTN_FWD(64, 2)
    } else {
        if (one) TIO_ATTN_FWD(128, 1) else TIO_ATTN_FWD(128, 2)
    }
#undef TIO_ATTN_FWD
}

void attn_bwd_mfma(hipStream_t s, const void *dO, const void *qkv, const void *O, const float *lse, float *delta, void *dqkv,
                   int64_t B, int64_t Tn, int64_t H, int64_t dh) {
    const float scale = 1.0f / sqrtf((float)dh);
    static bool attr_set = false;
    if (!attr_set) {
        (void)hipFuncSetAttribute((const void *)attn_bwd_dq_mfma_k<128>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kv_smem<128>());
        (void)hipFuncSetAttribute((const void *)attn_bwd_dkv_mfma_k<128>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<128, dkv_waves<128>(), 2>());
        (void)hipFuncSetAttribute((const void *)attn_bwd_both_mfma_k<128, 8, 2, false>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<128, 8, 2>());
        (void)hipFuncSetAttribute((const void *)attn_bwd_both_mfma_k<128, 4, 1, true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<128, 4, 1>());
        (void)hipFuncSetAttribute((const void *)attn_bwd_both_mfma_k<128, 4, 1, false>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<128, 4, 1>());
        attr_set = true;
    }
    // One launch for both gradients while its workgroups are at most a little more than the chip holds at once, with 16 rows to a
    // wavefront as in the forward pass while it holds about twice the workgroups of 64 rows (and up to 256 rows of a sequence nearly twice as
    // many of them: a block of 128 or 256 rows is a whole sequence or half of one there, most of whose products the mask throws away).
    // Forward and backward, us (workgroups of 64 rows on either side):
    //   32 rows, as in the launches below them / 16 rows
    //     heads of 64:  5 x 145, 22 19.1 / 16.1 (330)    8 x 512, 12 38.9 / 34.2 (768)    1 x 4096, 8 150 / 120 (512)    8 x 300, 20 34.4 / 30.7 (800)
    //                   8 x 256, 52 59.0 / 56.0 (1664)   6 x 512, 24 52.1 / 53.0 (1152)   8 x 1024, 8 64.1 / 66.1 (1024)
    //     of 128:       4 x 333,  6 32.9 / 24.6 (144)    1 x 2048, 8 112 / 83 (256)       3 x 700, 25 80.6 / 77.6 (880)    4 x 512, 16 53.1 / 44.5 (512)
    //                   8 x 256, 40 87.2 / 85.7 (1280)   8 x 512, 16 78.4 / 84.0 (1024)   1 x 4096, 16 311 / 335 (1024)
    //   32 rows, two launches / one
    //     heads of 64:  1 x 4096, 16 203 / 182           8 x 1024, 8 62.4 / 57.9          4 x 500, 31 41.1 / 39.5
    //     of 128:       4 x 1024, 16 112 / 104           1 x 4096, 16 362 / 304           2 x 2000, 15 191 / 165
    // Delta inside that launch while the tiles are few: the products are done over by every block of keys, the launch they replace
    // takes 3 us and two more between launches.  us, a launch of its own / inside: 5 x 145, 22 heads of 64 16.3 / 13.6, 8 x 512, 12 37.9 / 35.0,
    // 1 x 1024, 12 35.8 / 35.1, 1 x 4096, 8 123 / 131; 4 x 100, 6 heads of 128 14.9 / 12.8, 4 x 512, 16 47.5 / 44.8, 1 x 1024, 5 42.5 / 45.9.
    constexpr int64_t OWN_DELTA = 65536;                  // sequence length times head size
#define TIO_ATTN_BOTH_AS(DH, NW, NG, DELTA)                                                                                                    \
    attn_bwd_both_mfma_k<DH, NW, NG, DELTA><<<2 * l.grid.x, NW * 64, dkv_smem<DH, NW, NG>(), s>>>(                                             \
        (const uint16_t *)dO, (const uint16_t *)qkv, (const uint16_t *)O, lse, delta, (uint16_t *)dqkv, B, Tn, H, scale, l.order, l.grid.x)
#define TIO_ATTN_BOTH(DH, NW, NG, WORKGROUPS)                                                                                                  \
    {                                                                                                                                          \
        const Launch l(B * H, Tn, DH, NW * 16 * NG, NG == 1 ? 2 : DH == 64 ? 3 : 1);                                                           \
        if (2 * (int64_t)l.grid.x <= WORKGROUPS) {                                                                                             \
            if (NG == 1 && O && Tn * DH <= OWN_DELTA) {                                                                                        \
                TIO_ATTN_BOTH_AS(DH, NW, NG, (NG == 1));                                                                                       \
                return;                                                                                                                        \
            }                                                                                                                                  \
            if (O) attn_bwd_pre(s, TIO_PREC_BF16, dO, O, delta, B, Tn, H, DH);                                                                 \
            TIO_ATTN_BOTH_AS(DH, NW, NG, false);                                                                                               \
            return;                                                                                                                            \
        }                                                                                                                                      \
    }
#define TIO_ATTN_BWD(DH, DQ_PER_CU, DKV_PER_CU)                                                                                                \
    {                                                                                                                                          \
        const Launch q(B * H, Tn, DH, 128, DQ_PER_CU), kv(B * H, Tn, DH, dkv_waves<DH>() * 32, DKV_PER_CU);                                    \
        attn_bwd_dq_mfma_k<DH><<<q.grid, NT, kv_smem<DH>(), s>>>((const uint16_t *)dO, (const uint16_t *)qkv, (const uint16_t *)O, lse, delta, \
                                                                 (uint16_t *)dqkv, B, Tn, H, scale, q.order);                                  \
        attn_bwd_dkv_mfma_k<DH><<<kv.grid, dkv_waves<DH>() * 64, dkv_smem<DH, dkv_waves<DH>(), 2>(), s>>>(                                        \
            (const uint16_t *)dO, (const uint16_t *)qkv, lse, delta, (uint16_t *)dqkv, B, Tn, H, scale, kv.order);                             \
    }
    if (dh == 64) {
        TIO_ATTN_BOTH(64, 4, 1, 2 * (Tn <= 256 ? 1664 : 896))
        TIO_ATTN_BOTH(64, 4, 2, 1024)
        TIO_ATTN_BWD(64, 3, 3)
    } else {
        TIO_ATTN_BOTH(128, 4, 1, 2 * (Tn <= 256 ? 1664 : 896))
        TIO_ATTN_BOTH(128, 8, 2, 512)
        TIO_ATTN_BWD(128, 2, 1)
    }
#undef TIO_ATTN_BOTH
#undef TIO_ATTN_BOTH_AS
#undef TIO_ATTN_BWD
}

}  // namespace k
}  // namespace tio
