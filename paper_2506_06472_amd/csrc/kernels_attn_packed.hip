// Causal attention over a packed batch on the matrix cores (bf16, head size 64 or 128): sequences of different lengths one behind the other, query
// heads in groups that share a key and value head.  The loops are those of attn_mfma_rows.h; here is where their rows lie and how the batch is cut.
//
// The G query heads of a key head count as G rows for each row of the sequence (row r, head i: r * G + i).  A block of query rows then reads K
// and V once for all its heads, has G times fewer keys between its first and last row's diagonals, and a short sequence fills it G times
// better; a block of keys takes the query rows of all its heads in one chain of tiles, so that dK and dV need no sums over heads.
// Workgroups are dealt longest first (attn_packed.h).  A block of keys whose chain would outlast the others is cut into pieces, whose fp32 sums
// a launch behind them adds in order: no atomics, and results that depend on nothing but the lengths and heads.
#include "../../include/teraio.h"
#include "attn_mfma_rows.h"
#include "attn_packed.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

struct PackedRows {
    static constexpr bool GROUPED = true;
    const uint16_t *qkv;
    int64_t ld, ldg;
    int32_t H, G;
    PackedPlaces places;

    template <int DH, typename P> __device__ __forceinline__ bool start(unsigned block, P &at, int &hk, const int32_t *&item) const {
        if (!places.find(block, hk, item)) return false;
        const int64_t first = item[0];
        at.q = qkv + first * ld + (int64_t)hk * G * DH;
        at.k = qkv + first * ld + (int64_t)(H + hk) * DH;
        at.v = at.k + (int64_t)places.heads * DH;
        at.ld = ld;
        at.row = first * ldg + (int64_t)hk * G * DH;
        at.ldg = ldg;
        at.stat = (int64_t)hk * G * places.rows + first;
        at.heads_ld = places.rows;
        at.Tn = item[1];
        at.G = G;
        return true;
    }
    template <int DH, int ROWS> __device__ __forceinline__ bool place(unsigned block, QueryPlace &at) const {
        const int32_t *item;
        int hk;
        if (!start<DH>(block, at, hk, item)) return false;
        at.v0 = item[2];
        return at.v0 >= 0 && at.v0 < at.Tn * G;
    }
    // hk: the key head; part: of its partial sums, or -1
    template <int DH, int KEYS> __device__ __forceinline__ bool place(unsigned block, KeyPlace &at, int &hk, int &part, int &pieces) const {
        const int32_t *item;
        if (!start<DH>(block, at, hk, item)) return false;
        at.kv0 = item[2];
        at.t0 = item[3];
        const int per_tile = 64 / G, tiles = (at.Tn - at.kv0 + per_tile - 1) / per_tile;
        at.t1 = item[4] < tiles ? item[4] : tiles;
        part = item[5];
        pieces = item[6];
        return at.kv0 >= 0 && at.kv0 < at.Tn && at.t0 >= 0;
    }
};

// Both gradients in one launch: the blocks of keys, then those of queries, which fill what the first leave empty at their end (in two launches, with
// delta in that of dQ: 32 heads in 8 groups, 128, 8192 rows 499 us forward and backward, in one 484; 40 in 8, 4 x 2048: 769 / 782; 32 in 8 of
// 64, 6096 rows: 418 / 394).  DELTA: delta is computed by both kinds of blocks, O is read for it; otherwise it comes from a launch before.
template <int DH, int NW, int NG, bool DELTA, bool TAIL>
__global__ void __launch_bounds__(NW * 64, NG == 1 ? 2 : DH == 64 ? 3 : 2)
    attn_packed_both_mfma_k(const PackedRows keys, const PackedRows queries, unsigned key_blocks, const uint16_t *__restrict__ dO,
                            const uint16_t *__restrict__ O, const float *__restrict__ lse, float *__restrict__ delta, uint16_t *__restrict__ dqkv, float *__restrict__ partial, int parts,
                            float scale) {
    if (blockIdx.x < key_blocks) {
        KeyPlace at;
        int hk, part, pieces;
        if (!keys.place<DH, NW * 16 * NG>(blockIdx.x, at, hk, part, pieces) || at.t0 >= at.t1 || part >= parts) return;
        float *const mine = part < 0 ? nullptr : partial + ((int64_t)hk * parts + part) * key_partial<DH, NW, NG>();
        dkv_rows<DH, NW, NG, DELTA, true, TAIL>(at, dO + at.row, DELTA ? O + at.row : nullptr, lse + at.stat, delta + at.stat, dqkv + (at.k - keys.qkv),
                                                dqkv + (at.v - keys.qkv), mine, scale);
    } else {
        QueryPlace at;
        if (!queries.place<DH, NW * 16 * NG>(blockIdx.x - key_blocks, at)) return;
        dq_rows<DH, NW, NG, true>(at, dO + at.row, DELTA ? O + at.row : nullptr, lse + at.stat, delta + at.stat, dqkv + (at.q - queries.qkv), scale);
    }
}

template <int DH, int NW, int NG>
__global__ void __launch_bounds__(NW * 64) attn_packed_sums_k(const PackedRows where, const float *__restrict__ partial, int parts, uint16_t *__restrict__ dqkv,
                                                              float scale) {
    KeyPlace at;
    int hk, part, pieces;
    if (!where.place<DH, NW * 16 * NG>(blockIdx.x, at, hk, part, pieces) || part < 0 || pieces < 1 || part > parts - pieces) return;
    const int which = (int)blockIdx.y & 1;
    key_sums<DH, NW, NG>(at, partial + ((int64_t)hk * parts + part) * key_partial<DH, NW, NG>(), pieces, which, (int)blockIdx.y >> 1,
                         dqkv + ((which ? at.v : at.k) - where.qkv), scale);
}

template <int DH, int SPLIT> constexpr size_t fwd_smem() { return (size_t)3 * 2 * 32 * SPLIT * DH * 2; }      // three steps
template <int DH, int NW, int NG> constexpr size_t dkv_smem(int group) {         // tiles, V rows, then statistics and the first rows' delta
    return (size_t)2 * 2 * 64 * DH * 2 + (dkv_v_in_lds<DH, NG>() ? (size_t)NW * 16 * NG * DH * 2 : 0) + 2 * 128 * 4 + (size_t)EARLY * group * 4;
}

PackedRows rows_of(const Packing &p, const void *device, const ItemList &list, int words, const void *qkv, int64_t ld, int64_t ldg) {
    return PackedRows{(const uint16_t *)qkv, ld, ldg, p.H, p.group(), packed_places(p, device, list, words, p.Hkv)};
}
constexpr int QUERY_WORDS = sizeof(QueryItem) / 4, KEY_WORDS = sizeof(KeyItem) / 4;

template <int DH> void fwd(hipStream_t s, const Packing &p, const void *device, const void *qkv, int64_t ld, void *o, int64_t ldo, float *lse, float scale) {
    const PackedRows w = rows_of(p, device, p.fwd, QUERY_WORDS, qkv, ld, ldo);
    auto go = [&](auto NG, auto SPLIT) {
        const auto kernel = attn_fwd_mfma_k<DH, NG(), SPLIT(), PackedRows>;
        (void)hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)fwd_smem<DH, SPLIT()>());
        kernel<<<w.places.grid(), NT * SPLIT(), fwd_smem<DH, SPLIT()>(), s>>>(w, (uint16_t *)o, lse, scale);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    if (p.fwd_rows == 128) go(Two{}, One{});
    else if (p.fwd_sets == 1) go(One{}, One{});
    else go(One{}, Two{});
}

// The delta of short sequences is computed where it is needed, by every block of keys that a row meets, which saves a launch of 3 us (eight sequences of up
// to 100 rows, 12 heads of 64 in 4 groups: forward and backward 19.6 -> 17.8 us); the bound is that of the kernels of one length.  In fp32 arithmetic
// at head size 32.
bool own_delta(const Packing &p) { return p.mfma ? p.keys == 64 && (int64_t)p.max_len * p.group() * p.dh <= 65536 : p.dh == 32; }

// blocks of NW wavefronts of 16 NG keys or query rows
template <int DH, int NW, int NG>
void both(hipStream_t s, const Packing &p, const void *device, const void *qkv, int64_t ld, const void *o, const void *dO, int64_t ldo, const float *lse,
          float *delta, float *partial, void *dqkv, float scale) {
    const PackedRows keys = rows_of(p, device, p.key, KEY_WORDS, qkv, ld, ldo), queries = rows_of(p, device, p.dq, QUERY_WORDS, qkv, ld, ldo);
    const unsigned key_blocks = keys.places.grid();
    auto go = [&](auto DELTA, auto TAIL) {
        const auto kernel = attn_packed_both_mfma_k<DH, NW, NG, DELTA(), TAIL()>;
        (void)hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<DH, NW, NG>(64));
        kernel<<<key_blocks + queries.places.grid(), NW * 64, dkv_smem<DH, NW, NG>(p.group()), s>>>(keys, queries, key_blocks, (const uint16_t *)dO, (const uint16_t *)o,
                                                                                          lse, delta, (uint16_t *)dqkv, partial, p.parts, scale);
    };
    auto with = [&](auto DELTA) {
        if (rows_between_loads<DH, NW>() % p.group()) go(DELTA, std::true_type{});
        else go(DELTA, std::false_type{});
    };
    if (NG == 1 && own_delta(p)) {
        with(std::bool_constant<NG == 1>{});
    } else {
        attn_packed_pre(s, TIO_PREC_BF16, dO, o, ldo, delta, p.rows, p.H, DH);
        with(std::false_type{});
    }
    if (p.sums.n) {
        const PackedRows r = rows_of(p, device, p.sums, KEY_WORDS, qkv, ld, ldo);
        attn_packed_sums_k<DH, NW, NG><<<dim3(r.places.grid(), DH / 16), NW * 64, 0, s>>>(r, partial, p.parts, (uint16_t *)dqkv, scale);
    }
}

template <int DH> void bwd(hipStream_t s, const Packing &p, const void *device, const void *qkv, int64_t ld, const void *o, const void *dO, int64_t ldo,
                           const float *lse, float *delta, float *partial, void *dqkv, float scale) {
    if (p.keys == 64) both<DH, 4, 1>(s, p, device, qkv, ld, o, dO, ldo, lse, delta, partial, dqkv, scale);
    else both<DH, dkv_waves<DH>(), 2>(s, p, device, qkv, ld, o, dO, ldo, lse, delta, partial, dqkv, scale);
}

int64_t delta_bytes(const Packing &p) { return ((int64_t)p.H * p.rows * 4 + 255) / 256 * 256; }

}  // namespace

int64_t attn_packed_work(const Packing &p) {
    const int64_t part = (int64_t)p.keys * p.dh * 2 * 4;
    return delta_bytes(p) + (int64_t)p.parts * p.Hkv * part + 256;
}

// 32-bit offsets, as in kernels_attn_mfma.hip: a sequence's rows, and the rows past it that a block asks for, span less than 2 GiB
// (in fp32 arithmetic: 32 rows less than 4 GiB).
bool attn_packed_fits(const Packing &p, int64_t ld, int64_t ldo) {
    constexpr int64_t PAST = 512;
    const int64_t most = ld > ldo ? ld : ldo;
    return most < ((int64_t)1 << 24) && (!p.mfma || ((int64_t)p.max_len + PAST) * most * 2 < ((int64_t)1 << 31));
}

// The launch over all rows and heads for delta, where it is not the gradients' own: a grid has fewer than 2^32 threads.
bool attn_packed_bwd_fits(const Packing &p) {
    const int64_t lanes = p.dh / (p.dtype == TIO_PREC_BF16 ? 8 : 4);
    return own_delta(p) || (int64_t)p.rows * p.H * lanes < ((int64_t)1 << 32) - NT;
}

void attn_packed_fwd(hipStream_t s, const Packing &p, const void *device, const void *qkv, int64_t ld, void *o, int64_t ldo, float *lse) {
    const float scale = 1.0f / sqrtf((float)p.dh);
    if (!p.mfma) attn_packed_fwd_f32(s, p, device, qkv, ld, o, ldo, lse, scale);
    else if (p.dh == 64) fwd<64>(s, p, device, qkv, ld, o, ldo, lse, scale);
    else fwd<128>(s, p, device, qkv, ld, o, ldo, lse, scale);
}

void attn_packed_bwd(hipStream_t s, const Packing &p, const void *device, const void *qkv, int64_t ld, const void *o, const void *dO, int64_t ldo,
                     const float *lse, void *work, void *dqkv) {
    const float scale = 1.0f / sqrtf((float)p.dh);
    float *const delta = (float *)work, *const partial = (float *)((char *)work + delta_bytes(p));
    if (!p.mfma) attn_packed_bwd_f32(s, p, device, qkv, ld, o, dO, ldo, lse, delta, dqkv, scale);
    else if (p.dh == 64) bwd<64>(s, p, device, qkv, ld, o, dO, ldo, lse, delta, partial, dqkv, scale);
    else bwd<128>(s, p, device, qkv, ld, o, dO, ldo, lse, delta, partial, dqkv, scale);
}

}  // namespace k
}  // namespace tio
