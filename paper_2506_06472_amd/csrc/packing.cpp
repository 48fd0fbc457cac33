// How a packed batch is cut into workgroups.  Every list is sorted by the time its items take, the longest first: workgroups start in the order of
// their numbers, so that what is left when the chip runs empty are the shortest.
#include "packing.h"

#include <algorithm>
#include <cstring>
#include <stdexcept>
#include <string>

#include "../../include/teraio.h"

namespace tio {

namespace {

template <typename Item> ItemList append(Packing &p, std::vector<std::pair<int64_t, Item>> &items) {
    std::stable_sort(items.begin(), items.end(), [](const auto &a, const auto &b) { return a.first > b.first; });
    ItemList l;
    l.at = (int32_t)p.data.size();
    l.n = (int32_t)items.size();
    p.data.resize(p.data.size() + items.size() * (sizeof(Item) / 4));
    for (size_t i = 0; i < items.size(); ++i) std::memcpy(p.data.data() + l.at + i * (sizeof(Item) / 4), &items[i].second, sizeof(Item));
    return l;
}

// blocks of `rows` query rows; group heads' rows count as one sequence
ItemList query_items(Packing &p, const int32_t *offsets, int rows, int group) {
    std::vector<std::pair<int64_t, QueryItem>> items;
    for (int s = 0; s < p.n_seqs; ++s) {
        const int32_t first = offsets[s], len = offsets[s + 1] - first;
        for (int64_t v0 = 0; v0 < (int64_t)len * group; v0 += rows) {
            const int64_t last = std::min<int64_t>((v0 + rows - 1) / group, len - 1);
            items.push_back({last, QueryItem{first, len, (int32_t)v0, 0}});
        }
    }
    return append(p, items);
}

int64_t query_blocks(const Packing &p, const int32_t *offsets, int rows, int group) {
    int64_t n = 0;
    for (int s = 0; s < p.n_seqs; ++s) n += ((int64_t)(offsets[s + 1] - offsets[s]) * group + rows - 1) / rows;
    return n;
}

// into how many items a block of keys with that many tiles is cut
int64_t pieces_of(int64_t tiles, int64_t piece) { return tiles > piece + piece / 4 ? (tiles + piece - 1) / piece : 1; }
constexpr int64_t WHOLE = (int64_t)1 << 40;          // a piece that no block is larger than

// Blocks of `keys` key rows.  A block whose tiles are more than a piece's is shared by several items, whose sums are added afterwards.
void key_items(Packing &p, const int32_t *offsets, int keys, int per_tile, int64_t piece) {
    std::vector<std::pair<int64_t, KeyItem>> items, sums;
    for (int s = 0; s < p.n_seqs; ++s) {
        const int32_t first = offsets[s], len = offsets[s + 1] - first;
        for (int64_t kv0 = 0; kv0 < len; kv0 += keys) {
            const int64_t tiles = (len - kv0 + per_tile - 1) / per_tile, pieces = pieces_of(tiles, piece);
            if (pieces == 1) {
                items.push_back({tiles, KeyItem{first, len, (int32_t)kv0, 0, (int32_t)tiles, -1, 0, 0}});
                continue;
            }
            sums.push_back({pieces, KeyItem{first, len, (int32_t)kv0, 0, 0, p.parts, (int32_t)pieces, 0}});
            for (int64_t i = 0; i < pieces; ++i) {
                const int64_t t0 = tiles * i / pieces, t1 = tiles * (i + 1) / pieces;
                items.push_back({t1 - t0, KeyItem{first, len, (int32_t)kv0, (int32_t)t0, (int32_t)t1, p.parts++, 0, 0}});
            }
        }
    }
    p.key = append(p, items);
    p.sums = append(p, sums);
}

int64_t key_blocks(const Packing &p, const int32_t *offsets, int keys, int per_tile, int64_t piece) {
    int64_t n = 0;
    for (int s = 0; s < p.n_seqs; ++s)
        for (int64_t left = offsets[s + 1] - offsets[s]; left > 0; left -= keys) n += pieces_of((left + per_tile - 1) / per_tile, piece);
    return n;
}

// How the backward pass is cut: the keys of a block (64 of four wavefronts with 16 keys each; or 128 of four, head size 64, and 256 of eight,
// head size 128, with 32 each, which do a product for half the reads but are fewer and take longer for a tile) and the tiles of a piece.
// The time is estimated as that of the tiles, dealt evenly, or of the longest chain of them if that is longer, a quarter of the shorter of the two, and
// the partial sums' way to memory and back.  us; fitted to 480 ways to cut 30 batches (2 to 52 heads, groups of 1 to 13, 370 to 8192 rows), of which
// it picks the fastest or one within 6 %, 0.6 % behind on average.  Backward, us: 12 heads in 4 groups, 64, 8192 rows of 17 sequences: 128 keys whole 101,
// in pieces of 16 tiles 61, 64 keys whole 80, in pieces of 16 61; 32 heads in 8 groups, 128, 8192 rows of 8: 256 keys whole 398, in pieces of 64 364, 64 keys
// whole 421; 7 heads, 128, 2600 rows of two: 256 keys whole 524, in pieces of 16 73, 64 keys whole 265, in pieces of 16 52.
struct Way {
    int keys;
    double tile, chain, fixed;                       // a tile among others (per compute unit), a tile of a chain, the rest
};
constexpr Way WAYS[2][2] = {{{128, 0.78, 1.47, 9.1}, {64, 0.53, 1.02, 7.0}}, {{256, 3.0, 2.35, 12.0}, {64, 1.03, 1.32, 7.9}}};     // head size 64, 128
constexpr int64_t PIECES[] = {WHOLE, 96, 64, 48, 32, 24, 16, 12, 8, 6, 4};
constexpr int64_t MOST_PARTIAL = (int64_t)512 << 20;  // bytes of partial sums

int64_t cut_backward(Packing &p, const int32_t *offsets, int per_tile) {
    double best = 0.0;
    int64_t best_piece = WHOLE;
    p.keys = 0;
    for (const Way &way : WAYS[p.dh == 128]) {
        const int64_t group = p.group();
        int64_t tiles = 0, query_tiles = 0, longest_query = 0;
        std::vector<int64_t> blocks;                 // their tiles
        for (int s = 0; s < p.n_seqs; ++s) {
            const int64_t len = offsets[s + 1] - offsets[s];
            for (int64_t left = len; left > 0; left -= way.keys) {
                blocks.push_back((left + per_tile - 1) / per_tile);
                tiles += blocks.back();
            }
            for (int64_t v0 = 0; v0 < len * group; v0 += way.keys) {
                const int64_t t = std::min<int64_t>((v0 + way.keys - 1) / group, len - 1) / 64 + 1;
                query_tiles += t;
                longest_query = std::max(longest_query, t);
            }
        }
        const double work = ((double)tiles + 0.75 * (double)query_tiles) * p.Hkv * way.tile / 256.0;
        for (const int64_t piece : PIECES) {
            int64_t parts = 0, longest = 0;
            for (const int64_t t : blocks) {
                const int64_t n = pieces_of(t, piece);
                longest = std::max(longest, (t + n - 1) / n);
                if (n > 1) parts += n;
            }
            if (piece != WHOLE && !parts) continue;  // no block is that large
            const int64_t bytes = parts * p.Hkv * way.keys * p.dh * 8;
            if (bytes > MOST_PARTIAL) continue;
            const double chain = (double)longest * way.chain, rows = 0.75 * (double)longest_query * way.chain;
            const double us = way.fixed + std::max(std::max(work, chain), rows) + 0.25 * std::min(work, chain) + 0.5e-6 * (double)bytes + (parts ? 2.4 : 0.0);
            if (!p.keys || us < best) best = us, best_piece = piece, p.keys = way.keys;
        }
    }
    return best_piece;
}

// A grid has fewer than 2^32 threads, of which a workgroup here has at most 512 (and the kernels in fp32 arithmetic one for every query head).  Asked before the
// lists are built: those of a batch that is refused could be larger than the host's memory.
void check_grids(const Packing &p, int64_t fwd, int64_t dq, int64_t key) {
    const int64_t heads = p.mfma ? p.Hkv : p.H, items = std::max(fwd, dq + key) + 32;
    if (items * heads >= ((int64_t)1 << 23)) throw std::invalid_argument("too many blocks of rows: cut the batch");
}

}  // namespace

Packing build_packing(const int32_t *offsets, int32_t n_seqs, int32_t dtype, int64_t H, int64_t Hkv, int64_t dh) {
    if (n_seqs < 1) throw std::invalid_argument("a packing needs at least one sequence");
    if (n_seqs >= 1 << 28) throw std::invalid_argument("too many sequences");
    if (offsets[0] != 0) throw std::invalid_argument("the first offset must be 0");
    Packing p;
    p.n_seqs = n_seqs;
    for (int s = 0; s < n_seqs; ++s) {
        if (offsets[s + 1] < offsets[s]) throw std::invalid_argument("offset " + std::to_string(s + 1) + " is smaller than the one before it");
        p.max_len = std::max(p.max_len, offsets[s + 1] - offsets[s]);
    }
    p.rows = offsets[n_seqs];
    p.dtype = dtype;
    p.data.assign(offsets, offsets + n_seqs + 1);
    p.data.resize((p.data.size() + 3) / 4 * 4, 0);
    if (H == 0 && Hkv == 0 && dh == 0) return p;
    if (dtype != TIO_PREC_FP32 && dtype != TIO_PREC_BF16) throw std::invalid_argument("unknown element type");
    if (dh != 32 && dh != 64 && dh != 128) throw std::invalid_argument("head dimension must be 32, 64 or 128");
    if (H < 1 || Hkv < 1 || H % Hkv) throw std::invalid_argument("the query heads must be a multiple of the key heads");
    if (H / Hkv > 64) throw std::invalid_argument("at most 64 query heads to a key head");
    if (H > 65536) throw std::invalid_argument("too many heads");
    if ((int64_t)p.rows * H >= ((int64_t)1 << 31)) throw std::invalid_argument("rows times heads must stay below 2^31");
    p.H = (int32_t)H, p.Hkv = (int32_t)Hkv, p.dh = (int32_t)dh;
    p.mfma = dtype == TIO_PREC_BF16 && dh != 32;
    const int group = p.group();
    if (!p.mfma) {                                   // every query head by itself
        p.fwd_rows = p.dq_rows = p.keys = 32;
        const int64_t n = query_blocks(p, offsets, 32, 1);             // of keys as many
        check_grids(p, n, n, n);
        p.fwd = p.dq = query_items(p, offsets, 32, 1);
        key_items(p, offsets, 32, 32, WHOLE);
        return p;
    }
    // Forward pass: sixteen rows to a wavefront while there are few blocks of 64 rows, and two sets of wavefronts to a block, which take every other tile of
    // keys, while the longest chain of tiles is what counts.  us, 32 rows / 16 / two sets (blocks of 64 rows):
    //   heads of 64:  8192 rows of 17 sequences, 12/4 20.9 / 19.3 / 21.9 (1550)  4096, 32/8 81.8 / 85.0 / 87.8 (2048)  2 x 1024, 24 19.3 / 16.0 / 16.2 (768)
    //                 2 x 1024, 12 17.3 / 13.6 / 11.2 (384)    2048 and 1000, 8 29.4 / 22.5 / 17.2 (381)    4096, 4/1 52.9 / 39.5 / 27.5 (256)
    //   of 128:       3 x 1024, 32/8 35.0 / 37.5 / 58.8 (1536)  2048, 32/8 48.2 / 45.6 / 57.5 (1024)   1200 and 700, 16/4 26.6 / 22.2 / 22.7 (506)
    //                 1700 and 900, 7/1 33.6 / 25.8 / 21.4 (285)  4 x 300, 16/4 11.0 / 9.4 / 12.1 (304)  4096, 4/1 69.9 / 52.7 / 40.4 (256)
    const int64_t blocks = query_blocks(p, offsets, 64, group) * Hkv;
    p.fwd_rows = blocks <= (dh == 64 ? 1800 : 1024) ? 64 : 128;
    p.fwd_sets = blocks <= (dh == 64 ? 512 : p.max_len >= 700 ? 400 : 256) ? 2 : 1;
    const int per_tile = rows_per_tile(true, group);
    check_grids(p, 0, query_blocks(p, offsets, 256, group), query_blocks(p, offsets, 256, 1));           // the fewest there may be
    const int64_t piece = cut_backward(p, offsets, per_tile);
    p.dq_rows = p.keys;
    check_grids(p, query_blocks(p, offsets, p.fwd_rows, group), query_blocks(p, offsets, p.dq_rows, group), key_blocks(p, offsets, p.keys, per_tile, piece));
    p.fwd = query_items(p, offsets, p.fwd_rows, group);
    p.dq = p.fwd_rows == p.dq_rows ? p.fwd : query_items(p, offsets, p.dq_rows, group);
    key_items(p, offsets, p.keys, per_tile, piece);
    return p;
}

}  // namespace tio
