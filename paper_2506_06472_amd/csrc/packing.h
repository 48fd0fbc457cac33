// A packed batch: sequences of different lengths one behind the other, and how attention over them is cut into workgroups.
// Built on the host from the offsets; the kernels read a copy of `data` in device memory.
#pragma once
#include <cstdint>
#include <vector>

namespace tio {

// A list of work items in Packing::data: `n` items of `words` words each from word `at` (a multiple of four) on, the longest first.
struct ItemList {
    int32_t at = 0, n = 0;
};

// What the kernels read of an item
struct QueryItem {
    int32_t first, len;      // the sequence's first row, its rows
    int32_t v0, reserved;    // the block's first query row; all query heads of a key head together count as rows of one sequence
};
struct KeyItem {
    int32_t first, len;
    int32_t kv0;             // the block's first key row
    int32_t t0, t1;          // tiles of its query rows
    int32_t part;            // where its sums go: -1 to the gradients, otherwise to the partial sums
    int32_t pieces;          // of an item of Packing::sums: how many partial sums from `part` on are one block's
    int32_t reserved;
};

struct Packing {
    int32_t n_seqs = 0, rows = 0, max_len = 0;
    int32_t dtype = 0, H = 0, Hkv = 0, dh = 0;   // H = 0: no attention
    std::vector<int32_t> data;                   // the n_seqs + 1 offsets, padding to a multiple of four words, then the lists
    bool mfma = false;                           // bf16 matrix cores (head size 64 or 128); otherwise fp32 arithmetic
    int32_t fwd_rows = 0, dq_rows = 0, keys = 0; // rows of an item
    int32_t fwd_sets = 1;                        // sets of wavefronts that share a forward item's rows
    ItemList fwd, dq, key, sums;
    int32_t parts = 0;                           // blocks of partial sums for each key head
    int group() const { return Hkv ? H / Hkv : 1; }
};

// Query rows of a tile of the key items: whole rows of all heads of a group
inline int rows_per_tile(bool mfma, int group) { return mfma ? 64 / group : 32; }

// throws std::invalid_argument
Packing build_packing(const int32_t *offsets, int32_t n_seqs, int32_t dtype, int64_t H, int64_t Hkv, int64_t dh);

}  // namespace tio
