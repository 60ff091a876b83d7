// What the attentions over ranges of pages share (kv_ranges.hip, kv_prefix.hip).
#pragma once

#include "kv_tile.h"

namespace rift {

constexpr int kMaxParts = 64;   // of an item's tokens: a lane each where they are joined

// Rows of queries, one for each sequence and query head of a key head's group, over a prefix.
struct PrefixParams {
    const void* q;
    int64_t ld_q;
    TilePages pages;
    const int* table;
    int* status;
    float* slots;        // [key head][parts][rows][HD + 4]: weighted values, largest score (or another reference), sum
    int len, n_kv, n_pages, shift, group, rows, row_tiles, parts;
    float scale_log2;
};

int prefix_parts(int n_kv, int64_t rows, int len);
// pages of bf16 or 8 bits
hipError_t launch_prefix(const riftkv_cache& c, bool bf16, PrefixParams p, hipStream_t st);

}  // namespace rift
