// Internal launchers of the paged key-value cache (host side).  kv_capi.hip
// validates arguments and calls these; every launcher only enqueues work.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/rift_kv.h"
#include "launch.h"

namespace rift {

// RIFT_OK, or what is wrong with the pages' shape, and with `arrays` their pointers
rift_status kv_check_cache(const riftkv_cache* c, bool arrays);

constexpr int kMaxRotary = 256;
constexpr int64_t kMaxTokens = 1 << 30;   // of a table: a tile's end is within 31 bits

// One of the two row sets that a rotation takes: n heads a row.
struct RopeRows {
    const void* x;
    void* y;
    int64_t ld_x, ld_y;
    int n;
};
// Turns (not radians) a position of each pair: hi + lo, to about 2^-77 of it.
struct RopeFreqs {
    double hi[kMaxRotary / 2];
    float lo[kMaxRotary / 2];
};
hipError_t launch_kv_rope(const RopeRows& q, const RopeRows& k, bool bf16, const int* positions, int rows, int head_dim,
                          int rotary_dim, bool interleaved, const RopeFreqs& freqs, float magnitude, hipStream_t st);

// Where rows go, or come from: the page table and each row's sequence and position.
struct KvPlaces {
    const int* table;
    int n_seq, max_pages;
    const int* seq_ids;     // null: row i is of sequence i
    const int* positions;
    int rows;
    int* status;
};
hipError_t launch_kv_write(const riftkv_cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, bool bf16,
                           const KvPlaces& at, hipStream_t st);
hipError_t launch_kv_read(const riftkv_cache& c, void* k, int64_t ld_k, void* v, int64_t ld_v, bool bf16,
                          const KvPlaces& at, hipStream_t st);

// What a decode step over pages needs before its layers, per sequence: the row of
// (cos, sin) of its position [n_seq][hd / 2]; its length with the new token (0 for a negative
// position, -1 for one past `capacity`); its own number.
hipError_t launch_kv_decode_prep(const int* positions, int n_seq, int64_t capacity, int hd, float rope_base, float2* rope,
                                 int* lens, int* rows, hipStream_t st);

// The new tokens' q|k|v as a product's partial sums [slots][n][3 d] (launch_skinny_gemm): added up,
// q and k rotated by row i of rope, q as rows, k and v (rounded to bf16) to the places `at`
// of sequence i, as launch_kv_write would.  d = n_kv_heads * head_dim; pages of bf16 or 8 bits.
hipError_t launch_kv_decode_qkv(const riftkv_cache& c, const float* part, SkinnySplit sp, int d, const float2* rope,
                                const KvPlaces& at, uint16_t* q, hipStream_t st);

struct KvAttention {
    const void* q;
    void* out;
    int64_t ld_q, ld_out;
    int n_heads;
    bool bf16;              // type of q and out
    const int* table;
    int n_seq, max_pages;
    const int* lens;
    float scale;
    int* status;
    void* workspace;
};
size_t kv_attention_workspace(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages);
// whether 64-bit counts hold the call's tiles
bool kv_attention_counts(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages);
hipError_t launch_kv_attention(const riftkv_cache& c, const KvAttention& a, hipStream_t st);

}  // namespace rift
