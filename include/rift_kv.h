/*
 * rift_kv.h -- C ABI of the paged key-value cache (librift.so, gfx950).
 *
 * rift_prefill and rift_decode_step (rift.h) keep keys and values in dense
 * planes.  Here they live in pages of page_size tokens that any number of
 * sequences take from one pool, in 16 or 32 bits or quantised to 8, with one
 * key-value head for each group of query heads:
 *   riftkv_rope       rotary positions of query and key rows
 *   riftkv_rope_axes  the same with several positions a row (tile, row, column)
 *   riftkv_write      new key and value rows into their sequences' pages,
 *                     quantised as they are written
 *   riftkv_read       rows of the pages back, as dense rows
 *   riftkv_attention  one new token of every sequence over its pages
 *   riftkv_attention_shared  the same after a prefix that all sequences share,
 *                     read for many of them at a time
 *   riftkv_page_bounds, riftkv_select_pages, riftkv_attention_pages
 *                     the same over the pages that promise the largest scores
 *   riftkv_decode_step  a decode step of rift.h's model over them
 *
 * The conventions of rift.h hold: device pointers unless marked [host], buffers
 * and workspace owned by the caller, calls asynchronous and ordered on
 * `stream`, arguments checked on the host before anything is enqueued.
 * Base pointers of rows and pages are 16-byte aligned and row strides a
 * multiple of 16 bytes (RIFT_ERR_SHAPE), except in riftkv_rope and riftkv_rope_axes, which take any.
 * A call runs on the current device, to which `stream` and all memory belong.
 *
 * Pages
 *   page_table [n_seq][max_pages] i32: entry p of a sequence is the page of its
 *   tokens p page_size .. (p + 1) page_size - 1.  Entries past a sequence's
 *   length are not read.  Sequences may share pages that neither writes.
 *
 * Quantised pages (RIFTKV_FP8: OCP e4m3; RIFTKV_INT8)
 *   A row is one token's key or value of one head.  Its scale is a power of two,
 *   kept as a byte b, 2^(b - 127): the smallest that brings the row's largest
 *   magnitude to at most 448 (e4m3) or 127 (int8), 1 <= b <= 254; a row of zeros
 *   has b = 1.  A value is stored as x 2^(127 - b) rounded to nearest even and
 *   stands for code 2^(b - 127).  That product is exact in f32, and in bf16 for rows
 *   whose largest magnitude is at least 2^-110: a read back loses nothing, and
 *   writing it again gives the same values (e4m3: not always the same bytes, where the
 *   largest was rounded down to 448 times half the scale).  A row that holds NaN or
 *   infinity has b = 255 and codes 0, and reads back as NaN.
 *
 * Status word
 *   status [1] i32 is set to RIFT_ERR_SHAPE where a call finds an index or length
 *   out of range on the device, and is otherwise left as it is: clear it once,
 *   and any number of calls may share it.
 */
#ifndef RIFT_KV_H
#define RIFT_KV_H

#include "rift.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RIFTKV_ABI_VERSION 1

/* RIFTKV_ABI_VERSION that the loaded library was built with. */
RIFT_API int32_t riftkv_abi_version(void);

typedef enum { RIFTKV_F32 = 0, RIFTKV_BF16 = 1, RIFTKV_FP8 = 2, RIFTKV_INT8 = 3 } riftkv_dtype;

/* One layer's pages. */
typedef struct {
    void* k;            /* [n_pages][n_kv_heads][page_size][head_dim] dt */
    void* v;            /* the same */
    uint8_t* k_scale;   /* [n_pages][n_kv_heads][page_size], FP8 and INT8 only (else NULL) */
    uint8_t* v_scale;
    int32_t n_pages;    /* >= 1; n_pages * page_size <= INT32_MAX */
    int32_t page_size;  /* a power of two from 16 to 4096 */
    int32_t n_kv_heads; /* 1 to 1024 */
    int32_t head_dim;   /* 64 or 128 */
    riftkv_dtype dt;
} riftkv_cache;

/* ------------------------------------------------------------------ positions */

typedef enum {
    RIFTKV_ROPE_NONE = 0,   /* f_j = base^(-2j/R), R = rotary_dim                            */
    RIFTKV_ROPE_LINEAR = 1, /* f_j / factor                                                  */
    RIFTKV_ROPE_BASE = 2,   /* base factor^(R/(R-2)) in place of base; R > 2                 */
    RIFTKV_ROPE_RAMP = 3,   /* YaRN: f_j (1 - r_j) + (f_j / factor) r_j, r_j from 0 to 1 over
                               the pairs from a = floor(D(high)) to b = ceil(D(low)) (within
                               [0, R - 1]; b = a + 0.001 where they meet), D(n) = R
                               ln(original_len / (2 pi n)) / (2 ln base) the pair that turns
                               n times within original_len; magnitude 1 + 0.1 ln(factor)     */
    RIFTKV_ROPE_BANDS = 4   /* n_j = original_len f_j / (2 pi) turns: f_j for n_j > high,
                               f_j / factor for n_j < low, between them
                               f_j s + (f_j / factor)(1 - s), s = (n_j - low) / (high - low) */
} riftkv_rope_scaling;

typedef struct {
    int32_t rotary_dim;          /* even, 2 to 256                             */
    riftkv_rope_scaling scaling;
    double base;                 /* > 1                                        */
    double factor;               /* >= 1, except NONE                          */
    double original_len;         /* > 0, RAMP and BANDS                        */
    double low, high;            /* 0 < low < high, RAMP (1, 32) and BANDS (1, 4) */
} riftkv_rope_cfg;

/*
 * riftkv_rope_freqs -- [host only] the angle a position of each of the rotary_dim / 2
 * pairs, in float64, and the factor on the rotated pairs that goes with them.
 * freqs [host] out [rotary_dim / 2];  magnitude [host] out (1 except RAMP; may be NULL)
 * Errors: RIFT_ERR_NULL, RIFT_ERR_SHAPE (rotary_dim), RIFT_ERR_UNSUPPORTED (scaling),
 * RIFT_ERR_NONFINITE (a value out of range or not finite, a base that the factor makes so).
 */
RIFT_API rift_status riftkv_rope_freqs(const riftkv_rope_cfg* cfg, double* freqs, double* magnitude);

typedef enum {
    RIFTKV_ROPE_HALF = 0,        /* pair j: elements j and j + rotary_dim / 2 */
    RIFTKV_ROPE_INTERLEAVED = 1  /* pair j: elements 2 j and 2 j + 1          */
} riftkv_rope_layout;

/*
 * riftkv_rope -- rotary positions: for every row, head and pair (x1, x2) of the
 * head's first rotary_dim elements
 *   (y1, y2) = magnitude (x1 cos a - x2 sin a, x2 cos a + x1 sin a),
 * a = position * freqs[j], reduced in float64 whatever the position, the products
 * in float32; the other elements are copied.
 * q, k        [rows][n_q | n_k][head_dim] dt, rows ld_q | ld_k elements apart; either
 *             may be absent (n_q or n_k 0, its pointers NULL)
 * q_out, k_out  the same, ld_q_out | ld_k_out apart; may be q and k themselves (with the
 *             same stride); otherwise outputs overlap no input
 * positions   [rows] i32, any value
 * freqs       [host] [rotary_dim / 2], finite; read before the call returns
 * magnitude   finite in float32
 * Shape rules: rows >= 0, 0 <= n_q, n_k <= 4096, 1 <= head_dim <= 256,
 * rotary_dim even in [2, head_dim], every ld >= its heads * head_dim.
 */
RIFT_API rift_status riftkv_rope(const void* q, int64_t ld_q, int32_t n_q, void* q_out, int64_t ld_q_out,
                                 const void* k, int64_t ld_k, int32_t n_k, void* k_out, int64_t ld_k_out,
                                 rift_dtype dt, const int32_t* positions, int32_t rows, int32_t head_dim,
                                 int32_t rotary_dim, riftkv_rope_layout layout, const double* freqs,
                                 double magnitude, rift_stream stream);

/*
 * riftkv_rope_axes -- riftkv_rope with a position of every row on each of several axes (a tile's place
 * in the scene, row and column in the tile): pair j turns by positions[axes[j]][row] * freqs[j].
 * positions   [n_axes][rows] i32, any value
 * axes        [host] [rotary_dim / 2] i32 in [0, n_axes); read before the call returns
 * Everything else as for riftkv_rope, and with all positions of a row the same its results, bit for bit.
 * Shape rules: 1 <= n_axes <= 8.  Errors: RIFT_ERR_SHAPE also for an axis out of range.
 */
RIFT_API rift_status riftkv_rope_axes(const void* q, int64_t ld_q, int32_t n_q, void* q_out, int64_t ld_q_out,
                                      const void* k, int64_t ld_k, int32_t n_k, void* k_out, int64_t ld_k_out,
                                      rift_dtype dt, const int32_t* positions, int32_t n_axes, int32_t rows,
                                      int32_t head_dim, int32_t rotary_dim, riftkv_rope_layout layout,
                                      const double* freqs, const int32_t* axes, double magnitude, rift_stream stream);

/* ------------------------------------------------------------------ pages */

/*
 * riftkv_write -- rows of k and v into the pages of their sequences.
 * cache       [host] the pages (the struct; its arrays are device memory)
 * k, v        [rows][n_kv_heads][head_dim] dt, rows ld_k | ld_v elements apart
 * page_table  [n_seq][max_pages] i32
 * seq_ids     [rows] i32 the row's sequence, or NULL: row i is of sequence i
 * positions   [rows] i32 the row's position in it
 * A row whose sequence or position is negative is skipped (padding).  A row
 * whose sequence is >= n_seq, whose position is >= max_pages * page_size or
 * whose page is outside [0, n_pages) sets the status and is skipped.  Of two
 * rows of a call for the same place either may be there afterwards, or parts
 * of both.  f32 rows in bf16 pages are rounded to nearest even.
 * Shape rules: rows, n_seq, max_pages >= 0, max_pages * page_size <= 2^30, ld >=
 * n_kv_heads * head_dim.  Errors: RIFT_ERR_DTYPE also for bf16 rows in f32 pages.
 */
RIFT_API rift_status riftkv_write(const riftkv_cache* cache, const void* k, int64_t ld_k, const void* v,
                                  int64_t ld_v, rift_dtype dt, const int32_t* page_table, int32_t n_seq,
                                  int32_t max_pages, const int32_t* seq_ids, const int32_t* positions,
                                  int32_t rows, int32_t* status, rift_stream stream);

/*
 * riftkv_read -- rows of the pages, as riftkv_write addresses them, into dense
 * rows: k_out and v_out [rows][n_kv_heads][head_dim] dt, ld_k | ld_v elements apart.
 * Rows that are skipped or out of range are left as they are.  8-bit values are
 * exact in either dt; f32 pages read as bf16 are rounded to nearest even.
 */
RIFT_API rift_status riftkv_read(const riftkv_cache* cache, void* k_out, int64_t ld_k, void* v_out,
                                 int64_t ld_v, rift_dtype dt, const int32_t* page_table, int32_t n_seq,
                                 int32_t max_pages, const int32_t* seq_ids, const int32_t* positions,
                                 int32_t rows, int32_t* status, rift_stream stream);

/* ------------------------------------------------------------------ attention */

/* Workspace bytes of riftkv_attention for these heads and a table of n_seq sequences of
 * max_pages pages (0 for shapes that it refuses).  Not smaller for more sequences or
 * wider tables. */
RIFT_API size_t riftkv_attention_workspace_size(const riftkv_cache* cache, int32_t n_heads, int32_t n_seq,
                                                int32_t max_pages);

/*
 * riftkv_attention -- one query token of every sequence over the first lens[i]
 * tokens of its pages (its own among them, once written):
 *   out = sum_j softmax_j(scale q . k_j) v_j, j < lens[i],
 * query head h with key-value head h / (n_heads / n_kv_heads).  Scores, weights and
 * sums in float32 (with 8-bit pages the product of a weight, at most 1, and its row's
 * scale is cut off at 2^-133, fewer bits than float32 holds where the scale is below
 * 2^-110); a sequence of length 0 gives zeros.  With pages of bf16 an infinite value
 * gives an infinity or NaN, and an infinite key for f32 queries NaN where its weight
 * may be 0: their terms in the matrix products can be 0.
 * q        [n_seq][n_heads][head_dim] dt, sequences ld_q elements apart
 * out      [n_seq][n_heads][head_dim] dt, ld_out apart; overlaps no input
 * lens     [n_seq] i32 in [0, max_pages * page_size]
 * scale    1/sqrt(head_dim) as a rule; it and its product with log2(e) are finite
 * A length out of range, or a page outside [0, n_pages) among a sequence's tokens,
 * sets the status and makes that sequence's output NaN.
 * What lies in a page past a sequence's length has no effect, whatever its bits.
 * How the keys are dealt out depends on n_seq, max_pages and all sequences' lengths: a
 * result may differ in its last bits where any of these does, never between two calls
 * with the same.
 * dt bf16 with pages of bf16, fp8 or int8; dt f32 with any.
 * Shape rules: n_heads a multiple of n_kv_heads, at most 4096; 0 <= n_seq <= 65535; max_pages >=
 * 0, max_pages * page_size <= 2^30.  workspace >= riftkv_attention_workspace_size
 * bytes, 256-byte aligned; calls that may overlap in time need one each.
 */
RIFT_API rift_status riftkv_attention(const riftkv_cache* cache, const void* q, int64_t ld_q, int32_t n_heads,
                                      rift_dtype dt, const int32_t* page_table, int32_t n_seq, int32_t max_pages,
                                      const int32_t* lens, float scale, void* out, int64_t ld_out, int32_t* status,
                                      void* workspace, size_t ws_bytes, rift_stream stream);

/* ------------------------------------------------------------------ a shared prefix */

/* Workspace bytes of riftkv_attention_shared (0 for shapes that it refuses).  Not smaller for more
 * sequences, a longer prefix or wider tables. */
RIFT_API size_t riftkv_attention_shared_workspace_size(const riftkv_cache* cache, int32_t n_heads, int32_t n_seq,
                                                       int32_t prefix_len, int32_t max_pages);

/*
 * riftkv_attention_shared -- riftkv_attention of sequences that all begin with the same prefix_len tokens: each
 * attends to those and then to the first lens[i] tokens of its own pages, its own row i of page_table.  The prefix'
 * keys and values are read once for every 128 query rows of a key head (a sequence has n_heads / n_kv_heads), or every 16 where there
 * is little to do and where the pages are f32, or 8-bit with f32 queries; by every sequence if the prefix has 256 tokens at most.
 * prefix_table [ceil(prefix_len / page_size)] i32 pages of the prefix; its last page need not be full
 * prefix_len   [host] tokens of the prefix, >= 0
 * lens         [n_seq] i32 in [0, max_pages * page_size], the prefix not counted
 * A page of the prefix outside [0, n_pages) sets the status and makes every sequence's output NaN; a sequence
 * without any token gives zeros.  The largest weight of a query, before the sum divides them, is 1 in riftkv_attention and may here be as
 * small as 2^-8 for a prefix: 8-bit rows' scales lose bits below 2^-102, and sums of values below 2^-118 have fewer bits.  Everything
 * else as for riftkv_attention.
 * Shape rules: prefix_len <= 2^30, n_seq * n_heads <= 2^26.
 */
RIFT_API rift_status riftkv_attention_shared(const riftkv_cache* cache, const void* q, int64_t ld_q, int32_t n_heads,
                                             rift_dtype dt, const int32_t* prefix_table, int32_t prefix_len,
                                             const int32_t* page_table, int32_t n_seq, int32_t max_pages,
                                             const int32_t* lens, float scale, void* out, int64_t ld_out, int32_t* status,
                                             void* workspace, size_t ws_bytes, rift_stream stream);

/* ------------------------------------------------------------------ some pages of a long context */

/*
 * riftkv_page_bounds -- the smallest and largest value of every element of the keys of a page's tokens.
 * bounds      [n_pages][n_kv_heads][2][head_dim], f32 with f32 pages, else bf16: smallest, then largest; by page, as the
 *             cache is, so that sequences which share a page share its bounds
 * begins      [n_seq] i32, or NULL: all 0.  The pages of sequence i that hold its tokens begins[i] .. lens[i] - 1 are
 *             gone through anew, each from its first token on, up to lens[i]; the other bounds stay as they are.
 *             A decode step that wrote token n passes begins[i] = n, lens[i] = n + 1.  Below 0: as 0
 * lens        [n_seq] i32 in [0, max_pages * page_size]
 * The values are exact, 8-bit pages' but for those of rows whose largest magnitude is below 2^-110, which are rounded
 * to bf16; NaN among an element's values makes both its bounds NaN.
 * Where sequences share a page that is not full for all of them, its bounds are one of theirs, or parts of several.
 * A length out of range, or a page outside [0, n_pages), sets the status and is skipped.
 * Shape rules: 0 <= n_seq <= 65535, max_pages >= 0, max_pages * page_size <= 2^30.
 */
RIFT_API rift_status riftkv_page_bounds(const riftkv_cache* cache, void* bounds, const int32_t* page_table, int32_t n_seq,
                                        int32_t max_pages, const int32_t* begins, const int32_t* lens, int32_t* status,
                                        rift_stream stream);

/* Workspace bytes of riftkv_select_pages (0 for shapes that it refuses).  Not smaller for more sequences or wider
 * tables. */
RIFT_API size_t riftkv_select_pages_workspace_size(const riftkv_cache* cache, int32_t n_seq, int32_t max_pages);

/*
 * riftkv_select_pages -- for every sequence and key head the `top` pages that its new token's queries need most.
 * A page's score for a query is sum_d (min(q_d, 0) smallest_d + max(q_d, 0) largest_d), in float64: no key of
 * the page has a larger product with the query.  Its score for the key head is the largest of its group's queries'.
 * The first keep_first and the last keep_last pages of the sequence's ceil(lens[i] / page_size) are always taken, the
 * others by (score descending, page ascending) until there are `top`; a page with a score of NaN comes last.
 * bounds      as riftkv_page_bounds leaves them (of the sequences' pages)
 * q           [n_seq][n_heads][head_dim] dt, sequences ld_q elements apart
 * pages       [n_seq][n_kv_heads][top] i32 out: the places in the sequence's row of page_table, ascending; -1 behind the
 *             last where the sequence has fewer pages.  Overlaps no input
 * A length out of range sets the status and gives -1 throughout; a page outside [0, n_pages) sets the status and comes last.
 * Shape rules: those of riftkv_attention; 1 <= top <= 2^20, keep_first, keep_last >= 0, keep_first + keep_last <= top.
 * dt as for riftkv_attention.  workspace 256-byte aligned; calls that may overlap in time need one each.
 */
RIFT_API rift_status riftkv_select_pages(const riftkv_cache* cache, const void* bounds, const void* q, int64_t ld_q,
                                         int32_t n_heads, rift_dtype dt, const int32_t* page_table, int32_t n_seq,
                                         int32_t max_pages, const int32_t* lens, int32_t keep_first, int32_t keep_last,
                                         int32_t* pages, int32_t top, int32_t* status, void* workspace, size_t ws_bytes,
                                         rift_stream stream);

/* Workspace bytes of riftkv_attention_pages (0 for shapes that it refuses).  Not smaller for more sequences or
 * longer lists. */
RIFT_API size_t riftkv_attention_pages_workspace_size(const riftkv_cache* cache, int32_t n_heads, int32_t n_seq, int32_t top);

/*
 * riftkv_attention_pages -- riftkv_attention over the tokens of some pages only, a list for every sequence and key head.
 * pages       [n_seq][n_kv_heads][top] i32 places in the sequence's row of page_table, as riftkv_select_pages leaves them or
 *             in any order; negative ones are skipped.  Of each page the tokens before lens[i] count; a place that is listed
 *             twice counts twice
 * A list without tokens gives zeros.  A length out of range, a place >= max_pages or a page outside [0, n_pages) among the
 * listed tokens sets the status and makes the outputs of that sequence and key head NaN.
 * Shape rules: those of riftkv_attention; 1 <= top <= 2^20, top * page_size <= 2^30.
 */
RIFT_API rift_status riftkv_attention_pages(const riftkv_cache* cache, const void* q, int64_t ld_q, int32_t n_heads,
                                            rift_dtype dt, const int32_t* page_table, int32_t n_seq, int32_t max_pages,
                                            const int32_t* lens, const int32_t* pages, int32_t top, float scale, void* out,
                                            int64_t ld_out, int32_t* status, void* workspace, size_t ws_bytes,
                                            rift_stream stream);

/* ------------------------------------------------------------------ decode */

/* Workspace bytes of riftkv_decode_step (0 for shapes that it refuses).  Not smaller for
 * more sequences or wider tables. */
RIFT_API size_t riftkv_decode_workspace_size(const rift_model_cfg* cfg, const riftkv_cache* cache, int32_t n_seq,
                                             int32_t max_pages);

/*
 * riftkv_decode_step -- one generated token of every sequence through the decoder layers of
 * rift_prefill, keys and values in pages: rift_decode_step for prompts that come and go, any
 * length, and quantised caches.  Per layer the new token's rotated key and its value are
 * written (riftkv_write), and it attends to its sequence's tokens up to itself
 * (riftkv_attention).  A prompt's earlier rows are rift_prefill's kv_cache, written with
 * riftkv_write layer by layer (seq_ids and its position_ids say where); prompts with a shared
 * prefix may share the pages that the prefix fills.
 * cfg, layers  [host] as for rift_prefill; bfloat16 models
 * x_new        [n_seq][d] bf16  input embeddings of the new tokens
 * cache        [host] layer 0's pages; layer l's k, v, k_scale and v_scale follow those of layer
 *              l - 1 ([n_layers][n_pages]...).  n_kv_heads and head_dim are the model's;
 *              bf16, fp8 or int8
 * page_table   [n_seq][max_pages] i32, the same pages for every layer
 * positions    [n_seq] i32  the new token's position: the tokens that its sequence holds
 *              already.  Negative: no sequence here (padding); nothing is written for it
 *              and its hidden_out row means nothing
 * hidden_out   [n_seq][d] f32 out  residual stream of the new tokens after the last layer
 * status       as for riftkv_write and riftkv_attention; the row of a sequence that sets it is NaN
 * A sequence's last bits depend on the batch and the table's width as riftkv_attention's do.
 * Shape rules: those of rift_prefill's model and of riftkv_attention; n_seq * d and
 * n_seq * ffn < 2^31.
 * Errors: RIFT_ERR_UNSUPPORTED also for float32 models and pages.
 */
RIFT_API rift_status riftkv_decode_step(const rift_model_cfg* cfg, const rift_layer_weights* layers, const void* x_new,
                                        const riftkv_cache* cache, const int32_t* page_table, int32_t n_seq,
                                        int32_t max_pages, const int32_t* positions, float* hidden_out,
                                        int32_t* status, void* workspace, size_t ws_bytes, rift_stream stream);

#ifdef __cplusplus
}
#endif

#endif /* RIFT_KV_H */
