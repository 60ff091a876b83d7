// One query token of every sequence over its paged keys and values, split over the
// length and joined.
//
//   attention_kernel   Short heads: a workgroup takes one whole, its waves a share each.
//                      Otherwise the tiles (32 tokens of one sequence and head group) of
//                      all sequences, one after the other, are dealt out evenly to the
//                      waves, in runs: however uneven the lengths, waves finish
//                      together, and a wave writes at most two results of parts.
//                      Heads a wave finishes go straight to the output, the parts at
//                      its ends meet in LDS, and what a workgroup holds only a part
//                      of goes to its two slots of the workspace.
//   join_kernel        after a split: the parts of heads that several workgroups share;
//                      sequences without tokens.
//
// A head group is up to 16 query heads of one key head.  With the tile's tokens as rows,
// S^T = K Q^T leaves a lane the scores of one query and 8 tokens; they are the lane's
// own share of the second product's right operand, O^T = V^T P^T, if its token
// order is the lanes' (a sum's order is free), and a lane's own rows of V are, with two
// bytes or halfwords exchanged in registers, its share of the left one.  So nothing
// passes through LDS, and the softmax is a lane's own but for two swaps.  The bytes of keys
// and values bound this kernel, so that unused query columns cost nothing, except in 8-bit pages of
// 64 dimensions: there a tile's vector instructions, the softmax of 16 columns among them whatever the
// group, take longer than its bytes.  Groups of more than 16 are several head groups, each of which reads
// the key head's keys and values.
//
// Scores, weights and sums are float32: each weight, and each float32 query, goes into the
// matrix product as three bf16 terms that add up to it.  (Two terms, short by up to 2^-16 of a weight:
// 30 sequences of 29,813 tokens, 3 key heads of 64 dimensions, e4m3, 75.4 us and with three 76.2; 64 of
// 3,000 to 5,000, 8 of 128, int8, 97.3 and 99; 96 of 17 to 24,001, e4m3, 392.7 and 394; 128 of 32 to 512, 8 of 128,
// e4m3, 20.5 and 21.5; bf16 pages within 2%, the large ones 0.3%.)
#include <type_traits>

#include "kv_device.h"

namespace rift {

namespace {

constexpr int kTile = 32;                 // tokens of a tile
constexpr int kBegins = 1, kEnds = 2;     // a part holds a head's first, last tile
constexpr int kSplitWaves = 4;            // of a workgroup, where heads are split over workgroups
constexpr int kMaxWgs = 512;              // two workgroups a CU
constexpr int kFewSeqs = 256;             // sequences whose lengths a wave holds in registers

struct AttnParams {
    const void* q;
    void* out;
    int64_t ld_q, ld_out;
    const unsigned char *k, *v;
    const uint8_t *ks, *vs;
    const int* table;
    const int* lens;
    int* status;
    float* slots;          // [wgs][2][rows][HD + 4]: weighted values, max, sum
    int4* joins;           // [wgs][2]: of the head groups that end and that begin here, shared with others: sequence
                           // (-1: none), first head and heads (16 bits each), first and last workgroup
    int n_seq, max_pages, n_pages, n_kv, shift, group, q_tiles, rows;
    int few;               // at most kFewSeqs sequences, and 31 bits hold their tiles of all heads
    float scale_log2;
};

// A place in the sequence of tiles: of head group hq, the qt-th of key head kvh.
struct Place {
    int seq, hq, kvh, qt, tile, len;
};

__device__ __forceinline__ int tiles_of(int len) { return (len + kTile - 1) / kTile; }

// 0 for a length out of range.
__device__ __forceinline__ int length_of(int len, int max_pages, int shift) {
    return len < 0 || (int64_t)len > ((int64_t)max_pages << shift) ? 0 : len;
}

__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }

// a / b; most operands have 32 bits, and 64-bit division is long.
__device__ __forceinline__ unsigned long long quotient(unsigned long long a, unsigned long long b) {
    return ((a | b) >> 32) == 0 ? (unsigned)a / (unsigned)b : a / b;
}

// Inclusive sums over the wave.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
    return x;
}

// How N tiles are dealt to W waves (W <= N): wave w's run begins at w q + min(w, r).
struct Deal {
    unsigned long long q = 1, r = 0;
    __device__ __forceinline__ Deal() {}
    __device__ __forceinline__ Deal(unsigned long long N, unsigned W) {
        if (N != W) {
            q = quotient(N, W);
            r = N - q * W;
        }
    }
    __device__ __forceinline__ unsigned long long first(unsigned w) const { return w * q + (w < r ? w : r); }
    __device__ __forceinline__ int owner(unsigned long long tile) const {
        const unsigned long long longer = r * (q + 1);
        return (int)(tile < longer ? quotient(tile, q + 1) : r + quotient(tile - longer, q));
    }
};

// Maximum and sum over the four lanes that hold a query's tokens (16 lanes apart).
__device__ __forceinline__ float quad_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Two 8-bit codes (half `hi` of w) as two bf16 values, exact.
template <riftkv_dtype DT, bool HI>
__device__ __forceinline__ uint32_t widen(uint32_t w) {
    if constexpr (DT == RIFTKV_FP8)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    else {
        const float a = (float)(int8_t)(w >> (HI ? 16 : 0)), b = (float)(int8_t)(w >> (HI ? 24 : 8));
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
}

// Pairs of bf16 terms that add up to a and b: each takes the leading 8 of the bits that are left, so that
// three hold all 24 (of numbers from 2^-110 on; below, to 2^-133, the last bit of the smallest bf16).  Cut off, not
// rounded: no term can pass the largest number, and what is left is exact.
template <int N>
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        w[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        a -= __uint_as_float(x & 0xFFFF0000u);
        b -= __uint_as_float(y & 0xFFFF0000u);
    }
}

template <int N>
struct Words {
    typedef uint32_t type __attribute__((ext_vector_type(N)));
};
template <>
struct Words<1> {
    typedef uint32_t type;
};

// N words from p.
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const unsigned char* p) {
    constexpr int C = N < 4 ? N : 4;
    typedef typename Words<C>::type vec;
#pragma unroll
    for (int i = 0; i < N / C; ++i) {
        const vec x = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p) + i);
        if constexpr (C == 1) w[0] = x;
        else
#pragma unroll
            for (int j = 0; j < C; ++j) w[C * i + j] = x[j];
    }
}

// Output of a sequence without tokens, or of a length out of range: head group hq, or all (-1).
template <typename T>
__device__ void fill_heads(const AttnParams& p, int seq, int given, int hq, int hd, int tid, int threads) {
    const bool bad = given != 0;
    if (bad && tid == 0) *p.status = RIFT_ERR_SHAPE;
    int h0 = 0, heads = p.n_kv * p.group;
    if (hq >= 0) {
        const int kvh = hq / p.q_tiles, r0 = (hq - kvh * p.q_tiles) * 16;
        h0 = kvh * p.group + r0;
        heads = min(16, p.group - r0);
    }
    const size_t at = (size_t)seq * p.ld_out + (size_t)h0 * hd;
    for (int i = tid; i < heads * hd; i += threads) {
        if constexpr (sizeof(T) == 2) static_cast<bf16_t*>(p.out)[at + i] = bad ? 0x7FC0 : 0;
        else static_cast<float*>(p.out)[at + i] = bad ? NAN : 0.f;
    }
}

// T: type of queries and outputs.  WHOLE: a workgroup takes a head group of a sequence;
// otherwise a run of all tiles.
template <typename T, riftkv_dtype DT, int HD, int WAVES, bool WHOLE>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 8 ? 1 : 2)
attention_kernel(AttnParams p) {
    constexpr int kThreads = 64 * WAVES;
    constexpr int RECORDS = WHOLE ? WAVES : 2 * WAVES;   // a wave's parts of heads
    constexpr int B = DT == RIFTKV_F32 ? 4 : DT == RIFTKV_BF16 ? 2 : 1;   // bytes a value
    constexpr bool SCALED = B == 1, F32 = DT == RIFTKV_F32;
    // A load of keys takes E 64-byte pieces of 16 / E rows (whole 128-byte lines), so that
    // a row of the first product's left operand is one piece of one token: it meets each piece of
    // the query, in an accumulator of its own, and a score is the sum of what belongs
    // together.  Rows of 64 bytes, and float32 ones (whose products are not idle): E = 1.
    constexpr int E = F32 || HD * B == 64 ? 1 : 2;
    constexpr int KF = HD * B / (64 * E);    // loads of a lane for 16 / E keys
    constexpr int I = 4 / E;                 // a lane's scores of those
    constexpr int VW = HD * B / 64;          // words of a lane of one value row
    constexpr int C = HD / 16;               // columns of a lane of one value row
    constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = 3;
    constexpr int RS = HD + 4;               // floats of a part's row: values, max, sum (and odd to the banks)
    extern __shared__ __align__(16) float records[];   // [RECORDS][rows][RS]
    __shared__ int4 meta[RECORDS];           // sequence (-1: no record), first head, heads, which ends of their tiles it holds
    __shared__ unsigned long long head_end[RECORDS];   // the tile after the head's last
    __shared__ long long sums[WAVES];
    __shared__ int found_seq[WAVES];
    __shared__ long long found_at[WAVES];    // tiles before that sequence
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int HQ = p.n_kv * p.q_tiles;
    const int slot_floats = p.rows * RS;

    if (lane < RECORDS / WAVES) meta[wave * (RECORDS / WAVES) + lane] = make_int4(-1, 0, 0, 0);
    Place cur{};
    int left = 0;                       // tiles of this wave from cur on
    unsigned long long end = 0;         // and the tile after them, among all
    unsigned waves = 0;                 // waves with tiles, and their shares
    Deal deal;
    if constexpr (WHOLE) {
        cur.seq = blockIdx.x / HQ;
        cur.hq = blockIdx.x - cur.seq * HQ;
        const int given = p.lens[cur.seq];
        cur.len = length_of(given, p.max_pages, p.shift);
        if (cur.len == 0) {
            fill_heads<T>(p, cur.seq, given, cur.hq, HD, tid, kThreads);
            return;
        }
        const int t = tiles_of(cur.len);
        cur.tile = (int)((unsigned)(t * wave) / WAVES);
        left = (int)((unsigned)(t * (wave + 1)) / WAVES) - cur.tile;
    } else {
        const unsigned all = gridDim.x * WAVES, gw = blockIdx.x * WAVES + wave;
        if (p.few) {
            // Every wave by itself: the lengths in registers, scanned.
            constexpr int CH = kFewSeqs / 64;
            int len[CH], incl[CH], total = 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int s = 64 * c + lane;
                len[c] = s < p.n_seq ? length_of(p.lens[s], p.max_pages, p.shift) : 0;
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                incl[c] = 0;
                if (64 * c < p.n_seq) {
                    incl[c] = wave_scan(tiles_of(len[c])) + total;
                    total = __builtin_amdgcn_readlane(incl[c], 63);
                }
            }
            const unsigned long long N = (unsigned long long)total * HQ;
            waves = (unsigned)(N < all ? N : all);
            if (gw < waves) {
                deal = Deal(N, waves);
                const int at = (int)deal.first(gw);
                int before = 0, ch = 0;
                unsigned long long mask = 0;
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (mask == 0 && 64 * c < p.n_seq) {
                        mask = __ballot(incl[c] * HQ > at);
                        if (mask != 0) {
                            ch = c;
                            const int l = __ffsll(mask) - 1;
                            cur.len = __builtin_amdgcn_readlane(len[c], l);
                            before = (__builtin_amdgcn_readlane(incl[c], l) - tiles_of(cur.len)) * HQ;
                        }
                    }
                cur.seq = 64 * ch + __ffsll(mask) - 1;
                const unsigned t = tiles_of(cur.len), in = at - before;
                cur.hq = __builtin_amdgcn_readfirstlane(in / t);
                cur.tile = in - cur.hq * t;
            }
        } else {
            // A thread sums a run of sequences, the workgroup scans the sums, and whoever
            // holds a wave's first tile looks it up.
            const int per = (p.n_seq + kThreads - 1) / kThreads;
            const int s0 = min(tid * per, p.n_seq), s1 = min(s0 + per, p.n_seq);
            long long mine = 0;
            for (int s = s0; s < s1; ++s) mine += tiles_of(length_of(p.lens[s], p.max_pages, p.shift));
            long long incl = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const long long o = __shfl_up(incl, d);
                if (lane >= d) incl += o;
            }
            if (lane == 63) sums[wave] = incl;
            __syncthreads();
            long long before = incl - mine, total = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) before += sums[w];
                total += sums[w];
            }
            const unsigned long long N = (unsigned long long)total * HQ;
            waves = (unsigned)(N < all ? N : all);
            if (waves > 0) deal = Deal(N, waves);
            if (mine > 0) {
                for (int w = 0; w < WAVES; ++w) {
                    const unsigned other = blockIdx.x * WAVES + w;
                    if (other >= waves) break;
                    const long long a = (long long)deal.first(other);
                    if (a >= before * HQ && a < (before + mine) * HQ) {
                        long long at = before;
                        int s = s0;
                        for (;; ++s) {
                            const int t = tiles_of(length_of(p.lens[s], p.max_pages, p.shift));
                            if (a < (at + t) * HQ) break;
                            at += t;
                        }
                        found_seq[w] = s;
                        found_at[w] = at;
                    }
                }
            }
            __syncthreads();
            if (gw < waves) {
                cur.seq = __builtin_amdgcn_readfirstlane(found_seq[wave]);
                cur.len = __builtin_amdgcn_readfirstlane(p.lens[cur.seq]);
                const unsigned long long in = deal.first(gw) - (unsigned long long)found_at[wave] * HQ;
                const int t = tiles_of(cur.len);
                cur.hq = __builtin_amdgcn_readfirstlane((int)quotient(in, t));
                cur.tile = __builtin_amdgcn_readfirstlane((int)(in - (unsigned long long)cur.hq * t));
            }
        }
        if (gw < waves) {
            end = deal.first(gw + 1);
            left = __builtin_amdgcn_readfirstlane((int)(end - deal.first(gw)));
        }
    }

    if (left > 0) {
        cur.kvh = p.q_tiles == 1 ? cur.hq : cur.hq / p.q_tiles;
        cur.qt = cur.hq - cur.kvh * p.q_tiles;
        auto after = [&](Place c) __attribute__((always_inline)) {
            if ((c.tile + 1) * kTile < c.len) {
                ++c.tile;
                return c;
            }
            c.tile = 0;
            if (++c.qt == p.q_tiles) {
                c.qt = 0;
                ++c.kvh;
            }
            if (++c.hq == HQ) {
                c.hq = c.kvh = c.qt = 0;
                do {
                    ++c.seq;
                    c.len = length_of(p.lens[c.seq], p.max_pages, p.shift);
                } while (c.len == 0);
            }
            return c;
        };
        // pages of the two halves of a tile (the second's may be past the end: the first's)
        struct Pages {
            int a, b;
        };
        auto pages_at = [&](const Place& c) __attribute__((always_inline)) {
            const int* row = p.table + (size_t)c.seq * p.max_pages;
            const int t0 = c.tile * kTile, t1 = t0 + 16 < c.len ? t0 + 16 : t0;
            return Pages{row[t0 >> p.shift], row[t1 >> p.shift]};
        };
        uint32_t kr[2][E][KF][4], vr[2][4][VW], ksc[2], vsc[2];
        // Load x of the E takes tokens 4 r + I x + i (r = 0..3, i < I) of a half: lane (n, g) the piece n mod E of
        // row n / E.  Rows of values: 4 g + i.
        const int k_row = E == 1 ? n : 4 * (n >> 2) + ((n >> 1) & 1);
        const unsigned k_col = (n % E) * 64 + g * 16, v_col = n * VW * 4;
        // first row of a half's keys and values among the pages' rows
        auto row_of = [&](const Place& c, int page, int h) __attribute__((always_inline)) {
            page = (unsigned)page < (unsigned)p.n_pages ? page : 0;
            return ((((size_t)page * p.n_kv) + c.kvh) << p.shift) + ((c.tile * kTile + 16 * h) & ((1 << p.shift) - 1));
        };
        // Rows behind the last token are not read (3,200 heads of 131 to 643 tokens 103.4 -> 97.7 us): their
        // lanes take its row once more, and one line of the first row where there is nothing to load.
        auto last_of = [&](const Place& c, int h, bool live) __attribute__((always_inline)) {
            return live ? max(min(c.len - 1 - c.tile * kTile - 16 * h, 15), 0) : 0;
        };
        auto load_k = [&](const Place& c, const Pages& pg, bool live) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const size_t r = row_of(c, h ? pg.b : pg.a, h);
                const int last = last_of(c, h, live);
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    const unsigned off = min(k_row + x * I, last) * (HD * B) + (live ? k_col : 0);
#pragma unroll
                    for (int f = 0; f < KF; ++f) load_words<4>(kr[h][x][f], p.k + r * (HD * B) + off + 64 * E * f);
                }
                if constexpr (SCALED) ksc[h] = *reinterpret_cast<const uint32_t*>(p.ks + r + 4 * g);
            }
        };
        auto load_v = [&](const Place& c, const Pages& pg, bool live) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const size_t r = row_of(c, h ? pg.b : pg.a, h);
                const int last = last_of(c, h, live);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    load_words<VW>(vr[h][i], p.v + r * (HD * B) + (unsigned)(min(4 * g + i, last) * (HD * B) + (live ? v_col : 0)));
                if constexpr (SCALED) vsc[h] = *reinterpret_cast<const uint32_t*>(p.vs + r + 4 * g);
            }
        };

        // the next tile's pages are asked for with the first one's, and from then on a tile ahead
        Pages cur_pages = pages_at(cur);
        Place nxt = cur;
        Pages nxt_pages = cur_pages;
        if (left > 1) {
            nxt = after(cur);
            nxt_pages = pages_at(nxt);
        }
        load_k(cur, cur_pages, true);
        load_v(cur, cur_pages, true);

        bf16x8_t qf[F32 ? 1 : NQ][F32 ? 1 : HD / 32];
        float qs[F32 ? HD / 4 : 1];
        f32x4_t o[C];
        float m = -INFINITY, l = 0.f;
        bool bad = false;          // a page of the head is out of range
        int begin = cur.tile;      // this wave's first tile of the head
        int n_records = 0;
        auto start_head = [&](const Place& c) __attribute__((always_inline)) {
            const int r = 16 * c.qt + n;   // this lane's query
            const bool there = r < p.group;
            const size_t q0 = (size_t)c.seq * p.ld_q + (size_t)(c.kvh * p.group + (there ? r : 0)) * HD;
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.q) + q0 + 16 * i + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) qs[4 * i + e] = there ? x[e] : 0.f;
                }
            } else {
#pragma unroll
                for (int f = 0; f < HD / 32; ++f) {
                    const size_t at = q0 + (SCALED ? (f >> 1) * 64 + g * 16 + (f & 1) * 8 : f * 32 + g * 8);
                    if constexpr (NQ == 1) {
                        u32x4_t x = *reinterpret_cast<const u32x4_t*>(static_cast<const bf16_t*>(p.q) + at);
                        if (!there) x = u32x4_t{0, 0, 0, 0};
                        qf[0][f] = __builtin_bit_cast(bf16x8_t, x);
                    } else {
                        const float* src = static_cast<const float*>(p.q) + at;
                        u32x4_t x[NQ];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t w[NQ];
                            split_bf16<NQ>(there ? src[2 * e] : 0.f, there ? src[2 * e + 1] : 0.f, w);
#pragma unroll
                            for (int i = 0; i < NQ; ++i) x[i][e] = w[i];
                        }
#pragma unroll
                        for (int i = 0; i < NQ; ++i) qf[i][f] = __builtin_bit_cast(bf16x8_t, x[i]);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            m = -INFINITY;
            l = 0.f;
            bad = false;
        };
        start_head(cur);
        if constexpr (!WHOLE)
            if (wave == 0) {   // the head that an earlier workgroup began: worked out while the loads are under way
                int4 join = make_int4(-1, 0, 0, 0);
                if (cur.tile > 0 && p.rows > 1) {   // (a single row is joined where it begins)
                    const unsigned long long first = end - left - cur.tile;
                    join = make_int4(cur.seq, (cur.kvh * p.group + 16 * cur.qt) << 16 | min(16, p.group - 16 * cur.qt),
                                     deal.owner(first) / WAVES, deal.owner(first + tiles_of(cur.len) - 1) / WAVES);
                }
                if (lane == 0) p.joins[2 * blockIdx.x] = join;
            }

        for (;;) {
            const bool live = left > 1;
            bad |= (unsigned)cur_pages.a >= (unsigned)p.n_pages || (unsigned)cur_pages.b >= (unsigned)p.n_pages;
            // scores: s[4 h + i] of this lane's query and token 16 h + 4 g + i of the tile
            float s[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    f32x4_t acc[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int f = 0; f < KF; ++f) {
                        const uint32_t(&w)[4] = kr[h][x][f];
                        if constexpr (F32) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                acc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), qs[4 * f + j], acc[0], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int y = 0; y < (SCALED ? 2 : 1); ++y) {   // 16 bytes: 8 or 16 values
                                u32x4_t kw;
                                if constexpr (SCALED)
                                    kw = u32x4_t{widen<DT, false>(w[2 * y]), widen<DT, true>(w[2 * y]), widen<DT, false>(w[2 * y + 1]),
                                                 widen<DT, true>(w[2 * y + 1])};
                                else
                                    kw = u32x4_t{w[0], w[1], w[2], w[3]};
#pragma unroll
                                for (int e = 0; e < E; ++e)
#pragma unroll
                                    for (int i = 0; i < NQ; ++i)
                                        acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                            __builtin_bit_cast(bf16x8_t, kw), qf[i][SCALED ? 2 * (f * E + e) + y : f * E + e], acc[e], 0, 0, 0);
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < I; ++i) {
                        float a = acc[0][i * E];
                        if constexpr (E == 2) a += acc[1][i * E + 1];
                        const int j = 4 * h + I * x + i;
                        if constexpr (SCALED) a *= scale_of((ksc[h] >> (8 * (j & 3))) & 0xFFu);
                        s[j] = a * p.scale_log2;
                    }
                }
            }
            load_k(nxt, nxt_pages, live);
            const int there = cur.len - cur.tile * kTile - 4 * g;   // tokens from this lane's first on
            const bool tail = cur.len - cur.tile * kTile < kTile;
            if (tail) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (16 * (j >> 2) + (j & 3) >= there) s[j] = -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[j]);
            mx = quad_max(mx);
            if (__any(mx > m)) {
                const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - ref_of(mn));
                m = mn;
                l *= f;
#pragma unroll
                for (int c = 0; c < C; ++c) o[c] *= f;
            }
            const float ref = ref_of(m);
            float pr[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pr[j] = __builtin_amdgcn_exp2f(s[j] - ref);
                l += pr[j];
                if constexpr (SCALED) pr[j] *= scale_of((vsc[j >> 2] >> (8 * (j & 3))) & 0xFFu);
            }
            if (tail) {   // whatever lies behind the last token: no part of the sum, NaN or not
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (16 * (j >> 2) + (j & 3) >= there) {
                        pr[j] = 0.f;
#pragma unroll
                        for (int w = 0; w < VW; ++w) vr[j >> 2][j & 3][w] = 0;
                    }
            }
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[j >> 2][j & 3][c]), pr[j], o[c], 0, 0, 0);
            } else {
                u32x4_t pf[NP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t w[NP];
                    split_bf16<NP>(pr[2 * j], pr[2 * j + 1], w);
#pragma unroll
                    for (int i = 0; i < NP; ++i) pf[i][j] = w[i];
                }
                auto add = [&](int c, const u32x4_t& vw) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < NP; ++i)
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vw), __builtin_bit_cast(bf16x8_t, pf[i]),
                                                                        o[c], 0, 0, 0);
                };
#pragma unroll
                for (int c = 0; c < C; c += 2) {   // columns c and c + 1 of the lane's rows, tokens in pairs
                    u32x4_t v0, v1;
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const uint32_t(&x)[VW] = vr[d >> 1][2 * (d & 1)], (&y)[VW] = vr[d >> 1][2 * (d & 1) + 1];
                        if constexpr (SCALED) {
                            const uint32_t w = __builtin_amdgcn_perm(y[c >> 2], x[c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
                            v0[d] = widen<DT, false>(w);
                            v1[d] = widen<DT, true>(w);
                        } else {
                            v0[d] = __builtin_amdgcn_perm(y[c >> 1], x[c >> 1], 0x05040100u);
                            v1[d] = __builtin_amdgcn_perm(y[c >> 1], x[c >> 1], 0x07060302u);
                        }
                    }
                    add(c, v0);
                    add(c + 1, v1);
                }
            }
            load_v(nxt, nxt_pages, live);
            Place nn = nxt;
            Pages nn_pages = nxt_pages;
            if (left > 2) {
                nn = after(nxt);
                nn_pages = pages_at(nn);
            }

            const bool ends = (cur.tile + 1) * kTile >= cur.len;
            if (ends || !live) {   // the wave's last tile of this head: o[c][i] is column (4 g + i) C + c of query n
                float sum = quad_sum(l);
                if (bad) {
                    sum = NAN;
                    if (lane == 0) *p.status = RIFT_ERR_SHAPE;
                }
                const int h0 = cur.kvh * p.group + 16 * cur.qt, rows = min(16, p.group - 16 * cur.qt);   // first head, heads
                const bool valid = n < rows;
                if (begin == 0 && ends) {
                    if (valid) {
                        const float inv = 1.f / sum;
                        const size_t o0 = (size_t)cur.seq * p.ld_out + (size_t)(h0 + n) * HD;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int c = 0; c < C; c += 4) {
                                const size_t at = o0 + (4 * g + i) * C + c;
                                if constexpr (sizeof(T) == 2) {
                                    uint32_t w[2];
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        w[e] = (uint32_t)round_bf16(o[c + 2 * e][i] * inv) | (uint32_t)round_bf16(o[c + 2 * e + 1][i] * inv) << 16;
                                    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + at) = make_uint2(w[0], w[1]);
                                } else {
                                    *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) =
                                        f32x4_t{o[c][i] * inv, o[c + 1][i] * inv, o[c + 2][i] * inv, o[c + 3][i] * inv};
                                }
                            }
                    }
                } else {
                    const int rec = RECORDS / WAVES * wave + n_records++;
                    if (lane == 0) {
                        meta[rec] = make_int4(cur.seq, h0, rows, (begin == 0 ? kBegins : 0) | (ends ? kEnds : 0));
                        head_end[rec] = end - left - cur.tile + tiles_of(cur.len);
                    }
                    if (valid) {
                        float* dst = records + (size_t)rec * slot_floats + n * RS;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int c = 0; c < C; c += 4)
                                *reinterpret_cast<f32x4_t*>(dst + (4 * g + i) * C + c) = f32x4_t{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
                        if (g == 0) {
                            dst[HD] = m;
                            dst[HD + 1] = sum;
                        }
                    }
                }
                if (!live) break;
                start_head(nxt);
                begin = 0;
            }
            cur = nxt;
            cur_pages = nxt_pages;
            nxt = nn;
            nxt_pages = nn_pages;
            --left;
        }
    } else if (!WHOLE && tid == 0) {
        p.joins[2 * blockIdx.x] = make_int4(-1, 0, 0, 0);
    }
    __syncthreads();

    // Neighbouring records of one head are joined: a whole head goes to the output, the
    // end of one begun in an earlier workgroup to slot 0, the start of one that goes
    // on in the next to slot 1.
    // (All records are read, whether there or not, so that the reads follow each other.)
    int4 mt[RECORDS], join = make_int4(-1, 0, 0, 0);
    unsigned rest = 0;
    int last = 0;       // a record of the head that goes on
#pragma unroll
    for (int i = 0; i < RECORDS; ++i) mt[i] = meta[i];
#pragma unroll
    for (int i = 0; i < RECORDS; ++i) rest |= mt[i].x >= 0 ? 1u << i : 0u;
    rest = __builtin_amdgcn_readfirstlane(rest);
    while (rest != 0) {
        const int r = __ffs(rest) - 1;
        const int4 a = meta[r];
        unsigned mask = 0;
        int held = 0;
#pragma unroll
        for (int i = 0; i < RECORDS; ++i)
            if ((rest >> i & 1) && mt[i].x == a.x && mt[i].y == a.y) {
                mask |= 1u << i;
                held |= mt[i].w;
            }
        mask = __builtin_amdgcn_readfirstlane(mask);
        rest &= ~mask;
        held = __builtin_amdgcn_readfirstlane(held);
        float* slot = p.slots + ((size_t)blockIdx.x * 2 + (held & kBegins ? 1 : 0)) * slot_floats;
        if (held == kBegins) {
            join = a;
            last = r;
        }
        for (int item = tid; item < a.z * (HD / 4); item += kThreads) {
            const int row = item / (HD / 4), col = 4 * (item % (HD / 4));
            const float* src = records + row * RS;
            float m[RECORDS], mx = -INFINITY, L = 0.f;
            f32x4_t x[RECORDS], acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < RECORDS; ++i) {
                m[i] = src[i * slot_floats + HD];
                x[i] = *reinterpret_cast<const f32x4_t*>(src + i * slot_floats + col);
            }
#pragma unroll
            for (int i = 0; i < RECORDS; ++i)
                if (mask >> i & 1) mx = fmaxf(mx, m[i]);
#pragma unroll
            for (int i = 0; i < RECORDS; ++i)
                if (mask >> i & 1) {
                    const float f = __builtin_amdgcn_exp2f(m[i] - ref_of(mx));
                    L = fmaf(f, src[i * slot_floats + HD + 1], L);
                    acc += f * x[i];
                }
            if (held == (kBegins | kEnds)) {
                const size_t at = (size_t)a.x * p.ld_out + (size_t)(a.y + row) * HD + col;
                acc *= 1.f / L;
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + at) =
                        make_uint2((uint32_t)round_bf16(acc[0]) | (uint32_t)round_bf16(acc[1]) << 16,
                                   (uint32_t)round_bf16(acc[2]) | (uint32_t)round_bf16(acc[3]) << 16);
                else
                    *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = acc;
            } else {
                *reinterpret_cast<f32x4_t*>(slot + row * RS + col) = acc;
                if (col == 0) {
                    slot[row * RS + HD] = mx;
                    slot[row * RS + HD + 1] = L;
                }
            }
        }
    }
    if (!WHOLE && tid == 0)
        p.joins[2 * blockIdx.x + 1] = join.x < 0 ? join : make_int4(join.x, join.y << 16 | join.z, blockIdx.x, deal.owner(head_end[last] - 1) / WAVES);
}

// One workgroup for each of the first kernel's.  The rows of a head that several of those share are
// dealt out to them; a row's parts are slot 1 of the first and slot 0 of the others.  Half of the
// threads are for the head that ended in the workgroup, half for the one that went on; they
// take four columns of a row and every PG-th part, then join over LDS.
constexpr int kJoinThreads = 512;   // of a head

template <typename T, int HD>
__global__ void __launch_bounds__(2 * kJoinThreads)
join_kernel(AttnParams p) {
    constexpr int RS = HD + 4, CV = HD / 4;
    __shared__ __align__(16) f32x4_t accs[2 * kJoinThreads];
    __shared__ float2 mls[2 * kJoinThreads];
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x / kJoinThreads), tid = threadIdx.x % kJoinThreads;
    const int4 ended = p.joins[2 * blockIdx.x], went_on = p.joins[2 * blockIdx.x + 1], join = half ? went_on : ended;
    for (int s = blockIdx.x; s < p.n_seq; s += gridDim.x) {
        const int given = p.lens[s];
        if (length_of(given, p.max_pages, p.shift) == 0) fill_heads<T>(p, s, given, -1, HD, threadIdx.x, 2 * kJoinThreads);
    }
    if (ended.x < 0 && went_on.x < 0) return;
    const int first = join.z, parts = join.w - first + 1, heads = join.y & 0xFFFF;
    const int row0 = (int)blockIdx.x - first;                    // rows row0, row0 + parts, ... are this workgroup's
    const bool some = join.x >= 0 && row0 < heads;
    const int items = some && heads - row0 > parts ? ((heads - row0 + parts - 1) / parts) * CV : CV;   // of at most 8 rows
    const int PG = kJoinThreads / items;
    const int pg = tid / items, item = tid - pg * items, row = row0 + item / CV * parts, col = 4 * (item % CV);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (some && pg < PG) {
        const int slot_floats = p.rows * RS;
        constexpr int U = 2;   // parts in flight
        for (int i = pg; i < parts; i += U * PG) {
            f32x4_t x[U];
            float2 ml[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {   // past the last: its values, not used
                const int at = min(i + u * PG, parts - 1);
                const float* src = p.slots + ((size_t)(first + at) * 2 + (at == 0 ? 1 : 0)) * slot_floats + row * RS;
                x[u] = *reinterpret_cast<const f32x4_t*>(src + col);
                ml[u] = *reinterpret_cast<const float2*>(src + HD);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u * PG >= parts) continue;
                const float mn = fmaxf(m, ml[u].x);
                const float f = __builtin_amdgcn_exp2f(m - ref_of(mn)), fi = __builtin_amdgcn_exp2f(ml[u].x - ref_of(mn));
                acc = acc * f + x[u] * fi;
                l = l * f + ml[u].y * fi;
                m = mn;
            }
        }
    }
    accs[threadIdx.x] = acc;
    mls[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (!some || tid >= items) return;
    float mx = m;
    const int used = min(PG, parts);
    for (int i = 1; i < used; ++i) mx = fmaxf(mx, mls[i * items + threadIdx.x].x);
    float f = __builtin_amdgcn_exp2f(m - ref_of(mx));
    acc *= f;
    l *= f;
    for (int i = 1; i < used; ++i) {
        const float2 ml = mls[i * items + threadIdx.x];
        f = __builtin_amdgcn_exp2f(ml.x - ref_of(mx));
        acc += f * accs[i * items + threadIdx.x];
        l += f * ml.y;
    }
    acc *= 1.f / l;
    const size_t at = (size_t)join.x * p.ld_out + (size_t)((join.y >> 16) + row) * HD + col;
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + at) =
            make_uint2((uint32_t)round_bf16(acc[0]) | (uint32_t)round_bf16(acc[1]) << 16,
                       (uint32_t)round_bf16(acc[2]) | (uint32_t)round_bf16(acc[3]) << 16);
    else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = acc;
}

int q_tiles_of(const riftkv_cache& c, int n_heads) { return (n_heads / c.n_kv_heads + 15) / 16; }
int rows_of(const riftkv_cache& c, int n_heads) {
    const int group = n_heads / c.n_kv_heads;
    return group < 16 ? group : 16;
}
int64_t most_tiles(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages) {
    return n_seq * c.n_kv_heads * q_tiles_of(c, n_heads) * ((max_pages * c.page_size + kTile - 1) / kTile);
}
int workgroups(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages) {
    const int64_t wgs = (most_tiles(c, n_heads, n_seq, max_pages) + kSplitWaves - 1) / kSplitWaves;
    return (int)(wgs < 1 ? 1 : wgs > kMaxWgs ? kMaxWgs : wgs);
}

// Waves of a workgroup that takes a head whole, or 0: heads are split.  A split costs the
// scan of the lengths and the join, which short heads do not repay; a head taken whole is
// read at one CU's rate (and float32 ones multiplied at its rate), so it is bounded by what the
// table can hold.  Eight waves (a CU's worth of registers) where every head has a CU and tiles
// enough for them.  In us, split / whole with 1, 2, 4 and 8 waves, groups of 4 query heads if not
// said otherwise:
//   bf16, 128 dims:   8 heads of 256    8.7 / 10.2  7.1  5.8  6.5     8 of 512           9.0 / 17.8 11.1  8.1  8.1
//     8 of 640        9.1 / 21.6 13.1  9.2  9.6     8 of 1,024         9.4 / 32.7 19.2 12.5 11.3
//     96 of 512      12.6 / 23.3 14.2 10.2 10.1     96 of 1,024       16.3 / 45.1 26.0 17.3 16.0
//     192 of 768     19.8 / 35.4 21.0 15.6 15.5     256 of 768        22.9 / 36.2 21.8 18.5 18.7
//     512 of 64       9.6 /  5.5  6.1  6.0 10.2     512 of 1,024      46.5 / 52.5 43.8 43.6 45.5
//     4,096 of 64    29.7 / 25.8 29.0 39.5 71.9     2,048 of 256      46.1 / 43.7 45.7 46.1 64.1
//     3,200 of 50 to 1,024            151 / 155 146 141 162
//     group 1: 3,200 of 131 to 643    112 / 110 105 102 119             512 of 512 to 2,048    62.3 / 96.9 65.2 59.8 60.2
//              16,384 of 64          94.3 / 87.0 92.7 137 276           32 of 647              10.5 / 28.7 17.8 12.5 11.2
//   e4m3, 128 dims:   8 of 512          8.9 / 19.6 12.1  8.7  7.9     8 of 768           9.1 / 28.1 16.6 11.0  9.7
//     192 of 448     14.1 / 22.6 14.2 10.4 10.3     192 of 1,024      19.7 / 48.1 28.3 17.8 14.0
//     256 of 1,024   20.3 / 48.4 28.6 18.4 15.9     320 of 1,024      25.4 / 52.1 34.7 22.6 26.0
//     1,024 of 32 to 512  25.2 / 29.5 21.5 22.6 31.0  2,400 of 1 to 400, int8  41.7 / 42.1 37.2 37.3 66.6
//   bf16, 64 dims:    8 of 768          8.8 / 21.0 14.0  9.8  8.2     8 of 1,024         8.8 / 27.3 15.6 11.2  9.0
//     32 of 384       8.9 / 13.4  8.9  6.8  6.8     256 of 1,024      19.0 / 37.7 23.1 16.2 14.3
//     2,048 of 30 to 200  22.9 / 15.2 14.9 17.1 23.5
//   float32, 128 dims (no form with eight):  8 of 256  12.2 / 20.7 13.1 10.8     8 of 512     12.5 / 40.1 23.8 17.1
//     128 of 384     22.3 / 35.1 22.5 19.5          256 of 512        33.0 / 47.3 30.1 27.4
int whole_waves(const riftkv_cache& c, int64_t heads, int64_t max_pages) {
    const int64_t most = max_pages * c.page_size;
    const bool f32 = c.dt == RIFTKV_F32, wide = c.dt == RIFTKV_BF16 && c.head_dim == 128;
    int longest = 1024;
    if (f32 && heads < 256) longest = heads < 128 ? 256 : 384;
    if (!f32 && heads < 96) longest = c.head_dim == 64 ? 768 : 512;
    if (most > longest) return 0;
    if (most <= 64 || (most <= 256 && heads >= 2048)) return 1;
    int waves = 4;
    if (most <= 128 || (most <= 512 && heads >= 1024)) waves = 2;
    else if (!f32 && most > 384 && heads <= (wide ? 192 : 256)) waves = 8;
    return heads * waves < (1 << 26) ? waves : 1;   // a launch has less than 2^32 threads (at most 65,535 x 1,024 heads)
}

}  // namespace

size_t kv_attention_workspace(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages) {
    const size_t wgs = workgroups(c, n_heads, n_seq, max_pages);
    const size_t joins = (wgs * 2 * sizeof(int4) + 255) / 256 * 256;
    return joins + wgs * 2 * rows_of(c, n_heads) * (c.head_dim + 4) * sizeof(float);
}

bool kv_attention_counts(const riftkv_cache& c, int n_heads, int64_t n_seq, int64_t max_pages) {
    return most_tiles(c, n_heads, n_seq, max_pages) < (1ll << 41);   // a wave's share (one of 2,048) in 31 bits
}

hipError_t launch_kv_attention(const riftkv_cache& c, const KvAttention& a, hipStream_t st) {
    AttnParams p{};
    p.q = a.q;
    p.out = a.out;
    p.ld_q = a.ld_q;
    p.ld_out = a.ld_out;
    p.k = static_cast<const unsigned char*>(c.k);
    p.v = static_cast<const unsigned char*>(c.v);
    p.ks = c.k_scale;
    p.vs = c.v_scale;
    p.table = a.table;
    p.lens = a.lens;
    p.status = a.status;
    const int wgs = workgroups(c, a.n_heads, a.n_seq, a.max_pages);
    p.joins = static_cast<int4*>(a.workspace);
    p.slots = reinterpret_cast<float*>(static_cast<unsigned char*>(a.workspace) + (wgs * 2 * sizeof(int4) + 255) / 256 * 256);
    p.n_seq = a.n_seq;
    p.max_pages = a.max_pages;
    p.n_pages = c.n_pages;
    p.n_kv = c.n_kv_heads;
    p.shift = 31 - __builtin_clz(c.page_size);
    p.group = a.n_heads / c.n_kv_heads;
    p.q_tiles = q_tiles_of(c, a.n_heads);
    p.rows = rows_of(c, a.n_heads);
    p.few = a.n_seq <= kFewSeqs && most_tiles(c, a.n_heads, a.n_seq, a.max_pages) < (1ll << 31);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    const size_t record = (size_t)p.rows * (c.head_dim + 4) * sizeof(float);
    auto launch = [&](auto kernel, unsigned grid, int waves, size_t lds) {
        if (lds > 64 * 1024) {   // 16 query rows of 128 dimensions; the attribute is the current device's
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * waves), lds, st, p);
        return hipGetLastError();
    };
    const int64_t heads_of_all = (int64_t)a.n_seq * c.n_kv_heads * p.q_tiles;
    const int whole = whole_waves(c, heads_of_all, a.max_pages);
    auto run = [&](auto t, auto dt, auto hd) {
        using T = decltype(t);
        const unsigned all = (unsigned)heads_of_all;
        if (whole == 1) return launch(attention_kernel<T, dt.value, hd.value, 1, true>, all, 1, record);
        if (whole == 2) return launch(attention_kernel<T, dt.value, hd.value, 2, true>, all, 2, 2 * record);
        if constexpr (dt.value != RIFTKV_F32)
            if (whole == 8) return launch(attention_kernel<T, dt.value, hd.value, 8, true>, all, 8, 8 * record);
        if (whole == 4) return launch(attention_kernel<T, dt.value, hd.value, 4, true>, all, 4, 4 * record);
        const hipError_t e = launch(attention_kernel<T, dt.value, hd.value, kSplitWaves, false>, (unsigned)wgs, kSplitWaves, 2 * kSplitWaves * record);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((join_kernel<T, hd.value>), dim3(wgs), dim3(2 * kJoinThreads), 0, st, p);
        return hipGetLastError();
    };
    auto heads = [&](auto t, auto dt) {
        if (c.head_dim == 128) return run(t, dt, std::integral_constant<int, 128>{});
        return run(t, dt, std::integral_constant<int, 64>{});
    };
    auto types = [&](auto dt) {
        if constexpr (dt.value != RIFTKV_F32)
            if (a.bf16) return heads(bf16_t{}, dt);
        return heads(float{}, dt);
    };
    switch (c.dt) {
        case RIFTKV_F32: return types(std::integral_constant<riftkv_dtype, RIFTKV_F32>{});
        case RIFTKV_BF16: return types(std::integral_constant<riftkv_dtype, RIFTKV_BF16>{});
        case RIFTKV_FP8: return types(std::integral_constant<riftkv_dtype, RIFTKV_FP8>{});
        case RIFTKV_INT8: return types(std::integral_constant<riftkv_dtype, RIFTKV_INT8>{});
    }
    return hipErrorInvalidValue;
}

}  // namespace rift
