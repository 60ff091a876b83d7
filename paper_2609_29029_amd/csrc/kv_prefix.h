// Attention of many query rows over a prefix that they share (riftkv_attention_shared): the rows of a key head, one for
// each sequence and query head of the group, stand under each other, so that a tile of keys and values is read
// once for up to 128 of them.
//
// A workgroup takes 128 rows of a key head and a part of the prefix, a wave 32 of the rows.  Tiles of 64 tokens go through two LDS
// stages, by LDS DMA or, 8-bit ones, through registers where they are widened to bf16; the next tile is under way meanwhile.
// Weighted values, a reference and the sum of a part go to the workspace.
//
// S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16: a lane holds the scores of one query, and its weights are
// already its share of the second product's right operand, whose left one comes from transposing LDS reads.  Float32
// queries, and all weights, go into the products as three bf16 terms that add up to them.
//
// Bound by the products and the weights' vector instructions together, which overlap only in part: of a wave's tile 64 products of
// 32 cycles and some 270 vector instructions with 32 exponentials of 16.  64 sequences' 256 rows after 32,768 tokens, 8 key heads,
// bf16: 34 GFLOP in 76 us alone (134 MB), and 81.5 with the sequences' own 79 MB beside it (with two terms a weight, which are up
// to 2^-16 of it off, 66); every sequence on its own read the prefix 64 times and took 606.  Kept, measured with two terms: halves
// of a tile in a pipeline, a product and then two weights in turn (61 us a launch of 256 workgroups, 70 without); not kept: more of
// the next tiles touched ahead into L2, operands two products ahead (no change).
//
// Rows of a tile are 256 bytes (64 dimensions fill half of them); the 16-byte chunks of row r lie at chunk ^ (r & 15) for
// keys and at chunk ^ 4 (r & 3) for values, so that neither read meets a bank twice.
#pragma once

#include "kv_tile.h"
#include "lds_dma.h"

namespace rift {

// Rows of queries, one for each sequence and query head of a key head's group, over a prefix.
struct PrefixParams {
    const void* q;
    int64_t ld_q;
    TilePages pages;
    const int* table;
    int* status;
    float* slots;        // [key head][parts][rows][HD + 4]: weighted values, a reference, sum
    int len, n_kv, n_pages, shift, group, rows, row_tiles, parts;
    float scale_log2;
};

constexpr int kRows = 128, kTokens = 64;      // of a workgroup, of a tile
constexpr int kRowBytes = 256;
constexpr int kTileBytes = kTokens * kRowBytes;
constexpr int kStageBytes = 2 * kTileBytes;   // keys, then values
constexpr int kScaleFloats = 4 * 2 * kTokens; // of keys and values, four tiles
constexpr size_t kPrefixLds = 2 * kStageBytes + kScaleFloats * sizeof(float);
static_assert(kPrefixLds >= kRows * (128 + 4) * sizeof(float), "the rows of a workgroup");
constexpr float kLazy = 8.f;                  // log2 units that a reference is set above the largest score

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;

// Lane i of each 16-lane group g gets, in component j, the 16-bit element at (address of lane 16 g + 4 j + i / 4) + i % 4.
__device__ __forceinline__ v4s_t lds_read_tr16(const void* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p)); }

// A value that has to be there at this point of the program.
template <typename X>
__device__ __forceinline__ void hold(X& x) {
    asm volatile("" : "+v"(x));
}

// Workgroup `block` of n_kv * row_tiles * parts; lds: kPrefixLds bytes, two stages, then their scales.
template <typename T, riftkv_dtype DT, int HD>
__device__ __forceinline__ void prefix_body(const PrefixParams& p, int block, unsigned char* lds) {
    constexpr int B = DT == RIFTKV_BF16 ? 2 : 1;
    constexpr bool SCALED = B == 1;
    constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = 3;
    constexpr int CHUNKS = HD * B / 16;           // 16-byte chunks of a row in the pages
    constexpr int LOADS = kTokens * CHUNKS / 256; // of a thread, of keys or values
    constexpr int STEP = 256 / CHUNKS;            // rows between them
    constexpr int NK = HD / 16, NT = HD / 32;     // steps of the first product, 32-dimension blocks of the second
    constexpr int RS = HD + 4;
    float* scales = reinterpret_cast<float*>(lds + 2 * kStageBytes);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, n = lane & 31;
    const int part = block % p.parts, rest = block / p.parts;
    const int kvh = rest / p.row_tiles, r0 = (rest - kvh * p.row_tiles) * kRows + 32 * wave;
    const int tiles = (p.len + kTokens - 1) / kTokens;
    const int t0 = (int)((int64_t)tiles * part / p.parts), t1 = (int)((int64_t)tiles * (part + 1) / p.parts);
    const bool rows_here = r0 < p.rows;
    const int in_mask = (1 << p.shift) - 1;
    bool bad = false;

    // The pages' numbers, 64 at a time, one a lane.
    int first = (t0 * kTokens) >> p.shift, mine = 0;
    auto look = [&]() __attribute__((always_inline)) {
        const int e = first + lane;
        mine = t0 < t1 && e <= (p.len - 1) >> p.shift ? p.table[e] : 0;
        if ((unsigned)mine >= (unsigned)p.n_pages) {
            bad = true;
            mine = 0;
        }
    };
    // First row of 16 tokens among the pages' rows; token: the same for the whole wave, before the end.
    auto row_at = [&](int token) __attribute__((always_inline)) {
        const int page = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane((token >> p.shift) - first));
        return ((((size_t)page * p.n_kv) + kvh) << p.shift) + (token & in_mask);
    };
    look();

    // A bf16 tile comes by LDS DMA: a wave moves 16 of its rows, four an instruction; lane i the chunk that belongs at place
    // i mod 16 of row i / 16.
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    auto dma = [&](int t, bool v) __attribute__((always_inline)) {
        const int r = 16 * wave;
        if (t * kTokens + r >= p.len) return;
        const unsigned char* base = (v ? p.pages.v : p.pages.k) + row_at(t * kTokens + r) * (HD * B);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * i + (lane >> 4);
            const int c = (lane & 15) ^ (v ? 4 * (row & 3) : row);
            if (HD == 128 || c < CHUNKS)
                lds_dma16(base, (uint32_t)(row * (HD * B) + c * 16), lds0 + (t & 1) * kStageBytes + (v ? kTileBytes : 0) + (r + 4 * i) * kRowBytes);
        }
    };
    // An 8-bit tile goes through registers, where it is widened: chunk `chunk` of rows row, row + STEP, .. a thread.  All lanes
    // of a wave are in 16 rows of one page.
    const int row = tid / CHUNKS, chunk = tid % CHUNKS;
    u32x4_t kr[SCALED ? LOADS : 1], vr[SCALED ? LOADS : 1];
    uint32_t sr = 0;                               // scale bytes of 16 tokens a wave, of the keys and then of the values
    auto load = [&](u32x4_t(&x)[SCALED ? LOADS : 1], const unsigned char* pages, int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = t * kTokens + __builtin_amdgcn_readfirstlane((row + i * STEP) & ~15);
            const size_t at = ((r < p.len ? row_at(r) : 0) + ((row + i * STEP) & 15)) * (HD * B) + 16 * chunk;   // (past the end: any)
            x[i] = *reinterpret_cast<const u32x4_t*>(pages + at);
        }
    };
    auto store = [&](const u32x4_t(&x)[SCALED ? LOADS : 1], unsigned char* to, bool v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = row + i * STEP;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int c = (2 * chunk + y) ^ (v ? 4 * (r & 3) : r & 15);
                *reinterpret_cast<u32x4_t*>(to + r * kRowBytes + (c << 4)) =
                    u32x4_t{widen<DT, false>(x[i][2 * y]), widen<DT, true>(x[i][2 * y]), widen<DT, false>(x[i][2 * y + 1]), widen<DT, true>(x[i][2 * y + 1])};
            }
        }
    };
    // Keys of tile t + 1 (and the scales of its keys and values), and values of tile t, are asked for ..
    auto fetch = [&](int t) __attribute__((always_inline)) {
        if (t + 1 < t1) {
            if ((((t + 1) * kTokens + kTokens - 16) >> p.shift) - first >= 64) {
                first = (max(t, t0) * kTokens) >> p.shift;
                look();
            }
            if constexpr (SCALED) {
                load(kr, p.pages.k, t + 1);
                const int r = (t + 1) * kTokens + 16 * wave;
                const size_t at = r < p.len ? row_at(r) : 0;
                sr = lane < 32 && r + (lane & 15) < p.len ? (lane < 16 ? p.pages.ks : p.pages.vs)[at + (lane & 15)] : 127;   // (past the end: 1)
            } else dma(t + 1, false);
        }
        if (t >= t0 && t < t1) {
            if constexpr (SCALED) load(vr, p.pages.v, t);
            else dma(t, true);
        }
    };
    // .. and have arrived in LDS, for all waves.
    auto arrive = [&](int t) __attribute__((always_inline)) {
        if constexpr (SCALED) {
            if (t + 1 < t1) {
                store(kr, lds + ((t + 1) & 1) * kStageBytes, false);
                if (lane < 32) scales[((t + 1) & 3) * 2 * kTokens + (lane & 16) * (kTokens / 16) + 16 * wave + (lane & 15)] = scale_of(sr);
            }
            if (t >= t0) store(vr, lds + (t & 1) * kStageBytes + kTileBytes, true);
        } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    if (t0 < t1) fetch(t0 - 1);
    // this lane's query, 16 kk + 8 h .. of it; negated for a negative scale, so that the largest score is that of the largest
    // product, and nothing of it for a scale of 0
    bf16x8_t qf[NQ][NK];
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    const bool no_scale = p.scale_log2 == 0.f;
    const float scale = no_scale ? 1.f : fabsf(p.scale_log2);
    {
        const int r = min(r0 + n, p.rows - 1), seq = r / p.group;
        const T* q = static_cast<const T*>(p.q) + (size_t)seq * p.ld_q + (size_t)(kvh * p.group + r - seq * p.group) * HD + 8 * h;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            u32x4_t x[NQ];
            if constexpr (NQ == 1) x[0] = *reinterpret_cast<const u32x4_t*>(q + 16 * kk);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t w[NQ];
                    split_bf16<NQ>(q[16 * kk + 2 * e], q[16 * kk + 2 * e + 1], w);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) x[i][e] = w[i];
                }
            }
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[i][e] ^= flip;
                    if (no_scale)    // zeros, but for what is not a number, or infinite
                        x[i][e] = ((x[i][e] & 0x7F80u) == 0x7F80u ? 0x7FC0u : 0u) | ((x[i][e] & 0x7F800000u) == 0x7F800000u ? 0x7FC00000u : 0u);
                }
                qf[i][kk] = __builtin_bit_cast(bf16x8_t, x[i]);
            }
        }
        // (waited for here: the compiler does not count the DMA among what is under way)
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) asm volatile("" : "+v"(qf[i][kk]));
    }
    f32x16_t o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    // Half a tile at a time: s[i] is token 32 kb + 8 (i / 4) + 4 h + i % 4 of tile t.  Steps of one product each: `step` kk of
    // the first, `step` (x, c) of the second.
    // 8-bit tiles have no registers left for the places of all steps (spilled ones come back behind the next tile's loads, whose
    // order they share): there each is worked out where it is used.
    const int k_off = n * kRowBytes + ((h ^ (n & 15)) << 4);
    auto key_at = [&](int t, int kb, int kk) __attribute__((always_inline)) {
        int at = k_off;
        if constexpr (SCALED) hold(at);
        return *reinterpret_cast<const bf16x8_t*>(lds + (t & 1) * kStageBytes + kb * 32 * kRowBytes + (at ^ (kk << 5)));
    };
    auto score = [&](const bf16x8_t& kf, int kk, f32x16_t& s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i][kk], s, 0, 0, 0);
    };
    const int tg = lane >> 4, tj = (lane >> 2) & 3, tu = lane & 3;
    const int v_off = (4 * (tg >> 1) + tj) * kRowBytes + (2 * (tg & 1) + (tu >> 1)) * 16 + 8 * (tu & 1);
    auto value_at = [&](int t, int kb, int x, int c) __attribute__((always_inline)) {
        const unsigned char* at = lds + (t & 1) * kStageBytes + kTileBytes + (kb * 32 + 16 * x) * kRowBytes + v_off +
                                  ((c ^ tj) << 6);   // four chunks on, moved by the row's swizzle
        const v4s_t lo = lds_read_tr16(at), hi = lds_read_tr16(at + 8 * kRowBytes);
        return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 0, 1)), __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 2, 3)),
                       __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 0, 1)), __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 2, 3))};
    };
    auto value_term = [&](const u32x4_t& vv, int c, const u32x4_t& pf) __attribute__((always_inline)) {
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vv), __builtin_bit_cast(bf16x8_t, pf), o[c], 0, 0, 0);
    };
    auto scores = [&](int t, int kb, f32x16_t& s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) score(key_at(t, kb, kk), kk, s);
    };
    auto values = [&](int t, int kb, const u32x4_t(&pf)[2][NP]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const u32x4_t vv = value_at(t, kb, x, c);
#pragma unroll
                for (int i = 0; i < NP; ++i) value_term(vv, c, pf[x][i]);
            }
    };
    // No scores for tokens past the end.
    auto mask = [&](int t, int kb, f32x16_t& s) __attribute__((always_inline)) {
        const int there = p.len - t * kTokens;
        if (there < kTokens) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * kb + 8 * (i >> 2) + 4 * h + (i & 3) >= there) s[i] = -INFINITY;
        }
    };
    // The reference of half a tile's weights; what is added up so far is to be scaled by f.
    auto refer = [&](int t, int kb, f32x16_t& s) __attribute__((always_inline)) {
        if constexpr (SCALED) {
            const float* ks = scales + (t & 3) * 2 * kTokens + 32 * kb + 4 * h;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4_t f = *reinterpret_cast<const f32x4_t*>(ks + 2 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i + e] *= f[e];
            }
        }
        // A rounding of its own: fused with the reference's subtraction, scores past 2^31 would be whole exponents off it.
        {
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= scale;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        // It moves only when a score passes it, and then to kLazy above that: weights are 1 at most, the largest 2^-kLazy at
        // least, and the sums are rescaled for few tiles.  (Set at the largest score, to be passed by kLazy, weights of up to 2^kLazy
        // made sums of large values overflow that do not with a running maximum.)
        const float mn = mx > m ? mx + kLazy : m;
        const float f = __builtin_amdgcn_exp2f(m - ref_of(mn));
        m = mn;
        l *= f;
        return f;
    };
    auto weight = [&](float s, float neg_ref) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(s + neg_ref); };
    // The j-th two weights, as a word of each of the second product's operands.
    auto split_pair = [&](int t, int kb, int j, float a, float b, uint32_t(&y)[NP]) __attribute__((always_inline)) {
        l += a;
        l += b;
        if constexpr (SCALED) {
            const float2 f = *reinterpret_cast<const float2*>(scales + (t & 3) * 2 * kTokens + kTokens + 32 * kb + 4 * h + 8 * (j >> 1) + 2 * (j & 1));
            a *= f.x;
            b *= f.y;
        }
        split_bf16<NP>(a, b, y);
    };
    auto weights = [&](int t, int kb, f32x16_t& s, u32x4_t(&pf)[2][NP]) __attribute__((always_inline)) {
        const float f = refer(t, kb, s), neg_ref = -ref_of(m);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t y[NP];
            split_pair(t, kb, j, weight(s[2 * j], neg_ref), weight(s[2 * j + 1], neg_ref), y);
#pragma unroll
            for (int i = 0; i < NP; ++i) pf[j >> 2][i][j & 3] = y[i];
        }
        return f;
    };
    auto rescale = [&](float f) __attribute__((always_inline)) {
        if (__any(f != 1.f)) {
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[c][i] *= f;
        }
    };
    // scores(tn, kn, sn), values(tv, kv, pv) and weights(ts, ks, s, pf) in eight pieces, so that the vector unit makes two weights
    // while the matrix cores work on a piece of the products.
    auto half = [&](int tn, int kn, f32x16_t& sn, int tv, int kv, const u32x4_t(&pv)[2][NP], int ts, int ks, f32x16_t& s, u32x4_t(&pf)[2][NP])
        __attribute__((always_inline)) {
        constexpr int NV = 2 * NT;
        bf16x8_t kf[NK];
        u32x4_t vv[NV];
        float f = 1.f, neg_ref = 0.f;
        // The operands of piece j, a piece ahead (two ahead: the same, and 8-bit pages run out of registers): the scores' k0, the
        // values' v0, where it has one.
        auto ask = [&](int j) __attribute__((always_inline)) {
            const int k0 = j * NK / 8, k1 = (j + 1) * NK / 8, v0 = j * NV / 8, v1 = (j + 1) * NV / 8;
            if (k1 > k0) kf[k0] = key_at(tn, kn, k0);
            if (v1 > v0) vv[v0] = value_at(tv, kv, v0 / NT, v0 % NT);
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[i] = 0.f;
        ask(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k0 = j * NK / 8, k1 = (j + 1) * NK / 8, v0 = j * NV / 8, v1 = (j + 1) * NV / 8;
            // A product of the matrix cores holds the next one up: between two of them stands what the vector unit can do, and the
            // empty asm keeps it there.
            if (j < 7) ask(j + 1);
            bf16x8_t kf_now{};
            u32x4_t vv_now{};
            if (k1 > k0) kf_now = kf[k0];
            if (v1 > v0) vv_now = vv[v0];
            hold(kf_now);
            if (k1 > k0) score(kf_now, k0, sn);
            if (j == 0) {
                f = refer(ts, ks, s);
                neg_ref = -ref_of(m);
            }
            float w0 = s[2 * j], w1 = s[2 * j + 1];
            hold(w0);
            hold(w1);
            w0 = weight(w0, neg_ref);
            w1 = weight(w1, neg_ref);
            hold(w0);
            hold(w1);
            hold(vv_now);
            if (v1 > v0) value_term(vv_now, v0 % NT, pv[v0 / NT][0]);
            uint32_t y[NP];
            split_pair(ts, ks, j, w0, w1, y);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                hold(y[i]);
                pf[j >> 2][i][j & 3] = y[i];
            }
#pragma unroll
            for (int i = 1; i < NP; ++i)
                if (v1 > v0) value_term(vv_now, v0 % NT, pv[v0 / NT][i]);
        }
        return f;
    };
    // The halves of the tiles follow each other so that the matrix cores have work while one half's weights are made: the next
    // half's scores, and the values of the one before.  The keys of tile t + 1 and the values of tile t are needed from the
    // second half of tile t on: there the waves meet, and the stages that the keys of tile t and the values of
    // tile t - 1 lay in are filled anew.
    if (t0 < t1) {
        f32x16_t sa, sb;
        u32x4_t pa[2][NP], pb[2][NP];
        arrive(t0 - 1);
        fetch(t0);
        if (rows_here) {
            scores(t0, 0, sa);
            scores(t0, 1, sb);
            mask(t0, 0, sa);
            weights(t0, 0, sa, pa);
        }
        for (int t = t0; t + 1 < t1; ++t) {
            arrive(t);
            fetch(t + 1);
            if (!rows_here) continue;
            rescale(half(t + 1, 0, sa, t, 0, pa, t, 1, sb, pb));
            mask(t + 1, 0, sa);
            rescale(half(t + 1, 1, sb, t, 1, pb, t + 1, 0, sa, pa));
        }
        arrive(t1 - 1);
        const int there = p.len - (t1 - 1) * kTokens;
        if (there < kTokens) {     // values behind the last token: no part of a sum, whatever they are
            unsigned char* V = lds + ((t1 - 1) & 1) * kStageBytes + kTileBytes;
            for (int i = tid; i < (kTokens - there) * 16; i += 256)
                *reinterpret_cast<u32x4_t*>(V + (there + i / 16) * kRowBytes + (i % 16) * 16) = u32x4_t{0, 0, 0, 0};
            __syncthreads();
        }
        if (rows_here) {
            mask(t1 - 1, 1, sb);
            values(t1 - 1, 0, pa);
            rescale(weights(t1 - 1, 1, sb, pb));
            values(t1 - 1, 1, pb);
        }
    }
    l += __shfl_xor(l, 32);
    if (t0 == t1) l = kNoTokens;
    // every thread has looked at other pages
    if (__syncthreads_or(bad)) {
        l = NAN;
        if (tid == 0) *p.status = RIFT_ERR_SHAPE;
    }
    // The wave's rows lie together in the workspace: through LDS (all of it: four times 32 rows), so that whole lines are written.
    if (!rows_here) return;
    float* out = reinterpret_cast<float*>(lds) + wave * 32 * RS;
    float* dst = out + n * RS;
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4)   // dimensions 32 c + 2 i + 4 h ..
            *reinterpret_cast<f32x4_t*>(dst + 32 * c + 2 * i + 4 * h) = f32x4_t{o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]};
    if (h == 0) *reinterpret_cast<f32x4_t*>(dst + HD) = f32x4_t{m, l, 0.f, 0.f};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    f32x4_t* to = reinterpret_cast<f32x4_t*>(p.slots + (((size_t)kvh * p.parts + part) * p.rows + r0) * RS);
    const int quads = min(p.rows - r0, 32) * (RS / 4);
    for (int i = lane; i < quads; i += 64) to[i] = reinterpret_cast<const f32x4_t*>(out)[i];
}

}  // namespace rift
