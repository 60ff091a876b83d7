// One wave's pass over tiles of paged keys and values for up to 16 queries of one key head,
// and what kernels made of it share.
//
// With a tile's 32 tokens as rows, S^T = K Q^T leaves a lane the scores of one query and 8 tokens; they
// are the lane's own share of the second product's right operand, O^T = V^T P^T, if its token order is the
// lanes' (a sum's order is free), and a lane's own rows of V are, with two bytes or halfwords exchanged in
// registers, its share of the left one.  So nothing passes through LDS, and the softmax is a lane's own but
// for two swaps.
//
// Scores, weights and sums are float32: each weight, and each float32 query, goes into the matrix product
// as three bf16 terms that add up to it.
#pragma once

#include "kv_device.h"

namespace rift {

constexpr int kTile = 32;                 // tokens of a tile

__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }

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

// A whole of four columns: rounded to the type of the outputs.
template <typename T>
__device__ __forceinline__ void store_four(void* p, size_t at, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p) + at) =
            make_uint2((uint32_t)round_bf16(a) | (uint32_t)round_bf16(b) << 16, (uint32_t)round_bf16(c) | (uint32_t)round_bf16(d) << 16);
    else *reinterpret_cast<f32x4_t*>(static_cast<float*>(p) + at) = f32x4_t{a, b, c, d};
}

// Half a tile: its first row among the pages' rows (of a page that is there, whatever n), and how many
// of its 16 tokens count.
struct Half {
    size_t row;
    int n;
};

struct TilePages {
    const unsigned char *k, *v;
    const uint8_t *ks, *vs;
};

// T: type of the queries.  The calls of a tile: load_k, load_v; scores, which uses up the keys; softmax; values,
// which uses up the values.
template <typename T, riftkv_dtype DT, int HD>
struct TilePass {
    static constexpr int B = DT == RIFTKV_F32 ? 4 : DT == RIFTKV_BF16 ? 2 : 1;   // bytes a value
    static constexpr bool SCALED = B == 1, F32 = DT == RIFTKV_F32;
    // A load of keys takes E 64-byte pieces of 16 / E rows (whole 128-byte lines), so that
    // a row of the first product's left operand is one piece of one token: it meets each piece of
    // the query, in an accumulator of its own, and a score is the sum of what belongs
    // together.  Rows of 64 bytes, and float32 ones (whose products are not idle): E = 1.
    static constexpr int E = F32 || HD * B == 64 ? 1 : 2;
    static constexpr int KF = HD * B / (64 * E);    // loads of a lane for 16 / E keys
    static constexpr int I = 4 / E;                 // a lane's scores of those
    static constexpr int VW = HD * B / 64;          // words of a lane of one value row
    static constexpr int C = HD / 16;               // columns of a lane of one value row
    static constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = 3;

    int n, g;                                       // this lane's query, and its quarter of the tokens
    uint32_t kr[2][E][KF][4], vr[2][4][VW], ksc[2], vsc[2];
    bf16x8_t qf[F32 ? 1 : NQ][F32 ? 1 : HD / 32];
    float qs[F32 ? HD / 4 : 1];
    f32x4_t o[C];                                   // o[c][i] is column (4 g + i) C + c of query n
    float m, l;                                     // largest score (in log2 units), this lane's sum of weights
    float s[8];                                     // s[4 h + i]: token 4 g + i of half h

    __device__ __forceinline__ explicit TilePass(int lane) : n(lane & 15), g(lane >> 4) {}

    // q: this lane's query; absent (a column that no query has): zeros.
    __device__ __forceinline__ void start(const T* q, bool there) {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(q + 16 * i + 4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) qs[4 * i + e] = there ? x[e] : 0.f;
            }
        } else {
#pragma unroll
            for (int f = 0; f < HD / 32; ++f) {
                const T* src = q + (SCALED ? (f >> 1) * 64 + g * 16 + (f & 1) * 8 : f * 32 + g * 8);
                if constexpr (NQ == 1) {
                    u32x4_t x = *reinterpret_cast<const u32x4_t*>(src);
                    if (!there) x = u32x4_t{0, 0, 0, 0};
                    qf[0][f] = __builtin_bit_cast(bf16x8_t, x);
                } else {
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
    }

    // Rows behind the last token are not read: their lanes take its row once more, and one line of the
    // first row where no token counts.
    __device__ __forceinline__ void load_k(const TilePages& p, const Half (&half)[2]) {
        // Load x of the E takes tokens 4 r + I x + i (r = 0..3, i < I) of a half: lane (n, g) the piece n mod E of row n / E.
        const int k_row = E == 1 ? n : 4 * (n >> 2) + ((n >> 1) & 1);
        const unsigned k_col = (n % E) * 64 + g * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int last = max(half[h].n - 1, 0);
#pragma unroll
            for (int x = 0; x < E; ++x) {
                const unsigned off = min(k_row + x * I, last) * (HD * B) + (half[h].n > 0 ? k_col : 0);
#pragma unroll
                for (int f = 0; f < KF; ++f) load_words<4>(kr[h][x][f], p.k + half[h].row * (HD * B) + off + 64 * E * f);
            }
            if constexpr (SCALED) ksc[h] = *reinterpret_cast<const uint32_t*>(p.ks + half[h].row + 4 * g);
        }
    }
    __device__ __forceinline__ void load_v(const TilePages& p, const Half (&half)[2]) {
        const unsigned v_col = n * VW * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int last = max(half[h].n - 1, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_words<VW>(vr[h][i], p.v + half[h].row * (HD * B) + (unsigned)(min(4 * g + i, last) * (HD * B) + (half[h].n > 0 ? v_col : 0)));
            if constexpr (SCALED) vsc[h] = *reinterpret_cast<const uint32_t*>(p.vs + half[h].row + 4 * g);
        }
    }

    __device__ __forceinline__ void scores(float scale_log2) {
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
                    s[j] = a * scale_log2;
                }
            }
        }
    }

    // Weights in place of the scores.  na, nb: the tokens of the halves that count (the same for the whole
    // wave); whatever lies behind them is no part of a sum, NaN or not.
    __device__ __forceinline__ void softmax(int na, int nb) {
        const bool tail = na < 16 || nb < 16;
        if (tail) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((j & 3) >= (j < 4 ? na : nb) - 4 * g) s[j] = -INFINITY;
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
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[j] = __builtin_amdgcn_exp2f(s[j] - ref);
            l += s[j];
            if constexpr (SCALED) s[j] *= scale_of((vsc[j >> 2] >> (8 * (j & 3))) & 0xFFu);
        }
        if (tail) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((j & 3) >= (j < 4 ? na : nb) - 4 * g) {
                    s[j] = 0.f;
#pragma unroll
                    for (int w = 0; w < VW; ++w) vr[j >> 2][j & 3][w] = 0;
                }
        }
    }

    __device__ __forceinline__ void values() {
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[j >> 2][j & 3][c]), s[j], o[c], 0, 0, 0);
        } else {
            u32x4_t pf[NP];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[NP];
                split_bf16<NP>(s[2 * j], s[2 * j + 1], w);
#pragma unroll
                for (int i = 0; i < NP; ++i) pf[i][j] = w[i];
            }
            auto add = [&](int c, const u32x4_t& vw) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vw), __builtin_bit_cast(bf16x8_t, pf[i]), o[c], 0, 0, 0);
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
    }

    // Rows of a part: HD weighted values, the largest score, the sum.  rows: those that queries have.
    __device__ __forceinline__ void put(float* part, int rows, float sum) const {
        if (n >= rows) return;
        float* dst = part + n * (HD + 4);
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
};

// The sum of a part in which no token counts.  It adds to others like zero, and only a total
// of parts that are all like it has its sign: that row is zeros, where 0 from scores of -infinity gives NaN.
constexpr float kNoTokens = -0.f;
__device__ __forceinline__ float weight_of(float sum) { return __float_as_uint(sum) == 0x80000000u ? 0.f : 1.f / sum; }

}  // namespace rift
