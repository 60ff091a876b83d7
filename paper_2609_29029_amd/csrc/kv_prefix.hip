// Attention of many query rows over a prefix that they share (riftkv_attention_shared): the rows of a key head, one for
// each sequence and query head of the group, stand under each other, so that a tile of keys and values is read
// once for up to 128 of them.
//
//   prefix_kernel   a workgroup takes 128 rows of a key head and a part of the prefix, a wave 32 of the rows.  Tiles of
//                   64 tokens go through two LDS stages, widened to bf16 on the way; the next tile's loads are in
//                   flight meanwhile.  Weighted values, largest score and sum of a part go to the workspace,
//                   where ranges_kernel joins them with the sequences' own.
//
// S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16: a lane holds the scores of one query, and its weights are
// already its share of the second product's right operand, whose left one comes from transposing LDS reads.  Weights,
// and float32 queries, go into the products as three bf16 terms that add up to them, as in the attention of single sequences.
//
// Rows of a tile are 256 bytes (64 dimensions fill half of them); the 16-byte chunks of row r lie at chunk ^ (r & 15) for
// keys and at chunk ^ 4 (r & 3) for values, so that neither read meets a bank twice.
#include <type_traits>

#include "kv_ranges.h"

namespace rift {

namespace {

constexpr int kRows = 128, kTokens = 64;      // of a workgroup, of a tile
constexpr int kRowBytes = 256;
constexpr int kTileBytes = kTokens * kRowBytes;
constexpr int kStageBytes = 2 * kTileBytes;   // keys, then values
constexpr int kScaleFloats = 2 * 2 * kTokens; // of keys and values, two stages
constexpr float kLazy = 8.f;                  // log2 units by which a score may pass the reference

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;

// Lane i of each 16-lane group g gets, in component j, the 16-bit element at (address of lane 16 g + 4 j + i / 4) + i % 4.
__device__ __forceinline__ v4s_t lds_read_tr16(const void* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p)); }

// Two bf16 terms that add up to a and b but for 2^-17 of them: the first is cut off, what is left rounded.
__device__ __forceinline__ void round_split(float a, float b, uint32_t (&w)[2]) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    w[0] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    a -= __uint_as_float(x & 0xFFFF0000u);
    b -= __uint_as_float(y & 0xFFFF0000u);
    w[1] = (uint32_t)round_bf16(a) | (uint32_t)round_bf16(b) << 16;
}

// LDS DMA of 16 bytes a lane: from a wave-uniform base and a lane's offset to lds + 16 lane.
__device__ __forceinline__ void dma16(const unsigned char* base, uint32_t offset, uint32_t lds) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    const uint64_t ub = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b) |
                        ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32);
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(ub) : "memory", "m0");
}

template <typename T, riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1)
prefix_kernel(PrefixParams p) {
    constexpr int B = DT == RIFTKV_BF16 ? 2 : 1;
    constexpr bool SCALED = B == 1;
    constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = sizeof(T) == 2 ? 2 : 3;
    constexpr int CHUNKS = HD * B / 16;           // 16-byte chunks of a row in the pages
    constexpr int LOADS = kTokens * CHUNKS / 256; // of a thread, of keys or values
    constexpr int STEP = 256 / CHUNKS;            // rows between them
    constexpr int NK = HD / 16, NT = HD / 32;     // steps of the first product, 32-dimension blocks of the second
    constexpr int RS = HD + 4;
    extern __shared__ __align__(16) unsigned char lds[];   // two stages, then their scales
    float* scales = reinterpret_cast<float*>(lds + 2 * kStageBytes);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, n = lane & 31;
    const int part = blockIdx.x % p.parts, rest = blockIdx.x / p.parts;
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
        if (t0 < t1 && e <= (p.len - 1) >> p.shift) {
            mine = p.table[e];
            bad |= (unsigned)mine >= (unsigned)p.n_pages;
            if (bad) mine = 0;
        } else mine = 0;
    };
    // First row of 16 tokens among the pages' rows; token: the same for the whole wave, before the end.
    auto row_at = [&](int token) __attribute__((always_inline)) {
        const int page = __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane((token >> p.shift) - first));
        return ((((size_t)page * p.n_kv) + kvh) << p.shift) + (token & in_mask);
    };
    auto reach = [&](int t) __attribute__((always_inline)) {   // the pages of tile t
        if (((t * kTokens + kTokens - 16) >> p.shift) - first >= 64) {
            first = (t * kTokens) >> p.shift;
            look();
        }
    };
    look();

    // A bf16 tile comes by LDS DMA: waves 0 and 1 move 32 rows of keys each, waves 2 and 3 of values, four rows an instruction;
    // lane i the chunk that belongs at place i mod 16 of row i / 16.
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    auto dma = [&](int t) __attribute__((always_inline)) {
        reach(t);
        const bool v = wave >= 2;
        const unsigned char* pages = v ? p.pages.v : p.pages.k;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int r = 32 * (wave & 1) + 16 * x;            // the first of 16 rows
            if (t * kTokens + r >= p.len) continue;
            const unsigned char* base = pages + row_at(t * kTokens + r) * (HD * B);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 4 * i + (lane >> 4);
                const int c = (lane & 15) ^ (v ? 4 * (row & 3) : row);
                if (HD == 128 || c < CHUNKS)
                    dma16(base, (uint32_t)(row * (HD * B) + c * 16), lds0 + (t & 1) * kStageBytes + (v ? kTileBytes : 0) + (r + 4 * i) * kRowBytes);
            }
        }
    };
    // An 8-bit tile goes through registers, where it is widened: chunk `chunk` of rows row, row + STEP, .. a thread.  All lanes
    // of a wave are in 16 rows of one page.
    const int row = tid / CHUNKS, chunk = tid % CHUNKS;
    u32x4_t kr[SCALED ? LOADS : 1], vr[SCALED ? LOADS : 1];
    uint32_t sr = 0;
    auto load = [&](int t) __attribute__((always_inline)) {
        reach(t);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = t * kTokens + __builtin_amdgcn_readfirstlane((row + i * STEP) & ~15);
            const size_t at = ((r < p.len ? row_at(r) : 0) + ((row + i * STEP) & 15)) * (HD * B) + 16 * chunk;   // (past the end: any)
            kr[i] = *reinterpret_cast<const u32x4_t*>(p.pages.k + at);
            vr[i] = *reinterpret_cast<const u32x4_t*>(p.pages.v + at);
        }
        // the scale of a key (waves 0 and 1) or value of 32 tokens a wave, the upper lanes idle
        const int r = t * kTokens + 32 * (wave & 1);
        const size_t a = r < p.len ? row_at(r) : 0, b = r + 16 < p.len ? row_at(r + 16) : 0;
        sr = 0;
        if (lane < 32 && r + lane < p.len) sr = (wave < 2 ? p.pages.ks : p.pages.vs)[(lane & 16 ? b : a) + (lane & 15)];
    };
    auto store = [&](int t) __attribute__((always_inline)) {
        unsigned char* K = lds + (t & 1) * kStageBytes;
        unsigned char* V = K + kTileBytes;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = row + i * STEP;
            const u32x4_t v = t * kTokens + r < p.len ? vr[i] : u32x4_t{0, 0, 0, 0};   // behind the last token: no part of a sum
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int c = 2 * chunk + y;
                *reinterpret_cast<u32x4_t*>(K + r * kRowBytes + ((c ^ (r & 15)) << 4)) =
                    u32x4_t{widen<DT, false>(kr[i][2 * y]), widen<DT, true>(kr[i][2 * y]), widen<DT, false>(kr[i][2 * y + 1]), widen<DT, true>(kr[i][2 * y + 1])};
                *reinterpret_cast<u32x4_t*>(V + r * kRowBytes + ((c ^ (4 * (r & 3))) << 4)) =
                    u32x4_t{widen<DT, false>(v[2 * y]), widen<DT, true>(v[2 * y]), widen<DT, false>(v[2 * y + 1]), widen<DT, true>(v[2 * y + 1])};
            }
        }
        if (lane < 32) scales[(t & 1) * 2 * kTokens + 32 * wave + lane] = scale_of(sr);
    };

    if (t0 < t1) {
        if constexpr (SCALED) load(t0);
        else dma(t0);
    }
    // this lane's query, 16 kk + 8 h .. of it; negated for a negative scale, so that the largest score is that of the largest product
    bf16x8_t qf[NQ][NK];
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    const float scale = fabsf(p.scale_log2);
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
                for (int e = 0; e < 4; ++e) x[i][e] ^= flip;
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

    const int tg = lane >> 4, tj = (lane >> 2) & 3, tu = lane & 3;
    const int v_off = (4 * (tg >> 1) + tj) * kRowBytes + (2 * (tg & 1) + (tu >> 1)) * 16 + 8 * (tu & 1);
    if constexpr (SCALED) {
        if (t0 < t1) {
            store(t0);
            if (t0 + 1 < t1) load(t0 + 1);
        }
        __syncthreads();
    }
    for (int t = t0; t < t1; ++t) {
        unsigned char* K = lds + (t & 1) * kStageBytes;
        unsigned char* V = K + kTileBytes;
        const float* ks = scales + (t & 1) * 2 * kTokens;
        const int there = p.len - t * kTokens;
        if constexpr (SCALED) {
            if (t + 1 < t1) {       // into the stage that every wave left at the last barrier
                store(t + 1);
                if (t + 2 < t1) load(t + 2);
            }
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();        // tile t is there, and every wave is done with the one before
            if (there < kTokens) {  // values behind the last token: no part of a sum, whatever they are
                for (int i = tid; i < (kTokens - there) * 16; i += 256)
                    *reinterpret_cast<u32x4_t*>(V + (there + i / 16) * kRowBytes + (i % 16) * 16) = u32x4_t{0, 0, 0, 0};
                __syncthreads();
            }
            if (t + 1 < t1) dma(t + 1);
        }
        if (rows_here) {
            f32x16_t s[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
            for (int kk = 0; kk < NK; ++kk)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(K + (kb * 32 + n) * kRowBytes + (((2 * kk + h) ^ (n & 15)) << 4));
#pragma unroll
                    for (int i = 0; i < NQ; ++i) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i][kk], s[kb], 0, 0, 0);
                }
            // s[kb][i]: token 32 kb + 8 (i / 4) + 4 h + i % 4
            if constexpr (SCALED) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f32x4_t f = *reinterpret_cast<const f32x4_t*>(ks + 32 * kb + 2 * i + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[kb][i + e] *= f[e];
                    }
            }
            if (there < kTokens) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * kb + 8 * (i >> 2) + 4 * h + (i & 3) >= there) s[kb][i] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
            mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
            // The reference moves only when a score passes it by more than kLazy: weights stay below 2^kLazy, and the sums
            // are rescaled in few tiles.
            const float mn = mx > m + kLazy ? mx : m;
            if (__any(mn != m)) {
                const float f = __builtin_amdgcn_exp2f(m - ref_of(mn));
                l *= f;
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[c][i] *= f;
                m = mn;
            }
            const float neg_ref = -ref_of(m);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int ks_ = 0; ks_ < 2; ++ks_) {
                    // the values first: they arrive while the weights are worked out
                    const unsigned char* vb = V + (kb * 32 + 16 * ks_) * kRowBytes + v_off;
                    u32x4_t vv[NT];
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        const int at = (c ^ tj) << 6;   // four chunks on, moved by the row's swizzle
                        const v4s_t lo = lds_read_tr16(vb + at), hi = lds_read_tr16(vb + at + 8 * kRowBytes);
                        vv[c] = u32x4_t{__builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 0, 1)),
                                        __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 2, 3)),
                                        __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 0, 1)),
                                        __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 2, 3))};
                    }
                    float w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_exp2f(fmaf(s[kb][8 * ks_ + j], scale, neg_ref));
                    if (there < kTokens) {     // (-infinity times a scale of 0)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (32 * kb + 16 * ks_ + 8 * (j >> 2) + 4 * h + (j & 3) >= there) w[j] = 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) l += w[j];
                    if constexpr (SCALED) {
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const f32x4_t f = *reinterpret_cast<const f32x4_t*>(ks + kTokens + 32 * kb + 16 * ks_ + 2 * j + 4 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[j + e] *= f[e];
                        }
                    }
                    u32x4_t pf[NP];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x[NP];
                        if constexpr (NP == 2) round_split(w[2 * j], w[2 * j + 1], x);
                        else split_bf16<NP>(w[2 * j], w[2 * j + 1], x);
#pragma unroll
                        for (int i = 0; i < NP; ++i) pf[i][j] = x[i];
                    }
#pragma unroll
                    for (int i = 0; i < NP; ++i)
#pragma unroll
                        for (int c = 0; c < NT; ++c)
                            o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vv[c]), __builtin_bit_cast(bf16x8_t, pf[i]), o[c], 0, 0, 0);
                }
        }
        if constexpr (SCALED) __syncthreads();
    }
    l += __shfl_xor(l, 32);
    if (t0 == t1) l = kNoTokens;
    // every thread has looked at other pages
    if (__syncthreads_or(bad)) {
        l = NAN;
        if (tid == 0) *p.status = RIFT_ERR_SHAPE;
    }
    if (r0 + n < p.rows) {
        float* dst = p.slots + (((size_t)kvh * p.parts + part) * p.rows + r0 + n) * RS;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)   // dimensions 32 c + 2 i + 4 h ..
                *reinterpret_cast<f32x4_t*>(dst + 32 * c + 2 * i + 4 * h) = f32x4_t{o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]};
        if (h == 0) {
            dst[HD] = m;
            dst[HD + 1] = l;
        }
    }
}

}  // namespace

// a part has two tiles at least; two workgroups a CU
int prefix_parts(int n_kv, int64_t rows, int len) {
    const int64_t wgs = n_kv * ((rows + kRows - 1) / kRows), tiles = (len + kTokens - 1) / kTokens;
    int64_t parts = 512 / wgs;
    if (parts > tiles / 2) parts = tiles / 2;
    return parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : (int)parts;
}

hipError_t launch_prefix(const riftkv_cache& c, bool bf16, PrefixParams p, hipStream_t st) {
    p.row_tiles = (p.rows + kRows - 1) / kRows;
    const size_t lds = 2 * kStageBytes + kScaleFloats * sizeof(float);
    auto run = [&](auto kernel) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)p.n_kv * p.row_tiles * p.parts)), dim3(256), lds, st, p);
        return hipGetLastError();
    };
    auto types = [&](auto dt) {
        if (c.head_dim == 128) return bf16 ? run(prefix_kernel<bf16_t, dt.value, 128>) : run(prefix_kernel<float, dt.value, 128>);
        return bf16 ? run(prefix_kernel<bf16_t, dt.value, 64>) : run(prefix_kernel<float, dt.value, 64>);
    };
    switch (c.dt) {
        case RIFTKV_BF16: return types(std::integral_constant<riftkv_dtype, RIFTKV_BF16>{});
        case RIFTKV_FP8: return types(std::integral_constant<riftkv_dtype, RIFTKV_FP8>{});
        case RIFTKV_INT8: return types(std::integral_constant<riftkv_dtype, RIFTKV_INT8>{});
        default: return hipErrorInvalidValue;
    }
}

}  // namespace rift
