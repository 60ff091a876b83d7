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

template <typename T, riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1)
prefix_kernel(PrefixParams p) {
    constexpr int B = DT == RIFTKV_BF16 ? 2 : 1;
    constexpr bool SCALED = B == 1;
    constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = 3;
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

    // this lane's query, 16 kk + 8 h .. of it
    bf16x8_t qf[NQ][NK];
    {
        const int r = min(r0 + n, p.rows - 1), seq = r / p.group;
        const T* q = static_cast<const T*>(p.q) + (size_t)seq * p.ld_q + (size_t)(kvh * p.group + r - seq * p.group) * HD + 8 * h;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            if constexpr (NQ == 1) qf[0][kk] = *reinterpret_cast<const bf16x8_t*>(q + 16 * kk);
            else {
                u32x4_t x[NQ];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t w[NQ];
                    split_bf16<NQ>(q[16 * kk + 2 * e], q[16 * kk + 2 * e + 1], w);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) x[i][e] = w[i];
                }
#pragma unroll
                for (int i = 0; i < NQ; ++i) qf[i][kk] = __builtin_bit_cast(bf16x8_t, x[i]);
            }
        }
    }
    f32x16_t o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    bool bad = false;

    // A thread's share of a tile: chunk `chunk` of rows row, row + STEP, ..  All lanes of a wave are in rows of one page.
    const int row = tid / CHUNKS, chunk = tid % CHUNKS;
    u32x4_t kr[LOADS], vr[LOADS];
    uint32_t sr = 0;
    auto load = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int token = min(t * kTokens + row + i * STEP, p.len - 1);
            const int page = __builtin_amdgcn_readfirstlane(p.table[token >> p.shift]);
            const bool there = (unsigned)page < (unsigned)p.n_pages;
            bad |= !there;
            const size_t at = (((((size_t)(there ? page : 0) * p.n_kv) + kvh) << p.shift) + (token & ((1 << p.shift) - 1))) * (HD * B) + 16 * chunk;
            kr[i] = *reinterpret_cast<const u32x4_t*>(p.pages.k + at);
            vr[i] = *reinterpret_cast<const u32x4_t*>(p.pages.v + at);
        }
        if constexpr (SCALED) {
            if (tid < 2 * kTokens) {
                const int token = min(t * kTokens + (tid & (kTokens - 1)), p.len - 1);
                const int page = p.table[token >> p.shift];
                const size_t at = ((((size_t)((unsigned)page < (unsigned)p.n_pages ? page : 0) * p.n_kv) + kvh) << p.shift) + (token & ((1 << p.shift) - 1));
                sr = (tid < kTokens ? p.pages.ks : p.pages.vs)[at];
            }
        }
    };
    auto store = [&](int t) __attribute__((always_inline)) {
        unsigned char* K = lds + (t & 1) * kStageBytes;
        unsigned char* V = K + kTileBytes;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = row + i * STEP;
            const u32x4_t v = t * kTokens + r < p.len ? vr[i] : u32x4_t{0, 0, 0, 0};   // behind the last token: no part of a sum
            if constexpr (!SCALED) {
                *reinterpret_cast<u32x4_t*>(K + r * kRowBytes + ((chunk ^ (r & 15)) << 4)) = kr[i];
                *reinterpret_cast<u32x4_t*>(V + r * kRowBytes + ((chunk ^ (4 * (r & 3))) << 4)) = v;
            } else {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int c = 2 * chunk + y;
                    *reinterpret_cast<u32x4_t*>(K + r * kRowBytes + ((c ^ (r & 15)) << 4)) =
                        u32x4_t{widen<DT, false>(kr[i][2 * y]), widen<DT, true>(kr[i][2 * y]), widen<DT, false>(kr[i][2 * y + 1]), widen<DT, true>(kr[i][2 * y + 1])};
                    *reinterpret_cast<u32x4_t*>(V + r * kRowBytes + ((c ^ (4 * (r & 3))) << 4)) =
                        u32x4_t{widen<DT, false>(v[2 * y]), widen<DT, true>(v[2 * y]), widen<DT, false>(v[2 * y + 1]), widen<DT, true>(v[2 * y + 1])};
                }
            }
        }
        if constexpr (SCALED)
            if (tid < 2 * kTokens) scales[(t & 1) * 2 * kTokens + tid] = scale_of(sr);
    };

    const int tg = lane >> 4, tj = (lane >> 2) & 3, tu = lane & 3;
    const int v_off = (4 * (tg >> 1) + tj) * kRowBytes + (2 * (tg & 1) + (tu >> 1)) * 16 + 8 * (tu & 1);
    if (t0 < t1) {
        load(t0);
        store(t0);
        if (t0 + 1 < t1) load(t0 + 1);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const unsigned char* K = lds + (t & 1) * kStageBytes;
        const unsigned char* V = K + kTileBytes;
        const float* ks = scales + (t & 1) * 2 * kTokens;
        if (t + 1 < t1) {       // into the stage that every wave left at the last barrier
            store(t + 1);
            if (t + 2 < t1) load(t + 2);
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
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] *= p.scale_log2;
            const int there = p.len - t * kTokens;
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
            mx = fmaxf(mx, __shfl_xor(mx, 32));
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
            const float ref = ref_of(m);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int ks_ = 0; ks_ < 2; ++ks_) {
                    float w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        w[j] = __builtin_amdgcn_exp2f(s[kb][8 * ks_ + j] - ref);
                        l += w[j];
                    }
                    if constexpr (SCALED) {
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const f32x4_t f = *reinterpret_cast<const f32x4_t*>(ks + kTokens + 32 * kb + 16 * ks_ + 2 * j + 4 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[j + e] *= f[e];
                        }
                        if (there < kTokens) {   // (a last row's scale may be infinite)
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (32 * kb + 16 * ks_ + 8 * (j >> 2) + 4 * h + (j & 3) >= there) w[j] = 0.f;
                        }
                    }
                    u32x4_t pf[NP];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x[NP];
                        split_bf16<NP>(w[2 * j], w[2 * j + 1], x);
#pragma unroll
                        for (int i = 0; i < NP; ++i) pf[i][j] = x[i];
                    }
                    const unsigned char* vb = V + (kb * 32 + 16 * ks_) * kRowBytes + v_off;
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        const int at = (c ^ tj) << 6;   // four chunks on, moved by the row's swizzle
                        const v4s_t lo = lds_read_tr16(vb + at), hi = lds_read_tr16(vb + at + 8 * kRowBytes);
                        const u32x4_t vv = {__builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 0, 1)),
                                            __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 2, 3)),
                                            __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 0, 1)),
                                            __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 2, 3))};
#pragma unroll
                        for (int i = 0; i < NP; ++i)
                            o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vv), __builtin_bit_cast(bf16x8_t, pf[i]), o[c], 0, 0, 0);
                    }
                }
        }
        __syncthreads();
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
