// Rows of the paged key-value cache: rotary positions, rows into pages, rows out of
// them.  All three are bound by the bytes they move, so a lane moves 16 bytes of a row
// at a time, several of them in flight, and what belongs to a whole row (its sines,
// its place in the pages) is worked out once by the workgroup and passed in LDS.
#include <type_traits>

#include "kv_device.h"

namespace rift {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostThreads = (1ll << 32) - 1;   // of a launch along x: more rows take several launches

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ float load_f32(const void* p, size_t i) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(static_cast<const bf16_t*>(p)[i]);
    else return static_cast<const float*>(p)[i];
}
template <typename T>
__device__ __forceinline__ void store_f32(void* p, size_t i, float x) {
    if constexpr (sizeof(T) == 2) static_cast<bf16_t*>(p)[i] = round_bf16(x);
    else static_cast<float*>(p)[i] = x;
}

// 8 elements of a row, 16-byte aligned; read once, so past the caches (2 to 4% of every
// large call).
template <typename T>
struct Eight {
    u32x4_t w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const void* p, size_t i) {
    Eight<T> x;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j)
        x.w[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(static_cast<const T*>(p) + i) + j);
    return x;
}
template <typename T>
__device__ __forceinline__ void widen_eight(const Eight<T>& x, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) {
            f[2 * j] = bf16_lo(x.w[0][j]);
            f[2 * j + 1] = bf16_hi(x.w[0][j]);
        } else {
            f[j] = __uint_as_float(x.w[0][j]);
            f[4 + j] = __uint_as_float(x.w[1][j]);
        }
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return (uint32_t)round_bf16(a) | (uint32_t)round_bf16(b) << 16;
}
template <typename T>
__device__ __forceinline__ void store_eight(void* p, size_t i, const float (&f)[8]) {
    u32x4_t* q = reinterpret_cast<u32x4_t*>(static_cast<T*>(p) + i);
    if constexpr (sizeof(T) == 2) {
        *q = u32x4_t{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    } else {
        q[0] = u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
        q[1] = u32x4_t{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
    }
}

// ---------------------------------------------------------------- positions

// The angle in turns, reduced to [-1/2, 1/2] in float64: float32 holds it and its
// sine and cosine to their last bits however far the position is.  (The turns a position as one
// float64 are up to 1.3e-7 radians off at 2^31 positions of one radian, 1.2e-6 of 5.6 radians.)
__device__ __forceinline__ float2 rope_turn(int position, const RopeFreqs& freqs, int j, float magnitude) {
    const double p = position, whole = rint(p * freqs.hi[j]);
    const double t = fma(p, freqs.hi[j], -whole) + p * freqs.lo[j];
    float s, c;
    sincospif((float)(2.0 * t), &s, &c);
    return make_float2(c * magnitude, s * magnitude);
}

// Whose position turns pair j of a row: the row's one, or its axis' (22,204 rows of 40 heads, three axes, interleaved: 83 us, 455 MB
// at 5.5 TB/s; 100 rows of 64 heads 3.9 us).
struct OneAxis {
    __device__ __forceinline__ int position(const int* positions, int row, int) const { return positions[row]; }
};
struct SeveralAxes : RopeAxes {
    __device__ __forceinline__ int position(const int* positions, int row, int j) const { return positions[of[j] * stride + row]; }
};

// Any sizes, strides and alignment: a wave takes one head of one row.
template <typename T, typename Axes>
__global__ void __launch_bounds__(64)
rope_any_kernel(RopeRows q, RopeRows k, const int* __restrict__ positions, Axes axes, int head_dim, int rotary_dim, int interleaved,
                RopeFreqs freqs, float magnitude) {
    const int heads = q.n + k.n;
    const int row = blockIdx.x / heads, h = blockIdx.x - row * heads;
    const RopeRows& r = h < q.n ? q : k;
    const size_t hoff = (size_t)(h < q.n ? h : h - q.n) * head_dim;
    const size_t x0 = (size_t)row * r.ld_x + hoff, y0 = (size_t)row * r.ld_y + hoff;
    const int half = rotary_dim / 2;
    for (int j = threadIdx.x; j < half; j += 64) {
        const float2 cs = rope_turn(axes.position(positions, row, j), freqs, j, magnitude);
        const int i1 = interleaved ? 2 * j : j, i2 = interleaved ? 2 * j + 1 : j + half;
        const float2 y = rotate_pair(load_f32<T>(r.x, x0 + i1), load_f32<T>(r.x, x0 + i2), cs);
        store_f32<T>(r.y, y0 + i1, y.x);
        store_f32<T>(r.y, y0 + i2, y.y);
    }
    for (int j = rotary_dim + threadIdx.x; j < head_dim; j += 64) store_f32<T>(r.y, y0 + j, load_f32<T>(r.x, x0 + j));
}

// Eights of elements: a workgroup takes `per` heads of a row, or of several rows side by side whose threads have something to do
// at once.  (Rows that its threads take one after the other save launches of workgroups and lose more in the wait for the
// first sines: 16,384 rows of 40 heads, half layout, 57.5 us, in twos 60.6, in fours 63.6.)  A head's items are, in the half
// layout, rotary_dim / 16 pairs of eights, then the eights that are copied; interleaved,
// head_dim / 8 eights of four pairs each or copied.
template <typename T, bool INTERLEAVED, bool SIDE, typename Axes>
__global__ void __launch_bounds__(kThreads)
rope_kernel(RopeRows q, RopeRows k, const int* __restrict__ positions, int rows, Axes axes, int per, int threads_log2, int head_dim,
            int rotary_dim, RopeFreqs freqs, float magnitude) {
    __shared__ float2 turns_of[kThreads];
    static_assert(kThreads >= kMaxRotary / 2, "a row's pairs");
    const int threads = SIDE ? 1 << threads_log2 : kThreads, tid = SIDE ? threadIdx.x & (threads - 1) : threadIdx.x;
    const int nth = SIDE ? threadIdx.x >> threads_log2 : 0, row = SIDE ? blockIdx.x * (kThreads >> threads_log2) + nth : blockIdx.x;
    const int heads = q.n + k.n, h0 = blockIdx.y * per;
    const int half = rotary_dim / 2;
    float2* turns = turns_of + nth * half;
    const int turned = INTERLEAVED ? rotary_dim / 8 : rotary_dim / 16, items = turned + (head_dim - rotary_dim) / 8;
    // item v of head h; its values are asked for before they are needed, the first before
    // the sines
    int v = tid % items, h = h0 + tid / items;
    const int dv = threads % items, dh = threads / items, end = !SIDE || row < rows ? min(h0 + per, heads) : 0;
    Eight<T> xa, xb;
    void* y;
    size_t at;
    auto load = [&]() __attribute__((always_inline)) {
        const bool is_q = h < q.n;
        const void* x = is_q ? q.x : k.x;
        y = is_q ? q.y : k.y;
        const size_t hoff = (size_t)(is_q ? h : h - q.n) * head_dim;
        const size_t from = (size_t)row * (is_q ? q.ld_x : k.ld_x) + hoff;
        at = (size_t)row * (is_q ? q.ld_y : k.ld_y) + hoff;
        const int e = INTERLEAVED || v < turned ? 8 * v : rotary_dim + 8 * (v - turned);
        xa = load_eight<T>(x, from + e);
        if (!INTERLEAVED && v < turned) xb = load_eight<T>(x, from + half + e);
    };
    if (h < end) load();
    if (tid < half && (!SIDE || row < rows)) turns[tid] = rope_turn(axes.position(positions, row, tid), freqs, tid, magnitude);
    __syncthreads();
    while (h < end) {
        const int v0 = v;
        void* const y0 = y;
        const size_t at0 = at;
        float a[8], b[8];
        widen_eight<T>(xa, a);
        if constexpr (!INTERLEAVED) widen_eight<T>(xb, b);
        v += dv;
        h += dh;
        if (v >= items) {
            v -= items;
            ++h;
        }
        if (h < end) load();
        if (v0 >= turned) {
            store_eight<T>(y0, at0 + (INTERLEAVED ? 8 * v0 : rotary_dim + 8 * (v0 - turned)), a);
        } else if constexpr (INTERLEAVED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 o = rotate_pair(a[2 * j], a[2 * j + 1], turns[4 * v0 + j]);
                a[2 * j] = o.x;
                a[2 * j + 1] = o.y;
            }
            store_eight<T>(y0, at0 + 8 * v0, a);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 o = rotate_pair(a[j], b[j], turns[8 * v0 + j]);
                a[j] = o.x;
                b[j] = o.y;
            }
            store_eight<T>(y0, at0 + 8 * v0, a);
            store_eight<T>(y0, at0 + half + 8 * v0, b);
        }
    }
}

// A sequence a workgroup.  The angles are the prefill's, bit for bit.
__global__ void __launch_bounds__(64)
decode_prep_kernel(const int* __restrict__ positions, int64_t capacity, int hd, double base, float2* __restrict__ rope,
                   int* __restrict__ lens, int* __restrict__ rows) {
    const int i = blockIdx.x, pos = positions[i], half = hd / 2;
    if (threadIdx.x < half) rope[(size_t)i * half + threadIdx.x] = rope_entry(max(pos, 0), threadIdx.x, hd, base);
    if (threadIdx.x == 0) {
        lens[i] = pos < 0 ? 0 : pos >= capacity ? -1 : pos + 1;
        rows[i] = i;
    }
}

// ---------------------------------------------------------------- pages

// Index of (page, head 0, row in page) among the pages' rows; -1 where the row is
// skipped, or is out of range and the status set.
__device__ __forceinline__ int64_t page_row(const KvPlaces& at, int row, int n_pages, int shift, int n_kv) {
    const int seq = at.seq_ids ? at.seq_ids[row] : row, pos = at.positions[row];
    if (seq < 0 || pos < 0) return -1;
    int page = -1;
    if (seq < at.n_seq && (pos >> shift) < at.max_pages) page = at.table[(size_t)seq * at.max_pages + (pos >> shift)];
    if (page < 0 || page >= n_pages) {
        *at.status = RIFT_ERR_SHAPE;
        return -1;
    }
    return (((int64_t)page * n_kv) << shift) + (pos & ((1 << shift) - 1));
}

// Maximum over the G (8 or 16) lanes of a row.
template <int G>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, false));    // quad_perm 1, 0, 3, 2
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, false));    // quad_perm 2, 3, 0, 1
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, false));   // row_half_mirror
    if constexpr (G == 16) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, false));   // row_mirror
    return x;
}

// 8 values as codes: y = x up is exact, so that one addition rounds it to nearest even.
template <riftkv_dtype DT>
__device__ __forceinline__ uint2 codes_of(const float (&f)[8], float up) {
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float* x = f + 4 * j;
        if constexpr (DT == RIFTKV_FP8) {
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * up, x[1] * up, 0, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * up, x[3] * up, c, true);
            w[j] = (uint32_t)c;
        } else {
            constexpr float kOne = 12582912.f;   // 1.5 2^23: its last bit is worth 1
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(fmaf(x[e], up, kOne));   // the low byte is the code
            const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
            w[j] = lo | hi;
        }
    }
    return make_uint2(w[0], w[1]);
}
template <riftkv_dtype DT>
__device__ __forceinline__ void values_of(u32x2_t c, float scale, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t w = c[j];
        float* x = f + 4 * j;
        if constexpr (DT == RIFTKV_FP8) {
            const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
            x[0] = a[0] * scale;
            x[1] = a[1] * scale;
            x[2] = b[0] * scale;
            x[3] = b[1] * scale;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(w >> (8 * e)) * scale;
        }
    }
}

// A lane's 8 values of a row that G lanes hold, as codes, and the row's scale byte.
template <riftkv_dtype DT, int G>
__device__ __forceinline__ uint2 quantise_eight(const float (&f)[8], uint32_t& b) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    most = row_max<G>(most);
    const bool bad = most >= kNotFinite;
    b = bad ? 255u : scale_byte<DT>(most);
    const uint2 c = codes_of<DT>(f, __uint_as_float((254u - b) << 23));
    return bad ? make_uint2(0, 0) : c;
}

// Rows move as eights: HD / 8 lanes a row of a head, the rows of a tile under each other
// in a wave, which then writes (reads) several rows of a page in sequence.
struct MoveParams {
    unsigned char* pages[2];     // keys, values
    uint8_t* scales[2];
    void* rows_of[2];
    int64_t ld[2];
    int n_pages, shift, n_kv;
    int tile_log2, per;          // rows and heads of a workgroup
    int row0;                    // first row of the launch
    KvPlaces at;
};
constexpr int kTileRows = 16, kUnroll = 4;

template <typename T, riftkv_dtype DT, int HD, bool WRITE>
__global__ void __launch_bounds__(kThreads)
move_kernel(MoveParams p) {
    constexpr int G = HD / 8, E = DT == RIFTKV_F32 ? 4 : DT == RIFTKV_BF16 ? 2 : 1;
    constexpr bool SCALED = E == 1;
    __shared__ int64_t places[kTileRows];
    const int which = blockIdx.z, row0 = p.row0 + (blockIdx.x << p.tile_log2), h0 = blockIdx.y * p.per;
    const int n_heads = min(p.per, p.n_kv - h0);
    unsigned char* pages = p.pages[which];
    uint8_t* scales = p.scales[which];
    void* rows = p.rows_of[which];
    const int64_t ld = p.ld[which];
    const int items = n_heads << p.tile_log2;            // (head, row) pairs, the row running fastest
    const int lane = threadIdx.x % G, first = threadIdx.x / G;
    constexpr int STEP = kThreads / G;
    const int tile_mask = (1 << p.tile_log2) - 1;
    auto row_at = [&](int i) { return row0 + (i & tile_mask); };
    auto rows_index = [&](int i) { return (size_t)row_at(i) * ld + (size_t)(h0 + (i >> p.tile_log2)) * HD + 8 * lane; };
    Eight<T> x[kUnroll];
    auto load_rows = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * STEP;
            if (i < items && row_at(i) < p.at.rows) x[u] = load_eight<T>(rows, rows_index(i));
        }
    };
    if constexpr (WRITE) load_rows(first);
    if (threadIdx.x <= tile_mask) {
        const int row = row0 + threadIdx.x;
        places[threadIdx.x] = row < p.at.rows ? page_row(p.at, row, p.n_pages, p.shift, p.n_kv) : -1;
    }
    __syncthreads();
    for (int i0 = first; i0 < items; i0 += kUnroll * STEP) {
        if constexpr (WRITE) {
            if (i0 != first) load_rows(i0);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * STEP;
                const int64_t place = i < items ? places[i & tile_mask] : -1;
                if (place < 0) continue;      // all lanes of a row alike
                const size_t to = (size_t)place + ((size_t)(h0 + (i >> p.tile_log2)) << p.shift);
                float f[8];
                widen_eight<T>(x[u], f);
                if constexpr (DT == RIFTKV_F32) store_eight<float>(pages, to * HD + 8 * lane, f);
                else if constexpr (DT == RIFTKV_BF16) {
                    if constexpr (sizeof(T) == 2) reinterpret_cast<u32x4_t*>(pages)[(to * HD >> 3) + lane] = x[u].w[0];
                    else store_eight<bf16_t>(pages, to * HD + 8 * lane, f);
                } else {
                    uint32_t b;
                    reinterpret_cast<uint2*>(pages)[(to * HD >> 3) + lane] = quantise_eight<DT, G>(f, b);
                    if (lane == 0) scales[to] = (uint8_t)b;
                }
            }
        } else {
            Eight<std::conditional_t<DT == RIFTKV_F32, float, bf16_t>> y[kUnroll];
            u32x2_t c[kUnroll];
            uint32_t b[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * STEP;
                const int64_t place = i < items ? places[i & tile_mask] : -1;
                if (place < 0) continue;
                const size_t from = (size_t)place + ((size_t)(h0 + (i >> p.tile_log2)) << p.shift);
                if constexpr (SCALED) {
                    c[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(pages) + (from * HD >> 3) + lane);
                    b[u] = scales[from];
                } else {
                    y[u] = load_eight<std::conditional_t<DT == RIFTKV_F32, float, bf16_t>>(pages, from * HD + 8 * lane);
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * STEP;
                if (i >= items || places[i & tile_mask] < 0) continue;
                float f[8];
                if constexpr (SCALED) values_of<DT>(c[u], scale_of(b[u]), f);
                else widen_eight(y[u], f);
                if constexpr (DT == RIFTKV_BF16 && sizeof(T) == 2) reinterpret_cast<u32x4_t*>(rows)[rows_index(i) >> 3] = y[u].w[0];
                else store_eight<T>(rows, rows_index(i), f);
            }
        }
    }
}

// A decode step's q, k and v: lane j4 of the HD / 8 of a head owns its columns 4 j4 .. + 3 and
// their partners of the rotation, HD / 2 on, and finds the row's scale with its neighbours.
// One launch a layer for the sums and the pages (100 prompts of 131 to 643 rows, four
// layers, e4m3: 792 -> 776 us a step; one of 647, bf16: 437 -> 431).
constexpr int kQkvThreads = 64;

template <riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(kQkvThreads)
decode_qkv_kernel(const float* __restrict__ part, SkinnySplit sp, int d, const float2* __restrict__ rope, KvPlaces at,
                  bf16_t* __restrict__ q, riftkv_cache c, int shift) {
    constexpr int G = HD / 8, HALF = HD / 2;
    const int per_region = d / 8;                // (head, lane) pairs of q, of k, of v
    const long long idx = (long long)blockIdx.x * kQkvThreads + threadIdx.x;
    if (idx >= (long long)at.rows * 3 * per_region) return;      // whole heads: 3 d / 8 is a multiple of G
    const int m = (int)(idx / (3 * per_region)), rem = (int)(idx - (long long)m * (3 * per_region));
    const int region = rem / per_region, w = rem - region * per_region, head = w / G, j4 = w % G;
    const int col = region * d + head * HD + 4 * j4;
    int64_t place = -1;
    if (region > 0) place = page_row(at, m, c.n_pages, shift, c.n_kv_heads);
    f32x4_t cs0{}, cs1{};                        // (cos, sin) of columns j, j + 1 and j + 2, j + 3
    if (region < 2) {
        const f32x4_t* r = reinterpret_cast<const f32x4_t*>(rope + (size_t)m * HALF + 4 * j4);
        cs0 = r[0];
        cs1 = r[1];
    }
    const size_t N = 3 * (size_t)d, slot = (size_t)at.rows * N;
    const float* p0 = part + (size_t)m * N + col;
    const int S = sp.slots(col / 128);           // the product's tiles have 128 columns
    f32x4_t x1 = *reinterpret_cast<const f32x4_t*>(p0), x2 = *reinterpret_cast<const f32x4_t*>(p0 + HALF);
    for (int s = 1; s < S; ++s) {                // in slot order
        x1 += *reinterpret_cast<const f32x4_t*>(p0 + s * slot);
        x2 += *reinterpret_cast<const f32x4_t*>(p0 + s * slot + HALF);
    }
    if (region < 2) {
        const float cv[4] = {cs0[0], cs0[2], cs1[0], cs1[2]}, sv[4] = {cs0[1], cs0[3], cs1[1], cs1[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 y = rotate_pair(x1[e], x2[e], make_float2(cv[e], sv[e]));
            x1[e] = y.x;
            x2[e] = y.y;
        }
    }
    const uint2 lo = make_uint2(pack_bf16(x1[0], x1[1]), pack_bf16(x1[2], x1[3]));
    const uint2 hi = make_uint2(pack_bf16(x2[0], x2[1]), pack_bf16(x2[2], x2[3]));
    if (region == 0) {
        uint2* to = reinterpret_cast<uint2*>(q + (size_t)m * d + col);
        to[0] = lo;
        to[HALF / 4] = hi;
        return;
    }
    if (place < 0) return;
    const size_t to = (size_t)place + ((size_t)head << shift);
    unsigned char* pages = static_cast<unsigned char*>(region == 1 ? c.k : c.v);
    if constexpr (DT == RIFTKV_BF16) {
        uint2* row = reinterpret_cast<uint2*>(pages) + to * (HD / 4) + j4;
        row[0] = lo;
        row[HALF / 4] = hi;
    } else {
        const float f[8] = {bf16_lo(lo.x), bf16_hi(lo.x), bf16_lo(lo.y), bf16_hi(lo.y),
                            bf16_lo(hi.x), bf16_hi(hi.x), bf16_lo(hi.y), bf16_hi(hi.y)};
        uint32_t b;
        const uint2 codes = quantise_eight<DT, G>(f, b);
        uint32_t* row = reinterpret_cast<uint32_t*>(pages) + to * (HD / 4) + j4;
        row[0] = codes.x;
        row[HALF / 4] = codes.y;
        if (j4 == 0) (region == 1 ? c.k_scale : c.v_scale)[to] = (uint8_t)b;
    }
}

template <bool WRITE>
hipError_t launch_move(const riftkv_cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, bool bf16,
                       const KvPlaces& at, hipStream_t st) {
    MoveParams p{};
    p.pages[0] = static_cast<unsigned char*>(c.k);
    p.pages[1] = static_cast<unsigned char*>(c.v);
    p.scales[0] = c.k_scale;
    p.scales[1] = c.v_scale;
    p.rows_of[0] = const_cast<void*>(k);
    p.rows_of[1] = const_cast<void*>(v);
    p.ld[0] = ld_k;
    p.ld[1] = ld_v;
    p.n_pages = c.n_pages;
    p.shift = 31 - __builtin_clz(c.page_size);
    p.n_kv = c.n_kv_heads;
    p.at = at;
    // 8 rows of 16 heads a workgroup that writes, 16 of 8 one that reads (the scene's 32,987 rows of 32 heads
    // into e4m3 pages: 187 us and with 16 of 8 218; 120,001 rows of 8 heads out of int8 ones: 149 us
    // and with 8 of 8 160); fewer rows where that leaves CUs without work
    const int most = WRITE ? 16 : 8;
    p.per = c.n_kv_heads < most ? c.n_kv_heads : most;
    const unsigned splits = (c.n_kv_heads + p.per - 1) / p.per;
    p.tile_log2 = WRITE ? 3 : 4;
    while (p.tile_log2 > 0 && (int64_t)(at.rows >> p.tile_log2) * splits * 2 < 512) --p.tile_log2;
    const int64_t most_rows = (kMostThreads / kThreads) << p.tile_log2;
    auto launch = [&](auto kernel) {
        for (int64_t r = 0; r < at.rows; r += most_rows) {
            const int64_t n = at.rows - r < most_rows ? at.rows - r : most_rows;
            p.row0 = (int)r;
            hipLaunchKernelGGL(kernel, dim3((unsigned)((n + (1 << p.tile_log2) - 1) >> p.tile_log2), splits, 2), dim3(kThreads), 0, st, p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    auto heads = [&](auto t, auto dt) {
        using U = decltype(t);
        return c.head_dim == 128 ? launch(move_kernel<U, dt.value, 128, WRITE>) : launch(move_kernel<U, dt.value, 64, WRITE>);
    };
    auto types = [&](auto dt) {
        if constexpr (!(WRITE && dt.value == RIFTKV_F32))
            if (bf16) return heads(bf16_t{}, dt);
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

template <typename Axes>
hipError_t launch_rope(const RopeRows& q, const RopeRows& k, bool bf16, const int* positions, const Axes& axes, int rows, int head_dim,
                       int rotary_dim, bool interleaved, const RopeFreqs& freqs, float magnitude, hipStream_t st) {
    const int heads = q.n + k.n;
    // rows from r on
    auto from = [&](const RopeRows& x, int64_t r) {
        const int64_t e = bf16 ? 2 : 4;
        if (x.n == 0) return x;
        return RopeRows{static_cast<const unsigned char*>(x.x) + r * x.ld_x * e, static_cast<unsigned char*>(x.y) + r * x.ld_y * e,
                        x.ld_x, x.ld_y, x.n};
    };
    // launch(rows, first row), as often as the rows need
    auto in_pieces = [&](int64_t most, auto launch) {
        for (int64_t r = 0; r < rows; r += most) {
            launch((unsigned)(rows - r < most ? rows - r : most), r);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    auto aligned = [&](const RopeRows& r) {   // 16-byte eights
        const int64_t per = bf16 ? 8 : 4;
        return r.n == 0 || (((reinterpret_cast<uintptr_t>(r.x) | reinterpret_cast<uintptr_t>(r.y)) & 15) == 0 &&
                            r.ld_x % per == 0 && r.ld_y % per == 0);
    };
    if (head_dim % 8 != 0 || rotary_dim % 16 != 0 || !aligned(q) || !aligned(k)) {
        auto run = [&](auto kernel) {
            return in_pieces(kMostThreads / 64 / heads, [&](unsigned n, int64_t r) {
                hipLaunchKernelGGL(kernel, dim3(n * (unsigned)heads), dim3(64), 0, st, from(q, r), from(k, r), positions + r, axes,
                                   head_dim, rotary_dim, interleaved ? 1 : 0, freqs, magnitude);
            });
        };
        return bf16 ? run(rope_any_kernel<bf16_t, Axes>) : run(rope_any_kernel<float, Axes>);
    }
    // all heads of a row a workgroup, so that its sines are worked out once, or fewer where that
    // leaves CUs without work (32 rows of 40 heads: 2.6 us, with 512 workgroups 3.4)
    int per = heads;
    while (per > 4 && (int64_t)rows * ((heads + per - 1) / per) < 256) per = (per + 1) / 2;
    // Threads of a row: as few as take each no more than one item and one pair's sines, while workgroups stay for all CUs
    // (a workgroup a row and several side by side, us: 14,898 rows of 6 heads of 64, bf16 15.5 and 7.6, f32 19.5 and 12.7; 60,000
    // of 2 49 and 16; 20,000 of 10 of 128 28.2 and 23.7; 2,100 of 8 of 64 3.8 and 3.5; 1,000 of them 2.9 and 3.0).
    const int items = heads * ((interleaved ? rotary_dim / 8 : rotary_dim / 16) + (head_dim - rotary_dim) / 8);
    const int needed = items > rotary_dim / 2 ? items : rotary_dim / 2;
    int threads_log2 = 8;
    static_assert(kThreads == 1 << 8, "the threads of a workgroup");
    while (threads_log2 > 3 && 1 << (threads_log2 - 1) >= needed && rows >> (9 - threads_log2) >= 512) --threads_log2;
    const int side = kThreads >> threads_log2;
    auto run = [&](auto kernel) {
        return in_pieces(kMostThreads / kThreads * side, [&](unsigned n, int64_t r) {
            hipLaunchKernelGGL(kernel, dim3((n + side - 1) / side, (unsigned)((heads + per - 1) / per)), dim3(kThreads), 0, st, from(q, r),
                               from(k, r), positions + r, (int)n, axes, per, threads_log2, head_dim, rotary_dim, freqs, magnitude);
        });
    };
    auto types = [&](auto wide) {
        constexpr bool SIDE = decltype(wide)::value;
        if (bf16) return interleaved ? run(rope_kernel<bf16_t, true, SIDE, Axes>) : run(rope_kernel<bf16_t, false, SIDE, Axes>);
        return interleaved ? run(rope_kernel<float, true, SIDE, Axes>) : run(rope_kernel<float, false, SIDE, Axes>);
    };
    return side > 1 ? types(std::true_type{}) : types(std::false_type{});
}

}  // namespace

hipError_t launch_kv_rope(const RopeRows& q, const RopeRows& k, bool bf16, const int* positions, int rows, int head_dim,
                          int rotary_dim, bool interleaved, const RopeFreqs& freqs, float magnitude, hipStream_t st) {
    return launch_rope(q, k, bf16, positions, OneAxis{}, rows, head_dim, rotary_dim, interleaved, freqs, magnitude, st);
}

hipError_t launch_kv_rope_axes(const RopeRows& q, const RopeRows& k, bool bf16, const int* positions, const RopeAxes& axes, int rows,
                               int head_dim, int rotary_dim, bool interleaved, const RopeFreqs& freqs, float magnitude,
                               hipStream_t st) {
    return launch_rope(q, k, bf16, positions, SeveralAxes{axes}, rows, head_dim, rotary_dim, interleaved, freqs, magnitude, st);
}

hipError_t launch_kv_decode_prep(const int* positions, int n_seq, int64_t capacity, int hd, float rope_base, float2* rope,
                                 int* lens, int* rows, hipStream_t st) {
    hipLaunchKernelGGL(decode_prep_kernel, dim3((unsigned)n_seq), dim3(64), 0, st, positions, capacity, hd, (double)rope_base,
                       rope, lens, rows);
    return hipGetLastError();
}

hipError_t launch_kv_decode_qkv(const riftkv_cache& c, const float* part, SkinnySplit sp, int d, const float2* rope,
                                const KvPlaces& at, uint16_t* q, hipStream_t st) {
    const long long n = (long long)at.rows * 3 * (d / 8);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((n + kQkvThreads - 1) / kQkvThreads)), dim3(kQkvThreads), 0, st, part, sp, d,
                           rope, at, q, c, 31 - __builtin_clz(c.page_size));
        return hipGetLastError();
    };
    auto heads = [&](auto dt) {
        return c.head_dim == 128 ? launch(decode_qkv_kernel<dt.value, 128>) : launch(decode_qkv_kernel<dt.value, 64>);
    };
    switch (c.dt) {
        case RIFTKV_BF16: return heads(std::integral_constant<riftkv_dtype, RIFTKV_BF16>{});
        case RIFTKV_FP8: return heads(std::integral_constant<riftkv_dtype, RIFTKV_FP8>{});
        case RIFTKV_INT8: return heads(std::integral_constant<riftkv_dtype, RIFTKV_INT8>{});
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_kv_write(const riftkv_cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, bool bf16,
                           const KvPlaces& at, hipStream_t st) {
    return launch_move<true>(c, k, ld_k, v, ld_v, bf16, at, st);
}

hipError_t launch_kv_read(const riftkv_cache& c, void* k, int64_t ld_k, void* v, int64_t ld_v, bool bf16,
                          const KvPlaces& at, hipStream_t st) {
    return launch_move<false>(c, k, ld_k, v, ld_v, bf16, at, st);
}

}  // namespace rift
