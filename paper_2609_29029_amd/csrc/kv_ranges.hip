// One query token of every sequence over ranges of paged keys and values: the pages of a list
// (riftkv_attention_pages), or a prefix that all sequences share and then their own (riftkv_attention_shared).
//
//   ranges_kernel   a workgroup takes a part of the tokens of up to 16 query heads of one key head; its waves
//                   share the part's tiles and join in LDS.  Where the tokens are one part, the
//                   output is written here.
//   parts_kernel    otherwise: the sum of the parts.
#include <type_traits>

#include "kv_tile.h"

namespace rift {

namespace {

constexpr int kWaves = 4;

struct RangeParams {
    const void* q;
    void* out;
    int64_t ld_q, ld_out;
    TilePages pages;
    int* status;
    float* slots;            // [sequence][head group][parts][rows][HD + 4]: weighted values, largest score, sum
    int n_kv, group, q_tiles, rows, parts, n_pages, shift;
    float scale_log2;
};

// Tokens of the pages' table of a sequence, or what is wrong with their number.
struct OwnPages {
    const int* table;
    const int* lens;
    int max_pages;
    __device__ __forceinline__ bool length(int seq, int shift, int& len) const {
        len = lens[seq];
        const bool good = len >= 0 && (int64_t)len <= ((int64_t)max_pages << shift);
        if (!good) len = 0;
        return good;
    }
};

// Where the 16 tokens of half h of a tile are; false: at a page that is not there.
__device__ __forceinline__ bool half_at(const RangeParams& p, int page, int in_page, int kvh, int n, Half& out) {
    const bool there = (unsigned)page < (unsigned)p.n_pages;
    out.n = n;
    out.row = ((((size_t)(there ? page : 0) * p.n_kv) + kvh) << p.shift) + in_page;
    return there || n == 0;
}

// The tokens of the listed pages, in the list's order.
struct ListedPages {
    OwnPages own;
    const int* lists;        // [n_seq][n_kv][top]
    int top;
    struct At {
        const int *list, *table;
        int len, kvh;
    };
    __device__ __forceinline__ bool begin(const RangeParams& p, int seq, int kvh, At& at) const {
        at.list = lists + ((size_t)seq * p.n_kv + kvh) * top;
        at.table = own.table + (size_t)seq * own.max_pages;
        at.kvh = kvh;
        return own.length(seq, p.shift, at.len);
    }
    __device__ __forceinline__ int64_t tiles(const RangeParams& p, const At&) const { return (((int64_t)top << p.shift) + kTile - 1) / kTile; }
    __device__ __forceinline__ bool find(const RangeParams& p, const At& at, int64_t tile, Half (&half)[2]) const {
        bool good = true;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t v = tile * kTile + 16 * h;
            const int64_t entry = v >> p.shift;
            const int in_page = (int)v & ((1 << p.shift) - 1);
            const int place = entry < top ? at.list[entry] : -1;
            const bool known = place >= 0 && place < own.max_pages;
            const int64_t n = known ? (int64_t)at.len - ((int64_t)place << p.shift) - in_page : 0;
            const int page = known && n > 0 ? at.table[place] : 0;
            good &= place < own.max_pages;
            good &= half_at(p, page, in_page, at.kvh, (int)max((int64_t)0, min(n, (int64_t)16)), half[h]);
        }
        return good;
    }
};

// The prefix, then the sequence's own pages.
struct SharedPages {
    OwnPages own;
    const int* prefix;
    int prefix_len;
    struct At {
        const int* table;
        int len, kvh;
    };
    __device__ __forceinline__ bool begin(const RangeParams& p, int seq, int kvh, At& at) const {
        at.table = own.table + (size_t)seq * own.max_pages;
        at.kvh = kvh;
        return own.length(seq, p.shift, at.len);
    }
    __device__ __forceinline__ int64_t tiles(const RangeParams&, const At& at) const {
        return (int64_t)(prefix_len + kTile - 1) / kTile + (at.len + kTile - 1) / kTile;
    }
    __device__ __forceinline__ bool find(const RangeParams& p, const At& at, int64_t tile, Half (&half)[2]) const {
        const int before = (prefix_len + kTile - 1) / kTile;
        const bool in_prefix = tile < before;
        const int* table = in_prefix ? prefix : at.table;
        const int len = in_prefix ? prefix_len : at.len;
        const int t0 = (int)(in_prefix ? tile : tile - before) * kTile;
        bool good = true;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = t0 + 16 * h, n = max(0, min(len - t, 16));
            good &= half_at(p, n > 0 ? table[t >> p.shift] : 0, t & ((1 << p.shift) - 1), at.kvh, n, half[h]);
        }
        return good;
    }
};

template <typename T, riftkv_dtype DT, int HD, typename Where>
__global__ void __launch_bounds__(64 * kWaves, 2)
ranges_kernel(RangeParams p, Where where) {
    constexpr int RS = HD + 4;
    __shared__ __align__(16) float records[kWaves * 16 * RS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int HQ = p.n_kv * p.q_tiles;
    const int part = blockIdx.x % p.parts, item = blockIdx.x / p.parts;
    const int seq = item / HQ, hq = item - seq * HQ;
    const int kvh = hq / p.q_tiles, qt = hq - kvh * p.q_tiles;
    const int h0 = kvh * p.group + 16 * qt, rows = min(16, p.group - 16 * qt);   // first head, heads

    typename Where::At at;
    bool bad = !where.begin(p, seq, kvh, at);
    const int64_t all = where.tiles(p, at);
    const int64_t share = part * kWaves + wave, shares = (int64_t)p.parts * kWaves;
    int64_t tile = all * share / shares;
    int left = (int)(all * (share + 1) / shares - tile);

    TilePass<T, DT, HD> pass(lane);
    pass.start(static_cast<const T*>(p.q) + (size_t)seq * p.ld_q + (size_t)(h0 + min(pass.n, rows - 1)) * HD, pass.n < rows);
    bool any = false;
    if (left > 0) {
        Half cur[2], nxt[2];
        bad |= !where.find(p, at, tile, cur);
        pass.load_k(p.pages, cur);
        pass.load_v(p.pages, cur);
        for (; left > 0; --left) {
            ++tile;
            if (left > 1) bad |= !where.find(p, at, tile, nxt);
            else
                for (int h = 0; h < 2; ++h) nxt[h] = Half{cur[h].row, 0};
            pass.scores(p.scale_log2);
            pass.load_k(p.pages, nxt);
            any |= cur[0].n + cur[1].n > 0;
            pass.softmax(cur[0].n, cur[1].n);
            pass.values();
            pass.load_v(p.pages, nxt);
            for (int h = 0; h < 2; ++h) cur[h] = nxt[h];
        }
    }
    float sum = any ? quad_sum(pass.l) : kNoTokens;
    if (bad) {
        sum = NAN;
        if (lane == 0) *p.status = RIFT_ERR_SHAPE;
    }
    pass.put(records + wave * 16 * RS, rows, sum);
    __syncthreads();
    for (int i = tid; i < rows * (HD / 4); i += 64 * kWaves) {
        const int row = i / (HD / 4), col = 4 * (i % (HD / 4));
        const float* src = records + row * RS;
        float mx = -INFINITY, L = kNoTokens;
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, src[w * 16 * RS + HD]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(src[w * 16 * RS + HD] - ref_of(mx));
            L = fmaf(f, src[w * 16 * RS + HD + 1], L);
            acc += f * *reinterpret_cast<const f32x4_t*>(src + w * 16 * RS + col);
        }
        if (p.parts == 1) {
            acc *= weight_of(L);
            store_four<T>(p.out, (size_t)seq * p.ld_out + (size_t)(h0 + row) * HD + col, acc[0], acc[1], acc[2], acc[3]);
        } else {
            float* slot = p.slots + ((size_t)blockIdx.x * p.rows + row) * RS;
            *reinterpret_cast<f32x4_t*>(slot + col) = acc;
            if (col == 0) {
                slot[HD] = mx;
                slot[HD + 1] = L;
            }
        }
    }
}

// A query head's four columns a thread.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
parts_kernel(RangeParams p, int64_t n) {
    constexpr int RS = HD + 4, CV = HD / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t of = i / CV;            // sequence and head
    const int col = 4 * (int)(i % CV);
    const int heads = p.n_kv * p.group;
    const int64_t seq = of / heads;
    const int head = (int)(of - seq * heads), kvh = head / p.group, r = head - kvh * p.group, qt = r / 16;
    const float* src = p.slots + (((seq * p.n_kv + kvh) * p.q_tiles + qt) * p.parts * p.rows + (r - 16 * qt)) * RS;
    float m = -INFINITY, l = kNoTokens;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < p.parts; ++k, src += (size_t)p.rows * RS) {
        const float mk = src[HD], mn = fmaxf(m, mk);
        const float f = __builtin_amdgcn_exp2f(m - ref_of(mn)), fk = __builtin_amdgcn_exp2f(mk - ref_of(mn));
        acc = acc * f + *reinterpret_cast<const f32x4_t*>(src + col) * fk;
        l = fmaf(fk, src[HD + 1], l * f);
        m = mn;
    }
    acc *= weight_of(l);
    store_four<T>(p.out, (size_t)seq * p.ld_out + (size_t)head * HD + col, acc[0], acc[1], acc[2], acc[3]);
}

RangeParams params_of(const riftkv_cache& c, const KvAttention& a) {
    RangeParams p{};
    p.q = a.q;
    p.out = a.out;
    p.ld_q = a.ld_q;
    p.ld_out = a.ld_out;
    p.pages = TilePages{static_cast<const unsigned char*>(c.k), static_cast<const unsigned char*>(c.v), c.k_scale, c.v_scale};
    p.status = a.status;
    p.slots = static_cast<float*>(a.workspace);
    p.n_kv = c.n_kv_heads;
    p.group = a.n_heads / c.n_kv_heads;
    p.q_tiles = (p.group + 15) / 16;
    p.rows = p.group < 16 ? p.group : 16;
    p.n_pages = c.n_pages;
    p.shift = 31 - __builtin_clz(c.page_size);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    return p;
}

template <typename Where>
hipError_t launch_ranges(const riftkv_cache& c, const KvAttention& a, const RangeParams& p, const Where& where, hipStream_t st) {
    const int64_t items = (int64_t)a.n_seq * p.n_kv * p.q_tiles;
    auto run = [&](auto t, auto dt, auto hd) {
        using T = decltype(t);
        hipLaunchKernelGGL((ranges_kernel<T, dt.value, hd.value, Where>), dim3((unsigned)(items * p.parts)), dim3(64 * kWaves), 0, st, p, where);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.parts == 1) return e;
        const int64_t n = (int64_t)a.n_seq * a.n_heads * (hd.value / 4);
        hipLaunchKernelGGL((parts_kernel<T, hd.value>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p, n);
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

}  // namespace

size_t kv_shared_workspace(const riftkv_cache&, int, int64_t, int, int64_t) { return 256; }

size_t kv_listed_workspace(const riftkv_cache&, int, int64_t, int) { return 256; }

hipError_t launch_kv_attention_shared(const riftkv_cache& c, const KvAttention& a, const int* prefix_table, int prefix_len, hipStream_t st) {
    RangeParams p = params_of(c, a);
    p.parts = 1;
    return launch_ranges(c, a, p, SharedPages{OwnPages{a.table, a.lens, a.max_pages}, prefix_table, prefix_len}, st);
}

hipError_t launch_kv_attention_pages(const riftkv_cache& c, const KvAttention& a, const int* lists, int top, hipStream_t st) {
    RangeParams p = params_of(c, a);
    p.parts = 1;
    return launch_ranges(c, a, p, ListedPages{OwnPages{a.table, a.lens, a.max_pages}, lists, top}, st);
}

}  // namespace rift
