// One query token of every sequence over ranges of paged keys and values: the pages of a list
// (riftkv_attention_pages), or a prefix that all sequences share and then their own (riftkv_attention_shared).
//
//   ranges_kernel   a workgroup takes a part of the tokens of up to 16 query rows of one key head; its waves
//                   share the part's tiles and join in LDS.  Where the tokens are one part, it joins them with the
//                   prefix' parts, if there is one, and writes the output.
//   parts_kernel    otherwise: the sum of the parts.
// A shared prefix comes first, by prefix_kernel (kv_prefix.hip) or, for few rows and float32 pages, by ranges_kernel.
#include <type_traits>

#include "kv_ranges.h"

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
    const float* front;      // parts of a prefix, [key head][front_parts][n_seq * group][HD + 4]
    int n_kv, group, q_tiles, rows, parts, n_pages, shift, front_parts, item0;
    int64_t front_rows;      // n_seq * group
    float scale_log2;
};

// A page among an item's tokens, and how many of its tokens count: 0 too where there is none.
struct Entry {
    int page, count;
    bool bad;
};

// Tokens of a sequence's own pages; `bad` where their number is out of range.
struct OwnPages {
    const int* table;
    const int* lens;
    int max_pages;
    __device__ __forceinline__ int length(int seq, int shift, bool& bad) const {
        const int len = lens[seq];
        bad = len < 0 || (int64_t)len > ((int64_t)max_pages << shift);
        return bad ? 0 : len;
    }
    // page `place` of a sequence of len tokens
    __device__ __forceinline__ Entry at(const RangeParams& p, int seq, int place, int len) const {
        Entry e{0, 0, place >= max_pages};
        if (place < 0 || e.bad) return e;
        e.count = (int)max((int64_t)0, min((int64_t)len - ((int64_t)place << p.shift), (int64_t)1 << p.shift));
        if (e.count == 0) return e;
        e.page = table[(size_t)seq * max_pages + place];
        e.bad = (unsigned)e.page >= (unsigned)p.n_pages;
        if (e.bad) e.page = 0;
        return e;
    }
};

// What a workgroup's item is made of: `n` entries, and `tiles` of 32 tokens of them, one after the other.
struct Item {
    int len, n, tiles;
};

// The listed pages, in the list's order.
struct ListedPages {
    OwnPages own;
    const int* lists;        // [n_seq][n_kv][top]
    int top;
    static constexpr bool kFront = false;
    __device__ __forceinline__ const int* list(const RangeParams& p, int seq, int kvh) const { return lists + ((size_t)seq * p.n_kv + kvh) * top; }
    __device__ __forceinline__ Item item(const RangeParams& p, int seq, int kvh, int lane, bool& bad) const {
        Item it;
        it.len = own.length(seq, p.shift, bad);
        it.n = top;
        // A sequence of fewer pages: up to the last entry with tokens, so that the waves share those.
        if ((int64_t)it.len <= ((int64_t)(top - 1) << p.shift)) {
            const int* l = list(p, seq, kvh);
            it.n = 0;
            for (int e0 = 0; e0 < top; e0 += 64) {
                const int place = e0 + lane < top ? l[e0 + lane] : -1;
                const unsigned long long mask = __ballot(place >= 0 && (place >= own.max_pages || ((int64_t)place << p.shift) < it.len));
                if (mask != 0) it.n = e0 + 64 - __clzll(mask);
            }
        }
        it.tiles = ((it.n << p.shift) + kTile - 1) / kTile;
        return it;
    }
    __device__ __forceinline__ Entry entry(const RangeParams& p, const Item& it, int seq, int kvh, int e) const {
        return own.at(p, seq, e < it.n ? list(p, seq, kvh)[e] : -1, it.len);
    }
};

// A sequence's own pages.
struct WholePages {
    OwnPages own;
    static constexpr bool kFront = false;
    __device__ __forceinline__ Item item(const RangeParams& p, int seq, int, int, bool& bad) const {
        Item it;
        it.len = own.length(seq, p.shift, bad);
        it.n = it.len > 0 ? ((it.len - 1) >> p.shift) + 1 : 0;
        it.tiles = (it.len + kTile - 1) / kTile;
        return it;
    }
    __device__ __forceinline__ Entry entry(const RangeParams& p, const Item& it, int seq, int, int e) const {
        return own.at(p, seq, e < it.n ? e : -1, it.len);
    }
};

// A prefix' pages; its items are 16 rows of a key head, of whatever sequences, and write their parts for the others to join.
struct PrefixPages {
    OwnPages own;            // the prefix as sequence 0
    int len;
    static constexpr bool kFront = true;
    __device__ __forceinline__ Item item(const RangeParams& p, int, int, int, bool& bad) const {
        bad = false;
        return Item{len, own.max_pages, (len + kTile - 1) / kTile};
    }
    __device__ __forceinline__ Entry entry(const RangeParams& p, const Item& it, int, int, int e) const {
        return own.at(p, 0, e < it.n ? e : -1, it.len);
    }
};

template <typename T, riftkv_dtype DT, int HD, typename Where>
__global__ void __launch_bounds__(64 * kWaves, 2)
ranges_kernel(RangeParams p, Where where) {
    constexpr int RS = HD + 4;
    extern __shared__ __align__(16) float records[];   // [kWaves][rows][RS]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // blocks: item by item, each with its parts
    const int part = blockIdx.x % p.parts, item = blockIdx.x / p.parts + p.item0;
    int seq, kvh, r0, rows;                    // sequence, key head, first of its group's rows (of all rows) and how many
    if constexpr (Where::kFront) {
        const int tiles = (int)((p.front_rows + 15) / 16);
        seq = 0;
        kvh = item / tiles;
        r0 = 16 * (item - kvh * tiles);
        rows = (int)min(p.front_rows - r0, (int64_t)16);
    } else {
        const int HQ = p.n_kv * p.q_tiles;
        seq = item / HQ;
        const int hq = item - seq * HQ;
        kvh = hq / p.q_tiles;
        r0 = 16 * (hq - kvh * p.q_tiles);
        rows = min(16, p.group - r0);
    }

    bool bad;
    const Item it = where.item(p, seq, kvh, lane, bad);
    const int share = part * kWaves + wave, shares = p.parts * kWaves;
    int tile = (int)((int64_t)it.tiles * share / shares);
    int left = __builtin_amdgcn_readfirstlane((int)((int64_t)it.tiles * (share + 1) / shares) - tile);

    TilePass<T, DT, HD> pass(lane);
    {
        int of = seq, r = r0 + min(pass.n, rows - 1);
        if constexpr (Where::kFront) {
            of = r / p.group;
            r -= of * p.group;
        }
        pass.start(static_cast<const T*>(p.q) + (size_t)of * p.ld_q + (size_t)(kvh * p.group + r) * HD, pass.n < rows);
    }
    bool any = false;
    if (left > 0) {
        // 64 entries at a time, one a lane: what a tile needs of them is read from its lane, without a load to wait for
        // behind those of keys and values.
        const int in_mask = (1 << p.shift) - 1;
        int first = (tile * kTile) >> p.shift;
        Entry mine;
        auto look = [&]() __attribute__((always_inline)) {
            mine = where.entry(p, it, seq, kvh, first + lane);
            bad |= __any(mine.bad);
        };
        auto find = [&](int t, Half (&half)[2]) __attribute__((always_inline)) {
            if (((t * kTile + 16) >> p.shift) - first >= 64) {
                first = (t * kTile) >> p.shift;
                look();
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int v = t * kTile + 16 * h, in_page = v & in_mask;
                const int of = __builtin_amdgcn_readfirstlane((v >> p.shift) - first);
                const int page = __builtin_amdgcn_readlane(mine.page, of), count = __builtin_amdgcn_readlane(mine.count, of);
                half[h].row = ((((size_t)page * p.n_kv) + kvh) << p.shift) + in_page;
                half[h].n = max(0, min(count - in_page, 16));
            }
        };
        look();
        Half cur[2], nxt[2];
        find(tile, cur);
        pass.load_k(p.pages, cur);
        pass.load_v(p.pages, cur);
        for (; left > 0; --left) {
            ++tile;
            if (left > 1) find(tile, nxt);
            else
                for (int h = 0; h < 2; ++h) nxt[h] = Half{cur[h].row, 0};
            const bool full = cur[0].n + cur[1].n > 0;
            if (full) {
                any = true;
                pass.scores(p.scale_log2);
            }
            pass.load_k(p.pages, nxt);
            if (full) {
                pass.softmax(cur[0].n, cur[1].n);
                pass.values();
            }
            pass.load_v(p.pages, nxt);
            for (int h = 0; h < 2; ++h) cur[h] = nxt[h];
        }
    }
    float sum = any ? quad_sum(pass.l) : kNoTokens;
    if (bad) {
        sum = NAN;
        if (lane == 0) *p.status = RIFT_ERR_SHAPE;
    }
    const int record = p.rows * RS;
    pass.put(records + wave * record, rows, sum);
    __syncthreads();
    for (int i = tid; i < rows * (HD / 4); i += 64 * kWaves) {
        const int row = i / (HD / 4), col = 4 * (i % (HD / 4));
        const float* src = records + row * RS;
        float mx = -INFINITY, L = kNoTokens;
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, src[w * record + HD]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(src[w * record + HD] - ref_of(mx));
            L = fmaf(f, src[w * record + HD + 1], L);
            acc += f * *reinterpret_cast<const f32x4_t*>(src + w * record + col);
        }
        if constexpr (Where::kFront) {
            float* slot = p.slots + (((size_t)kvh * p.parts + part) * p.front_rows + r0 + row) * RS;
            *reinterpret_cast<f32x4_t*>(slot + col) = acc;
            if (col == 0) *reinterpret_cast<float2*>(slot + HD) = make_float2(mx, L);
        } else if (p.parts == 1) {
            if (p.front_parts > 0) {
                const size_t next = (size_t)p.front_rows * RS;
                const float* src = p.front + (size_t)kvh * p.front_parts * next + ((size_t)seq * p.group + r0 + row) * RS;
                constexpr int U = 4;   // parts in flight
                for (int k0 = 0; k0 < p.front_parts; k0 += U) {
                    float2 ml[U];
                    f32x4_t x[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {   // past the last: its values, not used
                        const float* at = src + min(k0 + u, p.front_parts - 1) * next;
                        ml[u] = *reinterpret_cast<const float2*>(at + HD);
                        x[u] = *reinterpret_cast<const f32x4_t*>(at + col);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (k0 + u >= p.front_parts) continue;
                        const float mn = fmaxf(mx, ml[u].x);
                        const float f = __builtin_amdgcn_exp2f(mx - ref_of(mn)), fk = __builtin_amdgcn_exp2f(ml[u].x - ref_of(mn));
                        acc = acc * f + x[u] * fk;
                        L = fmaf(fk, ml[u].y, L * f);
                        mx = mn;
                    }
                }
            }
            acc *= weight_of(L);
            store_four<T>(p.out, (size_t)seq * p.ld_out + (size_t)(kvh * p.group + r0 + row) * HD + col, acc[0], acc[1], acc[2], acc[3]);
        } else {
            float* slot = p.slots + (((size_t)item * p.parts + part) * p.rows + row) * RS;
            *reinterpret_cast<f32x4_t*>(slot + col) = acc;
            if (col == 0) *reinterpret_cast<float2*>(slot + HD) = make_float2(mx, L);
        }
    }
}

// A query head a wave: lane k finds the weight of part k, then the parts' values are added up, PG of them side by side, as
// many loads in flight as there are parts.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
parts_kernel(RangeParams p, int64_t n) {
    constexpr int RS = HD + 4, CV = HD / 4, PG = 64 / CV, U = 8;
    const int lane = threadIdx.x & 63;
    const int64_t of = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // sequence and head
    if (of >= n) return;
    const int heads = p.n_kv * p.group;
    const int64_t seq = of / heads;
    const int head = (int)(of - seq * heads), kvh = head / p.group, r = head - kvh * p.group, qt = r / 16;
    const int pg = lane / CV, col = 4 * (lane % CV);
    struct Set {                          // parts a fixed number of floats apart
        const float* at;
        size_t next;
        int n;
    };
    const Set sets[2] = {
        {p.slots + (((seq * p.n_kv + kvh) * p.q_tiles + qt) * p.parts * p.rows + (r - 16 * qt)) * RS, (size_t)p.rows * RS, p.parts},
        {p.front + ((int64_t)kvh * p.front_parts * p.front_rows + seq * p.group + r) * RS, (size_t)p.front_rows * RS, p.front_parts}};
    float2 ml[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        ml[i] = lane < sets[i].n ? *reinterpret_cast<const float2*>(sets[i].at + lane * sets[i].next + HD) : make_float2(-INFINITY, kNoTokens);
    f32x4_t x[U];
    auto load = [&](const Set& set, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const f32x4_t*>(set.at + min(k0 + u * PG + pg, set.n - 1) * set.next + col);
    };
    load(sets[0], 0);
    float mx = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = __builtin_amdgcn_exp2f(ml[i].x - ref_of(mx));
    float l = f[0] * ml[0].y + f[1] * ml[1].y;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        for (int k0 = 0; k0 < sets[i].n; k0 += U * PG) {
            if (i + k0 > 0) load(sets[i], k0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = k0 + u * PG + pg;
                const float fk = __shfl(f[i], k & 63);
                if (k < sets[i].n) acc += fk * x[u];
            }
        }
#pragma unroll
    for (int d = CV; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
    acc *= weight_of(l);
    if (pg == 0) store_four<T>(p.out, (size_t)seq * p.ld_out + (size_t)head * HD + col, acc[0], acc[1], acc[2], acc[3]);
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

constexpr int64_t kMostWorkgroups = ((1ll << 32) - 1) / 256;   // of a launch; more take several

template <typename Where>
hipError_t launch_ranges(const riftkv_cache& c, const KvAttention& a, RangeParams p, int64_t items, const Where& where, hipStream_t st) {
    const size_t lds = (size_t)kWaves * p.rows * (c.head_dim + 4) * sizeof(float);
    auto run = [&](auto t, auto dt, auto hd) {
        using T = decltype(t);
        const int64_t most = kMostWorkgroups / p.parts;
        for (int64_t i = 0; i < items; i += most) {
            p.item0 = (int)i;
            hipLaunchKernelGGL((ranges_kernel<T, dt.value, hd.value, Where>), dim3((unsigned)((items - i < most ? items - i : most) * p.parts)),
                               dim3(64 * kWaves), lds, st, p, where);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (Where::kFront || p.parts == 1) return hipSuccess;
        const int64_t n = (int64_t)a.n_seq * a.n_heads;
        hipLaunchKernelGGL((parts_kernel<T, hd.value>), dim3((unsigned)((n + 3) / 4)), dim3(256), 0, st, p, n);
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

constexpr int kMostSplit = 512;   // items times parts, where items are split

// Parts of an item of at most `tiles` tiles: a split costs a launch, which pays for long items that are few.
int parts_of(int64_t items, int64_t tiles) {
    if (items > 128 || tiles < 24) return 1;
    const int64_t parts = kMostSplit / items < tiles / 4 ? kMostSplit / items : tiles / 4;
    return parts > kMaxParts ? kMaxParts : (int)parts;
}

size_t part_bytes(const riftkv_cache& c) { return (size_t)(c.head_dim + 4) * sizeof(float); }

// How the call of a prefix is made: its parts and those of the sequences' own tokens.
struct SharedPlan {
    bool by_rows;            // prefix_kernel
    int64_t rows, items;     // rows of a key head; items of the sequences' own tokens
    int front_parts, parts;
    SharedPlan(const riftkv_cache& c, int n_heads, int64_t n_seq, int prefix_len, int64_t max_pages) {
        const int group = n_heads / c.n_kv_heads;
        rows = n_seq * group;
        items = n_seq * c.n_kv_heads * ((group + 15) / 16);
        by_rows = c.dt != RIFTKV_F32 && rows > 32;
        front_parts = 0;
        if (prefix_len > 0 && rows > 0) {
            const int64_t tiles = (prefix_len + kTile - 1) / kTile;
            if (by_rows) front_parts = prefix_parts(c.n_kv_heads, rows, prefix_len);
            else {
                const int64_t wgs = c.n_kv_heads * ((rows + 15) / 16);
                const int64_t n = kMostSplit / wgs < tiles / 4 ? kMostSplit / wgs : tiles / 4;
                front_parts = n < 1 ? 1 : n > kMaxParts ? kMaxParts : (int)n;
            }
        }
        parts = items > 0 ? parts_of(items, (max_pages * c.page_size + kTile - 1) / kTile) : 1;
    }
};

}  // namespace

size_t kv_shared_workspace(const riftkv_cache& c, int n_heads, int64_t n_seq, int prefix_len, int64_t) {
    // The prefix' parts: rows of 128 for each of 512 workgroups, or one part of every row; fewer where rows and their parts
    // are few.  Then those of the sequences' own tokens.
    const int64_t group = n_heads / c.n_kv_heads, rows = n_seq * n_heads;
    const int64_t split = rows * kMaxParts < 512 * 128 ? rows * kMaxParts : 512 * 128;
    return ((prefix_len > 0 ? split + rows : 0) + kMostSplit * (group < 16 ? group : 16)) * part_bytes(c);
}

size_t kv_listed_workspace(const riftkv_cache& c, int n_heads, int64_t, int) {
    const int group = n_heads / c.n_kv_heads;
    return (size_t)kMostSplit * (group < 16 ? group : 16) * part_bytes(c);
}

hipError_t launch_kv_attention_shared(const riftkv_cache& c, const KvAttention& a, const int* prefix_table, int prefix_len, hipStream_t st) {
    const SharedPlan plan(c, a.n_heads, a.n_seq, prefix_len, a.max_pages);
    RangeParams p = params_of(c, a);
    p.front_rows = plan.rows;
    if (plan.front_parts > 0) {
        float* front = static_cast<float*>(a.workspace);
        hipError_t e;
        if (plan.by_rows) {
            const PrefixParams f{a.q, a.ld_q, p.pages, prefix_table, a.status, front, prefix_len, p.n_kv, p.n_pages, p.shift, p.group,
                                 (int)plan.rows, 0, plan.front_parts, p.scale_log2};
            e = launch_prefix(c, a.bf16, f, st);
        } else {
            RangeParams f = p;
            f.slots = front;
            f.parts = plan.front_parts;
            f.rows = plan.rows < 16 ? (int)plan.rows : 16;
            const int pages = (int)(((int64_t)prefix_len + c.page_size - 1) / c.page_size);
            e = launch_ranges(c, a, f, p.n_kv * ((plan.rows + 15) / 16), PrefixPages{OwnPages{prefix_table, nullptr, pages}, prefix_len}, st);
        }
        if (e != hipSuccess) return e;
        p.front = front;
        p.front_parts = plan.front_parts;
        p.slots = front + (size_t)p.n_kv * plan.front_parts * plan.rows * (c.head_dim + 4);
    }
    p.parts = plan.parts;
    return launch_ranges(c, a, p, plan.items, WholePages{OwnPages{a.table, a.lens, a.max_pages}}, st);
}

hipError_t launch_kv_attention_pages(const riftkv_cache& c, const KvAttention& a, const int* lists, int top, hipStream_t st) {
    RangeParams p = params_of(c, a);
    const int64_t items = (int64_t)a.n_seq * p.n_kv * p.q_tiles;
    p.parts = parts_of(items, ((int64_t)top * c.page_size + kTile - 1) / kTile);
    return launch_ranges(c, a, p, items, ListedPages{OwnPages{a.table, a.lens, a.max_pages}, lists, top}, st);
}

}  // namespace rift
