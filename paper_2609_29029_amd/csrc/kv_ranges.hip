// One query token of every sequence over ranges of paged keys and values: the pages of a list
// (riftkv_attention_pages), or a prefix that all sequences share and then their own (riftkv_attention_shared).
//
//   listed_kernel   a workgroup takes a part of the tokens of up to 16 query heads of one key head; its waves share the
//                   part's tiles and join in LDS.  Where the tokens are one part, the output is written here.
//   shared_kernel   the same for a sequence's own tokens, and beside them, in the same launch, workgroups for the prefix:
//                   prefix_body (kv_prefix.h), or where there is little to do, and for float32 pages, as above, 16 rows of a
//                   key head whatever their sequences.  A short prefix is walked by every sequence itself.
//   parts_kernel    the sum of the parts.
//
// The items' tokens are bound by their bytes (64 sequences, 64 heads in groups of 8, 128 e4m3 pages of 32 a key head: 504 MB in 84 us,
// 6.0 TB/s), where they are few by the latency of a tile's loads, 1.2 us, and of a second launch, 4.
#include <type_traits>

#include "kv_prefix.h"

namespace rift {

namespace {

constexpr int kWaves = 4;
constexpr int kMaxParts = 64;   // of an item's tokens: a lane each where they are joined

struct RangeParams {
    const void* q;
    void* out;
    int64_t ld_q, ld_out;
    TilePages pages;
    int* status;
    float* slots;            // [sequence][head group][parts][rows][HD + 4]: weighted values, largest score, sum
    float* front;            // parts of a prefix, [key head][front_parts][front_rows][HD + 4]
    int64_t front_rows;      // n_seq * group
    int n_kv, group, q_tiles, rows, parts, n_pages, shift, front_parts;
    int front_wgs;           // workgroups for the prefix, the first of the launch
    int item0;               // first item of the others
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

// Where 16 tokens are: in an entry, at a row of its page, and how many of them there can be.
struct Place {
    int entry, in_page, most;
};

// The listed pages, in the list's order.
struct ListedPages {
    OwnPages own;
    const int* lists;        // [n_seq][n_kv][top]
    int top;
    __device__ __forceinline__ const int* list(const RangeParams& p, int seq, int kvh) const { return lists + ((size_t)seq * p.n_kv + kvh) * top; }
    __device__ __forceinline__ Item item(const RangeParams& p, int seq, int kvh, bool, int lane, bool& bad) const {
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
    __device__ __forceinline__ Entry entry(const RangeParams& p, const Item& it, int seq, int kvh, bool, int e) const {
        return own.at(p, seq, e < it.n ? list(p, seq, kvh)[e] : -1, it.len);
    }
    __device__ __forceinline__ Place place(const RangeParams& p, bool, int tile, int half) const {
        const int v = tile * kTile + 16 * half;
        return Place{v >> p.shift, v & ((1 << p.shift) - 1), 16};
    }
};

// The prefix (front items); a sequence's own pages, after the first `walked` tokens of the prefix: all or none.
struct SharedPages {
    OwnPages own, prefix;    // (the prefix as sequence 0)
    int prefix_len, walked;
    __device__ __forceinline__ int walked_pages(int shift) const { return walked > 0 ? prefix.max_pages : 0; }
    __device__ __forceinline__ Item item(const RangeParams& p, int seq, int, bool front, int, bool& bad) const {
        bad = false;
        if (front) return Item{prefix_len, prefix.max_pages, (prefix_len + kTile - 1) / kTile};
        const int len = own.length(seq, p.shift, bad);
        return Item{len, walked_pages(p.shift) + (len > 0 ? ((len - 1) >> p.shift) + 1 : 0), (walked + kTile - 1) / kTile + (len + kTile - 1) / kTile};
    }
    __device__ __forceinline__ Entry entry(const RangeParams& p, const Item& it, int seq, int, bool front, int e) const {
        const int before = walked_pages(p.shift);
        if (front || e < before) return prefix.at(p, 0, e < (front ? it.n : before) ? e : -1, prefix_len);
        return own.at(p, seq, e < it.n ? e - before : -1, it.len);
    }
    __device__ __forceinline__ Place place(const RangeParams& p, bool front, int tile, int half) const {
        const int before = front ? 0 : (walked + kTile - 1) / kTile, mask = (1 << p.shift) - 1;
        if (tile < before) {
            const int v = tile * kTile + 16 * half;
            return v < walked ? Place{v >> p.shift, v & mask, 16} : Place{0, 0, 0};
        }
        const int v = (tile - before) * kTile + 16 * half;
        return Place{(front ? 0 : walked_pages(p.shift)) + (v >> p.shift), v & mask, 16};
    }
};

// Workgroup `block` of the items' or, front, of the prefix'.
template <typename T, riftkv_dtype DT, int HD, typename Where>
__device__ __forceinline__ void ranges_body(const RangeParams& p, const Where& where, bool front, int block, float* records) {
    constexpr int RS = HD + 4;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // item by item, each with its parts
    const int n_parts = front ? p.front_parts : p.parts;
    const int part = block % n_parts, item = block / n_parts + (front ? 0 : p.item0);
    int seq, kvh, r0, rows;                    // sequence, key head, first of its group's rows (of all rows) and how many
    if (front) {
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
    const Item it = where.item(p, seq, kvh, front, lane, bad);
    const int share = part * kWaves + wave, shares = n_parts * kWaves;
    int tile = (int)((int64_t)it.tiles * share / shares);
    int left = __builtin_amdgcn_readfirstlane((int)((int64_t)it.tiles * (share + 1) / shares) - tile);

    TilePass<T, DT, HD> pass(lane);
    {
        int of = seq, r = r0 + min(pass.n, rows - 1);
        if (front) {
            of = r / p.group;
            r -= of * p.group;
        }
        pass.start(static_cast<const T*>(p.q) + (size_t)of * p.ld_q + (size_t)(kvh * p.group + r) * HD, pass.n < rows);
    }
    bool any = false;
    if (left > 0) {
        // 64 entries at a time, one a lane: what a tile needs of them is read from its lane, without a load to wait for
        // behind those of keys and values.
        int first = where.place(p, front, tile, 0).entry;
        Entry mine;
        auto look = [&]() __attribute__((always_inline)) {
            mine = where.entry(p, it, seq, kvh, front, first + lane);
            bad |= __any(mine.bad);
        };
        auto find = [&](int t, Half (&half)[2]) __attribute__((always_inline)) {
            const Place at[2] = {where.place(p, front, t, 0), where.place(p, front, t, 1)};
            if (max(at[0].entry, at[1].entry) - first >= 64) {
                first = at[0].entry;
                look();
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int of = __builtin_amdgcn_readfirstlane(max(at[h].entry - first, 0));
                const int page = __builtin_amdgcn_readlane(mine.page, of), count = __builtin_amdgcn_readlane(mine.count, of);
                half[h].row = ((((size_t)page * p.n_kv) + kvh) << p.shift) + at[h].in_page;
                half[h].n = max(0, min(count - at[h].in_page, at[h].most));
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
    const int record = (p.front_wgs > 0 ? 16 : p.rows) * RS;
    pass.put(records + wave * record, rows, sum);
    __syncthreads();
    const bool direct = !front && p.parts == 1 && p.front_parts == 0;
    float* slots = front ? p.front + (((size_t)kvh * n_parts + part) * p.front_rows + r0) * RS
                         : p.slots + ((size_t)item * n_parts + part) * p.rows * RS;
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
        if (direct) {
            acc *= weight_of(L);
            store_four<T>(p.out, (size_t)seq * p.ld_out + (size_t)(kvh * p.group + r0 + row) * HD + col, acc[0], acc[1], acc[2], acc[3]);
        } else {
            *reinterpret_cast<f32x4_t*>(slots + row * RS + col) = acc;
            if (col == 0) *reinterpret_cast<float2*>(slots + row * RS + HD) = make_float2(mx, L);
        }
    }
}

template <typename T, riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(64 * kWaves, 2)
listed_kernel(RangeParams p, ListedPages where) {
    extern __shared__ __align__(16) unsigned char lds[];
    ranges_body<T, DT, HD>(p, where, false, blockIdx.x, reinterpret_cast<float*>(lds));
}

// BY_ROWS: the prefix by prefix_body.
template <typename T, riftkv_dtype DT, int HD, bool BY_ROWS>
__global__ void __launch_bounds__(64 * kWaves, BY_ROWS && sizeof(T) == 4 ? 1 : 2)
shared_kernel(RangeParams p, SharedPages where, PrefixParams f) {
    extern __shared__ __align__(16) unsigned char lds[];
    const bool front = (int)blockIdx.x < p.front_wgs;
    if constexpr (BY_ROWS)
        if (front) {
            prefix_body<T, DT, HD>(f, blockIdx.x, lds);
            return;
        }
    ranges_body<T, DT, HD>(p, where, !BY_ROWS && front, front ? blockIdx.x : blockIdx.x - p.front_wgs, reinterpret_cast<float*>(lds));
}

// A query head a wave: lane k finds the weight of part k, then the parts' values are added up, PG of them side by side, as
// many loads in flight as there are parts.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
parts_kernel(RangeParams p, int64_t first, int64_t n) {
    constexpr int RS = HD + 4, CV = HD / 4, PG = 64 / CV, U = 8;
    const int lane = threadIdx.x & 63;
    const int64_t of = first + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // sequence and head
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
        for (int u = 0; u < U; ++u)
            if (k0 + u * PG < set.n) x[u] = *reinterpret_cast<const f32x4_t*>(set.at + min(k0 + u * PG + pg, set.n - 1) * set.next + col);
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
    p.parts = 1;
    p.n_kv = c.n_kv_heads;
    p.group = a.n_heads / c.n_kv_heads;
    p.q_tiles = (p.group + 15) / 16;
    p.rows = p.group < 16 ? p.group : 16;
    p.n_pages = c.n_pages;
    p.shift = 31 - __builtin_clz(c.page_size);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    return p;
}

constexpr int64_t kMostWorkgroups = ((1ll << 32) - 1) / (64 * kWaves);   // of a launch; more take several
constexpr int kMostSplit = 512;                                        // items times parts, where items are split
constexpr int kMostPrefixWgs = 384;

// run(row type, page type, head_dim)
template <typename Run>
hipError_t by_types(const riftkv_cache& c, bool bf16, Run run) {
    auto heads = [&](auto t, auto dt) {
        if (c.head_dim == 128) return run(t, dt, std::integral_constant<int, 128>{});
        return run(t, dt, std::integral_constant<int, 64>{});
    };
    auto types = [&](auto dt) {
        if constexpr (dt.value != RIFTKV_F32)
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

// launch(workgroups) for the items, as often as they need; the first time with the prefix' workgroups.
template <typename Launch>
hipError_t by_items(RangeParams& p, int64_t items, Launch launch) {
    const int64_t most = (kMostWorkgroups - p.front_wgs) / p.parts;
    for (int64_t i = 0; i < items; i += most) {
        p.item0 = (int)i;
        const hipError_t e = launch((unsigned)((items - i < most ? items - i : most) * p.parts + p.front_wgs));
        if (e != hipSuccess) return e;
        p.front_wgs = 0;
    }
    return hipSuccess;
}

template <typename T, int HD>
hipError_t join_parts(const KvAttention& a, const RangeParams& p, hipStream_t st) {
    const int64_t n = (int64_t)a.n_seq * a.n_heads, most = kMostWorkgroups * 4;   // a wave each
    for (int64_t i = 0; i < n; i += most) {
        const int64_t m = n - i < most ? n - i : most;
        hipLaunchKernelGGL((parts_kernel<T, HD>), dim3((unsigned)((m + 3) / 4)), dim3(256), 0, st, p, i, n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Parts of an item of at most `tiles` tiles, four of them at least a part.  In us, with 1, 4, 8 and 16 parts (bf16, 128 dimensions, groups
// of 4): 8 items of 64 tiles 19.9 12.0 9.8 8.9; 32 of 64 21.9 13.3 11.2 11.6; 64 of 32 13.5 11.3 11.6 14.1; 128 of 64 30.2 27.4 29.6
// 35.3, e4m3 128 of 128 47.9 28.3 29.7 32.2; one of 512 156 47 26.6 17.1, with 64 parts 12.5; whole: 160 of 32 16.1 (21.2 with 4), 512 of
// 128 87 (99), 8 of 8 5.3 (7.5), 8 of 16 6.6 (7.1).  Eight waves a workgroup instead of four: within 10% either way.
int parts_of(int64_t items, int64_t tiles) {
    const int64_t parts = kMostSplit / items < tiles / 4 ? kMostSplit / items : tiles / 4;
    return parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : (int)parts;
}

// The same where a split alone costs a launch to join the parts, which pays for long items that are few.  In us, whole and in parts:
// 96 items of 20 tiles 12.2 and 13.2, e4m3 of 64 dimensions 7.9 and 8.7; 32 of 20 9.5 and 8.8, e4m3 10.6 and 8.6; 16 of 12 6.9 and 8.1.  Float32
// pages, whose products take longer, of 128 (and 64) dimensions: 64 of 10 14.3 and 14.5 (9.5 and 11.0), of 12 14.9 and 12.4 (9.4 and
// 9.7), of 20 24.3 and 18.3 (12.3 and 11.2); 96 of 12 17.4 and 18.2 (9.0 and 11.1), of 20 26.8 and 19.7 (13.9 and 12.2); 160 of 16 23.9 and 24.9,
// of 20 29.4 and 27.9 (16.1 and 16.7), of 30 41.8 and 35.3 (23.7 and 21.7); in two parts 176 of 20 29.4 and 33.5, 192 of up to 31 40.9 and
// 44.4, 256 of 64 91.9 and 97.0.
int parts_alone(riftkv_dtype dt, int64_t items, int64_t tiles) {
    const bool split = dt == RIFTKV_F32 ? items <= kMostSplit / 3 && tiles >= (items <= 64 ? 12 : 20) : items <= 128 && tiles >= (items <= 64 ? 20 : 24);
    return split ? parts_of(items, tiles) : 1;
}

size_t part_bytes(const riftkv_cache& c) { return (size_t)(c.head_dim + 4) * sizeof(float); }

// How the call of a prefix is made.
struct SharedPlan {
    int64_t rows, items;     // rows of a key head; items of the sequences' own tokens
    bool walk, by_rows;      // the prefix by every sequence itself; by prefix_body
    int front_parts, front_wgs, row_tiles, parts;
    SharedPlan(const riftkv_cache& c, int n_heads, bool bf16, int64_t n_seq, int prefix_len, int64_t max_pages) {
        const int group = n_heads / c.n_kv_heads;
        const int64_t own = (max_pages * c.page_size + kTile - 1) / kTile;
        rows = n_seq * group;
        items = n_seq * c.n_kv_heads * ((group + 15) / 16);
        walk = prefix_len <= kWalked;
        // 16 rows at a time keep more CUs busy and wait less; 128 read less and use larger products, which pays from so many (16
        // rows, token) pairs on.  In us, 16 and 128 rows at a time (bf16 queries, 128 dimensions, 8 key heads, 16 or 64 sequences in
        // groups of 4): bf16 pages, 48,000 pairs 14.6 and 13.8 or 20.3 and 17.5, 64,000 17.1 and 14.3 or 20.6 and 17.9, 128,000 17.5 and
        // 19.7 or 23.5 and 21.3, 384,000 26.7 and 25.2 or 29.5 and 28.2, 4.2 million 194 and 92; 8 bits, 512,000 26.7 and 35.3 or 28.9 and
        // 34.5, 768,000 34.1 and 43.2 or 34.5 and 37.3, 1.0 million 41.5 and 40.0 (int8 48.2 and 41.3), 2.0 million 68.5 and 56.4, 4.2
        // million 138 and 102 (158 and 98).  Float32 queries: bf16 pages alike; 8 bits, two times three terms of widened rows, 29
        // and 45, 57 and 66, 170 and 180.
        const int64_t pairs = (int64_t)c.n_kv_heads * ((rows + 15) / 16) * prefix_len;
        by_rows = !walk && rows_kernel(c.dt, bf16) && pairs > (c.dt == RIFTKV_BF16 ? 56 : 900) * 1000;
        front_parts = front_wgs = 0;
        row_tiles = (int)((rows + kRows - 1) / kRows);
        parts = parts_alone(c.dt, items, own);
        if (walk) return;
        parts = parts_of(items, own);
        const int64_t wgs = c.n_kv_heads * (by_rows ? row_tiles : (rows + 15) / 16);
        if (by_rows) {
            const int64_t tiles = (prefix_len + kTokens - 1) / kTokens;
            // A workgroup a CU, so that the sequences' own tokens have the other half of it; more where a tile has few bytes or
            // is widened (64 sequences after 32,768 tokens, groups of 4, with 256 and 384: bf16 91.0 and 91.7 us, 8,192 tokens in
            // groups of 1 38.1 and 40.3; e4m3 108 and 106, int8 111 and 105, e4m3 of 64 dimensions 79 and 71).
            int64_t n = (c.dt == RIFTKV_BF16 && c.head_dim == 128 ? 256 : kMostPrefixWgs) / wgs;
            if (n > tiles / 2) n = tiles / 2;
            front_parts = n < 1 ? 1 : n > kMaxParts ? kMaxParts : (int)n;
        } else front_parts = parts_of(wgs, (prefix_len + kTile - 1) / kTile);
        front_wgs = (int)(wgs * front_parts);
    }
    static constexpr bool rows_kernel(riftkv_dtype dt, bool bf16) { return dt == RIFTKV_BF16 || (dt != RIFTKV_F32 && bf16); }
    // Tokens of a prefix that every sequence walks itself, walked / in workgroups of its own: 100 sequences of 96 to 608 tokens
    // and 32 heads 92 / 100 us (65 tokens), 101 / 103 (200), 109 / 103 (300); 64 of 1 to 300 in groups of 4 11.7 / 18.6 (65),
    // 13.8 / 18.9 (200), 15.2 / 19.0 (300); 8 of them 10.1 / 10.6 (256), 13.0 / 11.0 (500).
    static constexpr int kWalked = 256;
};

}  // namespace

size_t kv_shared_workspace(const riftkv_cache& c, int n_heads, int64_t n_seq, int prefix_len, int64_t) {
    // The prefix' parts: 128 rows for each of its workgroups, or one part of every row; fewer where rows and their parts are
    // few.  Those of the sequences' own tokens: one of every row (groups of more than 16 may leave some unused), or as many
    // as where they are split.
    const int64_t group = n_heads / c.n_kv_heads, rows = n_seq * n_heads;
    const int64_t split = rows * kMaxParts < kMostPrefixWgs * kRows ? rows * kMaxParts : kMostPrefixWgs * kRows;
    return ((prefix_len > 0 ? split + 3 * rows : 0) + kMostSplit * (group < 16 ? group : 16)) * part_bytes(c);
}

size_t kv_listed_workspace(const riftkv_cache& c, int n_heads, int64_t, int) {
    const int group = n_heads / c.n_kv_heads;
    return (size_t)kMostSplit * (group < 16 ? group : 16) * part_bytes(c);
}

hipError_t launch_kv_attention_shared(const riftkv_cache& c, const KvAttention& a, const int* prefix_table, int prefix_len, hipStream_t st) {
    const SharedPlan plan(c, a.n_heads, a.bf16, a.n_seq, prefix_len, a.max_pages);
    RangeParams p = params_of(c, a);
    p.parts = plan.parts;
    p.front_rows = plan.rows;
    p.front_parts = plan.front_parts;
    p.front_wgs = plan.front_wgs;
    p.front = static_cast<float*>(a.workspace);
    p.slots = p.front + (size_t)p.n_kv * plan.front_parts * plan.rows * (c.head_dim + 4);
    const int pages = (int)(((int64_t)prefix_len + c.page_size - 1) / c.page_size);
    const SharedPages where{OwnPages{a.table, a.lens, a.max_pages}, OwnPages{prefix_table, nullptr, pages}, prefix_len, plan.walk ? prefix_len : 0};
    const PrefixParams f{a.q, a.ld_q, p.pages, prefix_table, a.status, p.front, prefix_len, p.n_kv, p.n_pages, p.shift, p.group,
                         (int)plan.rows, plan.row_tiles, plan.front_parts, p.scale_log2};
    return by_types(c, a.bf16, [&](auto t, auto dt, auto hd) {
        using T = decltype(t);
        auto launch = [&](auto kernel, size_t lds) {
            if (lds > 64 * 1024) {   // the attribute is the current device's
                const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (e != hipSuccess) return e;
            }
            return by_items(p, plan.items, [&](unsigned wgs) {
                hipLaunchKernelGGL(kernel, dim3(wgs), dim3(64 * kWaves), lds, st, p, where, f);
                return hipGetLastError();
            });
        };
        hipError_t e;
        bool done = false;
        if constexpr (SharedPlan::rows_kernel(dt.value, sizeof(T) == 2))
            if (plan.by_rows) {
                e = launch(shared_kernel<T, dt.value, hd.value, true>, kPrefixLds);
                done = true;
            }
        if (!done) e = launch(shared_kernel<T, dt.value, hd.value, false>, (size_t)kWaves * (plan.front_wgs > 0 ? 16 : p.rows) * (hd.value + 4) * sizeof(float));
        if (e != hipSuccess || (plan.walk && p.parts == 1)) return e;
        return join_parts<T, hd.value>(a, p, st);
    });
}

hipError_t launch_kv_attention_pages(const riftkv_cache& c, const KvAttention& a, const int* lists, int top, hipStream_t st) {
    RangeParams p = params_of(c, a);
    const int64_t items = (int64_t)a.n_seq * p.n_kv * p.q_tiles, tiles = ((int64_t)top * c.page_size + kTile - 1) / kTile;
    p.parts = parts_alone(c.dt, items, tiles);
    const ListedPages where{OwnPages{a.table, a.lens, a.max_pages}, lists, top};
    const size_t lds = (size_t)kWaves * p.rows * (c.head_dim + 4) * sizeof(float);
    return by_types(c, a.bf16, [&](auto t, auto dt, auto hd) {
        using T = decltype(t);
        const hipError_t e = by_items(p, items, [&](unsigned wgs) {
            hipLaunchKernelGGL((listed_kernel<T, dt.value, hd.value>), dim3(wgs), dim3(64 * kWaves), lds, st, p, where);
            return hipGetLastError();
        });
        return e != hipSuccess || p.parts == 1 ? e : join_parts<T, hd.value>(a, p, st);
    });
}

}  // namespace rift
