// Which pages of a long context a new token needs: the smallest and largest key values of every page
// (riftkv_page_bounds), and the pages whose bounds promise the largest scores (riftkv_select_pages).
#include <type_traits>

#include "kv_device.h"

namespace rift {

namespace {

constexpr int kThreads = 256;
constexpr int kBoundWgs = 2048;
constexpr int kScoreWgs = 4096;

// The smaller of two numbers; NaN if either is.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// Tokens of a sequence, -1 for a number out of range.
__device__ __forceinline__ int length_of(int len, int max_pages, int shift) {
    return len < 0 || (int64_t)len > ((int64_t)max_pages << shift) ? -1 : len;
}
// Pages of n tokens
__device__ __forceinline__ int pages_of(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// ---------------------------------------------------------------- bounds

struct BoundParams {
    const unsigned char* k;
    const uint8_t* ks;
    void* bounds;
    const int *table, *begins, *lens;
    int* status;
    int n_seq, max_pages, n_pages, n_kv, shift;
};

// 16 bytes of a row as values
template <riftkv_dtype DT>
struct Values {
    static constexpr int N = DT == RIFTKV_F32 ? 4 : DT == RIFTKV_BF16 ? 8 : 16;
    float x[N];
    __device__ __forceinline__ Values(const u32x4_t& w, float scale) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (DT == RIFTKV_F32) x[j] = __uint_as_float(w[j]);
            else if constexpr (DT == RIFTKV_BF16) {
                x[2 * j] = bf16_lo(w[j]);
                x[2 * j + 1] = bf16_hi(w[j]);
            } else if constexpr (DT == RIFTKV_FP8) {
                const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
                x[4 * j] = a[0] * scale;
                x[4 * j + 1] = a[1] * scale;
                x[4 * j + 2] = b[0] * scale;
                x[4 * j + 3] = b[1] * scale;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * j + e] = (float)(int8_t)(w[j] >> (8 * e)) * scale;
            }
        }
    }
};

// The new pages of a sequence: from the one that holds its first new token.
struct NewPages {
    int first, n;
};
__device__ __forceinline__ NewPages new_pages(const BoundParams& p, int seq, int& len) {
    len = length_of(p.lens[seq], p.max_pages, p.shift);
    const int from = p.begins ? max(p.begins[seq], 0) : 0;
    return from < len ? NewPages{from >> p.shift, pages_of(len, p.shift) - (from >> p.shift)} : NewPages{0, 0};
}

// Values joined over the rows of a load: of two lanes each keeps one half of them, the first time the smallest or
// the negated largest, so that in the end all of a page's are spread over the wave.  at: the place of what this lane keeps.
template <int D, int HALF, int FIRST, int N>
__device__ __forceinline__ void join_rows(float (&x)[N], int lane, int& at) {
    if constexpr (D < 64) {
        const bool upper = lane & D;
#pragma unroll
        for (int e = 0; e < HALF; ++e) {
            const float give = upper ? x[e] : x[HALF + e], keep = upper ? x[HALF + e] : x[e];
            x[e] = least(keep, __shfl_xor(give, D));
        }
        if (upper) at += FIRST;
        join_rows<2 * D, HALF / 2, HALF / 2>(x, lane, at);
    }
}

// The pages of all sequences and heads, one after the other, are dealt out evenly to the workgroups, however uneven
// the lengths (a workgroup a sequence: 14.2 ms where this takes 104 us); a wave takes a page of a head at a time, 16 bytes of a
// row a lane.  Bound by the keys' bytes: 12 prompts of 3,001 to 65,536 tokens, 8 heads of 128 e4m3 values, 421 MB and 27 MB of bounds
// in 104 us, 4.6 TB/s; 64 new tokens' pages of 32 rows 5.0 us, the chain of lengths, table and keys.  A large page is one wave's loop: for 1 and 64
// new tokens in pages of 256 rows (bf16) 7.8 and 12.9 us, of 4,096 69 and 172.
template <riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(kThreads, 4)
bounds_kernel(BoundParams p) {
    constexpr int B = DT == RIFTKV_F32 ? 4 : DT == RIFTKV_BF16 ? 2 : 1, N = 16 / B;
    constexpr int LANES = HD / N, ROWS = 64 / LANES;   // lanes of a row, rows of a load
    constexpr int U = 4;                               // loads in flight
    __shared__ long long sums[kThreads / 64], found_before;
    __shared__ int found_seq;
    const int tid = threadIdx.x, lane = tid & 63, col = lane % LANES, sub = lane / LANES;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // A thread sums a run of sequences, the workgroup scans the sums, and whoever holds the first page looks it up.
    const int per = (p.n_seq + kThreads - 1) / kThreads;
    const int s0 = min(tid * per, p.n_seq), s1 = min(s0 + per, p.n_seq);
    long long mine = 0;
    int len;
    for (int s = s0; s < s1; ++s) {
        mine += new_pages(p, s, len).n;
        if (len < 0 && blockIdx.x == 0) *p.status = RIFT_ERR_SHAPE;
    }
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
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    total *= p.n_kv;
    // items begin .. end - 1: page of a sequence, head
    const long long q = total / gridDim.x, r = total - q * gridDim.x, b = blockIdx.x;
    const long long begin = b * q + (b < r ? b : r), end = begin + q + (b < r);
    if (begin == end) return;
    if (mine > 0 && begin >= before * p.n_kv && begin < (before + mine) * p.n_kv) {
        int s = s0;
        for (;; ++s) {
            const int n = new_pages(p, s, len).n;
            if (begin < (before + n) * p.n_kv) break;
            before += n;
        }
        found_seq = s;
        found_before = before;
    }
    __syncthreads();
    int seq = __builtin_amdgcn_readfirstlane(found_seq);
    long long base = found_before * p.n_kv;      // items before this sequence's
    NewPages pages = new_pages(p, seq, len);
    for (long long i = begin + wave; i < end; i += kThreads / 64) {
        while (i >= base + (long long)pages.n * p.n_kv) {
            base += (long long)pages.n * p.n_kv;
            pages = new_pages(p, ++seq, len);
        }
        const unsigned long long in = i - base;
        const int nth = (int)((in >> 32) == 0 ? (unsigned)in / (unsigned)p.n_kv : in / p.n_kv);
        const int head = __builtin_amdgcn_readfirstlane((int)(in - (unsigned long long)nth * p.n_kv));
        const int place = __builtin_amdgcn_readfirstlane(pages.first + nth);
        const int page = __builtin_amdgcn_readfirstlane(p.table[(size_t)seq * p.max_pages + place]);
        if ((unsigned)page >= (unsigned)p.n_pages) {
            if (lane == 0) *p.status = RIFT_ERR_SHAPE;
            continue;
        }
        const int n = (int)min((int64_t)len - ((int64_t)place << p.shift), (int64_t)1 << p.shift);
        const size_t row = (((size_t)page * p.n_kv) + head) << p.shift;
        float x[2 * N];                       // the smallest values, and the smallest of the negated ones
#pragma unroll
        for (int e = 0; e < 2 * N; ++e) x[e] = INFINITY;
        for (int r0 = 0; r0 < n; r0 += U * ROWS) {
            u32x4_t w[U];
            uint32_t scale[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {     // past the last token: its row once more
                const int at = min(r0 + u * ROWS + sub, n - 1);
                w[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p.k + (row + at) * (HD * B) + col * 16));
                if constexpr (B == 1) scale[u] = p.ks[row + at];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Values<DT> v(w[u], B == 1 ? scale_of(scale[u]) : 1.f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    x[e] = least(x[e], v.x[e]);
                    x[N + e] = least(x[N + e], -v.x[e]);
                }
            }
        }
        constexpr int M = 2 * N / ROWS;
        int to_col = col * N;
        join_rows<LANES, N, HD>(x, lane, to_col);
        const size_t to = ((size_t)page * p.n_kv + head) * (2 * HD) + to_col;
        const float sign = sub & 1 ? -1.f : 1.f;
        if constexpr (B == 4) {
#pragma unroll
            for (int e = 0; e < M; ++e) static_cast<float*>(p.bounds)[to + e] = sign * x[e];
        } else {
            uint32_t w[M / 2];
#pragma unroll
            for (int e = 0; e < M / 2; ++e) w[e] = (uint32_t)round_bf16(sign * x[2 * e]) | (uint32_t)round_bf16(sign * x[2 * e + 1]) << 16;
            if constexpr (M == 4) *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.bounds) + to) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(static_cast<bf16_t*>(p.bounds) + to) = w[0];
        }
    }
}

// ---------------------------------------------------------------- selection

struct SelectParams {
    const void *q, *bounds;
    int64_t ld_q;
    const int *table, *lens;
    int *lists, *status;
    unsigned long long* keys;   // [n_seq][n_kv][max_pages]
    int n_seq, max_pages, n_pages, n_kv, group, shift, first, last, top;
    int seq0, blocks;           // first sequence of the launch; workgroups of each of its key heads
};

// Order of the scores as whole numbers; NaN above every number.
constexpr unsigned long long kNanKey = ~0ull;
__device__ __forceinline__ unsigned long long key_of(double x) {
    const long long b = __double_as_longlong(x + 0.0);   // -0 as 0
    return x != x ? kNanKey : b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

// Eight values; of float32 four, and four `apart` elements on.
template <typename BT>
struct EightOf {
    u32x4_t w[sizeof(BT) / 2];
    __device__ __forceinline__ void load(const void* p, size_t i, int apart) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(BT) / 2; ++j) w[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(static_cast<const BT*>(p) + i + j * apart));
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(BT) == 2) return e & 1 ? bf16_hi(w[0][e / 2]) : bf16_lo(w[0][e / 2]);
        else return __uint_as_float(w[e / 4][e % 4]);
    }
};

template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
    const long long b = __double_as_longlong(x);
    const int lo = __builtin_amdgcn_mov_dpp((int)b, CTRL, 0xf, 0xf, false), hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 0xf, 0xf, false);
    return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}
template <int CTRL>
__device__ __forceinline__ unsigned long long dpp(unsigned long long x) {
    const int lo = __builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, false), hi = __builtin_amdgcn_mov_dpp((int)(x >> 32), CTRL, 0xf, 0xf, false);
    return ((unsigned long long)(unsigned)hi << 32) | (unsigned)lo;
}
// Lanes whose numbers differ in one bit; the lane eight or four on, among sixteen in a ring.
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kTurn8 = 0x128, kTurn4 = 0x124;

// Scores, on v_mfma_f64_4x4x4: four products of 4 pages x 4 elements and 4 elements x 4 queries.  In lane 16 k + 4 b + i (of the
// right operand: 4 b + j) of product b is page i's (query j's) element k, in lane 16 i + 4 b + j of the result page i's sum for
// query j.  A lane holds eight elements of a page's bounds, one for each of eight steps, which are the element k of product b:
// the order of a sum is free.  128 dimensions take the four products for one group of four pages, 64 two products for each of
// two.  Negative and positive query values are operands of their own, with the smallest and the largest keys, so that no
// product needs a choice.  Float64, because float32 sums would order pages otherwise than the definition does.
// NS: sets of four queries that share the bounds' conversions (groups of 8: 74.6 us with two, 80.8 with one).
//
// Between the bounds' bytes and the float64 unit, which has the products and the conversions: of a wave's 16 pages of 128
// dimensions 64 products (18.7 cycles each, measured, the rate of as many multiply-adds) and 64 conversions (8.3).  48 contexts of 17
// to 65,001 tokens, 32 heads in groups of 4, pages of 32: 200 MB, with the selection 52.4 us; 40 of loads alone.  Multiply-adds
// with queries in registers of float32 took 66.7: their conversions, 15 exchanges of a sum's parts, and two waves a SIMD
// instead of five.  256 to 8,192 workgroups: within 8%; a page's key heads in workgroups next to each other 3 to 5%; loads that
// stay in the caches 58 (float32 bounds too, 32 bytes a lane, until each load took whole pieces of 64: 114 us, 94 now).
constexpr int kQueries = 4;

template <typename T, typename BT, int HD, int NS>
__global__ void __launch_bounds__(kThreads, NS == 1 ? 4 : 3)
scores_kernel(SelectParams p) {
    constexpr int G = HD / 8, PW = 64 / G;           // lanes of a page, pages of a load
    constexpr int ITERS = G / 4, PAGES = PW * ITERS; // loads of a wave's turn: as many as products of a page
    constexpr int WAVES = kThreads / 64;
    const int lane = threadIdx.x & 63, k = lane >> 4, b = (lane >> 2) & 3;
    // product of the page that this lane's bounds belong to, and first page of its group of four
    const int part = HD == 128 ? b : b >> 1, group4 = HD == 128 ? 0 : 4 * (b & 1);
    constexpr int APART = sizeof(BT) == 2 ? 4 : HD / 2;
    const int d0 = (HD / 4 * k + 8 * part) / (sizeof(BT) / 2), sub = group4 + (lane & 3);   // its first element; its page of a load
    const int got = group4 + k;                      // the page, of load `part`, whose sum it has in the end
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a block of pages after the other, each with all key heads: what lies together in memory is read together
    const int of = blockIdx.x / p.n_kv, kvh = blockIdx.x - of * p.n_kv;
    const int seq = of / p.blocks + p.seq0, block = of % p.blocks, item = seq * p.n_kv + kvh;
    const int len = length_of(p.lens[seq], p.max_pages, p.shift);
    const int held = pages_of(max(len, 0), p.shift);
    if (held <= p.top) return;                       // all of them
    const int begin = p.first, end = held - p.last;  // the pages to choose from
    const int* table = p.table + (size_t)seq * p.max_pages;
    unsigned long long* keys = p.keys + (size_t)item * p.max_pages;
    const T* q = static_cast<const T*>(p.q) + (size_t)seq * p.ld_q + (size_t)kvh * p.group * HD + d0;
    double neg[NS][8], pos[NS][8];
    auto load_q = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NS; ++n) {               // past the last: it once more
            EightOf<T> x;
            x.load(q, (size_t)min(j0 + kQueries * n + (lane & 3), p.group - 1) * HD, APART);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = x.at(e);
                neg[n][e] = f > 0.f ? 0.f : f;       // (NaN is in both)
                pos[n][e] = f < 0.f ? 0.f : f;
            }
        }
    };
    load_q(0);
    const int64_t step = (int64_t)p.blocks * WAVES * PAGES;
    for (int64_t p0 = begin + (int64_t)(block * WAVES + wave) * PAGES; p0 < end; p0 += step) {
        EightOf<BT> lo[ITERS], hi[ITERS];
        bool good = true;
#pragma unroll
        for (int i = 0; i < ITERS; ++i) {            // past the last: it once more
            const int page = table[min((int)p0 + i * PW + sub, end - 1)];
            const bool is = (unsigned)page < (unsigned)p.n_pages;
            const unsigned long long there = __ballot(is);
            if (part == i) good = there >> got & 1;
            const size_t at = ((size_t)(is ? page : 0) * p.n_kv + kvh) * (2 * HD) + d0;
            lo[i].load(p.bounds, at, APART);
            hi[i].load(p.bounds, at + HD, APART);
        }
        unsigned long long best = 0;
        for (int j0 = 0; j0 < p.group; j0 += kQueries * NS) {
            if (p.group > kQueries * NS) load_q(j0);
#pragma unroll
            for (int i = 0; i < ITERS; ++i)          // converted where a step needs them, not for all steps before the loop
#pragma unroll
                for (int j = 0; j < (int)sizeof(BT) / 2; ++j) asm volatile("" : "+v"(lo[i].w[j]), "+v"(hi[i].w[j]));
            double s[NS][ITERS];
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < ITERS; ++i) s[n][i] = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < ITERS; ++i)
#pragma unroll
                    for (int n = 0; n < NS; ++n) s[n][i] = __builtin_amdgcn_mfma_f64_4x4x4f64(lo[i].at(e), neg[n][e], s[n][i], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < ITERS; ++i)
#pragma unroll
                    for (int n = 0; n < NS; ++n) s[n][i] = __builtin_amdgcn_mfma_f64_4x4x4f64(hi[i].at(e), pos[n][e], s[n][i], 0, 0, 0);
            }
            // Over the products of a page, whose numbers differ by two, then by one, in turn: all its lanes have its sum then, and
            // each takes that of one load.
#pragma unroll
            for (int n = 0; n < NS; ++n) {
#pragma unroll
                for (int i = 0; i < ITERS; ++i) {
                    s[n][i] += dpp<kTurn8>(s[n][i]);
                    if constexpr (HD == 128) s[n][i] += dpp<kTurn4>(s[n][i]);
                }
                double mine = s[n][0];
#pragma unroll
                for (int i = 1; i < ITERS; ++i)
                    if (part == i) mine = s[n][i];
                best = max(best, key_of(mine));
            }
        }
        best = max(best, dpp<kXor1>(best));          // over the queries
        best = max(best, dpp<kXor2>(best));
        const int64_t place = p0 + part * PW + got;
        if ((lane & 3) == 0 && place < end) {
            keys[place] = good && best != kNanKey ? best : 0;
            if (!good) *p.status = RIFT_ERR_SHAPE;
        }
    }
}

// A workgroup takes a key head of a sequence, a thread a run of its pages (of every 4,096): the key of the last page to take, eleven bits of it
// at a time from the first that differs between pages (so that few pages are left in a bucket of the first time, often the
// one that is looked for), then the list.  A chain of waits: 6.9 us for 8 key heads of 1,024 pages, 8.2 for 384 of up to 2,032.
// (A run of all of its pages, however many, took a thread through memory in long steps: 2 key heads of 62,500 pages, with the scores,
// 190 us, in turns 92; every 512th page: 133, and 2% more below 4,096.)
constexpr int kPickThreads = 512, kHeldKeys = 8;   // keys that a thread keeps in registers
constexpr int kTurnKeys = kPickThreads * kHeldKeys;  // more pages are gone through in turns
constexpr int kBucketBits = 11, kBuckets = 1 << kBucketBits;

// TURNS: there can be more pages than the threads hold.
template <bool TURNS>
__global__ void __launch_bounds__(kPickThreads)
pick_kernel(SelectParams p) {
    constexpr int WAVES = kPickThreads / 64;
    __shared__ __align__(16) int counts[kBuckets];
    __shared__ uint2 ends_of[WAVES];                // largest of the keys' upper words, and of their complements
    __shared__ int sums[WAVES][2];
    __shared__ int found, above, inside;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int item = blockIdx.x + p.seq0 * p.n_kv, seq = item / p.n_kv;
    int* list = p.lists + (size_t)item * p.top;
    const int len = length_of(p.lens[seq], p.max_pages, p.shift);
    if (len < 0 && tid == 0) *p.status = RIFT_ERR_SHAPE;
    const int held = pages_of(max(len, 0), p.shift);
    const int* table = p.table + (size_t)seq * p.max_pages;
    auto check = [&](int place) {
        if ((unsigned)table[place] >= (unsigned)p.n_pages) *p.status = RIFT_ERR_SHAPE;
    };
    if (held <= p.top) {
        for (int i = tid; i < p.top; i += kPickThreads) {
            list[i] = i < held ? i : -1;
            if (i < held) check(i);
        }
        return;
    }
    for (int i = tid; i < p.first; i += kPickThreads) {
        list[i] = i;
        check(i);
    }
    for (int i = tid; i < p.last; i += kPickThreads) {
        list[p.top - p.last + i] = held - p.last + i;
        check(held - p.last + i);
    }
    int need = p.top - p.first - p.last;
    if (need == 0) {                                                 // no score was worked out
        for (int i = p.first + tid; i < held - p.last; i += kPickThreads) check(i);
        return;
    }
    const int begin = p.first, n = held - p.first - p.last;          // the pages to choose from, more than need
    const unsigned long long* keys = p.keys + (size_t)item * p.max_pages + begin;
    const int per = ((TURNS ? min(n, kTurnKeys) : n) + kPickThreads - 1) / kPickThreads;
    unsigned long long mine[kHeldKeys];
    // this thread's run of the turn that begins at page `first`: i0 .. i1 - 1
    int i0 = 0, i1 = 0;
    auto load = [&](int first) __attribute__((always_inline)) {
        i0 = min(first + tid * per, n);
        i1 = min(i0 + per, n);
#pragma unroll
        for (int i = 0; i < kHeldKeys; ++i) mine[i] = i0 + i < i1 ? keys[i0 + i] : 0;
    };
    load(0);
    // f(key) of every page of this thread
    auto each = [&](auto f) __attribute__((always_inline)) {
        for (int first = 0;;) {
#pragma unroll
            for (int i = 0; i < kHeldKeys; ++i)
                if (i0 + i < i1) f(mine[i]);
            if (!TURNS || n <= kTurnKeys) break;
            first = first + kTurnKeys < n ? first + kTurnKeys : 0;
            load(first);
            if (first == 0) break;
        }
    };
    uint32_t highest = 0, complement = 0;
    each([&](unsigned long long k) {
        highest = max(highest, (uint32_t)(k >> 32));
        complement = max(complement, ~(uint32_t)(k >> 32));
    });
    highest = wave_most(highest);
    complement = wave_most(complement);
    if (lane == 0) ends_of[wave] = make_uint2(highest, complement);
    for (int i = tid; i < kBuckets; i += kPickThreads) counts[i] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        highest = max(highest, ends_of[w].x);
        complement = max(complement, ends_of[w].y);
    }
    // Keys of a bucket share the bits from `bit` on; those of higher buckets are all taken.  Upper words that are all alike: from
    // the lower ones on.
    const uint32_t differ = highest ^ ~complement;
    int bit = (differ == 0 ? 32 : 64 - __clz(differ)) - kBucketBits;
    unsigned long long bucket = ((unsigned long long)highest << 32) >> bit;
    int width = kBuckets;
    for (;;) {
        const unsigned long long base = bucket & ~(unsigned long long)(width - 1);   // the first of the buckets looked at
        each([&](unsigned long long k) {
            const unsigned long long in = (k >> bit) - base;
            if (in < (unsigned long long)width) atomicAdd(&counts[in], 1);
        });
        __syncthreads();
        if (wave == 0) {
            // a run of buckets a lane, the highest first
            constexpr int RUN = kBuckets / 64;
            int c[RUN], sum = 0;
#pragma unroll
            for (int i = 0; i < RUN; i += 4) {
                const int4 x = *reinterpret_cast<const int4*>(counts + kBuckets - RUN * (lane + 1) + i);
                c[RUN - 1 - i] = x.x;
                c[RUN - 2 - i] = x.y;
                c[RUN - 3 - i] = x.z;
                c[RUN - 4 - i] = x.w;
                sum += x.x + x.y + x.z + x.w;
            }
            const int incl = wave_scan(sum);
            int before = incl - sum, at = 0, in = 0;
            if (before < need && need <= incl) {
                bool past = false;
#pragma unroll
                for (int i = 0; i < RUN; ++i) {
                    if (!past && before + c[i] >= need) {
                        past = true;
                        at = i;
                        in = c[i];
                    }
                    if (!past) before += c[i];
                }
                found = kBuckets - 1 - RUN * lane - at;
                above = before;
                inside = in;
            }
        }
        __syncthreads();
        bucket = base + found;
        need -= above;
        if (bit == 0 || inside == need) break;
        const int step = min(bit, kBucketBits);
        width = 1 << step;
        bit -= step;
        bucket <<= step;
        __syncthreads();            // (found, above and inside have been read)
        for (int i = tid; i < kBuckets; i += kPickThreads) counts[i] = 0;
        __syncthreads();
    }
    // places in the list: of the pages above, and of the bucket's first ones
    int higher = 0, equal = 0;                       // in the turns before
    for (int first = 0; first == 0 || (TURNS && first < n); first += kTurnKeys) {
        if (TURNS && first > 0) {
            load(first);
            __syncthreads();                         // (the sums have been read)
        }
        int hi = 0, eq = 0;
#pragma unroll
        for (int i = 0; i < kHeldKeys; ++i)
            if (i0 + i < i1) {
                hi += (mine[i] >> bit) > bucket;
                eq += (mine[i] >> bit) == bucket;
            }
        const int hi_incl = wave_scan(hi), eq_incl = wave_scan(eq);
        if (lane == 63) {
            sums[wave][0] = hi_incl;
            sums[wave][1] = eq_incl;
        }
        __syncthreads();
        hi = higher + hi_incl - hi;
        eq = equal + eq_incl - eq;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) {
                hi += sums[w][0];
                eq += sums[w][1];
            }
            higher += sums[w][0];
            equal += sums[w][1];
        }
#pragma unroll
        for (int i = 0; i < kHeldKeys; ++i)
            if (i0 + i < i1) {
                const unsigned long long b = mine[i] >> bit;
                if (b > bucket || (b == bucket && eq < need)) list[p.first + hi + min(eq, need)] = begin + i0 + i;
                hi += b > bucket;
                eq += b == bucket;
            }
    }
}

}  // namespace

hipError_t launch_kv_page_bounds(const riftkv_cache& c, void* bounds, const int* table, int n_seq, int max_pages, const int* begins,
                                 const int* lens, int* status, hipStream_t st) {
    const BoundParams p{static_cast<const unsigned char*>(c.k), c.k_scale, bounds, table, begins, lens, status, n_seq, max_pages,
                        c.n_pages, c.n_kv_heads, 31 - __builtin_clz(c.page_size)};
    // a wave an item as far as the table can hold them, and as many as are resident
    const int64_t items = (int64_t)n_seq * max_pages * c.n_kv_heads, most = (items + 3) / 4;
    const unsigned wgs = (unsigned)(most < 1 ? 1 : most > kBoundWgs ? kBoundWgs : most);
    auto run = [&](auto dt) {
        if (c.head_dim == 128) hipLaunchKernelGGL((bounds_kernel<dt.value, 128>), dim3(wgs), dim3(kThreads), 0, st, p);
        else hipLaunchKernelGGL((bounds_kernel<dt.value, 64>), dim3(wgs), dim3(kThreads), 0, st, p);
        return hipGetLastError();
    };
    switch (c.dt) {
        case RIFTKV_F32: return run(std::integral_constant<riftkv_dtype, RIFTKV_F32>{});
        case RIFTKV_BF16: return run(std::integral_constant<riftkv_dtype, RIFTKV_BF16>{});
        case RIFTKV_FP8: return run(std::integral_constant<riftkv_dtype, RIFTKV_FP8>{});
        case RIFTKV_INT8: return run(std::integral_constant<riftkv_dtype, RIFTKV_INT8>{});
    }
    return hipErrorInvalidValue;
}

size_t kv_select_workspace(const riftkv_cache& c, int64_t n_seq, int64_t max_pages) {
    const size_t n = (size_t)n_seq * c.n_kv_heads * max_pages * sizeof(unsigned long long);
    return n < 256 ? 256 : n;
}

hipError_t launch_kv_select_pages(const riftkv_cache& c, const KvSelect& s, hipStream_t st) {
    SelectParams p{s.q, s.bounds, s.ld_q, s.table, s.lens, s.lists, s.status, static_cast<unsigned long long*>(s.workspace),
                   s.n_seq, s.max_pages, c.n_pages, c.n_kv_heads, s.n_heads / c.n_kv_heads, 31 - __builtin_clz(c.page_size),
                   s.first, s.last, s.top, 0, 1};
    const int64_t items = (int64_t)s.n_seq * c.n_kv_heads;
    // Workgroups of 64 pages a (sequence, key head), as many as the table can need or as keep all CUs busy.
    const int64_t most = (s.max_pages + 63) / 64, enough = (kScoreWgs + items - 1) / items;
    p.blocks = (int)(most < 1 ? 1 : most < enough ? most : enough);
    // launch(workgroups), as often as the sequences need
    auto in_pieces = [&](int64_t wgs_of_head, int threads, auto launch) {
        const int64_t of_seq = wgs_of_head * c.n_kv_heads, most = ((1ll << 32) - 1) / threads / of_seq;
        for (int64_t i = 0; i < s.n_seq; i += most) {
            p.seq0 = (int)i;
            launch((unsigned)((s.n_seq - i < most ? s.n_seq - i : most) * of_seq));
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    auto scores = [&](auto kernel) {
        return in_pieces(p.blocks, kThreads, [&](unsigned wgs) { hipLaunchKernelGGL(kernel, dim3(wgs), dim3(kThreads), 0, st, p); });
    };
    auto types = [&](auto t, auto bt) {
        using T = decltype(t);
        using BT = decltype(bt);
        auto sets = [&](auto n) {
            return c.head_dim == 128 ? scores(scores_kernel<T, BT, 128, n.value>) : scores(scores_kernel<T, BT, 64, n.value>);
        };
        return p.group > kQueries ? sets(std::integral_constant<int, 2>{}) : sets(std::integral_constant<int, 1>{});
    };
    if (s.max_pages > s.top && s.top > s.first + s.last) {     // something to choose
        const hipError_t e = c.dt == RIFTKV_F32 ? types(float{}, float{}) : s.bf16 ? types(bf16_t{}, bf16_t{}) : types(float{}, bf16_t{});
        if (e != hipSuccess) return e;
    }
    const auto pick = s.max_pages > kTurnKeys ? pick_kernel<true> : pick_kernel<false>;
    return in_pieces(1, kPickThreads, [&](unsigned wgs) { hipLaunchKernelGGL(pick, dim3(wgs), dim3(kPickThreads), 0, st, p); });
}

}  // namespace rift
