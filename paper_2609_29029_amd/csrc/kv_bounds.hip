// Which pages of a long context a new token needs: the smallest and largest key values of every page
// (riftkv_page_bounds), and the pages whose bounds promise the largest scores (riftkv_select_pages).
#include <type_traits>

#include "kv_device.h"

namespace rift {

namespace {

constexpr int kThreads = 256;
constexpr int kBoundWgs = 2048;

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
// the lengths; a wave takes a page of a head at a time, 16 bytes of a row a lane.
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
};

constexpr int kQueries = 4;     // of a pass over the bounds
constexpr int kSelectThreads = 1024;

// Order of the scores as whole numbers; NaN before every number.
__device__ __forceinline__ unsigned long long key_of(double x) {
    if (x != x) return 0;
    const long long b = __double_as_longlong(x + 0.0);   // -0 as 0
    return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

template <typename T>
__device__ __forceinline__ double load_f64(const void* p, size_t i) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(static_cast<const bf16_t*>(p)[i]);
    else return static_cast<const float*>(p)[i];
}

// A workgroup takes a key head of a sequence: a page a thread, then the rank of the last page
// to take, eight bits of it at a time, then the list.
template <typename T, typename BT, int HD>
__global__ void __launch_bounds__(kSelectThreads)
select_kernel(SelectParams p) {
    __shared__ double qs[2][kQueries][HD];      // min(q, 0), max(q, 0)
    __shared__ int counts[256];
    __shared__ int waves[kSelectThreads / 64], waves_eq[kSelectThreads / 64];
    __shared__ int found, above;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seq = blockIdx.x / p.n_kv, kvh = blockIdx.x - seq * p.n_kv;
    int* list = p.lists + (size_t)blockIdx.x * p.top;
    const int given = p.lens[seq], len = length_of(given, p.max_pages, p.shift);
    if (len < 0 && tid == 0) *p.status = RIFT_ERR_SHAPE;
    const int held = len < 0 ? 0 : pages_of(len, p.shift);
    const int* table = p.table + (size_t)seq * p.max_pages;
    unsigned long long* keys = p.keys + (size_t)blockIdx.x * p.max_pages;
    for (int i = min(held, p.top) + tid; i < p.top; i += kSelectThreads) list[i] = -1;
    if (held <= p.top) {
        for (int i = tid; i < held; i += kSelectThreads) {
            list[i] = i;
            if ((unsigned)table[i] >= (unsigned)p.n_pages) *p.status = RIFT_ERR_SHAPE;
        }
        return;
    }
    // scores
    for (int j0 = 0; j0 < p.group; j0 += kQueries) {
        const int nq = min(kQueries, p.group - j0);
        __syncthreads();
        for (int i = tid; i < kQueries * HD; i += kSelectThreads) {
            const int j = i / HD, d = i % HD;
            const double x = j < nq ? load_f64<T>(p.q, (size_t)seq * p.ld_q + (size_t)(kvh * p.group + j0 + j) * HD + d) : 0.0;
            qs[0][j][d] = x < 0.0 ? x : x == x ? 0.0 : x;
            qs[1][j][d] = x > 0.0 ? x : x == x ? 0.0 : x;
        }
        __syncthreads();
        for (int i = tid; i < held; i += kSelectThreads) {
            const int page = table[i];
            unsigned long long best = 0;
            if ((unsigned)page < (unsigned)p.n_pages) {
                const size_t at = ((size_t)page * p.n_kv + kvh) * (2 * HD);
                double s[kQueries] = {};
                for (int d = 0; d < HD; ++d) {
                    const double lo = load_f64<BT>(p.bounds, at + d), hi = load_f64<BT>(p.bounds, at + HD + d);
#pragma unroll
                    for (int j = 0; j < kQueries; ++j) s[j] = fma(qs[1][j][d], hi, fma(qs[0][j][d], lo, s[j]));
                }
                bool nan = j0 > 0 && keys[i] == 0;
                if (j0 > 0) best = keys[i];
#pragma unroll
                for (int j = 0; j < kQueries; ++j)
                    if (j < nq) {
                        const unsigned long long k = key_of(s[j]);
                        nan |= k == 0;
                        best = max(best, k);
                    }
                if (nan) best = 0;
            } else {
                *p.status = RIFT_ERR_SHAPE;
            }
            keys[i] = best;
        }
    }
    __syncthreads();
    // the key of the last page to take among those between the ends, and how many of its equals
    const int begin = p.first, end = held - p.last;
    int need = p.top - p.first - p.last;
    unsigned long long prefix = 0;
    for (int bit = 56; need > 0 && bit >= 0; bit -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) counts[i] = 0;
        __syncthreads();
        for (int i = begin + tid; i < end; i += kSelectThreads) {
            const unsigned long long k = keys[i];
            if (bit == 56 || (k >> (bit + 8)) == (prefix >> (bit + 8))) atomicAdd(&counts[(k >> bit) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int sum = 0, b = 255;
            while (sum + counts[b] < need) sum += counts[b--];
            found = b;
            above = sum;
        }
        __syncthreads();
        prefix |= (unsigned long long)found << bit;
        need -= above;
        __syncthreads();
    }
    // the list, in the pages' order
    int out = 0, equal = 0;
    for (int i0 = 0; i0 < held; i0 += kSelectThreads) {
        const int i = i0 + tid;
        const bool between = i >= begin && i < end;
        const unsigned long long k = between ? keys[i] : 0;
        const bool eq = between && need > 0 && k == prefix;
        const unsigned long long eqs = __ballot(eq);
        if (lane == 0) waves_eq[wave] = __popcll(eqs);
        __syncthreads();
        int rank = equal + __popcll(eqs & ((1ull << lane) - 1));
        for (int w = 0; w < kSelectThreads / 64; ++w) {
            if (w < wave) rank += waves_eq[w];
            equal += waves_eq[w];
        }
        const bool take = i < held && (!between || (need > 0 && (k > prefix || (eq && rank < need))));
        const unsigned long long takes = __ballot(take);
        if (lane == 0) waves[wave] = __popcll(takes);
        __syncthreads();
        int at = out + __popcll(takes & ((1ull << lane) - 1));
        for (int w = 0; w < kSelectThreads / 64; ++w) {
            if (w < wave) at += waves[w];
            out += waves[w];
        }
        if (take) list[at] = i;
        __syncthreads();
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
    const SelectParams p{s.q, s.bounds, s.ld_q, s.table, s.lens, s.lists, s.status, static_cast<unsigned long long*>(s.workspace),
                         s.n_seq, s.max_pages, c.n_pages, c.n_kv_heads, s.n_heads / c.n_kv_heads, 31 - __builtin_clz(c.page_size),
                         s.first, s.last, s.top};
    auto run = [&](auto t, auto bt) {
        using T = decltype(t);
        using BT = decltype(bt);
        const dim3 grid((unsigned)s.n_seq * (unsigned)c.n_kv_heads);
        if (c.head_dim == 128) hipLaunchKernelGGL((select_kernel<T, BT, 128>), grid, dim3(kSelectThreads), 0, st, p);
        else hipLaunchKernelGGL((select_kernel<T, BT, 64>), grid, dim3(kSelectThreads), 0, st, p);
        return hipGetLastError();
    };
    if (c.dt == RIFTKV_F32) return run(float{}, float{});
    return s.bf16 ? run(bf16_t{}, bf16_t{}) : run(float{}, bf16_t{});
}

}  // namespace rift
