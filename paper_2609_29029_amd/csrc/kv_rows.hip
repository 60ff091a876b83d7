// Rows of the paged key-value cache: rotary positions, rows into pages, rows out
// of them.  A wave takes one head of one row.
#include <type_traits>

#include "kv_device.h"

namespace rift {

namespace {

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

// The angle in turns, reduced to [-1/2, 1/2] in float64: float32 holds it and its
// sine and cosine to their last bits however far the position is.
__device__ __forceinline__ float2 rope_turn(int position, double turns, float magnitude) {
    const double t = (double)position * turns;
    float s, c;
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
    return make_float2(c * magnitude, s * magnitude);
}

template <typename T>
__global__ void __launch_bounds__(64)
rope_kernel(RopeRows q, RopeRows k, const int* __restrict__ positions, int head_dim, int rotary_dim, int interleaved,
            RopeFreqs freqs, float magnitude) {
    const int heads = q.n + k.n;
    const int row = blockIdx.x / heads, h = blockIdx.x - row * heads;
    const RopeRows& r = h < q.n ? q : k;
    const size_t hoff = (size_t)(h < q.n ? h : h - q.n) * head_dim;
    const size_t x0 = (size_t)row * r.ld_x + hoff, y0 = (size_t)row * r.ld_y + hoff;
    const int half = rotary_dim / 2;
    for (int j = threadIdx.x; j < half; j += 64) {
        const float2 cs = rope_turn(positions[row], freqs.f[j], magnitude);
        const int i1 = interleaved ? 2 * j : j, i2 = interleaved ? 2 * j + 1 : j + half;
        const float2 y = rotate_pair(load_f32<T>(r.x, x0 + i1), load_f32<T>(r.x, x0 + i2), cs);
        store_f32<T>(r.y, y0 + i1, y.x);
        store_f32<T>(r.y, y0 + i2, y.y);
    }
    for (int j = rotary_dim + threadIdx.x; j < head_dim; j += 64) store_f32<T>(r.y, y0 + j, load_f32<T>(r.x, x0 + j));
}

// Index of (page, head, row in page) among the pages' rows; -1 where the row is
// skipped, or is out of range and the status set.
__device__ __forceinline__ int64_t page_row(const KvPlaces& at, int row, int head, int n_pages, int page_size, int n_kv) {
    const int seq = at.seq_ids ? at.seq_ids[row] : row, pos = at.positions[row];
    if (seq < 0 || pos < 0) return -1;
    const int shift = 31 - __clz(page_size);
    int page = -1;
    if (seq < at.n_seq && (pos >> shift) < at.max_pages) page = at.table[(size_t)seq * at.max_pages + (pos >> shift)];
    if (page < 0 || page >= n_pages) {
        *at.status = RIFT_ERR_SHAPE;
        return -1;
    }
    return (((int64_t)page * n_kv + head) << shift) + (pos & (page_size - 1));
}

template <typename T, riftkv_dtype DT, int HD>
__device__ void write_row(const void* x, size_t x0, void* pages, uint8_t* scales, int64_t to, int lane) {
    constexpr int E = HD / 64;
    float f[E];
    for (int e = 0; e < E; ++e) f[e] = load_f32<T>(x, x0 + lane + 64 * e);
    const size_t y0 = (size_t)to * HD;
    if constexpr (DT == RIFTKV_F32 || DT == RIFTKV_BF16) {
        for (int e = 0; e < E; ++e) {
            if constexpr (DT == RIFTKV_F32) static_cast<float*>(pages)[y0 + lane + 64 * e] = f[e];
            else static_cast<bf16_t*>(pages)[y0 + lane + 64 * e] = round_bf16(f[e]);
        }
    } else {
        uint32_t most = 0;
        for (int e = 0; e < E; ++e) most = max(most, __float_as_uint(f[e]) & 0x7FFFFFFFu);
        for (int s = 32; s >= 1; s >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
        const bool bad = most >= kNotFinite;
        const uint32_t b = bad ? 255u : scale_byte<DT>(most);
        const float up = bad ? 0.f : __uint_as_float((254u - b) << 23);
        for (int e = 0; e < E; ++e) {
            const float y = bad ? 0.f : f[e] * up;
            uint8_t code;
            if constexpr (DT == RIFTKV_FP8) code = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false);
            else code = (uint8_t)(int)rintf(y);
            static_cast<uint8_t*>(pages)[y0 + lane + 64 * e] = code;
        }
        if (lane == 0) scales[to] = (uint8_t)b;
    }
}

template <typename T, riftkv_dtype DT, int HD>
__device__ void read_row(void* y, size_t y0, const void* pages, const uint8_t* scales, int64_t from, int lane) {
    const size_t x0 = (size_t)from * HD;
    for (int e = lane; e < HD; e += 64) {
        float f;
        if constexpr (DT == RIFTKV_F32) f = static_cast<const float*>(pages)[x0 + e];
        else if constexpr (DT == RIFTKV_BF16) f = bf16_to_f32(static_cast<const bf16_t*>(pages)[x0 + e]);
        else {
            const uint32_t code = static_cast<const uint8_t*>(pages)[x0 + e];
            if constexpr (DT == RIFTKV_FP8) f = __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
            else f = (float)(int8_t)code;
            f *= scale_of(scales[from]);
        }
        store_f32<T>(y, y0 + e, f);
    }
}

template <typename T, riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(64)
write_kernel(riftkv_cache c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, KvPlaces at) {
    const int row = blockIdx.x / c.n_kv_heads, h = blockIdx.x - row * c.n_kv_heads;
    const int64_t to = page_row(at, row, h, c.n_pages, c.page_size, c.n_kv_heads);
    if (to < 0) return;
    write_row<T, DT, HD>(k, (size_t)row * ld_k + h * HD, c.k, c.k_scale, to, threadIdx.x);
    write_row<T, DT, HD>(v, (size_t)row * ld_v + h * HD, c.v, c.v_scale, to, threadIdx.x);
}

template <typename T, riftkv_dtype DT, int HD>
__global__ void __launch_bounds__(64)
read_kernel(riftkv_cache c, void* k, int64_t ld_k, void* v, int64_t ld_v, KvPlaces at) {
    const int row = blockIdx.x / c.n_kv_heads, h = blockIdx.x - row * c.n_kv_heads;
    const int64_t from = page_row(at, row, h, c.n_pages, c.page_size, c.n_kv_heads);
    if (from < 0) return;
    read_row<T, DT, HD>(k, (size_t)row * ld_k + h * HD, c.k, c.k_scale, from, threadIdx.x);
    read_row<T, DT, HD>(v, (size_t)row * ld_v + h * HD, c.v, c.v_scale, from, threadIdx.x);
}

// f<T, DT, HD>() for the types of a call; the C ABI has refused the others.
template <typename F>
hipError_t with_types(bool bf16, riftkv_dtype dt, int hd, F f) {
    auto heads = [&](auto t, auto d) {
        if (hd == 128) f(t, d, std::integral_constant<int, 128>{});
        else f(t, d, std::integral_constant<int, 64>{});
        return hipGetLastError();
    };
    auto types = [&](auto d) { return bf16 ? heads(bf16_t{}, d) : heads(float{}, d); };
    switch (dt) {
        case RIFTKV_F32: return types(std::integral_constant<riftkv_dtype, RIFTKV_F32>{});
        case RIFTKV_BF16: return types(std::integral_constant<riftkv_dtype, RIFTKV_BF16>{});
        case RIFTKV_FP8: return types(std::integral_constant<riftkv_dtype, RIFTKV_FP8>{});
        case RIFTKV_INT8: return types(std::integral_constant<riftkv_dtype, RIFTKV_INT8>{});
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv_rope(const RopeRows& q, const RopeRows& k, bool bf16, const int* positions, int rows, int head_dim,
                          int rotary_dim, bool interleaved, const RopeFreqs& freqs, float magnitude, hipStream_t st) {
    const dim3 grid((unsigned)rows * (unsigned)(q.n + k.n));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(64), 0, st, q, k, positions, head_dim, rotary_dim, interleaved ? 1 : 0,
                           freqs, magnitude);
    };
    if (bf16) launch(rope_kernel<bf16_t>);
    else launch(rope_kernel<float>);
    return hipGetLastError();
}

hipError_t launch_kv_write(const riftkv_cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, bool bf16,
                           const KvPlaces& at, hipStream_t st) {
    const dim3 grid((unsigned)at.rows * (unsigned)c.n_kv_heads);
    return with_types(bf16, c.dt, c.head_dim, [&](auto t, auto dt, auto hd) {
        hipLaunchKernelGGL((write_kernel<decltype(t), dt.value, hd.value>), grid, dim3(64), 0, st, c, k, ld_k, v, ld_v, at);
    });
}

hipError_t launch_kv_read(const riftkv_cache& c, void* k, int64_t ld_k, void* v, int64_t ld_v, bool bf16,
                          const KvPlaces& at, hipStream_t st) {
    const dim3 grid((unsigned)at.rows * (unsigned)c.n_kv_heads);
    return with_types(bf16, c.dt, c.head_dim, [&](auto t, auto dt, auto hd) {
        hipLaunchKernelGGL((read_kernel<decltype(t), dt.value, hd.value>), grid, dim3(64), 0, st, c, k, ld_k, v, ld_v, at);
    });
}

}  // namespace rift
