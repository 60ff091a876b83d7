// One query token of every sequence over its paged keys and values: a wave takes
// one query head of one sequence and walks the tokens with a running maximum and sum.
#include "kv_device.h"

namespace rift {

namespace {

template <riftkv_dtype DT>
__device__ __forceinline__ float cached(const void* pages, const uint8_t* scales, size_t row, int hd, int e) {
    const size_t i = row * hd + e;
    if constexpr (DT == RIFTKV_F32) return static_cast<const float*>(pages)[i];
    else if constexpr (DT == RIFTKV_BF16) return bf16_to_f32(static_cast<const bf16_t*>(pages)[i]);
    else {
        const uint32_t code = static_cast<const uint8_t*>(pages)[i];
        const float f = DT == RIFTKV_FP8 ? __builtin_amdgcn_cvt_f32_fp8((int)code, 0) : (float)(int8_t)code;
        return f * scale_of(scales[row]);
    }
}

template <typename T, riftkv_dtype DT>
__global__ void __launch_bounds__(64)
attention_kernel(riftkv_cache c, KvAttention a) {
    const int seq = blockIdx.x / a.n_heads, h = blockIdx.x - seq * a.n_heads, lane = threadIdx.x;
    const int kvh = h / (a.n_heads / c.n_kv_heads), hd = c.head_dim, shift = 31 - __clz(c.page_size);
    const int len = a.lens[seq];
    const size_t q0 = (size_t)seq * a.ld_q + (size_t)h * hd, o0 = (size_t)seq * a.ld_out + (size_t)h * hd;
    auto load_q = [&](int e) {
        if constexpr (sizeof(T) == 2) return bf16_to_f32(static_cast<const bf16_t*>(a.q)[q0 + e]);
        else return static_cast<const float*>(a.q)[q0 + e];
    };
    const float q1 = load_q(lane), q2 = hd == 128 ? load_q(lane + 64) : 0.f;
    bool bad = len < 0 || (int64_t)len > ((int64_t)a.max_pages << shift);
    float m = -INFINITY, l = 0.f, o1 = 0.f, o2 = 0.f;
    for (int j = 0; j < len && !bad; ++j) {
        const int page = a.table[(size_t)seq * a.max_pages + (j >> shift)];
        if (page < 0 || page >= c.n_pages) {
            bad = true;
            break;
        }
        const size_t row = ((((size_t)page * c.n_kv_heads) + kvh) << shift) + (j & (c.page_size - 1));
        float s = q1 * cached<DT>(c.k, c.k_scale, row, hd, lane);
        if (hd == 128) s = fmaf(q2, cached<DT>(c.k, c.k_scale, row, hd, lane + 64), s);
        s = wave_sum(s) * a.scale;
        const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn;
        const float f = expf(m - ref), p = expf(s - ref);
        l = fmaf(l, f, p);
        o1 = fmaf(o1, f, p * cached<DT>(c.v, c.v_scale, row, hd, lane));
        if (hd == 128) o2 = fmaf(o2, f, p * cached<DT>(c.v, c.v_scale, row, hd, lane + 64));
        m = mn;
    }
    if (bad) {
        *a.status = RIFT_ERR_SHAPE;
        l = NAN;
    }
    const float inv = len == 0 ? 0.f : 1.f / l;
    auto store = [&](int e, float x) {
        if constexpr (sizeof(T) == 2) static_cast<bf16_t*>(a.out)[o0 + e] = round_bf16(x);
        else static_cast<float*>(a.out)[o0 + e] = x;
    };
    store(lane, o1 * inv);
    if (hd == 128) store(lane + 64, o2 * inv);
}

}  // namespace

size_t kv_attention_workspace(const riftkv_cache&, int, int64_t, int64_t) { return 256; }

hipError_t launch_kv_attention(const riftkv_cache& c, const KvAttention& a, hipStream_t st) {
    const dim3 grid((unsigned)a.n_seq * (unsigned)a.n_heads);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64), 0, st, c, a); };
    switch (c.dt) {
        case RIFTKV_F32: launch(attention_kernel<float, RIFTKV_F32>); break;
        case RIFTKV_BF16: a.bf16 ? launch(attention_kernel<bf16_t, RIFTKV_BF16>) : launch(attention_kernel<float, RIFTKV_BF16>); break;
        case RIFTKV_FP8: a.bf16 ? launch(attention_kernel<bf16_t, RIFTKV_FP8>) : launch(attention_kernel<float, RIFTKV_FP8>); break;
        case RIFTKV_INT8: a.bf16 ? launch(attention_kernel<bf16_t, RIFTKV_INT8>) : launch(attention_kernel<float, RIFTKV_INT8>); break;
    }
    return hipGetLastError();
}

}  // namespace rift
