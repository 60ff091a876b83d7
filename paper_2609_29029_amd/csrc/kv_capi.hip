// C ABI of the paged key-value cache: argument validation and kernel launches.
#include <math.h>
#include <string.h>

#include "kv.h"

using namespace rift;

namespace {

// A caller may pass any integer as an enum: its first inspection reads the bits.
template <typename E>
inline int enum_bits(const E& e) {
    int v = 0;
    memcpy(&v, &e, sizeof v);
    return v;
}

inline bool rows_dt_valid(const rift_dtype& dt) {
    const int v = enum_bits(dt);
    return v == (int)RIFT_BF16 || v == (int)RIFT_F32;
}

inline bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

inline rift_status hip_status(hipError_t e) { return e == hipSuccess ? RIFT_OK : RIFT_ERR_HIP; }

}  // namespace

namespace rift {

rift_status kv_check_cache(const riftkv_cache* c, bool arrays) {
    if (c == nullptr) return RIFT_ERR_NULL;
    const int dt = enum_bits(c->dt);
    if (dt < (int)RIFTKV_F32 || dt > (int)RIFTKV_INT8) return RIFT_ERR_DTYPE;
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0 || c->n_pages < 1 ||
        (int64_t)c->n_pages * c->page_size > INT32_MAX || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->head_dim < 1)
        return RIFT_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return RIFT_ERR_UNSUPPORTED;
    if (!arrays) return RIFT_OK;
    const bool scaled = dt == (int)RIFTKV_FP8 || dt == (int)RIFTKV_INT8;
    if (c->k == nullptr || c->v == nullptr || (scaled && (c->k_scale == nullptr || c->v_scale == nullptr)))
        return RIFT_ERR_NULL;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || (scaled && (misaligned(c->k_scale, 16) || misaligned(c->v_scale, 16))))
        return RIFT_ERR_SHAPE;
    return RIFT_OK;
}

}  // namespace rift

namespace {

bool check_table(const riftkv_cache& c, int32_t n_seq, int32_t max_pages) {
    return n_seq >= 0 && max_pages >= 0 && (int64_t)max_pages * c.page_size <= kMaxTokens;
}

// A row set [rows][heads * head_dim], `ld` elements apart (16 bytes hold 8 or 4)
bool check_rows(const void* x, int64_t ld, int64_t width, rift_dtype dt) {
    const int64_t per = dt == RIFT_BF16 ? 8 : 4;
    return !misaligned(x, 16) && ld >= width && ld % per == 0;
}

// Shared by writes and reads.
rift_status check_places(const riftkv_cache* cache, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         const rift_dtype& dt, const int32_t* table, int32_t n_seq, int32_t max_pages,
                         const int32_t* positions, int32_t rows, int32_t* status) {
    const rift_status cs = kv_check_cache(cache, true);
    if (cs != RIFT_OK) return cs;
    if (!rows_dt_valid(dt)) return RIFT_ERR_DTYPE;
    if (rows < 0 || !check_table(*cache, n_seq, max_pages)) return RIFT_ERR_SHAPE;
    if (status == nullptr) return RIFT_ERR_NULL;
    if (rows == 0) return RIFT_OK;
    if (k == nullptr || v == nullptr || positions == nullptr || (table == nullptr && n_seq > 0 && max_pages > 0))
        return RIFT_ERR_NULL;
    const int64_t width = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (!check_rows(k, ld_k, width, dt) || !check_rows(v, ld_v, width, dt)) return RIFT_ERR_SHAPE;
    return RIFT_OK;
}

// a grid of this many small workgroups, or of blocks of them
constexpr int64_t kMostItems = 1ll << 31;

}  // namespace

extern "C" {

int32_t riftkv_abi_version(void) { return RIFTKV_ABI_VERSION; }

rift_status riftkv_rope_freqs(const riftkv_rope_cfg* cfg, double* freqs, double* magnitude) {
    if (cfg == nullptr || freqs == nullptr) return RIFT_ERR_NULL;
    const int kind = enum_bits(cfg->scaling);
    if (kind < (int)RIFTKV_ROPE_NONE || kind > (int)RIFTKV_ROPE_BANDS) return RIFT_ERR_UNSUPPORTED;
    const int R = cfg->rotary_dim;
    if (R < 2 || R > kMaxRotary || R % 2 != 0 || (kind == (int)RIFTKV_ROPE_BASE && R == 2)) return RIFT_ERR_SHAPE;
    const bool ranged = kind == (int)RIFTKV_ROPE_RAMP || kind == (int)RIFTKV_ROPE_BANDS;
    if (!(isfinite(cfg->base) && cfg->base > 1.0)) return RIFT_ERR_NONFINITE;
    if (kind != (int)RIFTKV_ROPE_NONE && !(isfinite(cfg->factor) && cfg->factor >= 1.0)) return RIFT_ERR_NONFINITE;
    if (ranged && !(isfinite(cfg->original_len) && cfg->original_len > 0.0 && isfinite(cfg->high) && cfg->low > 0.0 &&
                    cfg->low < cfg->high))
        return RIFT_ERR_NONFINITE;
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    double base = cfg->base, a = 0.0, b = 0.0;
    if (kind == (int)RIFTKV_ROPE_BASE) base *= pow(cfg->factor, (double)R / (double)(R - 2));
    if (!isfinite(base)) return RIFT_ERR_NONFINITE;
    if (kind == (int)RIFTKV_ROPE_RAMP) {
        auto pair_of = [&](double turns) { return R * log(cfg->original_len / (kTwoPi * turns)) / (2.0 * log(base)); };
        a = fmax(floor(pair_of(cfg->high)), 0.0);
        b = fmin(ceil(pair_of(cfg->low)), (double)(R - 1));
        if (b <= a) b = a + 0.001;
    }
    for (int j = 0; j < R / 2; ++j) {
        double f = pow(base, -2.0 * j / R);
        if (kind == (int)RIFTKV_ROPE_LINEAR) f /= cfg->factor;
        if (kind == (int)RIFTKV_ROPE_RAMP) {
            const double r = fmin(fmax((j - a) / (b - a), 0.0), 1.0);
            f = f * (1.0 - r) + f / cfg->factor * r;
        }
        if (kind == (int)RIFTKV_ROPE_BANDS) {
            const double n = cfg->original_len * f / kTwoPi;
            const double s = fmin(fmax((n - cfg->low) / (cfg->high - cfg->low), 0.0), 1.0);
            f = f * s + f / cfg->factor * (1.0 - s);
        }
        freqs[j] = f;
    }
    if (magnitude != nullptr) *magnitude = kind == (int)RIFTKV_ROPE_RAMP ? 1.0 + 0.1 * log(cfg->factor) : 1.0;
    return RIFT_OK;
}

rift_status riftkv_rope(const void* q, int64_t ld_q, int32_t n_q, void* q_out, int64_t ld_q_out, const void* k,
                        int64_t ld_k, int32_t n_k, void* k_out, int64_t ld_k_out, rift_dtype dt,
                        const int32_t* positions, int32_t rows, int32_t head_dim, int32_t rotary_dim,
                        riftkv_rope_layout layout, const double* freqs, double magnitude, rift_stream stream) {
    if (!rows_dt_valid(dt)) return RIFT_ERR_DTYPE;
    const int lay = enum_bits(layout);
    if (lay != (int)RIFTKV_ROPE_HALF && lay != (int)RIFTKV_ROPE_INTERLEAVED) return RIFT_ERR_UNSUPPORTED;
    if (rows < 0 || n_q < 0 || n_q > 4096 || n_k < 0 || n_k > 4096 || head_dim < 1 || head_dim > 256 || rotary_dim < 2 ||
        rotary_dim > head_dim || rotary_dim % 2 != 0)
        return RIFT_ERR_SHAPE;
    if (freqs == nullptr) return RIFT_ERR_NULL;
    RopeFreqs f;
    // 2 pi = kTwoPi + kTwoPiRest, to 2^-109 of it
    constexpr double kTwoPi = 6.283185307179586476925286766559, kTwoPiRest = 2.4492935982947064e-16;
    for (int j = 0; j < rotary_dim / 2; ++j) {
        if (!isfinite(freqs[j])) return RIFT_ERR_NONFINITE;
        f.hi[j] = freqs[j] / kTwoPi;
        f.lo[j] = (float)((fma(-f.hi[j], kTwoPi, freqs[j]) - f.hi[j] * kTwoPiRest) * (1.0 / kTwoPi));
    }
    if (!isfinite((float)magnitude)) return RIFT_ERR_NONFINITE;
    if (rows == 0 || n_q + n_k == 0) return RIFT_OK;
    if (positions == nullptr || (n_q > 0 && (q == nullptr || q_out == nullptr)) ||
        (n_k > 0 && (k == nullptr || k_out == nullptr)))
        return RIFT_ERR_NULL;
    const int64_t wq = (int64_t)n_q * head_dim, wk = (int64_t)n_k * head_dim;
    if ((n_q > 0 && (ld_q < wq || ld_q_out < wq)) || (n_k > 0 && (ld_k < wk || ld_k_out < wk))) return RIFT_ERR_SHAPE;
    if ((n_q > 0 && q == q_out && ld_q != ld_q_out) || (n_k > 0 && k == k_out && ld_k != ld_k_out)) return RIFT_ERR_SHAPE;
    if ((int64_t)rows * (n_q + n_k) >= kMostItems) return RIFT_ERR_UNSUPPORTED;
    const RopeRows rq{q, q_out, ld_q, ld_q_out, n_q}, rk{k, k_out, ld_k, ld_k_out, n_k};
    return hip_status(launch_kv_rope(rq, rk, dt == RIFT_BF16, positions, rows, head_dim, rotary_dim,
                                     lay == (int)RIFTKV_ROPE_INTERLEAVED, f, (float)magnitude,
                                     static_cast<hipStream_t>(stream)));
}

rift_status riftkv_write(const riftkv_cache* cache, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         rift_dtype dt, const int32_t* page_table, int32_t n_seq, int32_t max_pages,
                         const int32_t* seq_ids, const int32_t* positions, int32_t rows, int32_t* status,
                         rift_stream stream) {
    const rift_status cs = check_places(cache, k, ld_k, v, ld_v, dt, page_table, n_seq, max_pages, positions, rows, status);
    if (cs != RIFT_OK) return cs;
    if (dt == RIFT_BF16 && cache->dt == RIFTKV_F32) return RIFT_ERR_DTYPE;
    if (rows == 0) return RIFT_OK;
    if ((int64_t)rows * cache->n_kv_heads >= kMostItems) return RIFT_ERR_UNSUPPORTED;
    const KvPlaces at{page_table, n_seq, max_pages, seq_ids, positions, rows, status};
    return hip_status(launch_kv_write(*cache, k, ld_k, v, ld_v, dt == RIFT_BF16, at, static_cast<hipStream_t>(stream)));
}

rift_status riftkv_read(const riftkv_cache* cache, void* k_out, int64_t ld_k, void* v_out, int64_t ld_v, rift_dtype dt,
                        const int32_t* page_table, int32_t n_seq, int32_t max_pages, const int32_t* seq_ids,
                        const int32_t* positions, int32_t rows, int32_t* status, rift_stream stream) {
    const rift_status cs =
        check_places(cache, k_out, ld_k, v_out, ld_v, dt, page_table, n_seq, max_pages, positions, rows, status);
    if (cs != RIFT_OK) return cs;
    if (rows == 0) return RIFT_OK;
    if ((int64_t)rows * cache->n_kv_heads >= kMostItems) return RIFT_ERR_UNSUPPORTED;
    const KvPlaces at{page_table, n_seq, max_pages, seq_ids, positions, rows, status};
    return hip_status(launch_kv_read(*cache, k_out, ld_k, v_out, ld_v, dt == RIFT_BF16, at, static_cast<hipStream_t>(stream)));
}

namespace {
bool attention_shape(const riftkv_cache& c, int32_t n_heads, int32_t n_seq, int32_t max_pages) {
    return n_heads >= 1 && n_heads <= 4096 && n_heads % c.n_kv_heads == 0 && n_seq <= 65535 && check_table(c, n_seq, max_pages);
}
}  // namespace

size_t riftkv_attention_workspace_size(const riftkv_cache* cache, int32_t n_heads, int32_t n_seq, int32_t max_pages) {
    if (kv_check_cache(cache, false) != RIFT_OK || !attention_shape(*cache, n_heads, n_seq, max_pages)) return 0;
    return kv_attention_workspace(*cache, n_heads, n_seq, max_pages);
}

rift_status riftkv_attention(const riftkv_cache* cache, const void* q, int64_t ld_q, int32_t n_heads, rift_dtype dt,
                             const int32_t* page_table, int32_t n_seq, int32_t max_pages, const int32_t* lens,
                             float scale, void* out, int64_t ld_out, int32_t* status, void* workspace, size_t ws_bytes,
                             rift_stream stream) {
    const rift_status cs = kv_check_cache(cache, true);
    if (cs != RIFT_OK) return cs;
    if (!rows_dt_valid(dt) || (dt == RIFT_BF16 && cache->dt == RIFTKV_F32)) return RIFT_ERR_DTYPE;
    if (!attention_shape(*cache, n_heads, n_seq, max_pages)) return RIFT_ERR_SHAPE;
    if (!kv_attention_counts(*cache, n_heads, n_seq, max_pages)) return RIFT_ERR_UNSUPPORTED;
    if (!isfinite(scale * 1.4426950408889634f)) return RIFT_ERR_NONFINITE;   // the base-2 exponent's
    if (status == nullptr || workspace == nullptr) return RIFT_ERR_NULL;
    if (misaligned(workspace, 256) || ws_bytes < kv_attention_workspace(*cache, n_heads, n_seq, max_pages))
        return RIFT_ERR_WORKSPACE;
    if (n_seq == 0) return RIFT_OK;
    if (q == nullptr || out == nullptr || lens == nullptr || (page_table == nullptr && max_pages > 0)) return RIFT_ERR_NULL;
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    if (!check_rows(q, ld_q, width, dt) || !check_rows(out, ld_out, width, dt)) return RIFT_ERR_SHAPE;
    const KvAttention a{q, out, ld_q, ld_out, n_heads, dt == RIFT_BF16, page_table, n_seq, max_pages, lens, scale, status, workspace};
    return hip_status(launch_kv_attention(*cache, a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
