// Native driver of tests/test_kv_ranges_sanitize.py: the host layer of the paged cache's calls for long contexts.  Every call is
// given arguments that validation refuses, or nothing to do, so that none reaches a HIP call.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <vector>

#include "../../include/rift_kv.h"

static int g_checks = 0, g_failed = 0;
#define EXPECT(cond)                                                         \
    do {                                                                     \
        ++g_checks;                                                          \
        if (!(cond)) {                                                       \
            ++g_failed;                                                      \
            std::printf("FAILED %s:%d %s\n", __FILE__, __LINE__, #cond);     \
        }                                                                    \
    } while (0)

// An enum field with any bits, as a C caller may leave it.
template <typename E>
static void set_bits(E& e, int v) {
    std::memcpy(&e, &v, sizeof e);
}

static void* const P = reinterpret_cast<void*>(0x10000);
static int32_t* const PI = static_cast<int32_t*>(P);
static constexpr size_t kAll = ~(size_t)0;

static riftkv_cache pages(int dt = RIFTKV_FP8) {
    riftkv_cache c{};
    c.k = c.v = P;
    c.k_scale = c.v_scale = static_cast<uint8_t*>(P);
    c.n_pages = 8;
    c.page_size = 16;
    c.n_kv_heads = 4;
    c.head_dim = 128;
    set_bits(c.dt, dt);
    return c;
}

static rift_status rope(int R, int n_axes, const int32_t* axes, int rows) {
    std::vector<double> f(R > 0 ? R / 2 : 0, 1.0);
    return riftkv_rope_axes(P, 1 << 20, 1, P, 1 << 20, nullptr, 0, 0, nullptr, 0, RIFT_BF16, PI, n_axes, rows, 256, R,
                            RIFTKV_ROPE_HALF, f.data(), axes, 1.0, nullptr);
}
static rift_status shared(const riftkv_cache& c, int heads, int n_seq, int prefix, int max_pages, size_t ws = kAll) {
    return riftkv_attention_shared(&c, P, 1 << 20, heads, RIFT_F32, PI, prefix, PI, n_seq, max_pages, PI, 0.1f, P, 1 << 20,
                                   PI, P, ws, nullptr);
}
static rift_status choose(const riftkv_cache& c, int heads, int n_seq, int max_pages, int first, int last, int top, size_t ws = kAll) {
    return riftkv_select_pages(&c, P, P, 1 << 20, heads, RIFT_F32, PI, n_seq, max_pages, PI, first, last, PI, top, PI, P, ws, nullptr);
}
static rift_status listed(const riftkv_cache& c, int heads, int n_seq, int max_pages, int top, size_t ws = kAll) {
    return riftkv_attention_pages(&c, P, 1 << 20, heads, RIFT_F32, PI, n_seq, max_pages, PI, PI, top, 0.1f, P, 1 << 20, PI, P, ws, nullptr);
}

int main() {
    // positions of several axes: the arrays of every size are read to their ends and no further; every axis that is refused
    for (int R = -2; R <= 260; ++R) {
        std::vector<int32_t> axes(R > 0 ? R / 2 : 0, 0);
        const bool good = R >= 2 && R <= 256 && R % 2 == 0;
        EXPECT(rope(R, 3, axes.data(), 0) == (good ? RIFT_OK : RIFT_ERR_SHAPE));
        if (!good) continue;
        for (int bad : {-1, 3, INT32_MAX, INT32_MIN})
            for (size_t at : {(size_t)0, axes.size() - 1}) {
                std::vector<int32_t> x = axes;
                x[at] = bad;
                EXPECT(rope(R, 3, x.data(), 5) == RIFT_ERR_SHAPE);
            }
        EXPECT(rope(R, 3, nullptr, 5) == RIFT_ERR_NULL);
    }
    std::vector<int32_t> axes(64, 0);
    for (int n : {INT32_MIN, -1, 0, 9, INT32_MAX}) EXPECT(rope(128, n, axes.data(), 5) == RIFT_ERR_SHAPE);
    // pages: every size that is refused, in every call
    for (int dt = -2; dt <= 6; ++dt)
        for (int page : {0, 8, 16, 48, 4096, 8192})
            for (int n : {0, 1, 1 << 27})
                for (int hd : {0, 64, 96, 128}) {
                    riftkv_cache c = pages(dt);
                    c.page_size = page;
                    c.n_pages = n;
                    c.head_dim = hd;
                    const bool shape = (page == 16 || page == 4096) && n == 1 && hd > 0;
                    const rift_status want = dt < 0 || dt > 3 ? RIFT_ERR_DTYPE
                        : !shape ? RIFT_ERR_SHAPE : hd == 96 ? RIFT_ERR_UNSUPPORTED : RIFT_OK;
                    EXPECT((riftkv_attention_shared_workspace_size(&c, 8, 2, 100, 1) > 0) == (want == RIFT_OK));
                    EXPECT((riftkv_select_pages_workspace_size(&c, 2, 1) > 0) == (want == RIFT_OK));
                    EXPECT((riftkv_attention_pages_workspace_size(&c, 8, 2, 4) > 0) == (want == RIFT_OK));
                    EXPECT(shared(c, 8, 0, 100, 1) == want);
                    EXPECT(choose(c, 8, 0, 1, 1, 1, 4) == want);
                    EXPECT(listed(c, 8, 0, 1, 4) == want);
                    EXPECT(riftkv_page_bounds(&c, P, PI, 0, 1, nullptr, PI, PI, nullptr) == want);
                }
    // workspaces: no overflow at the largest shapes, never smaller for more, a byte too few refused
    const int many[] = {0, 1, 2, 3, 31, 33, 128, 1000, 16383, 16384};
    for (int dt = 0; dt < 4; ++dt)
        for (int hd : {64, 128}) {
            riftkv_cache c = pages(dt);
            c.head_dim = hd;
            for (int prefix : {0, 1, 256, 257, 1 << 20, 1 << 30}) {
                size_t last = 0;
                for (int n : many) {
                    const size_t s = riftkv_attention_shared_workspace_size(&c, 4096, n, prefix, 1 << 26);
                    EXPECT(s >= last && s > 0 && s < ((size_t)1 << 38));
                    if (n > 0) EXPECT(shared(c, 4096, n, prefix, 1 << 26, s - 1) == RIFT_ERR_WORKSPACE);
                    last = s;
                }
                EXPECT(riftkv_attention_shared_workspace_size(&c, 4096, 16385, prefix, 1) == 0);
                EXPECT(shared(c, 4096, 16385, prefix, 1) == RIFT_ERR_SHAPE);
            }
            size_t last = 0;
            for (int prefix : {0, 1, 256, 257, 1 << 20, 1 << 30}) {
                const size_t s = riftkv_attention_shared_workspace_size(&c, 64, 40, prefix, 100);
                EXPECT(s >= last);
                last = s;
            }
            for (int n : {1, 65535}) {
                const size_t s = riftkv_select_pages_workspace_size(&c, n, 1 << 26);
                EXPECT(s == (size_t)n * 4 * 8 * ((size_t)1 << 26));
                EXPECT(choose(c, 8, n, 1 << 26, 0, 0, 1 << 20, s - 1) == RIFT_ERR_WORKSPACE);
                const size_t l = riftkv_attention_pages_workspace_size(&c, 4096, n, 1 << 20);
                EXPECT(l > 0 && listed(c, 4096, n, 1 << 26, 1 << 20, l - 1) == RIFT_ERR_WORKSPACE);
            }
        }
    riftkv_cache c = pages();
    for (int v : {-1, (1 << 30) + 1, INT32_MAX, INT32_MIN}) {
        EXPECT(shared(c, 8, 1, v, 1) == RIFT_ERR_SHAPE);
        EXPECT(riftkv_attention_shared_workspace_size(&c, 8, 1, v, 1) == 0);
        EXPECT(choose(c, 8, 1, 1, v, 0, 4) == RIFT_ERR_SHAPE);
        EXPECT(choose(c, 8, 1, 1, 0, v, 4) == RIFT_ERR_SHAPE);
        EXPECT(choose(c, 8, 1, 1, 0, 0, v) == RIFT_ERR_SHAPE);
        EXPECT(listed(c, 8, 1, 1, v) == RIFT_ERR_SHAPE);
        EXPECT(riftkv_attention_pages_workspace_size(&c, 8, 1, v) == 0);
        EXPECT(riftkv_page_bounds(&c, P, PI, 1, v, nullptr, PI, PI, nullptr) == RIFT_ERR_SHAPE);
        EXPECT(riftkv_page_bounds(&c, P, PI, v, 1, nullptr, PI, PI, nullptr) == RIFT_ERR_SHAPE);
        EXPECT(riftkv_select_pages_workspace_size(&c, v, 1) == 0 && riftkv_select_pages_workspace_size(&c, 1, v) == 0);
        EXPECT(shared(c, v, 1, 100, 1) == RIFT_ERR_SHAPE && listed(c, v, 1, 1, 4) == RIFT_ERR_SHAPE);
    }
    EXPECT(choose(c, 8, 1, 1, INT32_MAX, INT32_MAX, 1 << 20) == RIFT_ERR_SHAPE);
    EXPECT(riftkv_attention_shared_workspace_size(nullptr, 8, 1, 1, 1) == 0 && riftkv_select_pages_workspace_size(nullptr, 1, 1) == 0 &&
           riftkv_attention_pages_workspace_size(nullptr, 8, 1, 1) == 0);
    EXPECT(riftkv_attention_shared(&c, P, 1024, 8, RIFT_F32, PI, 100, PI, 1, 1, PI, 3e38f, P, 1024, PI, P, kAll, nullptr) == RIFT_ERR_NONFINITE);
    EXPECT(riftkv_attention_pages(&c, P, 1024, 8, RIFT_F32, PI, 1, 1, PI, PI, 4, NAN, P, 1024, PI, P, kAll, nullptr) == RIFT_ERR_NONFINITE);
    EXPECT(riftkv_attention_shared(&c, P, 1024, 8, RIFT_F32, nullptr, 100, PI, 1, 1, PI, 0.1f, P, 1024, PI, P, kAll, nullptr) == RIFT_ERR_NULL);
    std::printf("%d checks, %d failed\n", g_checks, g_failed);
    return g_failed ? 1 : 0;
}
