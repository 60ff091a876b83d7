// Native driver of tests/test_kv_sanitize.py: the host layer of the paged key-value
// cache.  Host-only calls run over their range; device calls are given arguments that
// validation refuses, or nothing to do, so that none reaches a HIP call.
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

int main() {
    EXPECT(riftkv_abi_version() == RIFTKV_ABI_VERSION);
    // frequencies: every even size exactly fills its buffer
    for (int scaling = 0; scaling <= 4; ++scaling)
        for (int R = 2; R <= 256; R += 2) {
            riftkv_rope_cfg f{R, RIFTKV_ROPE_NONE, 10000.0, 4.0, 4096.0, 1.0, 32.0};
            set_bits(f.scaling, scaling);
            std::vector<double> out(R / 2);
            double mag = 0.0;
            const rift_status s = riftkv_rope_freqs(&f, out.data(), &mag);
            EXPECT(s == (scaling == RIFTKV_ROPE_BASE && R == 2 ? RIFT_ERR_SHAPE : RIFT_OK));
            if (s == RIFT_OK)
                for (double x : out) EXPECT(std::isfinite(x) && x > 0.0 && x <= 1.0);
            EXPECT(riftkv_rope_freqs(&f, out.data(), nullptr) == s);
        }
    double one[128];
    for (double& x : one) x = 1.0;
    for (int scaling : {-1, 5, 1 << 30}) {
        riftkv_rope_cfg f{64, RIFTKV_ROPE_NONE, 10000.0, 4.0, 4096.0, 1.0, 32.0};
        set_bits(f.scaling, scaling);
        EXPECT(riftkv_rope_freqs(&f, one, nullptr) == RIFT_ERR_UNSUPPORTED);
    }
    EXPECT(riftkv_rope_freqs(nullptr, one, nullptr) == RIFT_ERR_NULL);
    EXPECT(riftkv_rope(P, 64, 1, P, 64, P, 64, 1, P, 64, RIFT_BF16, PI, 0, 64, 64, RIFTKV_ROPE_HALF, one, 1.0, nullptr) == RIFT_OK);
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
                    EXPECT(riftkv_write(&c, P, 512, P, 512, RIFT_F32, PI, 1, 1, nullptr, PI, 0, PI, nullptr) == want);
                    EXPECT(riftkv_read(&c, P, 512, P, 512, RIFT_F32, PI, 1, 1, nullptr, PI, 0, PI, nullptr) == want);
                    const size_t ws = riftkv_attention_workspace_size(&c, 8, 2, 1);
                    EXPECT((ws > 0) == (want == RIFT_OK));
                    EXPECT(riftkv_attention(&c, P, 1024, 8, RIFT_F32, PI, 0, 1, PI, 0.1f, P, 1024, PI, P, 1u << 30, nullptr) == want);
                }
    // workspaces: no overflow at the largest shapes, never smaller for more
    riftkv_cache c = pages();
    size_t last = 0;
    for (int n = 0; n <= 65535; n = 2 * n + 1) {
        const size_t s = riftkv_attention_workspace_size(&c, 4096, n, 1 << 26);
        EXPECT(s >= last && s < (64u << 20));
        last = s;
    }
    EXPECT(riftkv_attention_workspace_size(&c, 4, INT32_MAX, INT32_MAX) == 0);
    EXPECT(riftkv_attention_workspace_size(&c, INT32_MAX, 1, 1) == 0);
    EXPECT(riftkv_attention(&c, P, 512, 4, RIFT_BF16, PI, 65535, 1 << 26, PI, 0.1f, P, 512, PI, P, 1u << 30, nullptr) ==
           RIFT_ERR_UNSUPPORTED);
    EXPECT(riftkv_attention(&c, P, 512, 4, RIFT_BF16, PI, 1, 1, PI, 3e38f, P, 512, PI, P, 1u << 30, nullptr) ==
           RIFT_ERR_NONFINITE);
    rift_model_cfg m{512, 4, 128, 1408, 2, 1e-6f, 1e4f, RIFT_BF16};
    last = 0;
    for (int n = 0; n <= 65535; n = 2 * n + 1) {
        const size_t s = riftkv_decode_workspace_size(&m, &c, n, 64);
        EXPECT(s >= last && s > 0);
        last = s;
    }
    EXPECT(riftkv_decode_workspace_size(&m, &c, INT32_MAX, 64) == 0);
    EXPECT(riftkv_decode_workspace_size(nullptr, &c, 1, 1) == 0 && riftkv_decode_workspace_size(&m, nullptr, 1, 1) == 0);
    rift_layer_weights w[2]{};
    EXPECT(riftkv_decode_step(&m, w, P, &c, PI, 1, 1, PI, static_cast<float*>(P), PI, P, 1u << 30, nullptr) == RIFT_ERR_NULL);
    EXPECT(riftkv_decode_step(&m, w, P, &c, PI, 0, 1, PI, static_cast<float*>(P), PI, P, 1u << 30, nullptr) == RIFT_OK);
    std::printf("%d checks, %d failed\n", g_checks, g_failed);
    return g_failed ? 1 : 0;
}
