// Host-side driver for the sanitizer build of the 4-bit caches' entry points, attention weights, eviction and 4-bit products (no GPU): validation over a
// sweep of sizes and extreme values. Device pointers are fake and never dereferenced: in every call something is wrong, so that it returns before a launch.
#include "sp.h"

#include <cstdio>
#include <vector>

static int g_fail = 0;
#define EXPECT(cond)                                                                                                        \
    do {                                                                                                                    \
        if (!(cond)) { std::printf("FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, #cond, sp_last_error()); ++g_fail; } \
    } while (0)

static bool bad(sp_status rc) { return rc == SP_ERR_INVALID_ARG || rc == SP_ERR_UNSUPPORTED; }

int main()
{
    void *fake = reinterpret_cast<void *>(0x10000), *odd = reinterpret_cast<void *>(0x10001);
    float *ff = static_cast<float *>(fake);
    int32_t *fi = static_cast<int32_t *>(fake);
    const int64_t *fo = static_cast<const int64_t *>(fake);
    const int64_t extremes[] = {INT64_MIN, -1, 0, 1, 31, 32, 64, 4096, (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX};
    std::vector<int64_t> off(4097 + 1);
    for (size_t i = 0; i < off.size(); ++i) off[i] = (int64_t)i;
    for (int d : {64, 96, 128})
        for (int kv : {1, 8, 4096, 4097})
            for (int64_t page : extremes)
                for (int64_t stride : extremes) {
                    sp_cache_desc c{kv, kv, d, SP_CACHE_MX4, 8, page, stride, stride, stride};
                    for (int32_t B : {-1, 0, 1, 64, 4096, 4097})
                        for (int64_t len : extremes) {
                            size_t n = 0;
                            const sp_status rc = sp_attend_workspace(&c, off.data(), B, len, &n);
                            EXPECT(rc == SP_OK || bad(rc));
                            if (rc == SP_OK) EXPECT(n % 256 == 0);
                            if (B == 0) continue;
                            // the pool's address is bad throughout, unless there is nothing to do
                            const sp_status w = sp_attend_weights(&c, fake, off.data(), fo, B, fi, len, fi, (int64_t)1 << 31, odd, fake, 1.f, 1, 0, ff, ff, ff,
                                                                  len < 0 ? 0 : len, nullptr);
                            EXPECT(len == 0 ? w == SP_OK || bad(w) : bad(w));
                            EXPECT(bad(sp_cache_evict(&c, B, fi, len, fi, len, 0, 0, ff, len < 0 ? 0 : len, fi, (int64_t)1 << 31, fi, 1, odd, fake, fake, fake, fi + 1, fi,
                                                      nullptr, nullptr)));
                        }
                }
    sp_cache_desc ok{8, 2, 64, SP_CACHE_MX4, 4, 64, 8192, 4096, 64};
    const int64_t two[] = {0, 3}, huge[] = {0, INT64_MAX}, down[] = {0, INT64_MIN}, over[] = {0, (1 << 26) + 1};
    for (int64_t s : extremes)
        for (int64_t t : extremes)
            for (int64_t u : extremes) {
                EXPECT(bad(sp_attend_weights(&ok, fake, two, fo, 1, fi, s, fi, t, odd, fake, 1.f, 1, u, ff, ff, ff, t, nullptr)) || s == 0);
                EXPECT(bad(sp_attend_weights(&ok, fake, two, fo, 1, fi, 64, fi, 1, fake, fake, 0.f, 1, u, ff, ff, ff, t, nullptr)));
                EXPECT(bad(sp_cache_evict(&ok, 1, fi, s, fi, t, u, u, ff, s, fi, t, fi, u, fake, fake, fake, odd, fi + 1, fi, ff + 1, nullptr)));
                for (int32_t type : {INT32_MIN, -1, 0, 1, 2, INT32_MAX}) {
                    EXPECT(bad(sp_mx4_quantise(odd, type, s, t, u, fake, fake, nullptr)) || s == 0);
                    EXPECT(bad(sp_mx4_matmul(fake, fake, s, odd, fake, t, u, fake, type, t, nullptr)) || s == 0 || t == 0);
                }
            }
    for (const int64_t *o : {huge, down, over}) EXPECT(bad(sp_attend_weights(&ok, fake, o, fo, 1, fi, 64, fi, 1, fake, fake, 1.f, 1, 0, ff, ff, ff, 64, nullptr)));
    EXPECT(bad(sp_attend_weights(nullptr, fake, two, fo, 1, fi, 64, fi, 1, fake, fake, 1.f, 1, 0, ff, ff, ff, 64, nullptr)));
    EXPECT(bad(sp_attend_weights(&ok, fake, nullptr, fo, 1, fi, 64, fi, 1, fake, fake, 1.f, 1, 0, ff, ff, ff, 64, nullptr)));
    EXPECT(bad(sp_cache_evict(nullptr, 1, fi, 64, fi, 64, 0, 0, ff, 64, fi, 1, fi, 1, fake, fake, fake, fake, fi + 1, fi, nullptr, nullptr)));
    EXPECT(sp_mx4_matmul(fake, fake, INT32_MAX, fake, fake, INT32_MAX, 32, fake, SP_LOGITS_F32, INT32_MAX, nullptr) == SP_ERR_UNSUPPORTED);
    EXPECT(sp_mx4_quantise(fake, SP_LOGITS_F32, INT32_MAX, ((int64_t)1 << 31) - 32, (int64_t)1 << 31, fake, fake, nullptr) == SP_ERR_UNSUPPORTED);
    if (g_fail) return 1;
    std::printf("all checks passed\n");
    return 0;
}
