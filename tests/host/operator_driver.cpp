// Host-side driver for the sanitizer build of the cache, attention and log-probability entry points (no GPU): workspace
// arithmetic and validation over a sweep of shapes, sizes and extreme values. Device pointers are fake and never dereferenced: every call returns before a
// launch.
#include "sp.h"

#include <cstdio>
#include <vector>

static int g_fail = 0;
#define EXPECT(cond)                                                                                                        \
    do {                                                                                                                    \
        if (!(cond)) { std::printf("FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, #cond, sp_last_error()); ++g_fail; } \
    } while (0)

int main()
{
    void *fake = reinterpret_cast<void *>(0x10000);
    float *ff = static_cast<float *>(fake);
    int32_t *fi = static_cast<int32_t *>(fake);
    const int64_t extremes[] = {INT64_MIN, -1, 0, 1, 31, 32, 64, 4096, (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX};
    std::vector<int64_t> off(4097 + 1);
    for (size_t i = 0; i < off.size(); ++i) off[i] = (int64_t)i;
    for (int d : {64, 96, 128})
        for (int kv : {1, 8, 4096, 4097})
            for (int g : {1, 4, 16, 17})
                for (int type : {0, 1, 2})
                    for (int64_t page : extremes)
                        for (int64_t stride : extremes) {
                            sp_cache_desc c{kv * g, kv, d, type, 8, page, stride, stride, d};
                            for (int32_t B : {-1, 0, 1, 64, 4096, 4097})
                                for (int64_t len : {(int64_t)0, (int64_t)1, (int64_t)100000, (int64_t)INT32_MAX, (int64_t)1 << 40, (int64_t)-1}) {
                                    size_t n = 0;
                                    const sp_status rc = sp_attend_workspace(&c, off.data(), B, len, &n);
                                    EXPECT(rc == SP_OK || rc == SP_ERR_INVALID_ARG || rc == SP_ERR_UNSUPPORTED);
                                    if (rc == SP_OK) EXPECT(n % 256 == 0);
                                }
                        }
    sp_cache_desc ok{8, 2, 64, SP_CACHE_E4M3, 4, 64, 8192, 4096, 64};
    const int64_t two[] = {0, 3}, huge[] = {0, INT64_MAX}, big[] = {0, 1 << 26}, over[] = {0, (1 << 26) + 1}, down[] = {0, INT64_MIN};
    size_t n = 0;
    EXPECT(sp_attend_workspace(&ok, huge, 1, 64, &n) == SP_ERR_INVALID_ARG);
    EXPECT(sp_attend_workspace(&ok, down, 1, 64, &n) == SP_ERR_INVALID_ARG);
    EXPECT(sp_attend_workspace(&ok, big, 1, 1 << 30, &n) == SP_OK && n % 256 == 0);
    EXPECT(sp_attend_workspace(&ok, big, 1, (1 << 30) + 1, &n) == SP_ERR_INVALID_ARG);
    EXPECT(sp_attend_workspace(&ok, over, 1, 64, &n) == SP_ERR_UNSUPPORTED);
    for (int64_t s : extremes)
        for (int64_t t : extremes)
            for (int64_t np : extremes)
                for (int32_t rot : {INT32_MIN, -16, 8, 80, INT32_MAX}) {
                    // rot_dim is bad throughout: nothing is launched whatever the rest says
                    EXPECT(sp_cache_append(&ok, fake, s, fake, s, fake, s, fake, two, (const int64_t *)fake, 1, fi, fi, fi, t, ff, ff, np, rot, 0,
                                           fake, fake, ff, ff, nullptr) == SP_ERR_INVALID_ARG);
                    EXPECT(sp_attend(&ok, fake, two, (const int64_t *)fake, 1, fi, s, fi, t, fake, fake, ff, ff, 0.f, 1, np, fake, ff, fake, 0,
                                     nullptr) == SP_ERR_INVALID_ARG);
                    EXPECT(sp_logprobs(fake, 7, s, t, np, fi, rot, ff, ff, fi, ff, fake, 0, nullptr) == SP_ERR_INVALID_ARG);
                }
    for (int64_t rows : extremes)
        for (int64_t vocab : extremes)
            for (int32_t top : {INT32_MIN, -1, 0, 1, 32, 33, INT32_MAX}) {
                const sp_status rc = sp_logprobs_workspace(rows, vocab, top, &n);
                EXPECT(rc == SP_OK || rc == SP_ERR_INVALID_ARG);
                if (rc == SP_OK) EXPECT(n % 256 == 0);
            }
    if (g_fail) return 1;
    std::printf("all checks passed\n");
    return 0;
}
