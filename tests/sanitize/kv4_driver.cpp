// Host-side walk over the 4-bit cache's calls -- argument validation, workspace carving, the plan of attention -- for a build of
// their sources with -fsanitize=address,undefined on the host pass (tests/test_kv4_sanitizers.py).  Needs no GPU: every call here returns before
// touching a device.
#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/st.h"

static char last[512];
namespace st {
int fail(int code, const char *fmt, ...) {  // the library's is in a source that this build does without
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(last, sizeof last, fmt, ap);
    va_end(ap);
    return code;
}
}  // namespace st

#define CHECK(c)                                                                         \
    do {                                                                                 \
        if (!(c)) {                                                                      \
            std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #c, last); \
            return 1;                                                                    \
        }                                                                                \
    } while (0)

int main() {
    void *const p = reinterpret_cast<void *>(0x10000);  // never followed
    const st_kv4_config shapes[] = {
        {28, 4, 12, 2, 128, 8192, 4096, 8192, 1e-6f},       {64, 64, 40, 8, 128, 1 << 17, 4096, 1 << 20, 1e-6f},
        {1, 1, 1, 1, 64, 1, 1, 1, 0.f},                     {1, 64, 4096, 256, 64, 1 << 20, 1 << 20, INT_MAX, 1.f},
        {65535, 1, 16, 1, 64, 1 << 24, 1 << 20, 5, 1e-5f},
    };
    for (const st_kv4_config &c : shapes) {
        size_t cb = 0, wb = 0;
        CHECK(st_kv4_query_sizes(&c, &cb, &wb) == ST_OK && cb > 0 && wb > 0);
        st_kv4 *h = nullptr;
        CHECK(st_kv4_create(&c, (const float *)p, p, cb, p, wb, nullptr, &h) == ST_OK && h);
        st_kv4_destroy(h);
        CHECK(st_kv4_create(&c, (const float *)p, p, cb, p, wb - 1, nullptr, &h) == ST_ENOMEM && !h);
        CHECK(st_kv4_create(&c, (const float *)p, p, cb, p, wb, nullptr, &h) == ST_OK && h);
        for (int n = 0; n <= c.n_seq && n <= ST_KV4_MAX_SPANS; n += n < 5 ? 1 : 59) {
            std::vector<st_kv4_span> s(n);
            std::vector<int32_t> ranges(n);
            for (int64_t len = 0; len < c.max_seq; len = 3 * len + 1)
                for (int64_t rows = 0; rows <= c.max_rows && len + rows <= c.max_seq; rows = 5 * rows + 1) {
                    for (int j = 0; j < n; ++j)
                        s[j] = {n - 1 - j, (int32_t)(j % 3 == 2 ? len / 2 : len), 0, (int32_t)(j % 4 == 3 ? 0 : rows)};
                    int32_t columns = -1, blocks = -1;
                    const int rc = st_kv4_attend_plan(&c, s.data(), n, len % 2, &columns, &blocks, ranges.data());
                    CHECK(rc == ST_OK || (rc == ST_ERANGE && rows * n > c.max_rows * 3 / 4));
                    CHECK(rc != ST_OK || (blocks >= 0 && (columns == 0) == (blocks == 0)));
                }
        }
        const int big[] = {INT_MIN, -1, 0, 1, c.max_seq, INT_MAX};
        const st_kv4_ledger led = {(float *)p, (int32_t *)p};
        for (int seq : big)
            for (int len : big)
                for (int rows : big)
                    for (int pos : big) {
                        const st_kv4_span s = {seq, len, pos, rows};
                        const bool fits = seq >= 0 && seq < c.n_seq && len >= 0 && rows >= 0 && (int64_t)len + rows <= c.max_seq && pos >= 0;
                        if (!fits) {
                            CHECK(st_kv4_append(h, 0, &s, 1, p, 1 << 20, nullptr, nullptr, p, 1 << 20, &led) == ST_ERANGE);
                            CHECK(st_kv4_attend(h, 0, &s, 1, p, 1 << 20, p, 1 << 20, &led) == ST_ERANGE);
                            CHECK(st_kv4_read(h, 0, 1, &s, 1, p, p) == ST_ERANGE);
                            CHECK(st_kv4_evict(h, 0, 1, &s, 1, 1, 0, &led, nullptr) == ST_ERANGE);
                            CHECK(st_kv4_attend_plan(&c, &s, 1, 0, nullptr, nullptr, nullptr) == ST_ERANGE);
                        } else if (rows) {
                            CHECK(st_kv4_evict(h, 0, 1, &s, 1, 1, 0, &led, nullptr) == (rows < 1 << 24 ? ST_EINVAL : ST_ERANGE));
                        }
                    }
        for (int layer : {INT_MIN, -1, (int)c.n_layers, INT_MAX}) {
            CHECK(st_kv4_append(h, layer, nullptr, 0, p, 1 << 20, nullptr, nullptr, p, 1 << 20, nullptr) == ST_ERANGE);
            CHECK(st_kv4_attend(h, layer, nullptr, 0, p, 1 << 20, p, 1 << 20, nullptr) == ST_ERANGE);
            CHECK(st_kv4_read(h, 0, layer == c.n_layers ? layer + 1 : layer, nullptr, 0, p, p) == ST_ERANGE);
        }
        CHECK(st_kv4_append(h, 0, nullptr, 0, p, INT64_MIN, nullptr, nullptr, p, 1 << 20, nullptr) == ST_EINVAL);
        CHECK(st_kv4_attend(h, 0, nullptr, 1, p, 1 << 20, p, 1 << 20, nullptr) == ST_EINVAL);
        CHECK(st_kv4_attend(h, 0, nullptr, ST_KV4_MAX_SPANS + 1, p, 1 << 20, p, 1 << 20, nullptr) == ST_EINVAL);
        CHECK(st_kv4_attend(h, 0, nullptr, INT_MIN, p, 1 << 20, p, 1 << 20, nullptr) == ST_EINVAL);
        st_kv4_destroy(h);
    }
    std::puts("ok");
    return 0;
}
