// The launches of the paged cache's calls and of the verdict over drafts on the CPU: the HIP runtime's functions are replaced by ones that note what is asked of them, so that
// grids, block sizes and LDS can be checked without a GPU (tests/test_paged_launches.py).  No pointer handed to the library is followed.
#include <hip/hip_runtime_api.h>

#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <set>
#include <utility>
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

struct Launch {
    const void *kernel;
    dim3 grid, block;
    size_t lds;
    int device;
};
static std::vector<Launch> launches;
static std::set<std::pair<int, const void *>> raised;  // (GPU, kernel) with a raised LDS limit
static int device = 0, asked = 0;
static bool refuse_attribute = false, refused = false;  // refused: a launch that the runtime would not take

extern "C" {
hipError_t hipGetDevice(int *d) { return *d = device, hipSuccess; }
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute, int) {
    ++asked;
    if (refuse_attribute) return hipErrorInvalidValue;
    raised.insert({device, f});
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
static dim3 next_grid, next_block;
static size_t next_lds;
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t) {
    next_grid = g, next_block = b, next_lds = lds;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, hipStream_t *s) {
    *g = next_grid, *b = next_block, *lds = next_lds, *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 g, dim3 b, void **, size_t lds, hipStream_t) {
    launches.push_back({f, g, b, lds, device});
    const uint64_t threads[] = {(uint64_t)g.x * b.x, (uint64_t)g.y * b.y, (uint64_t)g.z * b.z};
    for (uint64_t t : threads) refused |= t == 0 || t >> 32;
    refused |= (uint64_t)b.x * b.y * b.z > 1024 || g.y > 65535 || g.z > 65535;
    refused |= lds > 65536 && !raised.count({device, f});
    return hipSuccess;
}
void **__hipRegisterFatBinary(const void *) { static void *none; return &none; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
}

#define CHECK(c)                                                                         \
    do {                                                                                 \
        if (!(c)) {                                                                      \
            std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #c, last); \
            return 1;                                                                    \
        }                                                                                \
    } while (0)

static void *const p = reinterpret_cast<void *>(0x10000);  // never followed
static char *const far_away = reinterpret_cast<char *>(1ll << 46);
static const st_draft_tree tree = {(int32_t *)p, (int32_t *)p, (uint64_t *)p, 16, 4};

static st_paged *cache(const st_paged_config &c) {
    size_t cb = 0, wb = 0;
    st_paged *h = nullptr;
    if (st_paged_query_sizes(&c, &cb, &wb) != ST_OK || st_paged_create(&c, (const float *)p, (const int32_t *)p, p, cb, p, wb, nullptr, &h) != ST_OK) return nullptr;
    launches.clear(), refused = false, asked = 0;
    return h;
}

// Every call at the ends of its ranges: grids that the runtime takes, or a refusal before anything is launched
static int grids() {
    const st_paged_config shapes[] = {
        {28, 64, 12, 2, 128, 1 << 16, 16, 1 << 14, 1 << 16, 1 << 20, ST_BF16, 128, 0, 1e-6f}, {64, 64, 40, 8, 128, 1 << 20, 64, 1 << 18, 1 << 20, INT_MAX, ST_F16, 64, 1, 1e-6f},
        {1, 64, 1, 1, 64, 1, 16, 1, 16, 1, ST_BF16, 0, 0, 0.f},                               {65535, 64, 4096, 256, 64, 16, 1024, 1 << 14, 1 << 20, INT_MAX, ST_F16, 16, 1, 1.f},
    };
    for (const st_paged_config &c : shapes) {
        st_paged *h = cache(c);
        CHECK(h);
        const int64_t slots = (int64_t)c.page_size * c.max_pages;
        st_kv4_span s[64];
        for (int n : {1, 4, 5, 16, 17, 64})
            for (int64_t rows : {(int64_t)1, (int64_t)2, (int64_t)7, (int64_t)64, (int64_t)1000, (int64_t)1024, (int64_t)c.max_rows / n})
                for (int64_t len : {(int64_t)0, (int64_t)1, slots / 3, slots - rows}) {
                    if (rows < 1 || rows * n > c.max_rows || len < 0 || len + rows > slots || rows > c.max_pos) continue;
                    for (int j = 0; j < n; ++j) s[j] = {j, (int32_t)(j % 2 ? len / 2 : len), 0, (int32_t)(j % 5 == 4 ? 0 : rows)};
                    const int64_t width = (int64_t)(c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim;
                    for (const st_draft_tree *t : {(const st_draft_tree *)nullptr, &tree}) {
                        if (t && rows > 1024) continue;
                        launches.clear();
                        CHECK(st_paged_append(h, 0, s, n, t, p, width, p, p, far_away, width) == ST_OK && launches.size() == 1 && !refused);
                        launches.clear();
                        const int rc = st_paged_attend(h, 0, s, n, t, p, width, far_away, width);
                        CHECK(!refused && (rc == ST_OK ? !launches.empty() && launches.size() <= 2 : rc == ST_ERANGE && launches.empty()));
                        int32_t blocks = 0, columns = 0;
                        CHECK(st_paged_attend_plan(&c, s, n, t != nullptr, &columns, &blocks, nullptr) == ST_OK);
                        CHECK((rc == ST_ERANGE) == (blocks >= 1 << 24) && (rc != ST_OK || (int)launches[0].grid.x == blocks));
                    }
                    launches.clear();
                    CHECK(st_paged_keep(h, 0, c.n_layers, s, n, (int32_t *)p, INT_MAX, (int32_t *)p) == ST_OK && launches.size() == 1 && !refused);
                    CHECK((int64_t)launches[0].grid.x * 256 >= 2 * (int64_t)c.n_kv_heads * c.head_dim / 8 && (int)launches[0].grid.y == n && (int)launches[0].grid.z == c.n_layers);
                }
        st_paged_destroy(h);
    }
    return 0;
}

// Blocks that want more LDS than a kernel has without asking: on every GPU the limit is raised there, once, before the launch; where it cannot be, nothing is launched
static int lds() {
    for (int type : {ST_BF16, ST_F16}) {
        st_paged *h = cache({1, 64, 40, 8, 128, 64, 64, 64, 4096, 64, type, 0, 0, 0.f});
        CHECK(h);
        for (int n : {1, 9, 40}) {  // each size of the span table is a kernel of its own
            st_kv4_span s[64];
            for (int j = 0; j < n; ++j) s[j] = {j, 100, 0, 40};
            device = 3, refuse_attribute = true, launches.clear();
            CHECK(st_paged_attend(h, 0, s, n, nullptr, p, 5120, far_away, 5120) == ST_EHIP && launches.empty());
            refuse_attribute = false;
            for (int round = 0; round < 2; ++round)
                for (int gpu : {0, 1, 5, 70}) {
                    device = gpu, asked = 0;
                    CHECK(st_paged_attend(h, 0, s, n, nullptr, p, 5120, far_away, 5120) == ST_OK && !refused && launches.back().device == gpu);
                    CHECK(launches[0].lds > 65536 ? asked == (round == 0 || gpu >= 64) : asked == 0);
                }
        }
        device = 0;
        st_paged_destroy(h);
    }
    return 0;
}

static int verify() {
    for (int dtype : {ST_BF16, ST_F16, ST_F32})
        for (const st_verify_config &c : {st_verify_config{1, dtype, 32767, 1}, st_verify_config{152064, dtype, 2048, 64}, st_verify_config{1 << 24, dtype, 32767, 3}, st_verify_config{4097, dtype, 1, 2}}) {
            size_t wb = 0;
            st_verify *h = nullptr;
            CHECK(st_verify_query_sizes(&c, &wb) == ST_OK && st_verify_create(&c, p, wb, nullptr, &h) == ST_OK);
            for (int n : {1, 2, 64})
                for (int rows : {1, 2, 21, 500, 1024}) {
                    if (n * rows > c.max_rows) continue;
                    std::vector<int32_t> r(n, rows);
                    for (int greedy = 0; greedy < 3; ++greedy) {
                        std::vector<float> heat(n, greedy == 1 ? 0.f : 0.7f);
                        if (greedy == 2) heat[0] = 0.f;
                        st_draft_tree t = tree;
                        t.width = c.max_width;
                        for (int k = 0; k < 4; ++k) {
                            launches.clear(), refused = false;
                            CHECK(st_verify_drafts(h, r.data(), n, k & 1 ? &t : nullptr, (int32_t *)p, p, 1ll << 40, k & 2 ? p : nullptr, 1ll << 40, heat.data(), (double *)p, (double *)p,
                                                   (int32_t *)p, rows, (int32_t *)p, (int32_t *)p) == ST_OK);
                            const bool all = greedy == 1 || (greedy == 2 && n == 1);
                            const size_t left = (k & 2) && !all && (k & 1) && t.width > 1 ? t.width : 0;  // width - 1 looks, and the verdicts after them
                            const bool fused = !left && rows <= 8 && ((int64_t)c.vocab + 4095) / 4096 * n <= 256;  // (the verdicts in the launch that draws)
                            CHECK(!refused && launches.size() == 3 + left + (all ? 0 : 1) - fused);
                        }
                    }
                }
            st_verify_destroy(h);
        }
    return 0;
}

int main(int argc, char **argv) {
    const struct {
        const char *name;
        int (*f)();
    } tests[] = {{"grids", grids}, {"lds", lds}, {"verify", verify}};
    for (const auto &t : tests)
        if (argc == 2 && !std::strcmp(argv[1], t.name)) {
            if (t.f()) return 1;
            std::puts("ok");
            return 0;
        }
    return 2;
}
