// The launches of the 4-bit cache's calls on the CPU: the HIP runtime's functions are replaced by ones that note what is asked of them, so that
// grids, block sizes and LDS can be checked without a GPU (tests/test_kv4_launches.py).  No pointer handed to the library is followed.
#include <hip/hip_runtime_api.h>

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
static const st_kv4_ledger led = {(float *)p, (int32_t *)p};

static st_kv4 *cache(const st_kv4_config &c) {
    size_t cb = 0, wb = 0;
    st_kv4 *h = nullptr;
    if (st_kv4_query_sizes(&c, &cb, &wb) != ST_OK || st_kv4_create(&c, (const float *)p, p, cb, p, wb, nullptr, &h) != ST_OK) return nullptr;
    launches.clear(), refused = false, asked = 0;
    return h;
}

// Evictions whose blocks want more LDS than a kernel has without asking: on every GPU the limit is raised there, once, before the launch
static int lds_on_every_gpu() {
    for (int d : {64, 128}) {
        st_kv4 *h = cache({1, 20, 4, 2, d, 24576, 8, 64, 1e-6f});
        CHECK(h);
        for (int n : {1, 5, 20}) {  // each size of the span table is a kernel of its own
            st_kv4_span s[20];
            for (int j = 0; j < n; ++j) s[j] = {j, 24576 - j, 24576, 0};
            for (int round = 0; round < 2; ++round)
                for (int gpu : {0, 1, 5, 70}) {
                    device = gpu, asked = 0;
                    CHECK(st_kv4_evict(h, 0, 1, s, n, 20000, 100, &led, nullptr) == ST_OK);
                    CHECK(!refused && launches.back().device == gpu);
                    CHECK(asked == (round == 0 || gpu >= 64));
                }
        }
        st_kv4_destroy(h);
    }
    device = 0;
    return 0;
}

// A limit that cannot be raised is an error, and nothing is launched
static int lds_refused() {
    st_kv4 *h = cache({1, 1, 4, 2, 64, 24576, 8, 64, 1e-6f});
    const st_kv4_span s = {0, 24576, 24576, 0};
    CHECK(h);
    device = 9, refuse_attribute = true;
    CHECK(st_kv4_evict(h, 0, 1, &s, 1, 20000, 100, &led, nullptr) == ST_EHIP && launches.empty());
    refuse_attribute = false;
    CHECK(st_kv4_evict(h, 0, 1, &s, 1, 20000, 100, &led, nullptr) == ST_OK && !refused);
    device = 0;
    st_kv4_destroy(h);
    return 0;
}

// Whole contexts of 64 sequences with a ledger: a grid that the runtime would refuse is refused before anything is launched
static int grids_of_weights() {
    st_kv4 *h = cache({1, 64, 40, 8, 64, 1 << 21, 1 << 20, 64, 1e-6f});
    CHECK(h);
    st_kv4_span s[64];
    for (int rows : {1, 2, 6, 10, 13, 100, 1000})
        for (int n : {64, 63, 1})
            for (int short_by : {0, 63, 64, 65}) {  // the last sequence ends in a block of slots less, or not
                for (int j = 0; j < n; ++j) s[j] = {j, (1 << 21) - rows - (j == 63 ? short_by : 0), 0, rows};
                launches.clear();
                const int rc = st_kv4_attend(h, 0, s, n, p, 1 << 20, (char *)p + (1ll << 45), 1 << 20, &led);
                CHECK(!refused && (rc == ST_OK ? !launches.empty() : rc == ST_ERANGE && launches.empty()));
                CHECK((rc == ST_ERANGE) == (n == 64 && short_by < 64 && rows * 5 > 32));
                launches.clear();
                CHECK(st_kv4_attend(h, 0, s, n, p, 1 << 20, (char *)p + (1ll << 45), 1 << 20, nullptr) == ST_OK && !refused);
            }
    st_kv4_destroy(h);
    return 0;
}

// Where moves are a launch of their own, a block does 256 of them once: the grid has to have room for the most that a head can have
static int blocks_of_moves() {
    st_kv4 *h = cache({1, 4, 4, 2, 64, 1 << 20, 8, 64, 1e-6f});
    CHECK(h);
    int two = 0;
    for (int len : {2049, 2050, 2304, 2305, 5000, 24576, 24577, 40000, 131072, 131073, 1 << 20})
        for (int keep : {1, 1023, 1024, 1025, 1279, 1280, 1281, 2048, len / 2 - 1, len / 2, len / 2 + 1, len - 1281, len - 1280, len - 1025, len - 1}) {
            if (keep <= 0) continue;
            const st_kv4_span s[] = {{2, keep / 2, len, 0}, {0, len, len, 0}, {1, len / 2, len, 0}};
            launches.clear();
            CHECK(st_kv4_evict(h, 0, 1, s, 3, keep, 0, &led, nullptr) == ST_OK && !refused);
            const int moves = len - keep < keep ? len - keep : keep;
            CHECK(launches.size() == (moves > 1024 ? 2u : 1u));
            if (launches.size() == 2) {
                const dim3 g = launches[1].grid;
                CHECK(g.x % 2 == 0 && (int)(g.x / 2) * 256 >= moves && g.y == 3 && g.z == 1);
                ++two;
            }
        }
    CHECK(two > 20);
    st_kv4_destroy(h);
    return 0;
}

int main(int argc, char **argv) {
    const struct {
        const char *name;
        int (*f)();
    } tests[] = {{"lds_on_every_gpu", lds_on_every_gpu}, {"lds_refused", lds_refused}, {"grids_of_weights", grids_of_weights}, {"blocks_of_moves", blocks_of_moves}};
    for (const auto &t : tests)
        if (argc == 2 && !std::strcmp(argv[1], t.name)) {
            if (t.f()) return 1;
            std::puts("ok");
            return 0;
        }
    return 2;
}
