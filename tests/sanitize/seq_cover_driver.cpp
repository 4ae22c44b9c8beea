// Host driver of the cut of the paged attention (na_seq_api.cpp) under sanitizers: the splits of
// every row tile, as a kernel forms them from what it is handed, cover its key tiles once each and
// none is empty; for the number of tiles that the caller's bounds allow no split is left over.
// Linked against no device code.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "na_launch.h"
#include "na_seq.h"
#include "na_seq_kernels.h"

static long checks = 0, splits_seen = 0;
static int64_t max_context = 0;
static std::mt19937_64 rng(11);

#define CHECK(c)                                                          \
    do {                                                                  \
        ++checks;                                                         \
        if (!(c)) {                                                       \
            std::printf("%s:%d: %s\n", __FILE__, __LINE__, #c);           \
            std::exit(1);                                                 \
        }                                                                 \
    } while (0)

static void check_cover(const na::SeqGeo& g, int nT) {
    // as seq_splits, and e0, e1 of the kernels
    const int splits = std::max(1, std::min(g.nsplit, (nT + g.chunk - 1) / g.chunk));
    int at = 0;
    for (int s = 0; s < splits; ++s) {
        const int64_t e0 = (int64_t)s * g.chunk;
        const int e1 = s == splits - 1 ? nT : (int)e0 + g.chunk;
        CHECK(e0 == at && e1 > at && e1 <= nT);
        at = e1;
    }
    CHECK(at == nT);
    splits_seen += splits > 1;
}

namespace na {

hipError_t launch_seq_forward(const SeqGeo& g, int, int, bool paged, bool narrow, const void*,
                              const void*, const void*, void*, float*, float*, hipStream_t) {
    // a row is up to 31 positions before the last of its wave, and that one up to 32 before the
    // first of a tile of a stage; the masks form (such a distance, less 4) - W + 1 in 32 bits
    CHECK((int64_t)-31 - 32 - 4 - g.W + 1 >= INT32_MIN);
    if (!paged) return hipSuccess;
    const int64_t M = narrow ? 32 : 128, room = (int64_t)g.max_pages << g.lgps;
    const int64_t span = (int64_t)g.W + g.S + M + 64;
    const int64_t bound = max_context > 0 ? std::min(max_context, room) : room;
    const int64_t tiles = std::max<int64_t>(1, (std::min(bound, span) + 31) / 32 + 1);
    CHECK((int64_t)(g.nsplit - 1) * g.chunk < tiles && tiles <= (int64_t)g.nsplit * g.chunk);
    check_cover(g, (int)tiles);
    // fewer tiles, and more than the bounds say (they are not relied on)
    for (int nT = 1; nT <= 70; ++nT) check_cover(g, nT);
    for (int i = 0; i < 20; ++i) check_cover(g, 1 + (int)(rng() % (uint64_t(1) << (1 + rng() % 26))));
    for (int d = -1; d <= 1; ++d)
        for (int s = 1; s <= g.nsplit + 1; s += std::max(1, g.nsplit / 3))
            if ((int64_t)s * g.chunk + d >= 1 && (int64_t)s * g.chunk < (1 << 26))
                check_cover(g, s * g.chunk + d);
    return hipSuccess;
}

hipError_t launch_seq_backward(const SeqBwd&, int, int, const void*, const void*, const void*,
                               const void*, const float*, const void*, void*, void*, void*,
                               hipStream_t) {
    return hipSuccess;
}
hipError_t launch_cache_tables(int, int, int, int, int, const int32_t*, const int32_t*,
                               const int32_t*, const int32_t*, int32_t*, int32_t*, int64_t*,
                               int32_t*, int32_t*, hipStream_t) {
    return hipSuccess;
}
hipError_t launch_cache_write(int, int, int, int, int64_t, int64_t, int64_t, int64_t, int64_t,
                              const void*, const void*, const int64_t*, void*, void*, hipStream_t) {
    return hipSuccess;
}

}  // namespace na

static int64_t pick(std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); }
static int64_t near(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (hi - lo + 1)); }

int main() {
    alignas(16) static int32_t dummy[64];
    void* p = dummy;
    for (int it = 0; it < 40000; ++it) {
        na_cache_problem c;
        std::memset(&c, 0, sizeof c);
        c.kv_heads = near(1, 9);
        c.heads = c.kv_heads * near(1, 40);
        c.requests = near(1, it % 10 ? 100 : 100000);
        c.tokens = near(1, it % 10 ? 300 : 50000);
        c.head_dim = pick({32, 64, 128});
        c.page_size = pick({16, 32, 64, 256, 4096});
        c.pages = near(0, 100000);
        c.max_pages = near(0, it % 7 ? 2000 : 20000);
        c.kernel_size = pick({1, 7, 30, 255, 512, 4096, 1 << 20, (1u << 31) - 1, INT64_MAX});
        c.sinks = pick({0, 1, 4, 33, 500, 100000, INT64_MAX});
        c.max_new = pick({0, 1, 8, 5000});
        c.max_context = pick({0, 1, 100, 500, 3000, 30000, INT64_MAX});
        c.dtype = (int32_t)pick({0, 1, 2});
        c.scale = 0.1f;
        c.q = c.out = {0, c.head_dim, c.heads * c.head_dim};
        max_context = c.max_context;
        // (an address only: nothing is read or written)
        char* work = reinterpret_cast<char*>(uintptr_t(1) << 40);
        const na_status st = na_cache_attention(&c, p, p, p, dummy, dummy, dummy, p,
                                                reinterpret_cast<float*>(p), work,
                                                na_cache_attention_workspace(&c), nullptr);
        CHECK(st == NA_OK || c.requests * c.max_pages >= (int64_t(1) << 31));

        na_sink_problem q;
        std::memset(&q, 0, sizeof q);
        q.batch = 1;
        q.kv_heads = q.heads = 1;
        q.tokens = 100;
        q.head_dim = 64;
        q.kernel_size = c.kernel_size;
        q.scale = 0.1f;
        q.q = q.k = q.v = q.out = {0, 0, 64};
        CHECK(na_sink_forward(&q, p, p, p, nullptr, p, reinterpret_cast<float*>(p), nullptr) == NA_OK);
    }
    std::printf("ok cover %ld %ld\n", checks, splits_seen);
    return 0;
}
