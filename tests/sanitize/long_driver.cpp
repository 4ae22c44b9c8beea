// Host driver of the cache operators for long contexts (na_long_api.cpp) under sanitizers, with
// launchers that check what a kernel would be handed: grids within 2^32 threads, cuts that cover every
// key tile, workspaces that hold every part.  Linked against no device code.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "na_launch.h"
#include "na_seq.h"
#include "na_shared.h"

static long checks = 0, launches = 0;
static size_t work_bytes = 0;
static char* work_base = nullptr;

#define CHECK(c)                                                          \
    do {                                                                  \
        ++checks;                                                         \
        if (!(c)) {                                                       \
            std::printf("%s:%d: %s\n", __FILE__, __LINE__, #c);           \
            std::exit(1);                                                 \
        }                                                                 \
    } while (0)

static const int64_t kThreads = int64_t(1) << 32;

static void check_divisor(const na::FastDiv& f, int d) {
    na::FastDiv w;
    w.init(d);
    CHECK(f.mul == w.mul && f.shr == w.shr);
}

static void inside(const void* p, size_t bytes) {
    const char* c = static_cast<const char*>(p);
    CHECK(c >= work_base && c + bytes <= work_base + work_bytes);
}

static void check_paged(const na::SeqGeo& g, int D, int dtype) {
    CHECK(g.G >= 1 && g.Hkv >= 1 && g.B >= 1 && g.n >= 1 && g.W >= 1 && g.S >= 0);
    CHECK(D == 32 || D == 64 || D == 128);
    CHECK(dtype >= 0 && dtype <= 2);
    CHECK(g.lgps >= 4 && ((int64_t)g.max_pages << g.lgps) <= (1 << 30));
    CHECK(g.kb == g.kh * g.Hkv && g.kb < (int64_t(1) << 31));
    check_divisor(g.fd_G, g.G);
    check_divisor(g.fd_kv, g.Hkv);
}

namespace na {

hipError_t launch_shared_attention(const SharedGeo& s, int D, int dtype, const void*, const void*,
                                   const void*, void*, float*, hipStream_t) {
    ++launches;
    const SeqGeo& g = s.g;
    check_paged(g, D, dtype);
    const SharedSide* sides[2] = {&s.shared_side, &s.own_side};
    for (int i = 0; i < 2; ++i) {
        const SharedSide& x = *sides[i];
        const int64_t M = x.narrow ? 32 : 128;
        if (i == 0 && s.groups == 0) {
            CHECK(x.nsplit == 0 && s.shared_jobs == 0);
            continue;
        }
        CHECK(x.nsplit >= 1 && x.nsplit <= kSeqMaxSplit && x.chunk >= 1);
        CHECK(x.ntiles >= (int64_t)g.n * g.G / M + (i == 0 ? s.groups : g.B));
        check_divisor(x.fd_tiles, x.ntiles * g.Hkv);
        // splits of any number of tiles: each begins where the one before it ends, the last one ends
        // with the tiles
        for (int64_t nT : {int64_t(0), int64_t(1), int64_t(x.chunk), int64_t(x.chunk) * x.nsplit + 7,
                           int64_t(1) << 25}) {
            int64_t at = 0;
            for (int p = 0; p < x.nsplit; ++p) {
                const int64_t e0 = std::min<int64_t>((int64_t)p * x.chunk, nT);
                CHECK((int64_t)p * x.chunk < (int64_t(1) << 31));
                CHECK(e0 == at);
                at = p == x.nsplit - 1 ? nT : std::min<int64_t>(e0 + x.chunk, nT);
            }
            CHECK(at == nT);
        }
    }
    CHECK(g.ntiles == s.own_side.ntiles);
    const int64_t own = (int64_t)s.own_side.ntiles * g.Hkv * s.own_side.nsplit;
    CHECK(s.groups == 0 ||
          s.shared_jobs == (int64_t)s.shared_side.ntiles * g.Hkv * s.shared_side.nsplit);
    CHECK((s.shared_jobs + own) * 256 < kThreads);
    CHECK((int64_t)g.ntiles * g.Hkv * (s.own_side.narrow ? 1 : 4) * 256 < kThreads);
    const size_t rows = (size_t)(s.shared_side.nsplit + s.own_side.nsplit) * g.n * g.Hkv * g.G;
    inside(s.part, rows * D * 4);
    inside(s.part_lse, rows * 4);
    CHECK(reinterpret_cast<char*>(s.part_lse) >= reinterpret_cast<char*>(s.part) + rows * D * 4);
    return hipSuccess;
}

hipError_t launch_cache_weights(const WeightsGeo& w, int D, int dtype, const void*, const void*,
                                hipStream_t) {
    ++launches;
    const SeqGeo& g = w.g;
    check_paged(g, D, dtype);
    const int64_t slices = (int64_t)g.B * g.Hkv;
    CHECK(w.form == 0 || w.form == 1);
    CHECK(g.nsplit >= 1 && g.chunk >= 8 && g.chunk % 8 == 0 && w.shares >= 1 && w.capacity > 0);
    CHECK(w.shares == 1 << w.lgshares && (w.form == 1 || w.shares == 1));
    check_divisor(g.fd_tiles, g.nsplit);
    CHECK(slices * g.nsplit * w.shares * 256 < kThreads);
    if (w.shares > 1) {
        check_divisor(w.fd_joins, w.joins);
        CHECK((int64_t)w.joins * 8 == (int64_t)g.nsplit * g.chunk);
        CHECK(slices * w.joins * 256 < kThreads);
        CHECK(w.part_keys == (int64_t)g.nsplit * g.chunk * 32);
        inside(w.part, (size_t)w.shares * slices * w.part_keys * 4);
    }
    return hipSuccess;
}

hipError_t launch_cache_evict(const EvictGeo& v, void*, void*, hipStream_t) {
    ++launches;
    const int64_t slices = (int64_t)v.R * v.Hkv;
    CHECK(v.R >= 0 && v.Hkv >= 1 && v.budget >= 1 && v.recent >= 0 && v.recent <= v.budget);
    CHECK(v.lgps >= 4 && ((int64_t)v.max_pages << v.lgps) <= (1 << 30) && v.num_free >= 0);
    CHECK(v.lgslice >= 6 && v.lgslice <= v.lgrow && v.lgrow <= 9);
    CHECK((slices + 1) * 1024 < kThreads);
    CHECK(v.chunk >= 1 && v.chunks >= 1);
    CHECK(((slices << (v.lgrow - v.lgslice + 1)) + 2 * slices * v.chunks) * 256 < kThreads);
    CHECK(((slices << (v.lgrow - v.lgslice + 1)) + 2 * slices * v.chunks) < (int64_t(1) << 31));
    // every row that can move has a workgroup
    CHECK((int64_t)v.chunk * v.chunks >=
          std::min<int64_t>(v.budget, std::max<int64_t>(1, (int64_t)v.max_pages << v.lgps)));
    check_divisor(v.fd_kv, v.Hkv);
    check_divisor(v.fd_chunks, v.chunks);
    inside(v.moves, (size_t)slices * 8);
    inside(v.to, (size_t)slices * v.budget * 4);
    inside(v.from, (size_t)slices * v.budget * 4);
    CHECK(v.to == v.moves + 2 * slices && v.from == v.to + slices * v.budget);
    return hipSuccess;
}

}  // namespace na

static std::mt19937_64 rng(11);
static int64_t pick(std::initializer_list<int64_t> v) {
    return *(v.begin() + rng() % v.size());
}
static int64_t any() {
    if (rng() % 8 == 0) return pick({-1, 0, INT64_MAX, INT64_MIN, int64_t(1) << 62, 1 << 30});
    return (int64_t)(rng() % (int64_t(1) << (rng() % 40 + 1)));
}
static int64_t near(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (hi - lo + 1)); }

int main() {
    alignas(16) static int32_t dummy[64];
    void* p = dummy;
    float* f = reinterpret_cast<float*>(p);
    na_stream_t s = nullptr;
    for (int it = 0; it < 60000; ++it) {
        const bool wild = it % 2;
        na_shared_problem q;
        std::memset(&q, 0, sizeof q);
        na_cache_problem& c = q.cache;
        const int64_t D = pick({32, 64, 128, 128, wild ? 80 : 64});
        c.kv_heads = wild ? any() : near(1, 9);
        c.heads = wild ? any() : c.kv_heads * near(1, 40);
        c.requests = wild ? any() : near(0, it % 10 ? 100 : 100000);
        c.tokens = wild ? any() : near(0, it % 10 ? 300 : 50000);
        c.head_dim = D;
        c.page_size = wild ? any() : pick({16, 32, 64, 256, 4096});
        c.pages = wild ? any() : near(0, 100000);
        c.max_pages = wild ? any() : near(0, 2000);
        c.kernel_size = wild ? any() : pick({1, 7, 512, 4096, 1 << 20, INT64_MAX});
        c.sinks = wild ? any() : pick({0, 1, 4, 33, 500, 100000, INT64_MAX});
        c.max_new = wild ? any() : pick({0, 1, 8, 5000});
        c.max_context = wild ? any() : pick({0, 1, 100, 30000, INT64_MAX});
        c.dtype = (int32_t)pick({0, 1, 2, wild ? -5 : 1});
        c.scale = 0.1f;
        const int64_t ch = std::max<int64_t>(0, std::min<int64_t>(c.heads, 1 << 20));
        c.q = c.out = {0, D, ch * D};
        q.groups = wild ? any() : near(0, it % 10 ? 20 : 5000);
        q.max_shared = wild ? any() : pick({0, 1, 100, 30000, INT64_MAX});
        q.max_own = wild ? any() : pick({0, 1, 100, 30000, INT64_MAX});
        // (addresses only: nothing is read or written)
        work_base = reinterpret_cast<char*>(uintptr_t(1) << 40);
        work_bytes = na_cache_shared_attention_workspace(&q);
        const na_status st =
            na_cache_shared_attention(&q, p, p, p, dummy, dummy, dummy, dummy, dummy, p, f, work_base,
                                      work_bytes, s);
        const bool fits = !wild && c.requests * c.max_pages < (int64_t(1) << 31) &&
                          c.max_pages * c.page_size <= (1 << 30);
        if (!wild && it % 10 && fits) CHECK(st == NA_OK);
        if (work_bytes)
            CHECK(na_cache_shared_attention(&q, p, p, p, dummy, dummy, dummy, dummy, dummy, p, f,
                                            work_base, work_bytes - 1, s) == NA_ERR_WORKSPACE);

        na_weights_problem w;
        w.cache = c;
        w.capacity = wild ? any() : near(0, 100000);
        work_bytes = na_cache_weights_workspace(&w);
        CHECK(work_bytes <= (size_t(1) << 28));
        const na_status ws = na_cache_weights(&w, p, f, p, dummy, dummy, dummy, it % 3 ? dummy : nullptr,
                                              f, work_base, work_bytes, s);
        if (!wild && it % 10 && fits) CHECK(ws == NA_OK);

        na_evict_problem e;
        std::memset(&e, 0, sizeof e);
        e.requests = c.requests;
        e.kv_heads = c.kv_heads;
        e.head_dim = D;
        e.pages = c.pages;
        e.page_size = c.page_size;
        e.max_pages = c.max_pages;
        e.num_free = wild ? any() : near(0, 1000);
        e.capacity = w.capacity;
        e.budget = wild ? any() : near(1, it % 10 ? 5000 : 500000);
        e.recent = wild ? any() : pick({0, 1, 100, INT64_MAX});
        e.dtype = c.dtype;
        work_bytes = na_cache_evict_workspace(&e);
        const na_status es = na_cache_evict(&e, f, dummy, dummy, dummy, dummy, dummy, p, dummy + 4,
                                            dummy + 1, f + 1, dummy, dummy + 2, work_base, work_bytes, s);
        if (!wild && it % 10 && fits) CHECK(es == NA_OK);
    }
    std::printf("ok long %ld %ld\n", checks, launches);
    return 0;
}
