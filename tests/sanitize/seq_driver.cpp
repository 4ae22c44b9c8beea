// Host driver of the sequence operators' C ABI (na_seq_api.cpp) under sanitizers, with launchers
// that check the geometry a kernel would be handed: grids within 2^32 threads, splits that cover
// every key tile, workspaces that hold every part.  Linked against no device code.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "na_launch.h"
#include "na_seq.h"
#include "na_seq_kernels.h"

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

namespace na {

hipError_t launch_seq_forward(const SeqGeo& g, int D, int dtype, bool paged, bool narrow,
                              const void*, const void*, const void*, void*, float*, float* part,
                              hipStream_t) {
    ++launches;
    const int64_t M = narrow ? 32 : 128;
    CHECK(g.G >= 1 && g.Hkv >= 1 && g.B >= 1 && g.n >= 1 && g.W >= 1 && g.S >= 0);
    CHECK(D == 32 || D == 64 || D == 128);
    CHECK(dtype >= 0 && dtype <= 2 && g.nsplit >= 1 && g.nsplit <= kSeqMaxSplit && g.chunk >= 1);
    const int64_t tiles = (int64_t)g.ntiles * g.Hkv * (paged ? 1 : g.B);
    CHECK(tiles * g.nsplit * 256 < kThreads);
    check_divisor(g.fd_G, g.G);
    check_divisor(g.fd_kv, g.Hkv);
    if (paged) {
        check_divisor(g.fd_tiles, g.ntiles * g.Hkv);
        // every request's tiles fit, however the tokens fall
        CHECK(g.ntiles >= (int64_t)g.n * g.G / M + g.B);
        CHECK(g.lgps >= 4 && ((int64_t)g.max_pages << g.lgps) <= (1 << 30));
        if (g.nsplit > 1) {
            CHECK(tiles * 4 * 256 < kThreads);
            inside(part, (size_t)tiles * g.nsplit * M * (D + 1) * 4);
        }
    } else {
        check_divisor(g.fd_tiles, g.ntiles);
        check_divisor(g.fd_slices, g.B * g.Hkv);
        CHECK((int64_t)g.ntiles * 128 >= (int64_t)g.n * g.G && !narrow && g.nsplit == 1);
    }
    return hipSuccess;
}

hipError_t launch_seq_backward(const SeqBwd& b, int D, int dtype, const void*, const void*,
                               const void*, const void*, const float*, const void*, void*, void*,
                               void*, hipStream_t) {
    ++launches;
    const SeqGeo& g = b.g;
    const int64_t slices = (int64_t)g.B * g.Hkv;
    CHECK((int64_t)b.ktiles * 128 >= g.n && b.hsplit >= 1 && b.hsplit <= g.G && b.chunks >= 1);
    CHECK(b.first_jobs == slices * b.blocks * b.chunks);
    CHECK((b.first_jobs + slices * b.ktiles * b.hsplit) * 512 < kThreads);
    CHECK(slices * g.ntiles * 256 < kThreads);
    check_divisor(b.fd_ktiles, b.ktiles);
    check_divisor(b.fd_hsplit, b.hsplit);
    check_divisor(b.fd_chunks, b.chunks);
    // keys that rows outside their window see have parts
    if (g.S > 0 && g.n > g.W)
        CHECK((int64_t)b.blocks * 32 >= std::min<int64_t>(g.S, g.n - g.W));
    else
        CHECK(b.blocks == 0);
    const size_t rows = (size_t)slices * g.G * g.n * 4;
    inside(b.lse2, rows);
    inside(b.delta, rows);
    CHECK(reinterpret_cast<char*>(b.delta) >= reinterpret_cast<char*>(b.lse2) + rows);
    const size_t key = 2 * (size_t)D * 4;
    const size_t part = slices * key * (b.hsplit > 1 ? (size_t)b.hsplit * g.n : b.blocks * 32);
    const size_t first = (size_t)b.chunks * slices * b.blocks * 32 * key;
    if (part) inside(b.part, part);
    if (first) inside(b.first_part, first);
    CHECK(reinterpret_cast<char*>(b.part) >= reinterpret_cast<char*>(b.delta) + rows);
    CHECK(reinterpret_cast<char*>(b.first_part) >= reinterpret_cast<char*>(b.part) + part);
    (void)dtype;
    return hipSuccess;
}

hipError_t launch_cache_tables(int R, int tokens, int lgps, int max_pages, int num_free,
                               const int32_t*, const int32_t*, const int32_t*, const int32_t*,
                               int32_t*, int32_t*, int64_t*, int32_t*, int32_t*, hipStream_t) {
    ++launches;
    CHECK(R >= 0 && tokens >= 0 && lgps >= 4 && max_pages >= 0 && num_free >= 0);
    return hipSuccess;
}

hipError_t launch_cache_write(int tokens, int Hkv, int row_bytes, int lgps, int64_t slots_end,
                              int64_t, int64_t, int64_t, int64_t, const void*, const void*,
                              const int64_t*, void*, void*, hipStream_t) {
    ++launches;
    CHECK(tokens >= 1 && Hkv >= 1 && row_bytes >= 64 && lgps >= 4 && slots_end >= 16);
    CHECK((int64_t)tokens * Hkv * (row_bytes / 16) < (int64_t(1) << 31));
    return hipErrorNoDevice;  // a launch that fails is reported
}

}  // namespace na

static std::mt19937_64 rng(7);
static int64_t pick(std::initializer_list<int64_t> v) {
    return *(v.begin() + rng() % v.size());
}
// spread over magnitudes, extremes among them
static int64_t any() {
    if (rng() % 8 == 0) return pick({-1, 0, INT64_MAX, INT64_MIN, int64_t(1) << 62, 1 << 30});
    return (int64_t)(rng() % (int64_t(1) << (rng() % 40 + 1)));
}
static int64_t near(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (hi - lo + 1)); }

int main() {
    alignas(16) static int32_t dummy[64];
    void* p = dummy;
    na_stream_t s = nullptr;
    for (int it = 0; it < 60000; ++it) {
        na_sink_problem q;
        std::memset(&q, 0, sizeof q);
        const bool wild = it % 2;
        q.kv_heads = wild ? any() : near(1, 9);
        q.heads = wild ? any() : q.kv_heads * near(1, 40);
        q.batch = wild ? any() : near(0, 5);
        q.tokens = wild ? any() : near(0, it % 10 ? 5000 : 200000);
        q.head_dim = pick({32, 64, 128, 128, wild ? 80 : 64});
        q.kernel_size = wild ? any() : pick({1, 7, 512, 4096, 1 << 20, INT64_MAX});
        q.sinks = wild ? any() : pick({0, 1, 4, 33, 500, 100000, INT64_MAX});
        q.dtype = (int32_t)pick({0, 1, 2, wild ? -5 : 1});
        q.scale = 0.1f;
        const int64_t H = std::max<int64_t>(0, std::min<int64_t>(q.heads, 1 << 20));
        const int64_t K = std::max<int64_t>(0, std::min<int64_t>(q.kv_heads, 1 << 20));
        const int64_t N = std::max<int64_t>(0, std::min<int64_t>(q.tokens, 1 << 20));
        const int64_t D = q.head_dim;
        q.q = q.out = q.dout = q.dq = {H * N * D, N * D, D};
        q.k = q.v = q.dk = q.dv = {K * N * D, N * D, D};
        if (wild && rng() % 3 == 0) q.q = {any(), any(), any()};
        if (wild && rng() % 3 == 0) q.dk = {any(), any(), any()};
        na_sink_forward(&q, p, p, p, nullptr, p, reinterpret_cast<float*>(p), s);
        const size_t need = na_sink_backward_workspace(&q);
        // (addresses only: nothing is read or written)
        work_base = reinterpret_cast<char*>(uintptr_t(1) << 40);
        work_bytes = need;
        const na_status st = na_sink_backward(&q, p, p, p, nullptr, p, reinterpret_cast<float*>(p), p,
                                              p, p, p, work_base, need, s);
        if (!wild) CHECK(st == NA_OK);
        if (need)
            CHECK(na_sink_backward(&q, p, p, p, nullptr, p, reinterpret_cast<float*>(p), p, p, p, p,
                                   work_base, need - 1, s) == NA_ERR_WORKSPACE);

        na_cache_problem c;
        std::memset(&c, 0, sizeof c);
        c.kv_heads = wild ? any() : near(1, 9);
        c.heads = wild ? any() : c.kv_heads * near(1, 40);
        c.requests = wild ? any() : near(0, it % 10 ? 100 : 100000);
        c.tokens = wild ? any() : near(0, it % 10 ? 300 : 50000);
        c.head_dim = D;
        c.page_size = wild ? any() : pick({16, 32, 64, 256, 4096});
        c.pages = wild ? any() : near(0, 100000);
        c.max_pages = wild ? any() : near(0, 2000);
        c.kernel_size = q.kernel_size;
        c.sinks = q.sinks;
        c.max_new = wild ? any() : pick({0, 1, 8, 5000});
        c.max_context = wild ? any() : pick({0, 1, 100, 30000, INT64_MAX});
        c.dtype = q.dtype;
        c.scale = 0.1f;
        const int64_t ch = std::max<int64_t>(0, std::min<int64_t>(c.heads, 1 << 20));
        const int64_t ck = std::max<int64_t>(0, std::min<int64_t>(c.kv_heads, 1 << 20));
        c.q = c.out = {0, D, ch * D};
        c.k = c.v = {0, D, ck * D};
        const size_t cn = na_cache_attention_workspace(&c);
        work_bytes = cn;
        const na_status cs = na_cache_attention(&c, p, p, p, dummy, dummy, dummy, p,
                                                reinterpret_cast<float*>(p), work_base, cn, s);
        if (!wild && c.requests * c.max_pages < (int64_t(1) << 31) &&
            c.max_pages * c.page_size <= (1 << 30))
            CHECK(cs == NA_OK);
        const na_status ws = na_cache_write(&c, p, p, reinterpret_cast<int64_t*>(p), p, p, s);
        if (!wild) CHECK(ws == NA_ERR_HIP || c.tokens == 0 || c.pages == 0);
        na_cache_tables(c.requests, c.tokens, c.page_size, c.max_pages, near(0, 10), dummy, dummy,
                        dummy, dummy, dummy, dummy, reinterpret_cast<int64_t*>(p), dummy, dummy + 1,
                        s);
    }
    std::printf("ok sequence %ld %ld\n", checks, launches);
    return 0;
}
