// The cache operators for long contexts at the ends of what their checks accept: row tiles, requests
// and groups by the million.  The launchers and their checks are long_driver.cpp's.
#define main long_driver_main
#include "long_driver.cpp"
#undef main

// A size up to 2^top, spread over its logarithm.
static int64_t spread(int top) {
    const int bits = (int)(rng() % (top + 1));
    return (int64_t(1) << bits) + (int64_t)(rng() % (int64_t(1) << bits));
}

int main() {
    alignas(16) static int32_t dummy[64];
    void* p = dummy;
    float* f = reinterpret_cast<float*>(p);
    work_base = reinterpret_cast<char*>(uintptr_t(1) << 40);  // (addresses only)
    long taken = 0, full = 0;
    auto attend = [&](na_shared_problem& q) {
        q.cache.q = q.cache.out = {0, q.cache.head_dim, q.cache.heads * q.cache.head_dim};
        work_bytes = na_cache_shared_attention_workspace(&q);
        const long before = launches;
        const na_status st =
            na_cache_shared_attention(&q, p, p, p, dummy, dummy, dummy, dummy, dummy, p, f,
                                      work_base, work_bytes, nullptr);
        CHECK(st == NA_OK || st == NA_ERR_SHAPE);
        CHECK((st == NA_OK) == (launches > before));
        return st;
    };
    na_shared_problem q;
    std::memset(&q, 0, sizeof q);
    na_cache_problem& c = q.cache;
    c.head_dim = 32;
    c.heads = c.kv_heads = 1;
    c.kernel_size = INT64_MAX;
    c.scale = 0.1f;
    c.pages = 10;
    // every split that one side could have for itself, beside as many tiles of the other
    c.tokens = 1;
    c.requests = 1 << 21;
    q.groups = (1 << 23) - 1;
    c.page_size = 4096;
    c.max_pages = 1;
    CHECK(attend(q) == NA_OK);
    // narrow tiles on both sides, of rows that a hint says to be few
    q.groups = (1 << 23) - 1024;
    c.tokens = 32 * q.groups - 64;
    c.requests = 1;
    c.max_new = 1;
    CHECK(attend(q) == NA_OK);
    q.groups = 1;
    c.tokens = (int64_t(1) << 29) - 100000;
    CHECK(attend(q) == NA_OK);
    for (int it = 0; it < 400000; ++it) {
        std::memset(&q, 0, sizeof q);
        c.head_dim = pick({32, 64, 128});
        c.dtype = (int32_t)pick({0, 1, 2});
        c.kv_heads = it % 2 ? 1 : spread(7);
        c.heads = c.kv_heads * (it % 3 ? 1 : spread(6));
        c.requests = spread(23);
        c.tokens = spread(29);
        q.groups = it % 16 ? spread(23) : 0;
        c.page_size = int64_t(16) << (rng() % 10);
        c.max_pages = spread(10);
        c.pages = 1000;
        c.kernel_size = pick({1, 4096, INT64_MAX});
        c.sinks = pick({0, 64, INT64_MAX});
        c.scale = 0.1f;
        c.max_new = pick({0, 1, 1000});
        q.max_shared = pick({0, 1, 1000, 1 << 20});
        q.max_own = pick({0, 1, 1000, 1 << 20});
        const bool ok = attend(q) == NA_OK;
        taken += ok;
        full += ok && (c.requests + q.groups) * c.kv_heads > (1 << 22);
    }
    CHECK(taken > 40000 && full > 4000);
    long gathered = 0, cut = 0;
    for (int it = 0; it < 400000; ++it) {
        na_weights_problem w;
        std::memset(&w, 0, sizeof w);
        na_cache_problem& a = w.cache;
        a.head_dim = 32;
        a.kv_heads = spread(7);
        a.heads = a.kv_heads * (it % 3 ? 1 : spread(6));
        a.requests = spread(20);
        a.tokens = spread(29);
        a.page_size = int64_t(16) << (rng() % 10);
        a.max_pages = spread(20);
        a.pages = 1000;
        a.kernel_size = pick({1, 4096, INT64_MAX});
        a.sinks = pick({0, 64, INT64_MAX});
        a.scale = 0.1f;
        a.max_new = pick({0, 1, 1000});
        a.max_context = pick({0, 1, 1000, 1 << 20});
        a.q = {0, 32, a.heads * 32};
        w.capacity = spread(26);
        work_bytes = na_cache_weights_workspace(&w);
        long before = launches;
        na_status st = na_cache_weights(&w, p, f, p, dummy, dummy, dummy, nullptr, f, work_base,
                                        work_bytes, nullptr);
        CHECK(st == NA_OK || st == NA_ERR_SHAPE);
        CHECK((st == NA_OK) == (launches > before));
        gathered += st == NA_OK;

        na_evict_problem e;
        std::memset(&e, 0, sizeof e);
        e.requests = spread(20);
        e.kv_heads = spread(7);
        e.head_dim = pick({32, 64, 128});
        e.page_size = a.page_size;
        e.max_pages = a.max_pages;
        e.pages = 1000;
        e.num_free = spread(29);
        e.capacity = w.capacity;
        e.budget = spread(29);
        e.recent = spread(30);
        work_bytes = na_cache_evict_workspace(&e);
        before = launches;
        st = na_cache_evict(&e, f, dummy, dummy, dummy, dummy, dummy, p, dummy + 4, dummy + 1, f + 1,
                            dummy, dummy + 2, work_base, work_bytes, nullptr);
        CHECK(st == NA_OK || st == NA_ERR_SHAPE);
        CHECK((st == NA_OK) == (launches > before));
        cut += st == NA_OK;
    }
    CHECK(gathered > 40000 && cut > 40000);
    std::printf("ok limits %ld %ld\n", checks, launches);
    return 0;
}
