// na_long_api.cpp -- the C ABI of the cache operators for long contexts (na_seq.h): attention with
// shared first tokens, gathered weights, eviction.  Validation, the split of the work and
// dispatch; nothing allocates, synchronises or keeps state.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>

#include "na_launch.h"
#include "na_seq_host.h"
#include "na_shared.h"

namespace {

using namespace na::host;

bool nothing(const na_cache_problem& p) {
    return p.heads == 0 || p.tokens == 0 || p.requests == 0;
}

// ---- attention with shared first tokens ----
na_status check_shared(const na_shared_problem& s) {
    const na_cache_problem& p = s.cache;
    const na_status st = check_attention(p);
    if (st != NA_OK) return st;
    if (s.groups < 0 || s.groups >= kMaxGrid || s.max_shared < 0 || s.max_own < 0)
        return NA_ERR_SHAPE;
    if (nothing(p)) return NA_OK;
    const int64_t G = p.heads / p.kv_heads;
    const int64_t tiles = p.tokens * G / 32 + 4 * p.requests + s.groups;
    if (tiles >= kMaxGrid || tiles * p.kv_heads >= kMaxGrid) return NA_ERR_SHAPE;
    return NA_OK;
}

// The cut of the keys of one side over workgroups.  keys: the most that a row tile has;
// busy: row tiles that are expected to have rows; room: the most workgroups.  The least lengths
// are those of cache_attention's splits; a join there is in any case.  256 workgroups of the wide
// form are aimed at and 512 of the narrow one.  us a call, of 64 requests behind 8192 shared tokens,
// proposed tokens behind three prompts, and chunks of prompts: 28.0, 20.0 and 215; with 512 and 1024
// 31.7, 20.7 and 215, with 128 wide 28.4, 23.5 and 215, with 1536 wide 30.6, 20.8 and 225.
void cut_side(na::SharedSide& side, int64_t keys, int64_t busy, int64_t Hkv, bool half,
              int64_t room) {
    const bool narrow = side.narrow;
    const int64_t tiles = std::max<int64_t>(1, (keys + 31) / 32 + 1);
    int64_t split = std::max<int64_t>(1, (narrow ? 512 : 256) / std::max<int64_t>(1, busy * Hkv));
    split = std::min<int64_t>(split, na::kSeqMaxSplit);
    split = std::min(split, std::max<int64_t>(1, room / ((int64_t)side.ntiles * Hkv)));
    const int64_t least = half ? (narrow ? 12 : 8) : (narrow ? 8 : 2);
    const int64_t step = narrow ? 4 : 2;
    int64_t chunk = split == 1 ? tiles : std::max<int64_t>(least, (tiles + split - 1) / split);
    chunk = (chunk + step - 1) / step * step;
    side.chunk = (int)chunk;
    side.nsplit = (int)((tiles + chunk - 1) / chunk);
    side.fd_tiles.init((int)(side.ntiles * Hkv));
}

void fill_shared(const na_shared_problem& s, na::SharedGeo& x) {
    const na_cache_problem& p = s.cache;
    std::memset(&x, 0, sizeof x);
    na::SeqGeo& g = x.g;
    fill_common(g, p.heads, p.kv_heads, p.kernel_size, p.sinks, p.scale);
    fill_paged(p, g);
    const int64_t rows = p.tokens * g.G, room = p.max_pages * p.page_size;
    const bool half = p.dtype != NA_FP32;
    x.groups = (int)s.groups;

    na::SharedSide &own = x.own_side, &shared = x.shared_side;
    own.narrow = cache_narrow(p);
    // (the narrow form where a group's rows are expected to fill one block of 32)
    shared.narrow = rows <= 32 * s.groups;
    auto tiles = [&](bool narrow, int64_t n) { return n ? rows / (narrow ? 32 : 128) + n : 0; };
    // One grid for both sides.  Where narrow tiles of both would not fit it: wide ones, for which
    // check_shared has left room.
    if ((tiles(own.narrow, p.requests) + tiles(shared.narrow, s.groups)) * g.Hkv >= kMaxGrid)
        own.narrow = shared.narrow = false;
    own.ntiles = g.ntiles = (int)tiles(own.narrow, p.requests);
    shared.ntiles = (int)tiles(shared.narrow, s.groups);

    const int64_t M = own.narrow ? 32 : 128;
    int64_t keys = s.max_own > 0 ? std::min(s.max_own, room) : room;
    keys = std::min(keys, (int64_t)g.W + g.S + M + 64);
    cut_side(own, keys, std::max((rows + M - 1) / M, std::min(p.requests, p.tokens)), g.Hkv, half,
             kMaxGrid - 1 - (int64_t)shared.ntiles * g.Hkv);

    shared.fd_tiles.init(1);
    if (s.groups == 0) return;
    const int64_t Ms = shared.narrow ? 32 : 128;
    keys = s.max_shared > 0 ? std::min(s.max_shared, room) : room;
    cut_side(shared, keys, std::max((rows + Ms - 1) / Ms, std::min(s.groups, p.tokens)), g.Hkv,
             half, kMaxGrid - 1 - (int64_t)own.ntiles * g.Hkv * own.nsplit);
    x.shared_jobs = shared.ntiles * g.Hkv * shared.nsplit;
}

size_t shared_bytes(const na_shared_problem& s, const na::SharedGeo& x) {
    return (size_t)(x.shared_side.nsplit + x.own_side.nsplit) * s.cache.tokens * s.cache.heads *
           (s.cache.head_dim + 1) * 4;
}

}  // namespace

extern "C" {

size_t na_cache_shared_attention_workspace(const na_shared_problem* problem) {
    if (!problem || check_shared(*problem) != NA_OK || nothing(problem->cache)) return 0;
    na::SharedGeo x;
    fill_shared(*problem, x);
    return shared_bytes(*problem, x);
}

na_status na_cache_shared_attention(const na_shared_problem* problem, const void* q,
                                    const void* k_pages, const void* v_pages,
                                    const int32_t* page_table, const int32_t* context_lens,
                                    const int32_t* cu_new, const int32_t* cu_groups,
                                    const int32_t* shared_lens, void* out, float* logsumexp,
                                    void* workspace, size_t workspace_bytes, na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_cache_problem& p = problem->cache;
    const na_status st = check_shared(*problem);
    if (st != NA_OK) return st;
    if (nothing(p)) return NA_OK;
    if (!q || !context_lens || !cu_new || !out || !logsumexp ||
        (problem->groups > 0 && (!cu_groups || !shared_lens)) ||
        (p.pages > 0 && (!k_pages || !v_pages)) || (p.max_pages > 0 && !page_table))
        return NA_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) ||
        !aligned(logsumexp, 16) || !aligned(workspace, 16) || !aligned(page_table, 4) ||
        !aligned(context_lens, 4) || !aligned(cu_new, 4) || !aligned(cu_groups, 4) ||
        !aligned(shared_lens, 4))
        return NA_ERR_ALIGNMENT;
    na::SharedGeo x;
    fill_shared(*problem, x);
    const size_t need = shared_bytes(*problem, x);
    if (workspace_bytes < need) return NA_ERR_WORKSPACE;
    if (!workspace) return NA_ERR_NULL;
    x.g.context = context_lens;
    x.g.cu = cu_new;
    x.g.table = page_table;
    x.cu_groups = cu_groups;
    x.shared = shared_lens;
    x.part = static_cast<float*>(workspace);
    x.part_lse = x.part + (size_t)(x.shared_side.nsplit + x.own_side.nsplit) * p.tokens * p.heads *
                              p.head_dim;
    return na::launch_shared_attention(x, (int)p.head_dim, p.dtype, q, k_pages, v_pages, out,
                                       logsumexp, reinterpret_cast<hipStream_t>(stream)) ==
                   hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

static na_status check_weights(const na_weights_problem& w) {
    const na_cache_problem& p = w.cache;
    const na_status st = check_attention(p, false);
    if (st != NA_OK) return st;
    const int64_t slices = p.requests * p.kv_heads;
    if (w.capacity < 0 || w.capacity >= (int64_t(1) << 40) || slices >= (int64_t(1) << 20) ||
        (__int128)slices * w.capacity >= ((__int128)1 << 40))
        return NA_ERR_SHAPE;
    return NA_OK;
}

// The cut of the work.  Few rows: chunks of 8 to 64 key tiles (what a workgroup sums up at a time),
// 8192 workgroups if every request had the most keys (32 requests of 8k to 32k tokens 109 us a call,
// with 4096 115).  Many: 8 key tiles to a workgroup, whose rows are shared by as many as leave each
// 1024 rows, or 128 where there would be fewer than 1024 workgroups (chunks of 1500 tokens over 2k to
// 7k: 195 us; with 512 rows 189, at twice the workspace; with 2048 221, unshared 225.  Windowed chunks of up
// to 400 tokens 15.3, unshared 27).
static void fill_weights(const na_weights_problem& problem, na::WeightsGeo& w) {
    const na_cache_problem& p = problem.cache;
    std::memset(&w, 0, sizeof w);
    na::SeqGeo& g = w.g;
    fill_common(g, p.heads, p.kv_heads, p.kernel_size, p.sinks, p.scale);
    fill_paged(p, g);
    w.form = cache_narrow(p) ? 0 : 1;
    w.capacity = problem.capacity;
    const int64_t slices = p.requests * p.kv_heads, busy = std::min(p.requests, p.tokens) * p.kv_heads;
    const int64_t room = p.max_pages * p.page_size;
    const int64_t most = p.max_new > 0 ? std::min(p.max_new, p.tokens) : p.tokens;
    int64_t keys = p.max_context > 0 ? std::min(p.max_context, room) : room;
    keys = std::min(keys, (int64_t)g.W + g.S + most + 64);
    const int64_t tiles = std::max<int64_t>(1, (keys + 31) / 32 + 1);
    int64_t chunk = 8;
    if (w.form == 0) {
        const int64_t split = std::max<int64_t>(1, 8192 / busy);
        chunk = std::min<int64_t>(64, std::max<int64_t>(8, (tiles + split - 1) / split));
    }
    chunk = std::max(chunk, (tiles * slices + kMaxGrid / 2 - 1) / (kMaxGrid / 2));
    chunk = (chunk + 7) / 8 * 8;
    g.chunk = (int)chunk;
    g.nsplit = (int)((tiles + chunk - 1) / chunk);
    g.fd_tiles.init(g.nsplit);
    int64_t shares = 1;
    w.part_keys = (int64_t)g.nsplit * g.chunk * 32;
    w.joins = (int)((int64_t)g.nsplit * g.chunk / 8);
    w.fd_joins.init(w.joins);
    if (w.form == 1 && slices * w.joins < kMaxGrid) {
        // (rows that see any of the 256 keys of a workgroup)
        const int64_t rows = std::min(most, (int64_t)g.W + 256) * g.G;
        const int64_t fill = 1024 / (busy * g.nsplit);
        shares = std::max(rows / 1024, std::min(fill, rows / 128));
        shares = std::min<int64_t>(std::max<int64_t>(shares, 1), 32);
        shares = std::min(shares, std::max<int64_t>(1, (kMaxGrid - 1) / (slices * g.nsplit)));
        // (the shares' sums take no more than 256 MiB; with no bound of the context they are as long
        // as the table)
        shares = std::min(shares, std::max<int64_t>(1, (int64_t(1) << 26) / (slices * w.part_keys)));
        while (shares & (shares - 1)) shares &= shares - 1;
    }
    w.shares = (int)shares;
    w.lgshares = __builtin_ctz(w.shares);
}

static size_t weights_bytes(const na::WeightsGeo& w) {
    return w.shares == 1 ? 0 : (size_t)w.shares * w.g.B * w.g.Hkv * w.part_keys * 4;
}

size_t na_cache_weights_workspace(const na_weights_problem* problem) {
    if (!problem || check_weights(*problem) != NA_OK || nothing(problem->cache)) return 0;
    na::WeightsGeo w;
    fill_weights(*problem, w);
    return weights_bytes(w);
}

na_status na_cache_weights(const na_weights_problem* problem, const void* q,
                           const float* logsumexp, const void* k_pages, const int32_t* page_table,
                           const int32_t* context_lens, const int32_t* cu_new,
                           const int32_t* first, float* weights, void* workspace,
                           size_t workspace_bytes, na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_cache_problem& p = problem->cache;
    const na_status st = check_weights(*problem);
    if (st != NA_OK) return st;
    if (nothing(p) || problem->capacity == 0) return NA_OK;
    if (!q || !logsumexp || !context_lens || !cu_new || !weights || (p.pages > 0 && !k_pages) ||
        (p.max_pages > 0 && !page_table))
        return NA_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(logsumexp, 4) ||
        !aligned(weights, 4) || !aligned(page_table, 4) || !aligned(context_lens, 4) ||
        !aligned(cu_new, 4) || !aligned(first, 4) || !aligned(workspace, 4))
        return NA_ERR_ALIGNMENT;
    na::WeightsGeo w;
    fill_weights(*problem, w);
    const size_t need = weights_bytes(w);
    if (workspace_bytes < need) return NA_ERR_WORKSPACE;
    if (need && !workspace) return NA_ERR_NULL;
    w.first = first;
    w.lse = logsumexp;
    w.weights = weights;
    w.part = static_cast<float*>(workspace);
    w.g.context = context_lens;
    w.g.cu = cu_new;
    w.g.table = page_table;
    return na::launch_cache_weights(w, (int)p.head_dim, p.dtype, q, k_pages,
                                    reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

// ---- eviction ----
static na_status check_evict(const na_evict_problem& p) {
    const na_status st = check_types(p.head_dim, p.dtype, 1.f);
    if (st != NA_OK) return st;
    if (p.requests < 0 || p.requests >= kMaxGrid || p.kv_heads < 1 || p.kv_heads >= kMaxGrid ||
        p.requests * p.kv_heads >= (int64_t(1) << 20))
        return NA_ERR_SHAPE;
    if (p.pages < 0 || p.pages >= kMaxRows || p.page_size < 16 || p.page_size > (1 << 20) ||
        (p.page_size & (p.page_size - 1)) || p.max_pages < 0 || p.max_pages >= kMaxRows ||
        p.max_pages * p.page_size > kMaxRows || p.requests * p.max_pages >= (int64_t(1) << 31) ||
        p.num_free < 0 || p.num_free >= kMaxRows)
        return NA_ERR_SHAPE;
    if (p.budget < 1 || p.budget >= kMaxRows || p.recent < 0 || p.capacity < 0 ||
        p.capacity >= (int64_t(1) << 40) ||
        (__int128)p.requests * p.kv_heads * p.capacity >= ((__int128)1 << 40))
        return NA_ERR_SHAPE;
    if (p.kv_heads * p.page_size * p.head_dim * elem_bytes(p.dtype) >= (int64_t(1) << 31))
        return NA_ERR_SHAPE;
    return NA_OK;
}

size_t na_cache_evict_workspace(const na_evict_problem* problem) {
    if (!problem || check_evict(*problem) != NA_OK) return 0;
    const size_t slices = (size_t)(problem->requests * problem->kv_heads);
    return slices * (2 * (size_t)problem->budget + 2) * 4;
}

na_status na_cache_evict(const na_evict_problem* problem, const float* weights,
                         const int32_t* context_lens, const int32_t* first,
                         const int32_t* page_table, const int32_t* head, int32_t* free_pages,
                         void* k_pages, void* v_pages, int32_t* new_context, float* new_weights,
                         int32_t* kept, int32_t* new_head, void* workspace,
                         size_t workspace_bytes, na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_evict_problem& p = *problem;
    const na_status st = check_evict(p);
    if (st != NA_OK) return st;
    if (!head || !new_head || (p.num_free && !free_pages)) return NA_ERR_NULL;
    const bool some = p.requests > 0;
    if (some && (!context_lens || !new_context || !kept || (p.max_pages && !page_table) ||
                 (p.capacity && (!weights || !new_weights)) ||
                 (p.pages && (!k_pages || !v_pages))))
        return NA_ERR_NULL;
    const void* words[] = {weights, context_lens, first,       page_table, head,
                           free_pages, new_context, new_weights, kept,       new_head};
    for (const void* x : words)
        if (!aligned(x, 4)) return NA_ERR_ALIGNMENT;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(workspace, 4))
        return NA_ERR_ALIGNMENT;
    if (head == new_head || (some && new_context == context_lens) ||
        (some && p.capacity && new_weights == weights) || (some && p.pages && k_pages == v_pages))
        return NA_ERR_SHAPE;
    const size_t need = na_cache_evict_workspace(problem);
    if (workspace_bytes < need) return NA_ERR_WORKSPACE;
    if (need && !workspace) return NA_ERR_NULL;
    na::EvictGeo v;
    std::memset(&v, 0, sizeof v);
    v.R = (int)p.requests;
    v.Hkv = (int)p.kv_heads;
    v.budget = (int)p.budget;
    v.recent = (int)std::min(p.recent, p.budget);
    v.lgps = __builtin_ctzll(p.page_size);
    v.pages = (int)p.pages;
    v.max_pages = (int)p.max_pages;
    v.num_free = (int)p.num_free;
    const int64_t row = p.head_dim * elem_bytes(p.dtype);
    v.lgrow = v.lgslice = __builtin_ctzll(row);
    const int64_t slices = p.requests * p.kv_heads;
    while (v.lgslice > 6 && (slices * 2 << (v.lgrow - v.lgslice)) < 1024) --v.lgslice;
    // (8192 workgroups, most of which may find nothing to move: 8 long prompts 147 us a call, with
    // 2048 157)
    const int64_t most = std::max<int64_t>(1, std::min(p.budget, p.max_pages * p.page_size));
    const int64_t chunks = std::min(
        (most + 127) / 128, std::max<int64_t>(1, 4096 / std::max<int64_t>(1, slices)));
    v.chunk = (int)((most + chunks - 1) / chunks);
    v.chunks = (int)((most + v.chunk - 1) / v.chunk);
    v.fd_chunks.init(v.chunks);
    v.capacity = p.capacity;
    v.fd_kv.init(v.Hkv);
    v.weights = reinterpret_cast<const uint32_t*>(weights);
    v.context = context_lens;
    v.first = first;
    v.table = page_table;
    v.head = head;
    v.free_pages = free_pages;
    v.new_context = new_context;
    v.kept = kept;
    v.new_head = new_head;
    v.new_weights = reinterpret_cast<uint32_t*>(new_weights);
    v.moves = static_cast<int32_t*>(workspace);
    v.to = v.moves + 2 * slices;
    v.from = v.to + slices * p.budget;
    return na::launch_cache_evict(v, k_pages, v_pages, reinterpret_cast<hipStream_t>(stream)) ==
                   hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

}  // extern "C"
