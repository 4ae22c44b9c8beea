// na_seq_api.cpp -- the C ABI of the sequence operators (na_seq.h): validation, the split of
// the work and dispatch.  Host code; nothing allocates, synchronises or keeps state.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "na_launch.h"
#include "na_seq.h"
#include "na_seq_kernels.h"

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 30;   // rows of a (sequence, key/value head), positions
constexpr int64_t kMaxGrid = int64_t(1) << 24;   // workgroups of 256 threads in 2^32 threads
constexpr int64_t kMaxToken = int64_t(1) << 26;  // bytes of a token stride

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int elem_bytes(int dtype) { return dtype == NA_FP32 ? 4 : 2; }

na_status check_types(int64_t head_dim, int32_t dtype, float scale) {
    if (head_dim != 32 && head_dim != 64 && head_dim != 128) return NA_ERR_HEAD_DIM;
    if (dtype != NA_FP32 && dtype != NA_FP16 && dtype != NA_BF16) return NA_ERR_DTYPE;
    return std::isfinite(scale) ? NA_OK : NA_ERR_SCALE;
}

// Heads in whole groups (a key head without a query head has none: its gradients would be 0 that
// no launch writes), a window and first tokens that are counts.
na_status check_heads(int64_t heads, int64_t kv_heads, int64_t kernel_size, int64_t sinks) {
    if (heads < 0 || kv_heads < 0 || heads >= kMaxRows) return NA_ERR_SHAPE;
    if ((heads == 0) != (kv_heads == 0)) return NA_ERR_SHAPE;
    if (heads > 0 && heads % kv_heads != 0) return NA_ERR_SHAPE;
    if (kernel_size < 1) return NA_ERR_KERNEL_SIZE;
    return sinks < 0 ? NA_ERR_SHAPE : NA_OK;
}

// Strides as they are used: 0 on axes of one entry, whatever the caller has there.
na_strides used(const na_strides& s, int64_t batch, int64_t heads, int64_t tokens) {
    return {batch == 1 ? 0 : s.batch, heads == 1 ? 0 : s.head, tokens == 1 ? 0 : s.token};
}

// Strides of a [batch, heads, tokens, head_dim] tensor (see na_seq.h), its axes of more than one
// entry.  Outputs: those, ordered by stride, do not overlap.
bool good_strides(const na_strides& all, int es, int64_t batch, int64_t heads, int64_t tokens,
                  int64_t head_dim, bool output) {
    const na_strides s = used(all, batch, heads, tokens);
    const int64_t st[3] = {s.batch, s.head, s.token}, n[3] = {batch, heads, tokens};
    for (int i = 0; i < 3; ++i) {
        if (st[i] < 0 || st[i] >= (int64_t(1) << 40) || (st[i] * es) % 16 != 0) return false;
    }
    if (s.token * es >= kMaxToken) return false;
    if (!output) return true;
    __int128 reach = head_dim;  // entries that the axes so far cover
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return st[a] < st[b]; });
    for (int i : order) {
        if (n[i] <= 1) continue;
        if (st[i] < reach) return false;
        reach += (__int128)st[i] * (n[i] - 1);
    }
    return true;
}

// A window in 32 bits.  Positions stay below kMaxRows + kMaxRows - 256, so the clamp keeps every
// distance inside it, and the masks may take it from a distance down to -127 (a row lies at most
// 31 before its wave's last, that one 32 before a stage's second tile, entries start 4 later).
int clamp_window(int64_t x) { return (int)std::min<int64_t>(x, INT32_MAX - 128); }

// The fields that both forms of the attention share.
void fill_common(na::SeqGeo& g, int64_t heads, int64_t kv_heads, int64_t kernel_size,
                 int64_t sinks, float scale) {
    std::memset(&g, 0, sizeof g);
    g.G = (int)(heads / kv_heads);
    g.Hkv = (int)kv_heads;
    g.W = clamp_window(kernel_size);
    g.S = (int)std::min<int64_t>(sinks, kMaxRows);
    g.c = scale * na::kLog2e;
    g.nsplit = 1;
    g.chunk = INT32_MAX;
    g.fd_G.init(g.G);
    g.fd_kv.init(g.Hkv);
}

// ---- contiguous sequences ----
na_status check_sink(const na_sink_problem& p, bool backward) {
    na_status st = check_types(p.head_dim, p.dtype, p.scale);
    if (st != NA_OK) return st;
    if ((st = check_heads(p.heads, p.kv_heads, p.kernel_size, p.sinks)) != NA_OK) return st;
    if (p.batch < 0 || p.tokens < 0 || p.batch >= kMaxRows || p.tokens >= kMaxRows)
        return NA_ERR_SHAPE;
    if (p.batch == 0 || p.heads == 0 || p.tokens == 0) return NA_OK;
    const int64_t rows = p.tokens * (p.heads / p.kv_heads);
    if (rows >= kMaxRows) return NA_ERR_SHAPE;
    // row tiles of every slice fit a launch (checked without overflow)
    if (p.batch * p.kv_heads >= kMaxGrid ||
        p.batch * p.kv_heads * ((rows + 127) / 128) >= kMaxGrid)
        return NA_ERR_SHAPE;
    const int es = elem_bytes(p.dtype);
    auto q_like = [&](const na_strides& s, bool o) {
        return good_strides(s, es, p.batch, p.heads, p.tokens, p.head_dim, o);
    };
    auto k_like = [&](const na_strides& s, bool o) {
        return good_strides(s, es, p.batch, p.kv_heads, p.tokens, p.head_dim, o);
    };
    if (!q_like(p.q, false) || !k_like(p.k, false) || !k_like(p.v, false)) return NA_ERR_SHAPE;
    if (!backward) return q_like(p.out, true) ? NA_OK : NA_ERR_SHAPE;
    if (!q_like(p.out, false) || !q_like(p.dout, false) || !q_like(p.dq, true) ||
        !k_like(p.dk, true) || !k_like(p.dv, true))
        return NA_ERR_SHAPE;
    return NA_OK;
}

bool empty_sink(const na_sink_problem& p) { return p.batch == 0 || p.heads == 0 || p.tokens == 0; }

// Byte strides of one tensor of the problem.
void put_strides(const na_sink_problem& p, const na_strides& all, int64_t heads, int64_t& b,
                 int64_t& h, int64_t& t) {
    const na_strides s = used(all, p.batch, heads, p.tokens);
    const int64_t es = elem_bytes(p.dtype);
    b = s.batch * es;
    h = s.head * es;
    t = s.token * es;
}

void fill_sink(const na_sink_problem& p, const int32_t* lengths, na::SeqGeo& g) {
    fill_common(g, p.heads, p.kv_heads, p.kernel_size, p.sinks, p.scale);
    g.n = (int)p.tokens;
    g.B = (int)p.batch;
    g.ntiles = (int)((p.tokens * g.G + 127) / 128);
    g.fd_tiles.init(g.ntiles);
    g.fd_slices.init((int)(p.batch * p.kv_heads));
    g.runs = 2 * (int64_t)g.W < p.tokens;
    put_strides(p, p.q, p.heads, g.qb, g.qh, g.qt);
    put_strides(p, p.k, p.kv_heads, g.kb, g.kh, g.kt);
    put_strides(p, p.v, p.kv_heads, g.vb, g.vh, g.vt);
    put_strides(p, p.out, p.heads, g.ob, g.oh, g.ot);
    g.lb = p.heads * p.tokens;
    g.lh = p.tokens;
    g.lt = 1;
    g.lengths = lengths;
}

// The cut of dk, dv over workgroups, and the workspace: logsumexp and delta per row, then the
// fp32 parts.  Key tiles share the heads of a group among workgroups where they are fewer than
// the CUs, or, where windows are so long that the first key tiles have many times the rows of
// the last (1024 workgroups even that out: gradients of 16 heads on 4, 8192 tokens, full causal,
// bf16 D = 128 in 1000 us, with 256 aimed at 1370).  The rows behind the windows of first
// tokens are cut into short chunks, no more of them than fill the GPU four times over.
// False: too large to launch.
bool fill_backward(const na_sink_problem& p, const int32_t* lengths, na::SeqBwd& b, size_t& bytes) {
    std::memset(&b, 0, sizeof b);
    fill_sink(p, lengths, b.g);
    const na::SeqGeo& g = b.g;
    const int64_t n = p.tokens, slices = p.batch * p.kv_heads;
    b.scale = p.scale;
    const int64_t ktiles = (n + 127) / 128, base = slices * ktiles;
    const int64_t want = 2 * (int64_t)g.W >= n ? 1024 : 256;
    const int64_t hsplit = std::min<int64_t>(g.G, (want + base - 1) / base);
    int64_t blocks = 0, chunks = 1;
    if (g.S > 0 && n > g.W) {
        blocks = (std::min<int64_t>(g.S, n - g.W) + 31) / 32;
        const int64_t tiles = g.G * ((n - g.W) / 32 + 1);
        const int64_t share = 8 * 4;  // tiles of a workgroup: four for each of eight waves
        chunks = std::min((tiles + share - 1) / share,
                          std::max<int64_t>(1, 1024 / (slices * blocks)));
    }
    const int64_t first_jobs = slices * blocks * chunks;
    if (first_jobs + base * hsplit >= kMaxGrid / 2) return false;  // (up to 512 threads each)
    b.ktiles = (int)ktiles;
    b.hsplit = (int)hsplit;
    b.blocks = (int)blocks;
    b.chunks = (int)chunks;
    b.first_jobs = (int)first_jobs;
    b.fd_ktiles.init(b.ktiles);
    b.fd_hsplit.init(b.hsplit);
    b.fd_blocks.init(std::max(1, b.blocks));
    b.fd_chunks.init(b.chunks);
    const size_t rows = ((size_t)(p.batch * p.heads * n) + 3) / 4 * 4;
    const size_t key = 2 * (size_t)p.head_dim;
    const size_t part = (size_t)slices * key *
                        (hsplit > 1 ? (size_t)(hsplit * n) : (size_t)blocks * 32);
    const size_t first = (size_t)chunks * slices * blocks * 32 * key;
    bytes = (2 * rows + part + first) * 4;
    return true;
}

void place_workspace(const na_sink_problem& p, float* w, na::SeqBwd& b) {
    const size_t rows = ((size_t)(p.batch * p.heads * p.tokens) + 3) / 4 * 4;
    const size_t key = 2 * (size_t)p.head_dim;
    b.lse2 = w;
    b.delta = w + rows;
    b.part = w + 2 * rows;
    b.first_part = b.part + (size_t)(p.batch * p.kv_heads) * key *
                                (b.hsplit > 1 ? (size_t)b.hsplit * p.tokens : (size_t)b.blocks * 32);
}

// ---- paged cache ----
na_status check_cache(const na_cache_problem& p) {
    if (p.requests < 0 || p.tokens < 0 || p.requests >= kMaxGrid || p.tokens >= kMaxRows)
        return NA_ERR_SHAPE;
    if (p.pages < 0 || p.pages >= kMaxRows) return NA_ERR_SHAPE;
    if (p.page_size < 16 || p.page_size > (1 << 20) || (p.page_size & (p.page_size - 1)))
        return NA_ERR_SHAPE;
    return NA_OK;
}

na_status check_attention(const na_cache_problem& p) {
    na_status st = check_types(p.head_dim, p.dtype, p.scale);
    if (st != NA_OK) return st;
    if ((st = check_heads(p.heads, p.kv_heads, p.kernel_size, p.sinks)) != NA_OK) return st;
    if ((st = check_cache(p)) != NA_OK) return st;
    if (p.max_pages < 0 || p.max_pages >= kMaxRows || p.max_pages * p.page_size > kMaxRows ||
        p.requests * p.max_pages >= (int64_t(1) << 31) || p.max_new < 0 || p.max_context < 0)
        return NA_ERR_SHAPE;
    if (p.heads == 0 || p.tokens == 0 || p.requests == 0) return NA_OK;
    const int64_t G = p.heads / p.kv_heads;
    // (a page's bytes, and a row's offset in it, fit 32 bits)
    if (p.kv_heads * p.page_size * p.head_dim * elem_bytes(p.dtype) >= (int64_t(1) << 31))
        return NA_ERR_SHAPE;
    if (p.tokens * G >= kMaxRows - 256 || (p.tokens * G / 32 + p.requests) >= kMaxGrid ||
        (p.tokens * G / 32 + p.requests) * p.kv_heads >= kMaxGrid)
        return NA_ERR_SHAPE;
    const int es = elem_bytes(p.dtype);
    if (!good_strides(p.q, es, 1, p.heads, p.tokens, p.head_dim, false) ||
        !good_strides(p.out, es, 1, p.heads, p.tokens, p.head_dim, true))
        return NA_ERR_SHAPE;
    return NA_OK;
}

// Few new tokens per request (their rows fill one block of 32): the narrow form.
bool cache_narrow(const na_cache_problem& p) {
    const int64_t most = p.max_new > 0 ? std::min(p.max_new, p.tokens) : p.tokens;
    return most * (p.heads / p.kv_heads) <= 32;
}

// Splits the keys of a row tile when the row tiles alone would leave the 256 CUs idle (the wide
// form: two workgroups a CU) or, in the narrow form, unevenly loaded: the bound is the longest
// request's length, so requests of mixed lengths fill about half of the splits.
//   A split costs a second launch (4 us) that joins, so 16-bit types have at least 8 key tiles a
// split and split no fewer than 24 (narrow, whose four waves share a split's tiles: 12 and 40);
// the products of fp32 take sixteen times as long, and 2 (8) tiles are enough.  bf16, 16 heads
// on 4, D = 128, 64 new tokens over 8000: 37 us with 32 tiles a split at least, 27 with 16, 21
// with 8, 24 with 4; one new token for each of 8 requests of 3000: 19 with 32, 15 with 12, 17
// with 8.  fp32, 6 heads on 1, D = 64, 100 tokens of 5 requests, window 255: 32, 22 and 18 us
// with 8, 4 and 2.
//   fp32 over its range (captured; 4 requests of 64 new tokens or 8 of one, 6 heads on 1; wide with 2,
// 4, 8 tiles a split at least, unsplit): 3 tiles, D = 32 11.0, 12.4, 10.6, 10.6 us, D = 128 25.9, 33.3,
// 31.5, 31.4; 8 tiles 11.1, 14.3, 20.2, 18.3 and 27, 39, 60, 60; 38 tiles 17, 16, 21, 67 and 55, 44, 63,
// 241.  Narrow with 4, 8, 16: 19 tiles, D = 32 8.3, 9.9, 12.9, D = 128 21, 33, 57; 75 tiles at 16
// heads on 4 14.9, 13.1, 13.3 and 57, 64, 61.
//   The bounds of 24 and 40 tiles, bf16 (split, unsplit): wide, 21 tiles 13.4 and 18.7 us at D = 32, 21
// and 26 at D = 128, 40 tiles 13 and 32, 21 and 43; narrow, 38 tiles 8.1 and 10.2, 10.4 and 16, 75 tiles
// 9 and 16, 11.5 and 27.  (So lower ones would pay; those of half the size were right at 9 tiles,
// where nothing was split either way.)
//   Decoding over 8k to 32k contexts (32 requests, 4 key heads, fp16 D = 128) with 512, 1024,
// 2048 and 4096 splits aimed at: 254, 224, 236, 252 us.
void fill_split(const na_cache_problem& p, bool narrow, na::SeqGeo& g) {
    const int64_t M = narrow ? 32 : 128;
    const int64_t rows = p.tokens * g.G;
    g.ntiles = (int)(rows / M + p.requests);
    const int64_t room = p.max_pages * p.page_size;
    int64_t keys = p.max_context > 0 ? std::min(p.max_context, room) : room;
    keys = std::min(keys, (int64_t)g.W + g.S + M + 64);
    const int64_t tiles = std::max<int64_t>(1, (keys + 31) / 32 + 1);
    const int64_t busy = std::max<int64_t>((rows + M - 1) / M, std::min(p.requests, p.tokens)) * g.Hkv;
    int64_t split = std::min<int64_t>(na::kSeqMaxSplit,
                                      std::max<int64_t>(1, (narrow ? 1024 : 512) / busy));
    // (the joining launch has four workgroups a row tile)
    split = std::min(split, std::max<int64_t>(1, (kMaxGrid - 1) / (4 * (int64_t)g.ntiles * g.Hkv)));
    if (4 * (int64_t)g.ntiles * g.Hkv >= kMaxGrid) split = 1;
    const bool half = p.dtype != NA_FP32;
    const int64_t least = half ? (narrow ? 12 : 8) : (narrow ? 8 : 2);
    if (half && tiles < (narrow ? 40 : 24)) split = 1;
    const int64_t step = narrow ? 4 : 2;
    int64_t chunk = split == 1 ? tiles : std::max<int64_t>(least, (tiles + split - 1) / split);
    chunk = (chunk + step - 1) / step * step;
    g.chunk = (int)chunk;
    g.nsplit = (int)((tiles + chunk - 1) / chunk);
    g.fd_tiles.init(g.ntiles * g.Hkv);
}

size_t split_bytes(const na_cache_problem& p, bool narrow, const na::SeqGeo& g) {
    if (g.nsplit == 1) return 0;
    return (size_t)g.ntiles * g.Hkv * g.nsplit * (narrow ? 32 : 128) * (p.head_dim + 1) * 4;
}

}  // namespace

extern "C" {

na_status na_sink_forward(const na_sink_problem* problem, const void* q, const void* k,
                          const void* v, const int32_t* lengths, void* out, float* logsumexp,
                          na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_sink_problem& p = *problem;
    const na_status st = check_sink(p, false);
    if (st != NA_OK) return st;
    if (empty_sink(p)) return NA_OK;
    if (!q || !k || !v || !out || !logsumexp) return NA_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) ||
        !aligned(logsumexp, 16) || !aligned(lengths, 4))
        return NA_ERR_ALIGNMENT;
    na::SeqGeo g;
    fill_sink(p, lengths, g);
    return na::launch_seq_forward(g, (int)p.head_dim, p.dtype, false, false, q, k, v, out,
                                  logsumexp, nullptr, reinterpret_cast<hipStream_t>(stream)) ==
                   hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

size_t na_sink_backward_workspace(const na_sink_problem* problem) {
    na::SeqBwd b;
    size_t bytes = 0;
    if (!problem || check_sink(*problem, true) != NA_OK || empty_sink(*problem) ||
        !fill_backward(*problem, nullptr, b, bytes))
        return 0;
    return bytes;
}

na_status na_sink_backward(const na_sink_problem* problem, const void* q, const void* k,
                           const void* v, const int32_t* lengths, const void* out,
                           const float* logsumexp, const void* dout, void* dq, void* dk, void* dv,
                           void* workspace, size_t workspace_bytes, na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_sink_problem& p = *problem;
    const na_status st = check_sink(p, true);
    if (st != NA_OK) return st;
    if (empty_sink(p)) return NA_OK;
    const void* ptrs[] = {q, k, v, out, logsumexp, dout, dq, dk, dv};
    for (const void* x : ptrs)
        if (!x) return NA_ERR_NULL;
    for (const void* x : ptrs)
        if (!aligned(x, 16)) return NA_ERR_ALIGNMENT;
    if (!aligned(workspace, 16) || !aligned(lengths, 4)) return NA_ERR_ALIGNMENT;
    na::SeqBwd b;
    size_t need = 0;
    if (!fill_backward(p, lengths, b, need)) return NA_ERR_SHAPE;
    if (workspace_bytes < need) return NA_ERR_WORKSPACE;
    if (!workspace) return NA_ERR_NULL;
    place_workspace(p, static_cast<float*>(workspace), b);
    put_strides(p, p.dout, p.heads, b.gb, b.gh, b.gt);
    put_strides(p, p.dq, p.heads, b.qb, b.qh, b.qt);
    put_strides(p, p.dk, p.kv_heads, b.kb, b.kh, b.kt);
    put_strides(p, p.dv, p.kv_heads, b.vb, b.vh, b.vt);
    return na::launch_seq_backward(b, (int)p.head_dim, p.dtype, q, k, v, out, logsumexp, dout, dq,
                                   dk, dv, reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

na_status na_cache_tables(int64_t requests, int64_t tokens, int64_t page_size, int64_t max_pages,
                          int64_t num_free, const int32_t* context_lens, const int32_t* new_lens,
                          const int32_t* free_pages, const int32_t* head, int32_t* page_table,
                          int32_t* cu_new, int64_t* slots, int32_t* positions, int32_t* new_head,
                          na_stream_t stream) {
    if (requests < 0 || requests >= kMaxRows || tokens < 0 || tokens >= kMaxRows || num_free < 0 ||
        num_free >= kMaxRows || page_size < 16 || page_size > (1 << 20) ||
        (page_size & (page_size - 1)) || max_pages < 0 || max_pages >= kMaxRows ||
        max_pages * page_size > kMaxRows || requests * max_pages >= (int64_t(1) << 31))
        return NA_ERR_SHAPE;
    if (!cu_new || !new_head || (requests && (!context_lens || !new_lens)) ||
        (requests && max_pages && !page_table) || (num_free && !free_pages) ||
        (tokens && (!slots || !positions)))
        return NA_ERR_NULL;
    if (!aligned(context_lens, 4) || !aligned(new_lens, 4) || !aligned(free_pages, 4) ||
        !aligned(head, 4) || !aligned(page_table, 4) || !aligned(cu_new, 4) ||
        !aligned(slots, 8) || !aligned(positions, 4) || !aligned(new_head, 4))
        return NA_ERR_ALIGNMENT;
    if (head == new_head) return NA_ERR_SHAPE;
    return na::launch_cache_tables((int)requests, (int)tokens, __builtin_ctzll(page_size),
                                   (int)max_pages, (int)num_free, context_lens, new_lens,
                                   free_pages, head, page_table, cu_new, slots, positions,
                                   new_head, reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

na_status na_cache_write(const na_cache_problem* problem, const void* k, const void* v,
                         const int64_t* slots, void* k_pages, void* v_pages, na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_cache_problem& p = *problem;
    na_status st = check_types(p.head_dim, p.dtype, 1.f);
    if (st != NA_OK) return st;
    if ((st = check_cache(p)) != NA_OK) return st;
    if (p.kv_heads < 0 || p.kv_heads >= kMaxGrid) return NA_ERR_SHAPE;
    if (p.tokens == 0 || p.kv_heads == 0 || p.pages == 0) return NA_OK;
    const int es = elem_bytes(p.dtype);
    const int64_t row = p.head_dim * es;
    if (p.tokens * p.kv_heads >= kMaxRows || p.tokens * p.kv_heads * (row / 16) >= 2 * kMaxRows)
        return NA_ERR_SHAPE;
    if (!good_strides(p.k, es, 1, p.kv_heads, p.tokens, p.head_dim, false) ||
        !good_strides(p.v, es, 1, p.kv_heads, p.tokens, p.head_dim, false))
        return NA_ERR_SHAPE;
    if (!k || !v || !slots || !k_pages || !v_pages) return NA_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
        !aligned(slots, 8))
        return NA_ERR_ALIGNMENT;
    const na_strides ks = used(p.k, 1, p.kv_heads, p.tokens), vs = used(p.v, 1, p.kv_heads, p.tokens);
    return na::launch_cache_write((int)p.tokens, (int)p.kv_heads, (int)row,
                                  __builtin_ctzll(p.page_size), p.pages * p.page_size,
                                  ks.token * es, ks.head * es, vs.token * es, vs.head * es, k, v,
                                  slots, k_pages, v_pages,
                                  reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

size_t na_cache_attention_workspace(const na_cache_problem* problem) {
    if (!problem || check_attention(*problem) != NA_OK) return 0;
    const na_cache_problem& p = *problem;
    if (p.heads == 0 || p.tokens == 0 || p.requests == 0) return 0;
    na::SeqGeo g;
    fill_common(g, p.heads, p.kv_heads, p.kernel_size, p.sinks, p.scale);
    fill_split(p, cache_narrow(p), g);
    return split_bytes(p, cache_narrow(p), g);
}

na_status na_cache_attention(const na_cache_problem* problem, const void* q, const void* k_pages,
                             const void* v_pages, const int32_t* page_table,
                             const int32_t* context_lens, const int32_t* cu_new, void* out,
                             float* logsumexp, void* workspace, size_t workspace_bytes,
                             na_stream_t stream) {
    if (!problem) return NA_ERR_NULL;
    const na_cache_problem& p = *problem;
    const na_status st = check_attention(p);
    if (st != NA_OK) return st;
    if (p.heads == 0 || p.tokens == 0 || p.requests == 0) return NA_OK;
    // (a pool or a table without entries is never read)
    if (!q || !context_lens || !cu_new || !out || !logsumexp ||
        (p.pages > 0 && (!k_pages || !v_pages)) || (p.max_pages > 0 && !page_table))
        return NA_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) ||
        !aligned(logsumexp, 16) || !aligned(workspace, 16) || !aligned(page_table, 4) ||
        !aligned(context_lens, 4) || !aligned(cu_new, 4))
        return NA_ERR_ALIGNMENT;
    const bool narrow = cache_narrow(p);
    na::SeqGeo g;
    fill_common(g, p.heads, p.kv_heads, p.kernel_size, p.sinks, p.scale);
    fill_split(p, narrow, g);
    const size_t need = split_bytes(p, narrow, g);
    if (workspace_bytes < need) return NA_ERR_WORKSPACE;
    if (need && !workspace) return NA_ERR_NULL;
    const int64_t es = elem_bytes(p.dtype);
    g.n = (int)p.tokens;
    g.B = (int)p.requests;
    g.pages = (int)p.pages;
    g.max_pages = (int)p.max_pages;
    g.lgps = __builtin_ctzll(p.page_size);
    const na_strides qs = used(p.q, 1, p.heads, p.tokens), os = used(p.out, 1, p.heads, p.tokens);
    g.qh = qs.head * es;
    g.qt = qs.token * es;
    g.oh = os.head * es;
    g.ot = os.token * es;
    g.kt = g.vt = p.head_dim * es;
    g.kh = g.vh = g.kt << g.lgps;
    g.kb = g.vb = g.kh * p.kv_heads;
    g.lh = 1;
    g.lt = p.heads;
    g.context = context_lens;
    g.cu = cu_new;
    g.table = page_table;
    return na::launch_seq_forward(g, (int)p.head_dim, p.dtype, true, narrow, q, k_pages, v_pages,
                                  out, logsumexp, static_cast<float*>(workspace),
                                  reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? NA_OK
               : NA_ERR_HIP;
}

}  // extern "C"
