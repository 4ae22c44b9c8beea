// na_seq_host.h -- checks and fields that the host code of the sequence operators shares.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "na_seq.h"
#include "na_seq_kernels.h"

namespace na {
namespace host {

constexpr int64_t kMaxRows = int64_t(1) << 30;   // rows of a (sequence, key/value head), positions
constexpr int64_t kMaxGrid = int64_t(1) << 24;   // workgroups of 256 threads in 2^32 threads
constexpr int64_t kMaxToken = int64_t(1) << 26;  // bytes of a token stride

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline int elem_bytes(int dtype) { return dtype == NA_FP32 ? 4 : 2; }

inline na_status check_types(int64_t head_dim, int32_t dtype, float scale) {
    if (head_dim != 32 && head_dim != 64 && head_dim != 128) return NA_ERR_HEAD_DIM;
    if (dtype != NA_FP32 && dtype != NA_FP16 && dtype != NA_BF16) return NA_ERR_DTYPE;
    return std::isfinite(scale) ? NA_OK : NA_ERR_SCALE;
}

// Heads in whole groups (a key head without a query head has none: its gradients would be 0 that
// no launch writes), a window and first tokens that are counts.
inline na_status check_heads(int64_t heads, int64_t kv_heads, int64_t kernel_size, int64_t sinks) {
    if (heads < 0 || kv_heads < 0 || heads >= kMaxRows) return NA_ERR_SHAPE;
    if ((heads == 0) != (kv_heads == 0)) return NA_ERR_SHAPE;
    if (heads > 0 && heads % kv_heads != 0) return NA_ERR_SHAPE;
    if (kernel_size < 1) return NA_ERR_KERNEL_SIZE;
    return sinks < 0 ? NA_ERR_SHAPE : NA_OK;
}

// Strides as they are used: 0 on axes of one entry, whatever the caller has there.
inline na_strides used(const na_strides& s, int64_t batch, int64_t heads, int64_t tokens) {
    return {batch == 1 ? 0 : s.batch, heads == 1 ? 0 : s.head, tokens == 1 ? 0 : s.token};
}

// Strides of a [batch, heads, tokens, head_dim] tensor (see na_seq.h), its axes of more than one
// entry.  Outputs: those, ordered by stride, do not overlap.
inline bool good_strides(const na_strides& all, int es, int64_t batch, int64_t heads, int64_t tokens,
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
inline int clamp_window(int64_t x) { return (int)std::min<int64_t>(x, INT32_MAX - 128); }

// The fields that both forms of the attention share.
inline void fill_common(na::SeqGeo& g, int64_t heads, int64_t kv_heads, int64_t kernel_size,
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

inline na_status check_cache(const na_cache_problem& p) {
    if (p.requests < 0 || p.tokens < 0 || p.requests >= kMaxGrid || p.tokens >= kMaxRows)
        return NA_ERR_SHAPE;
    if (p.pages < 0 || p.pages >= kMaxRows) return NA_ERR_SHAPE;
    if (p.page_size < 16 || p.page_size > (1 << 20) || (p.page_size & (p.page_size - 1)))
        return NA_ERR_SHAPE;
    return NA_OK;
}

// out: whether the problem has one.
inline na_status check_attention(const na_cache_problem& p, bool out = true) {
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
        (out && !good_strides(p.out, es, 1, p.heads, p.tokens, p.head_dim, true)))
        return NA_ERR_SHAPE;
    return NA_OK;
}

// Few new tokens per request (their rows fill one block of 32): the narrow form.
inline bool cache_narrow(const na_cache_problem& p) {
    const int64_t most = p.max_new > 0 ? std::min(p.max_new, p.tokens) : p.tokens;
    return most * (p.heads / p.kv_heads) <= 32;
}

// The paged form's fields, of the tensors that a problem has.
inline void fill_paged(const na_cache_problem& p, na::SeqGeo& g) {
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
}

}  // namespace host
}  // namespace na
