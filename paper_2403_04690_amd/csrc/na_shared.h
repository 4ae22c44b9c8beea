// na_shared.h -- what the host hands to the kernels of the cache operators for long contexts
// (na_shared.hip, na_weights.hip, na_evict.hip).
#pragma once

#include "na_seq_kernels.h"

namespace na {

// One of the two problems of the attention with shared first tokens: row tiles, and the cut of
// their keys.
struct SharedSide {
    int ntiles;  // row tiles of a key/value head, of all groups or requests
    int nsplit;  // key splits of a row tile (0: the problem does not exist)
    int chunk;   // key tiles of a split
    int narrow;  // tiles of 32 rows instead of 128
    FastDiv fd_tiles;  // divides by the row tiles of all key/value heads
};

struct SharedGeo {
    SeqGeo g;  // the requests (paged form); ntiles as own_side's
    int groups;
    SharedSide shared_side, own_side;
    int shared_jobs;  // workgroups of shared_side
    const int32_t *cu_groups, *shared;
    float *part, *part_lse;  // [parts][tokens][heads] of D values, and of logsumexps
};

hipError_t launch_shared_attention(const SharedGeo& s, int D, int dtype, const void* q,
                                   const void* k, const void* v, void* out, float* lse,
                                   hipStream_t st);

// Gathered weights: g's ntiles are unused, its nsplit and chunk cut the key tiles of a request.
struct WeightsGeo {
    SeqGeo g;
    int64_t capacity;      // weights of a (request, key/value head)
    int form;              // 0: few rows, 1: many
    int shares, lgshares;  // workgroups that share the rows of the same keys (form 1)
    int joins;             // workgroups that add up the shares of a (request, key/value head)
    FastDiv fd_joins;
    int64_t part_keys;     // sums of a (request, key/value head) in part[shares][..][part_keys]
    float* part;
    const int32_t* first;  // keys before it gather nothing, or null
    const float* lse;
    float* weights;
};

hipError_t launch_cache_weights(const WeightsGeo& w, int D, int dtype, const void* q, const void* k,
                                hipStream_t st);

struct EvictGeo {
    int R, Hkv, budget, recent, lgps, pages, max_pages, num_free;
    int lgrow;    // log2 of a key's bytes
    int lgslice;  // log2 of the bytes of a row that a workgroup moves in order
    int chunk, chunks;  // rows that a workgroup moves in any order, such workgroups of K or V
    int64_t capacity;
    FastDiv fd_kv, fd_chunks;
    const uint32_t* weights;  // (the bits of fp32)
    uint32_t* new_weights;
    const int32_t *context, *first, *table, *head;
    int32_t *free_pages, *new_context, *kept, *new_head;
    // by (request, key/value head): how many rows move to the place of another, and how many of
    // them from positions below the budget; [.][budget] the places that they get, where they are
    int32_t *moves, *to, *from;
};

hipError_t launch_cache_evict(const EvictGeo& v, void* k_pages, void* v_pages, hipStream_t st);

}  // namespace na
