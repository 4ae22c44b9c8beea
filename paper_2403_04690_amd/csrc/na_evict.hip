// na_evict.hip -- eviction from a paged cache by gathered attention weight (gfx950).
//
// Of a request with n > budget tokens a key/value head keeps its first f and its last l tokens, and of
// those between the k = budget - f - l of largest weight.  The places 0 .. budget - 1 then hold
//   the first tokens and, at their own places, the heavy ones below end = budget - l;
//   at the others below end ("holes"), in order, the heavy tokens from end on;
//   the last l tokens, in order, from end on.
// So only what has to moves: the last tokens, and the heavy ones that lie behind the places.
//
//   The k-th largest weight is found by its digits, from the upper end: a histogram of 11 bits of
// the weights that share the digits so far, three times (11, 11 and 10 bits).  Everything is
// whole numbers from there on, so the same weights always keep the same tokens.
#include "na_launch.h"
#include "na_shared.h"

namespace na {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kPer = 4;  // tokens of a thread in a pass in order
constexpr int kBins = 2048;

// Order of weights (by their bits) as whole numbers: equal for equal weights (-0 and 0 too), NaN
// below all.  (Weights are moved and compared as whole numbers throughout: the compiler may take a
// float for no NaN.)
__device__ __forceinline__ uint32_t weight_key(uint32_t u) {
    if ((u << 1) == 0) u = 0;
    if ((u << 1) > 0xff000000u) return 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_context(const EvictGeo& v, int r) {
    return min(max(v.context[r], 0), v.max_pages << v.lgps);
}

// What a request keeps: its first f and last l tokens, k of the others.
struct EvictSplit {
    int n, f, l, k, end;
    __device__ __forceinline__ void init(const EvictGeo& v, int r) {
        n = evict_context(v, r);
        f = v.first ? min(max(v.first[r], 0), v.budget) : 0;
        l = min(v.recent, v.budget - f);
        k = v.budget - f - l;
        end = v.budget - l;
    }
};

// Exclusive sum of x over the workgroup's threads, and the sum of all.  Two barriers.
__device__ __forceinline__ int block_scan(int x, int* waves, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int y = __shfl_up(s, d, kWave);
        s += lane >= d ? y : 0;
    }
    __syncthreads();  // (what was there is read)
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int c = waves[w];
        before += w < wave ? c : 0;
        total += c;
    }
    return before + s - x;
}

// The weights of one (request, key/value head): those behind the capacity are 0.
struct EvictRow {
    const uint32_t* w;
    int64_t capacity;
    __device__ __forceinline__ uint32_t at(int i) const { return i < capacity ? w[i] : 0u; }
};

// The k-th largest key of the tokens [lo, hi) (0 < k < hi - lo), how many tokens of that key
// belong to the k, and how many there are.
__device__ __forceinline__ void select_key(const EvictRow& row, int lo, int hi, int k, int* hist,
                                           int* waves, uint32_t& key, int& need, int& equal) {
    __shared__ uint32_t s_key;
    __shared__ int s_need, s_equal;
    key = 0;
    need = k;
    int shift = 32;
    for (int digit = 0; digit < 3; ++digit) {
        const int bits = digit < 2 ? 11 : 10;
        const uint32_t above = digit == 0 ? 0u : key >> shift;  // the digits so far
        for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
            const uint32_t x = weight_key(row.at(i));
            if (digit == 0 || x >> shift == above)
                atomicAdd(&hist[(x >> (shift - bits)) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
        // bins from the upper end: thread x has 2047 - 2 x and the one below
        const int b = kBins - 1 - 2 * (int)threadIdx.x;
        const int c0 = hist[b], c1 = hist[b - 1];
        int all;
        const int before = block_scan(c0 + c1, waves, all);
        if (before < need && need <= before + c0 + c1) {
            const bool second = need > before + c0;
            s_key = key | (uint32_t)(second ? b - 1 : b) << (shift - bits);
            s_need = need - before - (second ? c0 : 0);
            s_equal = second ? c1 : c0;
        }
        __syncthreads();
        key = s_key;
        need = s_need;
        equal = s_equal;
        shift -= bits;
    }
}

// Pages behind the budget's go back to the free list, request by request below its head.
__device__ __forceinline__ void return_pages(const EvictGeo& v, int* counts) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int page = 1 << v.lgps;
    const int keep = (int)(((int64_t)v.budget + page - 1) >> v.lgps);
    // the freed pages of request r that exist, visited by the wave
    auto visit = [&](int r, auto each) {
        int found = 0;
        if (r >= v.R) return found;
        const int n = evict_context(v, r);
        const int held = n > v.budget ? (int)(((int64_t)n + page - 1) >> v.lgps) : 0;
        for (int col = keep; col < held; col += 64) {
            int id = -1;
            if (col + lane < held) id = v.table[(int64_t)r * v.max_pages + col + lane];
            const bool ok = (unsigned)id < (unsigned)v.pages;
            const uint64_t m = __builtin_amdgcn_ballot_w64(ok);
            if (ok) each(found + __builtin_popcountll(m & ((1ull << lane) - 1)), id);
            found += __builtin_popcountll(m);
        }
        return found;
    };
    int64_t total = 0;
    for (int base = 0; base < v.R; base += kWaves)
        total += visit(base + wave, [](int, int) {});
    int64_t* sums = reinterpret_cast<int64_t*>(counts);  // of each wave
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kWaves; ++w) total += sums[w];
    int64_t at = (int64_t)*v.head - total;
    if (threadIdx.x == 0) *v.new_head = (int)max(at, (int64_t)0);
    __syncthreads();
    for (int base = 0; base < v.R; base += kWaves) {
        const int mine = visit(base + wave, [](int, int) {});
        if (lane == 0) sums[wave] = mine;
        __syncthreads();
        int64_t to = at;
        for (int w = 0; w < kWaves; ++w) {
            to += w < wave ? sums[w] : 0;
            at += sums[w];
        }
        visit(base + wave, [&](int x, int id) {
            if (to + x >= 0 && to + x < v.num_free) v.free_pages[to + x] = id;
        });
        __syncthreads();
    }
}

// A workgroup for each (request, key/value head) finds what stays and where it goes; the last one
// returns the pages.
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictGeo v) {
    __shared__ int hist[kBins];
    __shared__ __align__(8) int waves[2 * kWaves];
    const int slice = blockIdx.x;
    if (slice == v.R * v.Hkv) {
        return_pages(v, waves);
        return;
    }
    const int r = v.fd_kv.div(slice), kvh = slice - r * v.Hkv;
    EvictSplit p;
    p.init(v, r);
    const EvictRow row{v.weights + (int64_t)slice * v.capacity, v.capacity};
    int32_t* kept = v.kept + (int64_t)slice * v.budget;
    uint32_t* out = v.new_weights + (int64_t)slice * v.capacity;
    const int left = min(p.n, v.budget);
    if (kvh == 0 && threadIdx.x == 0) v.new_context[r] = left;
    for (int64_t i = left + (int)threadIdx.x; i < v.capacity; i += kThreads) out[i] = 0u;
    auto stay = [&](int i, uint32_t w) {
        kept[i] = i;
        if (i < v.capacity) out[i] = w;
    };
    if (p.n <= v.budget) {
        for (int i = threadIdx.x; i < v.budget; i += kThreads) {
            if (i < p.n) stay(i, row.at(i));
            else kept[i] = -1;
        }
        if (threadIdx.x == 0) v.moves[slice] = 0;
        return;
    }
    for (int i = threadIdx.x; i < p.f; i += kThreads) stay(i, row.at(i));
    for (int i = threadIdx.x; i < p.l; i += kThreads) {
        kept[p.end + i] = p.n - p.l + i;
        if (p.end + i < v.capacity) out[p.end + i] = row.at(p.n - p.l + i);
    }
    const int last = p.n - p.l;
    if (p.k == 0) {  // (then there are no places but the first and the last ones')
        if (threadIdx.x == 0) v.moves[slice] = 0;
        return;
    }
    uint32_t key;
    int need, equal;
    select_key(row, p.f, last, p.k, hist, waves, key, need, equal);

    // In order: which tokens are heavy, the holes below end, and the heavy ones behind it.
    int32_t* to = v.to + (int64_t)slice * v.budget;
    int32_t* from = v.from + (int64_t)slice * v.budget;
    int ties = 0, holes = 0, movers = 0;
    for (int side = 0; side < 2; ++side) {
        const int lo = side ? p.end : p.f, hi = side ? last : p.end;
        for (int base = lo; base < hi; base += kThreads * kPer) {
            const int i0 = base + (int)threadIdx.x * kPer;
            uint32_t w[kPer];
            bool heavy[kPer], is_tie[kPer];
            int mine = 0;
#pragma unroll
            for (int x = 0; x < kPer; ++x) {
                const int i = i0 + x;
                w[x] = i < hi ? row.at(i) : 0u;
                const uint32_t y = weight_key(w[x]);
                heavy[x] = i < hi && y >= key;
                is_tie[x] = i < hi && y == key;
                mine += is_tie[x];
            }
            int all;
            if (need < equal) {  // (uniform) the first `need` of the equal ones
                int at = ties + block_scan(mine, waves, all);
                ties += all;
#pragma unroll
                for (int x = 0; x < kPer; ++x)
                    if (is_tie[x] && at++ >= need) heavy[x] = false;
            }
            mine = 0;
#pragma unroll
            for (int x = 0; x < kPer; ++x) mine += i0 + x < hi && heavy[x] == (side == 1);
            int at = (side ? movers : holes) + block_scan(mine, waves, all);
            (side ? movers : holes) += all;
#pragma unroll
            for (int x = 0; x < kPer; ++x) {
                const int i = i0 + x;
                if (i >= hi) continue;
                if (side == 0 && heavy[x]) stay(i, w[x]);
                if (side == 0 && !heavy[x]) to[at++] = i;
                if (side == 1 && heavy[x]) {
                    const int place = to[at];
                    from[at++] = i;
                    kept[place] = i;
                    if (place < v.capacity) out[place] = w[x];
                }
            }
        }
        __syncthreads();  // (the holes are written)
    }
    if (threadIdx.x == 0) v.moves[slice] = movers;
}

// Moves the rows of a (request, key/value head), a workgroup for each slice of their bytes, K and V
// alike, so that a slice's moves follow each other without waiting for another workgroup.  First the
// heavy ones into the holes (no place of one is where another one lies), then the last tokens,
// in order: every place lies before its source, so what a pass writes is read already.
constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 8;  // rows of a thread in flight

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(
    EvictGeo v, unsigned char* k_pages, unsigned char* v_pages) {
    const int lgs = v.lgrow - v.lgslice;  // log2 of the slices of a row
    const int id = blockIdx.x >> (lgs + 1), part = blockIdx.x & ((2 << lgs) - 1);
    const int r = v.fd_kv.div(id), kvh = id - r * v.Hkv;
    EvictSplit p;
    p.init(v, r);
    if (p.n <= v.budget) return;
    const int moves = v.moves[id];
    unsigned char* pages = (part & 1 ? v_pages : k_pages) + ((part >> 1) << v.lgslice);
    const int lgt = v.lgslice - 4;  // log2 of the threads of a row
    const int seg = (threadIdx.x & ((1 << lgt) - 1)) << 4;
    const int row = threadIdx.x >> lgt, rows = kMoveThreads >> lgt;
    const int32_t* table = v.table + (int64_t)r * v.max_pages;
    auto place = [&](int j) -> unsigned char* {
        const int page = table[j >> v.lgps];  // (j < max_pages pages)
        if ((unsigned)page >= (unsigned)v.pages) return nullptr;
        const int64_t at = ((((int64_t)page * v.Hkv + kvh) << v.lgps) + (j & ((1 << v.lgps) - 1)));
        return pages + (at << v.lgrow) + seg;
    };
    auto pass = [&](int base, int count, auto to, auto from, bool ordered) {
        i32x4 x[kMoveRows];
        unsigned char* dst[kMoveRows];
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            const int i = base + u * rows + row;
            dst[u] = nullptr;
            if (i < count) {
                const unsigned char* src = place(from(i));
                dst[u] = place(to(i));
                x[u] = src ? ld16<i32x4>(src) : i32x4{0, 0, 0, 0};
            }
        }
        if (ordered) __syncthreads();  // every thread's rows are read
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u)
            if (dst[u]) st16(dst[u], x[u]);
    };
    const int32_t* to = v.to + (int64_t)id * v.budget;
    const int32_t* from = v.from + (int64_t)id * v.budget;
    for (int base = 0; base < moves; base += kMoveRows * rows)
        pass(base, moves, [&](int i) { return to[i]; }, [&](int i) { return from[i]; }, false);
    __syncthreads();
    for (int base = 0; base < p.l; base += kMoveRows * rows)
        pass(base, p.l, [&](int i) { return p.end + i; }, [&](int i) { return p.n - p.l + i; }, true);
}

}  // namespace

hipError_t launch_cache_evict(const EvictGeo& v, void* k_pages, void* v_pages, hipStream_t st) {
    const unsigned slices = (unsigned)v.R * v.Hkv;
    hipLaunchKernelGGL(evict_select_kernel, dim3(slices + 1), dim3(kThreads), 0, st, v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || slices == 0 || v.pages == 0) return e;
    hipLaunchKernelGGL(evict_move_kernel, dim3(slices << (v.lgrow - v.lgslice + 1)),
                       dim3(kMoveThreads), 0, st, v, static_cast<unsigned char*>(k_pages),
                       static_cast<unsigned char*>(v_pages));
    return hipGetLastError();
}

}  // namespace na
