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
// the weights that share the digits so far, at most three times (11, 11 and 10 bits).  Everything
// is whole numbers from there on, so the same weights always keep the same tokens.
#include <type_traits>

#include "na_launch.h"
#include "na_shared.h"

namespace na {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;

// Order of weights (by their bits) as whole numbers from 1 on: equal for equal weights (-0 and 0
// too), NaN below all.  (Weights are moved and compared as whole numbers throughout: the compiler
// may take a float for no NaN.)
__device__ __forceinline__ uint32_t weight_key(uint32_t u) {
    if ((u << 1) == 0) u = 0;
    if ((u << 1) > 0xff000000u) return 1;
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

// Digits of the keys from the upper end: add(integral_constant<digit>, key) counts into hist the
// digits of that number of the keys whose digits before it are key's.  Leaves in key the k-th largest
// key, or one that just k keys are not below (need = equal); in need how many of that
// key belong to the k, in equal how many there are.
constexpr int digit_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }

template <typename Add>
__device__ __forceinline__ void select_digits(int k, int among, int* hist, int* waves,
                                              uint32_t* found, uint32_t& key, int& need, int& equal,
                                              Add add) {
    key = 0;
    need = k;
    equal = among;
    auto next = [&](auto digit) __attribute__((always_inline)) {
        constexpr int shift = digit_shift(decltype(digit)::value);
        for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        add(digit, key);
        __syncthreads();
        // bins from the upper end: thread x has 2047 - 2 x and the one below
        const int b = kBins - 1 - 2 * (int)threadIdx.x;
        const int c0 = hist[b], c1 = hist[b - 1];
        int all;
        const int before = block_scan(c0 + c1, waves, all);
        if (before < need && need <= before + c0 + c1) {
            const bool second = need > before + c0;
            found[0] = key | (uint32_t)(second ? b - 1 : b) << shift;
            found[1] = (uint32_t)(need - before - (second ? c0 : 0));
            found[2] = (uint32_t)(second ? c1 : c0);
        }
        __syncthreads();
        key = found[0];
        need = (int)found[1];
        equal = (int)found[2];
    };
    next(std::integral_constant<int, 0>{});
    if (need < equal) next(std::integral_constant<int, 1>{});
    if (need < equal) next(std::integral_constant<int, 2>{});
}

// Bits of the tokens lo .. hi - 1 in a block of 64 tokens from `base` on (all uniform).
__device__ __forceinline__ uint64_t block_bits(int base, int lo, int hi) {
    const int a = min(max(lo - base, 0), 64), b = min(max(hi - base, 0), 64);
    const uint64_t below_b = b == 64 ? ~0ull : (1ull << b) - 1;
    const uint64_t below_a = a == 64 ? ~0ull : (1ull << a) - 1;
    return below_b & ~below_a;
}
__device__ __forceinline__ int rank_in(uint64_t bits) {  // set bits of the lanes before this one
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
}

// f(u, weight(u)) for the blocks u of [first, m) of a wave.  SLOTS: m is at most that, unrolled;
// 0: any number, the weights of eight blocks read before the first is used (of sixteen: the same
// times, 67 us for 64 heads of 8k to 32k tokens).
template <int SLOTS, typename Weight, typename F>
__device__ __forceinline__ void each_block(int first, int m, Weight weight, F f) {
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int u = 0; u < SLOTS; ++u)
            if (u >= first && u < m) f(u, weight(u));
    } else {
        for (int u0 = first; u0 < m; u0 += 8) {
            uint32_t w[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) w[x] = weight(min(u0 + x, m - 1));
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (u0 + x < m) f(u0 + x, w[x]);
        }
    }
}

// Chooses the heavy ones of a context's tokens up to the last ones, and says where tokens go.
// Wave x has a run of m blocks of 64 tokens.  SLOTS: m is at most that, and the weights stay in
// registers; 0: they are read again for each of the up to six steps.
template <int SLOTS>
__device__ __forceinline__ void evict_choose(const EvictGeo& v, const EvictSplit& p, int slice,
                                             const uint32_t* __restrict__ weights,
                                             uint32_t* __restrict__ out, int32_t* __restrict__ kept,
                                             int* hist, int* waves, uint32_t* found) {
    const int lane = threadIdx.x & 63, last = p.n - p.l;
    const int m = (last + kThreads - 1) / kThreads;
    const int base = uniform(((int)threadIdx.x >> 6) * m * 64);
    const int cap = (int)min(v.capacity, (int64_t)last);  // (weights behind it are 0)
    int32_t* to = v.to + (int64_t)slice * v.budget;  // (holes are written, then read)
    int32_t* __restrict__ from = v.from + (int64_t)slice * v.budget;
    uint32_t held[SLOTS > 0 ? SLOTS : 1];
    auto read = [&](int u) __attribute__((always_inline)) {
        if (cap == 0) return 0u;  // (uniform)
        const int i = base + u * 64 + lane;
        const uint32_t w = weights[min(i, cap - 1)];  // (loads of several blocks in flight)
        return i < cap ? w : 0u;
    };
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int u = 0; u < SLOTS; ++u) held[u] = u < m ? read(u) : 0u;
    }
    auto weight = [&](int u) __attribute__((always_inline)) {
        if constexpr (SLOTS > 0) return held[u];
        else return read(u);
    };
    const int room = (int)min(v.capacity, (int64_t)v.budget);
    auto put = [&](int i, int j, uint32_t w) __attribute__((always_inline)) {
        kept[i] = j;
        if (i < room) out[i] = w;
    };
    // whether all of block u is to choose from (the others, at the ends, take their bits)
    auto inner = [&](int u) __attribute__((always_inline)) {
        return base + u * 64 >= p.f && base + u * 64 + 64 <= last;
    };
    uint32_t least;
    int need, equal;
    select_digits(p.k, last - p.f, hist, waves, found, least, need, equal,
                  [&](auto digit, uint32_t above) __attribute__((always_inline)) {
        constexpr int kDigit = decltype(digit)::value, kShift = digit_shift(kDigit);
        each_block<SLOTS>(0, m, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
            const uint32_t x = weight_key(w);
            bool count = true;
            if constexpr (kDigit > 0)
                count = (x ^ above) >> digit_shift(kDigit - 1) == 0;
            if (!inner(u)) {
                const int i = base + u * 64 + lane;
                count = count && i >= p.f && i < last;
            }
            if (count) atomicAdd(&hist[x >> kShift & (kDigit == 2 ? 1023 : 2047)], 1);
        });
    });
    // bits of the heavy ones of block u
    const bool some = need < equal;  // (uniform) not all of the equal ones
    int ties = 0;                    // equal ones before the block
    // (the least weight above 0: weights are not below it where their bits are from its on, up to
    // infinity's)
    const bool above_0 = least > 0x80000000u;
    const uint32_t first = least & 0x7fffffffu, range = 0x7f800000u - first;
    auto bits_of = [&](int u, uint64_t x) __attribute__((always_inline)) {
        return inner(u) ? x : x & block_bits(base + u * 64, p.f, last);
    };
    auto equal_to = [&](int u, uint32_t w) __attribute__((always_inline)) {
        return bits_of(u, __builtin_amdgcn_ballot_w64(weight_key(w) == least));
    };
    auto heavy = [&](int u, uint32_t w) __attribute__((always_inline)) {
        uint64_t h;
        if (above_0) h = __builtin_amdgcn_ballot_w64(w - first <= range);
        else h = __builtin_amdgcn_ballot_w64(weight_key(w) >= least);
        h = bits_of(u, h);
        if (some) {
            const uint64_t e = equal_to(u, w);
            h &= ~(e & __builtin_amdgcn_ballot_w64(ties + rank_in(e) >= need));
            ties += __builtin_popcountll(e);
        }
        return h;
    };
    int all, ties0 = 0;
    if (some) {
        int mine = 0;
        each_block<SLOTS>(0, m, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
            mine += __builtin_popcountll(equal_to(u, w));
        });
        ties = ties0 = uniform(block_scan(lane == 0 ? mine : 0, waves, all));
    }
    // How many heavy ones the wave has, and how many of them before end; the others of its tokens
    // there are holes.
    int heavies = 0, fronts = 0;
    if (SLOTS == 0 && above_0 && !some) {
        // (each lane its own count, and one sum of them all: 2 us for 32 blocks, by ballots 10)
        int back = 0;
        each_block<SLOTS>(0, m, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
            const int i = base + u * 64 + lane;
            const bool h = w - first <= range && i >= p.f && i < last;
            fronts += h && i < p.end;
            back += h && i >= p.end;
        });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            fronts += __shfl_xor(fronts, d, kWave);
            back += __shfl_xor(back, d, kWave);
        }
        heavies = fronts + back;
    } else {
        each_block<SLOTS>(0, m, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
            const int b = base + u * 64;
            const uint64_t h = heavy(u, w);
            heavies += __builtin_popcountll(h);
            if (b + 64 <= p.end) fronts += __builtin_popcountll(h);
            else if (b < p.end) fronts += __builtin_popcountll(h & block_bits(b, 0, p.end));
        });
    }
    const int mine = max(min(base + m * 64, p.end) - max(base, p.f), 0);
    int holes = uniform(block_scan(lane == 0 ? mine - fronts : 0, waves, all));
    if (threadIdx.x == 0) {
        v.moves[2 * slice] = all;
        found[0] = 0;
    }
    int movers = uniform(block_scan(lane == 0 ? heavies - fronts : 0, waves, all));
    ties = ties0;
    const int front = min(max((p.end - base + 63) >> 6, 0), m);  // blocks that begin before end
    each_block<SLOTS>(0, front, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
        const int b = base + u * 64, i = b + lane;
        uint64_t hole = ~heavy(u, w), range = ~0ull;
        if (!inner(u) || b + 64 > p.end) {
            range = block_bits(b, p.f, p.end);
            hole &= range;
        }
        if (hole >> lane & 1) to[holes + rank_in(hole)] = i;
        else if (range >> lane & 1) put(i, i, w);
        holes += __builtin_popcountll(hole);
    });
    __syncthreads();  // (every hole is written)
    // (ties: of the blocks before `back` too)
    const int back = some ? 0 : min(max((p.end - base) >> 6, 0), m);
    ties = ties0;
    each_block<SLOTS>(back, m, weight, [&](int u, uint32_t w) __attribute__((always_inline)) {
        const int b = base + u * 64, i = b + lane;
        uint64_t mover = heavy(u, w);
        if (b < p.end) mover &= ~block_bits(b, 0, p.end);
        if (mover >> lane & 1) {
            const int at = movers + rank_in(mover);
            from[at] = i;
            put(to[at], i, w);
            if (i < v.budget) atomicMax(&found[0], (uint32_t)at + 1);
        }
        movers += __builtin_popcountll(mover);
    });
    __syncthreads();
    if (threadIdx.x == 0) v.moves[2 * slice + 1] = (int)found[0];
}

// Pages behind the budget's go back to the free list, request by request below its head: the freed
// pages of 1024 requests at a time in one row, a thread each; first counted, then written.
__device__ __forceinline__ void return_pages(const EvictGeo& v, int* offsets, int* waves) {
    const int tid = threadIdx.x, page = 1 << v.lgps;
    const int keep = (int)(((int64_t)v.budget + page - 1) >> v.lgps);
    int64_t at = 0;
    int id = -1;
    bool have = false;  // (uniform) id holds this thread's page of all there are
    for (int step = 0; step < 2; ++step) {
        int64_t total = 0;
        for (int base = 0; base < v.R; base += kThreads) {
            int freed = 0, all, valid;
            if (!have) {
                if (base + tid < v.R) {
                    const int n = evict_context(v, base + tid);
                    const int held = (int)(((int64_t)n + page - 1) >> v.lgps);
                    freed = n > v.budget ? held - keep : 0;
                }
                const int before = block_scan(freed, waves, all);
                offsets[tid] = before;
                __syncthreads();
            } else {
                all = kThreads;
            }
            for (int s0 = 0; s0 < all; s0 += kThreads) {
                const int s = s0 + tid;
                if (!have) {
                    id = -1;
                    if (s < all) {
                        int x = 0;  // the last request whose pages begin at or before s
#pragma unroll
                        for (int bit = kThreads / 2; bit > 0; bit >>= 1)
                            x += offsets[x + bit] <= s ? bit : 0;
                        id = v.table[(int64_t)(base + x) * v.max_pages + keep + s - offsets[x]];
                    }
                }
                const bool ok = (unsigned)id < (unsigned)v.pages;
                const int rank = block_scan(ok, waves, valid);
                const int64_t to = at + total + rank;
                if (step == 1 && ok && to >= 0 && to < v.num_free) v.free_pages[to] = id;
                total += valid;
            }
            have = v.R <= kThreads && all <= kThreads;
            __syncthreads();
        }
        if (step == 0) {
            at = (int64_t)*v.head - total;
            if (tid == 0) *v.new_head = (int)max(at, (int64_t)0);
        }
    }
}

// A workgroup for each (request, key/value head) finds what stays and where it goes; the last one
// returns the pages.  Bound by a chain of loads, barriers and scans: 18 us for 256 heads of 2100 tokens,
// 67 us for 64 heads of 8k to 32k tokens (74 % of the waves' cycles wait).  Registers for the weights
// of all 32 blocks of a long context instead of reading them again: 61 us and 5 us more for short
// ones, whose code it was too.
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictGeo v) {
    __shared__ int hist[kBins];
    __shared__ int waves[kWaves];
    __shared__ uint32_t found[3];
    const int slice = blockIdx.x;
    if (slice == v.R * v.Hkv) {
        return_pages(v, hist, waves);
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
    // token `from` with weight w goes to place i
    auto put = [&](int i, int from, uint32_t w) __attribute__((always_inline)) {
        kept[i] = from;
        if (i < v.capacity) out[i] = w;
    };
    const int last = p.n - p.l;
    // (read now, written at the end: the loads' latency passes meanwhile)
    const int tid = threadIdx.x;
    const uint32_t front = p.n > v.budget && tid < p.f ? row.at(tid) : 0u;
    const uint32_t back = p.n > v.budget && tid < p.l ? row.at(last + tid) : 0u;
    if (p.n > v.budget && p.k > 0) {
        if (last <= 4 * kThreads)
            evict_choose<4>(v, p, slice, row.w, out, kept, hist, waves, found);
        else
            evict_choose<0>(v, p, slice, row.w, out, kept, hist, waves, found);
    } else if (threadIdx.x < 2) {  // (k = 0: there are no places but the first and the last ones')
        v.moves[2 * slice + threadIdx.x] = 0;
    }
    for (int64_t i = left + (int)threadIdx.x; i < v.capacity; i += kThreads) out[i] = 0u;
    if (p.n <= v.budget) {
        for (int i = threadIdx.x; i < v.budget; i += kThreads) {
            if (i < p.n) put(i, i, row.at(i));
            else kept[i] = -1;
        }
        return;
    }
    for (int i = tid; i < p.f; i += kThreads) put(i, i, i == tid ? front : row.at(i));
    for (int i = tid; i < p.l; i += kThreads)
        put(p.end + i, last + i, i == tid ? back : row.at(last + i));
}

constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 8;  // rows of a thread in flight

// A workgroup's share of the rows of a (request, key/value head): 16 bytes a thread.
struct EvictMover {
    unsigned char* pages;  // the first byte of the thread's segment in the head's first row
    const int32_t* table;
    int lgps, count;
    int64_t head_rows, kvh_rows;
    int lgrow, row, rows;  // this thread's row of a pass, rows of a pass

    __device__ __forceinline__ void init(const EvictGeo& v, int r, int kvh, unsigned char* p, int byte,
                                         int lgslice) {
        const int lgt = lgslice - 4;  // log2 of the threads of a row
        pages = p + byte + ((threadIdx.x & ((1 << lgt) - 1)) << 4);
        table = v.table + (int64_t)r * v.max_pages;
        lgps = v.lgps;
        count = v.pages;
        head_rows = (int64_t)v.Hkv << lgps;
        kvh_rows = (int64_t)kvh << lgps;
        lgrow = v.lgrow;
        row = threadIdx.x >> lgt;
        rows = kMoveThreads >> lgt;
    }
    __device__ __forceinline__ unsigned char* place(int j) const {
        const int page = table[j >> lgps];  // (j < max_pages pages)
        if ((unsigned)page >= (unsigned)count) return nullptr;
        return pages + ((page * head_rows + kvh_rows + (j & ((1 << lgps) - 1))) << lgrow);
    }
    // rows base .. base + kMoveRows * rows - 1 (below end) of those that `from` and `to` name
    template <bool ORDERED, typename To, typename From>
    __device__ __forceinline__ void pass(int base, int end, To to, From from) const {
        i32x4 x[kMoveRows];
        unsigned char* dst[kMoveRows];
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u) {
            const int i = base + u * rows + row;
            dst[u] = nullptr;
            if (i < end) {
                const unsigned char* src = place(from(i));
                dst[u] = place(to(i));
                x[u] = src ? ld16<i32x4>(src) : i32x4{0, 0, 0, 0};
            }
        }
        if constexpr (ORDERED) __syncthreads();  // every thread's rows are read
#pragma unroll
        for (int u = 0; u < kMoveRows; ++u)
            if (dst[u]) st16(dst[u], x[u]);
    }
};

// Rows to their places.  Heavy tokens from position `budget` on lie where nothing is written, and
// go to holes that nobody reads: any order, `chunk` of them to a workgroup of whole rows.  Those
// before it, and the last tokens, are in each other's way: a workgroup for each slice of the
// bytes of K and of V moves its slice of them all, first the heavy ones, then the last ones in
// order (a place lies before its source, so what a pass writes is read already).  Slices
// let few requests fill the GPU; whole rows are read faster where many move (8 prompts of 8k to 32k tokens
// cut to 4096, 8 heads, bf16 D = 128: 113 us with slices alone, 80 with both, 2.6 TB/s; trimming
// 64 requests of 2049 to 2304 tokens to 2048, 4 heads: 26 us, 3.6 TB/s).
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictGeo v, unsigned char* k_pages,
                                                                  unsigned char* v_pages) {
    const int lgs = v.lgrow - v.lgslice;  // log2 of the slices of a row
    const int ordered = v.R * v.Hkv << (lgs + 1);
    EvictMover m;
    EvictSplit p;
    if ((int)blockIdx.x < ordered) {
        const int id = blockIdx.x >> (lgs + 1), part = blockIdx.x & ((2 << lgs) - 1);
        const int r = v.fd_kv.div(id), kvh = id - r * v.Hkv;
        p.init(v, r);
        if (p.n <= v.budget) return;
        const int moves = v.moves[2 * id + 1];
        m.init(v, r, kvh, part & 1 ? v_pages : k_pages, (part >> 1) << v.lgslice, v.lgslice);
        const int32_t* to = v.to + (int64_t)id * v.budget;
        const int32_t* from = v.from + (int64_t)id * v.budget;
        for (int base = 0; base < moves; base += kMoveRows * m.rows)
            m.pass<false>(base, moves, [&](int i) { return to[i]; }, [&](int i) { return from[i]; });
        __syncthreads();
        for (int base = 0; base < p.l; base += kMoveRows * m.rows)
            m.pass<true>(base, p.l, [&](int i) { return p.end + i; },
                         [&](int i) { return p.n - p.l + i; });
        return;
    }
    const int share = v.fd_chunks.div(blockIdx.x - ordered);
    const int chunk = blockIdx.x - ordered - share * v.chunks;
    const int id = share >> 1, r = v.fd_kv.div(id), kvh = id - r * v.Hkv;
    if (evict_context(v, r) <= v.budget) return;
    const int first = v.moves[2 * id + 1] + chunk * v.chunk;
    const int end = min(v.moves[2 * id], first + v.chunk);
    if (first >= end) return;
    m.init(v, r, kvh, share & 1 ? v_pages : k_pages, 0, v.lgrow);
    const int32_t* to = v.to + (int64_t)id * v.budget;
    const int32_t* from = v.from + (int64_t)id * v.budget;
    for (int base = first; base < end; base += kMoveRows * m.rows)
        m.pass<false>(base, end, [&](int i) { return to[i]; }, [&](int i) { return from[i]; });
}

}  // namespace

hipError_t launch_cache_evict(const EvictGeo& v, void* k_pages, void* v_pages, hipStream_t st) {
    const unsigned slices = (unsigned)v.R * v.Hkv;
    hipLaunchKernelGGL(evict_select_kernel, dim3(slices + 1), dim3(kThreads), 0, st, v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || slices == 0 || v.pages == 0) return e;
    const unsigned ordered = slices << (v.lgrow - v.lgslice + 1);
    hipLaunchKernelGGL(evict_move_kernel, dim3(ordered + 2 * slices * (unsigned)v.chunks),
                       dim3(kMoveThreads), 0, st, v, static_cast<unsigned char*>(k_pages),
                       static_cast<unsigned char*>(v_pages));
    return hipGetLastError();
}

}  // namespace na
