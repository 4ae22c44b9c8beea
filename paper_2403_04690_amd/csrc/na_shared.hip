// na_shared.hip -- attention of new tokens over a paged cache in which groups of requests share their
// first tokens: the shared keys are read once for all rows of a group (gfx950).
//
//   With a row's keys in two sets A and B, lse = log(e^lse_A + e^lse_B) and
//   out = e^(lse_A - lse) out_A + e^(lse_B - lse) out_B,
// so the shared keys are one problem of all the rows of a group (every request's new tokens times
// the heads of a key/value head), the keys behind them one problem a request, and a second
// launch joins the parts.  Each of the problems is cut into splits of its keys; every
// split of every row leaves a logsumexp (-inf where the row sees nothing of it, NaN where a score
// is NaN or +inf) and, unless it is -inf, its mean of the values, both in fp32.
//   64 requests of one token behind 8192 shared ones and 16 to 1024 of their own, 16 heads on 4, bf16
// D = 128: 28 us a call; read request by request (cache_attention over tables that list the shared
// pages) 97.  Chunks of 64 to 300 tokens of 16 requests behind 4k and 6k shared ones: 208 to 215 us
// (0.68 to 0.71 PFLOP/s), kernels 191 and 24; there the products bound both, the parts and their join come
// on top, and cache_attention takes 202.
#include <cmath>
#include <type_traits>

#include "na_launch.h"
#include "na_seq_state.h"
#include "na_shared.h"

namespace na {

namespace {

// A tile of rows against the keys [from, end) of a request, or of those that a group shares.
// (Where its rows are is SeqTile's, as seq_locate and seq_row take it.)
struct SharedTile : SeqTile {
    int r0, r1;       // requests that its rows belong to
    int from, end;    // keys of this side
    int s0;           // first tile of the first tokens
    // Requests stand at different positions: with a window shorter than they are apart there may be
    // keys between lo and end that no row sees.  Then `seen` has those of the tile that is staged
    // next (bit e: its key e), otherwise all bits.
    bool gaps;
    unsigned seen;

    // Rows at positions rmin .. rmax, keys [from, to).
    __device__ __forceinline__ void span(const SeqGeo& g, int rmin, int rmax, int to) {
        end = min(to, rmax + 1);
        pmax = end - 1;
        lo = max(rmin - g.W + 1, from);
        w0 = lo >> 5;
        s0 = from >> 5;
        gaps = rmax - rmin >= g.W;
        seen = ~0u;
        nS = nT = 0;
        if (end <= from) return;
        // (first tokens in the window's first tile come with it, if there is a window here)
        const bool window = lo < end;
        const int stop = (min(g.S, end) + 31) >> 5;
        nS = max(0, (window ? min(stop, w0) : stop) - s0);
        nT = nS + (window ? (pmax >> 5) - w0 + 1 : 0);
    }
    __device__ __forceinline__ int tile(int e) const { return (e < nS ? s0 + e : w0 + e - nS) << 5; }
    __device__ __forceinline__ bool sees(const SeqGeo& g, int j) const {
        return (j >= lo || j < g.S) && j >= from && j < end && (seen >> (j & 31) & 1);
    }
    __device__ __forceinline__ bool whole(const SeqGeo& g, int j0) const {
        return j0 >= from && j0 + 31 < end && (j0 >= lo || j0 + 31 < g.S) && seen == ~0u;
    }
    // Keys of the tile from j0 on that the rows at positions pos (N a lane) of the wave see.
    template <int N>
    __device__ __forceinline__ void look(const SeqGeo& g, int j0, const int (&pos)[N]) {
        unsigned m = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int d = pos[n] - j0;
            m |= below32(d + 1) & (~below32(d - g.W + 1) | below32(g.S - j0));
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) m |= __shfl_xor(m, x, kWave);
        seen = uniform((int)m);
    }
    __device__ __forceinline__ static unsigned below32(int x) {
        return x >= 32 ? ~0u : (1u << max(x, 0)) - 1u;
    }
};

// The last x of [lo, lo + span) with at(x) <= v (at does not decrease; lo where there is none): the
// lanes probe 64 places at a time.
template <typename At>
__device__ __forceinline__ int last_at(int lo, int span, int v, int lane, At at) {
    while (span > 1) {
        const int step = (span + 63) >> 6;
        const bool in = lane * step < span && at(lo + lane * step) <= v;
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
        const int skip = (n > 0 ? n - 1 : 0) * step;
        lo += skip;
        span = min(step, span - skip);
    }
    return uniform(lo);
}

__device__ __forceinline__ int context_of(const SeqGeo& g, int c) {
    return min(max(c, 0), g.max_pages << g.lgps);
}
// What every lane reads first, for all that follows: group `lane` (where there are at most 64).
struct Groups {
    int begin, end, shared;
    __device__ __forceinline__ void load(const SharedGeo& s, int lane) {
        begin = end = INT32_MAX;
        shared = 0;
        if (s.groups > 64 || lane >= s.groups) return;
        begin = s.cu_groups[lane];
        end = s.cu_groups[lane + 1];
        shared = s.shared[lane];
    }
};

// Row tile `tile` of M = 2^lgM rows of the groups -> its rows.  False: no such tile.  Group x has
// tiles from floor(first row / M) + x on, at least as many as it needs.
__device__ __forceinline__ bool locate_group(const SharedGeo& s, const Groups& all, int tile, int lgM,
                                             int lane, SharedTile& t, int& to) {
    const SeqGeo& g = s.g;
    auto request = [&](int r) { return min(max(r, 0), g.B); };
    auto token = [&](int r) { return min(max(g.cu[request(r)], 0), g.n); };
    int x, start, n, shared;
    if (s.groups <= 64) {  // (two loads after each other)
        const bool in = lane < s.groups;
        const int a = in ? token(all.begin) : 0, b = in ? token(all.end) : 0;
        const uint64_t m = __builtin_amdgcn_ballot_w64(in && (a * g.G >> lgM) + lane <= tile);
        x = max(__builtin_popcountll(m) - 1, 0);
        t.r0 = __builtin_amdgcn_readlane(all.begin, x);
        t.r1 = __builtin_amdgcn_readlane(all.end, x);
        start = __builtin_amdgcn_readlane(a, x);
        n = __builtin_amdgcn_readlane(b, x) - start;
        shared = __builtin_amdgcn_readlane(all.shared, x);
    } else {
        x = last_at(0, s.groups, tile, lane,
                    [&](int i) { return (token(s.cu_groups[i]) * g.G >> lgM) + i; });
        t.r0 = uniform(s.cu_groups[x]);
        t.r1 = uniform(s.cu_groups[x + 1]);
        start = uniform(token(t.r0));
        n = uniform(token(t.r1)) - start;
        shared = uniform(s.shared[x]);
    }
    t.r0 = request(t.r0);
    t.r1 = request(t.r1);
    if (t.r0 >= t.r1 || n <= 0) return false;
    const int at = tile - (start * g.G >> lgM) - x;
    if (at < 0 || at >= kSeqMaxTiles) return false;
    t.row0 = at << lgM;
    if (t.row0 < 0 || t.row0 >= n * g.G) return false;
    t.b = t.r0;
    t.rows = min(n * g.G - t.row0, 1 << lgM);
    t.qtok = start;
    t.pos0 = 0;
    t.valid = n;
    t.from = 0;
    to = context_of(g, shared);
    return true;
}

// Group of request r (-1: none) and the tokens that it shares.
__device__ __forceinline__ int group_of(const SharedGeo& s, const Groups& all, int r, int lane,
                                        int& shared) {
    shared = 0;
    if (s.groups == 0) return -1;
    int x, begin, end;
    if (s.groups <= 64) {
        const uint64_t m = __builtin_amdgcn_ballot_w64(all.begin <= r);  // (none behind the last)
        x = max(__builtin_popcountll(m) - 1, 0);
        begin = __builtin_amdgcn_readlane(all.begin, x);
        end = __builtin_amdgcn_readlane(all.end, x);
        shared = __builtin_amdgcn_readlane(all.shared, x);
    } else {
        x = last_at(0, s.groups, r, lane, [&](int i) { return s.cu_groups[i]; });
        begin = uniform(s.cu_groups[x]);
        end = uniform(s.cu_groups[x + 1]);
        shared = uniform(s.shared[x]);
    }
    shared = context_of(s.g, shared);
    if (begin <= r && r < end) return x;
    shared = 0;
    return -1;
}

// Position of row `tok` of q (each lane its own; `least` the wave's least) among the requests
// [r0, r1), whose offsets do not decrease.
__device__ __forceinline__ int position_of(const SeqGeo& g, int r0, int r1, int least, int tok,
                                           int lane) {
    int base = r0, pos = 0;
    if (r1 - r0 > 64)
        base = last_at(r0, r1 - r0, least, lane, [&](int i) { return g.cu[i]; });
    for (;;) {
        const int r = min(base + lane, r1 - 1);
        const int c = g.context[r];
        const int start = base + lane < r1 ? max(g.cu[r], 0) : INT32_MAX;
        int i = 0;  // the last of these requests that begins at or before tok
#pragma unroll
        for (int bit = 32; bit > 0; bit >>= 1) {
            const int at = __shfl(start, i + bit, kWave);
            i += at <= tok ? bit : 0;
        }
        const int begin = __shfl(start, i, kWave), cached = __shfl(c, i, kWave);
        if (begin <= tok) pos = context_of(g, cached) + tok - begin;
        base += 64;
        if (base >= r1 ||
            __builtin_amdgcn_ballot_w64(max(g.cu[base], 0) <= tok) == 0)
            return pos;
    }
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = min(x, __shfl_xor(x, d, kWave));
    return uniform(x);
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = max(x, __shfl_xor(x, d, kWave));
    return uniform(x);
}

// The rows of a workgroup of one side: where they are, and the keys [e0, e1) of its split.
// GROUP: of the shared keys; otherwise of a request's own ones.
template <bool GROUP, int LGM>
struct SharedJob {
    SharedTile t;
    int tile, kvh, split, part;  // part: place among all parts of a row
    int to, group;

    __device__ __forceinline__ bool locate(const SharedGeo& s, int bid, int lane) {
        const SeqGeo& g = s.g;
        const SharedSide& side = GROUP ? s.shared_side : s.own_side;
        split = side.fd_tiles.div(bid);
        const int id = bid - split * side.ntiles * g.Hkv;
        tile = g.fd_kv.div(id);
        kvh = id - tile * g.Hkv;
        part = split + (GROUP ? 0 : s.shared_side.nsplit);
        Groups all;
        all.load(s, lane);
        if constexpr (GROUP) {
            return locate_group(s, all, tile, LGM, lane, t, to);
        } else {
            if (!seq_locate(g, tile, LGM, lane, t)) return false;
            group = group_of(s, all, t.b, lane, t.from);
            t.span(g, t.pmin, t.pmax, INT32_MAX);
            return true;
        }
    }
    __device__ __forceinline__ void keys(const SharedGeo& s, int& e0, int& e1) const {
        const SharedSide& side = GROUP ? s.shared_side : s.own_side;
        e0 = min(split * side.chunk, t.nT);
        e1 = split == side.nsplit - 1 ? t.nT : min(e0 + side.chunk, t.nT);
    }
};

// The build takes floats for numbers, so whether one is NaN is asked of its bits, behind a point
// at which the compiler knows nothing of it.
constexpr uint32_t kNaN = 0x7fc00000u;
__device__ __forceinline__ uint32_t bits_of(float x) {
    settle(x);
    return __float_as_uint(x);
}
__device__ __forceinline__ bool is_nan(uint32_t bits) { return (bits & 0x7fffffffu) > 0x7f800000u; }

// x, or NaN where `nan`, for stores and conversions.
__device__ __forceinline__ float or_nan(float x, bool nan) {
    float y = __uint_as_float(nan ? kNaN : bits_of(x));
    settle(y);
    return y;
}

// Logsumexp in base 2 from its reference and its sum: -inf where the sum is 0.  (A score that is
// NaN or +inf leaves a sum of NaN; the row has no result then.)
__device__ __forceinline__ float logsumexp2(float mref, float sum) {
    return sum > 0.f ? mref + __log2f(sum) : -INFINITY;
}

// Place of a row's part: its logsumexp (base 2); D times that its mean of the values.
__device__ __forceinline__ int64_t part_row(const SharedGeo& s, int part, int tok, int64_t head) {
    return ((int64_t)part * s.g.n + tok) * ((int64_t)s.g.Hkv * s.g.G) + head;
}

// Requests without a group have no shared part: their rows' places there say so.
template <typename Job>
__device__ __forceinline__ void no_shared_part(const SharedGeo& s, const Job& job, int m, int tok,
                                               int head) {
    if (job.group >= 0 || job.split != 0 || m >= job.t.rows) return;
    for (int x = 0; x < s.shared_side.nsplit; ++x)
        s.part_lse[part_row(s, x, job.t.qtok + tok, (int64_t)job.kvh * s.g.G + head)] = -INFINITY;
}

// Stages key or value rows.  Where the rows of 64 tiles are, and which of them every row or no row of
// the wave sees, is found at a time, a lane each: found tile by tile it took the wide form 1 us of
// every 2.4 us stage (the first passes of a process, before the clocks are up).
template <typename T, int D, bool GROUP>
struct SharedStage {
    using R = SeqRows<T, D>;
    R rows;
    const unsigned char *kb, *vb;  // the head's rows of page 0
    uint32_t lane_rows;
    int pass;                 // tiles pass + lane:
    int64_t at0, at1;         // bytes of their two blocks of 16 rows from the head's rows of page 0
    uint64_t fast, ok0, ok1;  // (uniform) both blocks exist and every row is seen; a block exists
    uint64_t out, full;       // (uniform) no row of the wave sees any key, every row sees all

    __device__ __forceinline__ void init(const SeqGeo& g, int kvh, int lane, const void* k,
                                         const void* v) {
        rows.init(lane);
        kb = static_cast<const unsigned char*>(k) + kvh * g.kh;
        vb = static_cast<const unsigned char*>(v) + kvh * g.vh;
        lane_rows = rows.rowl * (uint32_t)g.kt;
    }
    // wmin, wmax: positions of the wave's rows.
    __device__ __forceinline__ void look_up(const SeqGeo& g, const SharedTile& t, int first, int e1,
                                            int lane, int wmin, int wmax) {
        pass = first;
        const int32_t* row = g.table + (int64_t)t.b * g.max_pages;
        const int j = t.tile(pass + lane), col0 = j >> g.lgps, col1 = (j + 16) >> g.lgps;
        const int in = (1 << g.lgps) - 1;
        const bool on = pass + lane < e1;
        const int id0 = on && col0 < g.max_pages ? row[col0] : -1;
        const int id1 = on && col1 < g.max_pages ? row[col1] : -1;
        const bool is0 = (unsigned)id0 < (unsigned)g.pages, is1 = (unsigned)id1 < (unsigned)g.pages;
        at0 = (int64_t)(is0 ? id0 : 0) * g.kb + (j & in) * g.kt;
        at1 = (int64_t)(is1 ? id1 : 0) * g.kb + ((j + 16) & in) * g.kt;
        ok0 = __builtin_amdgcn_ballot_w64(is0);
        ok1 = __builtin_amdgcn_ballot_w64(is1);
        fast = __builtin_amdgcn_ballot_w64(is0 && is1 && !(GROUP && t.gaps) && t.whole(g, j));
        out = __builtin_amdgcn_ballot_w64(!on || j > wmax ||
                                          (wmin - (j + 31) >= g.W && j >= g.S));
        full = __builtin_amdgcn_ballot_w64(on && j + 31 <= wmin &&
                                           (wmax - j < g.W || j + 31 < g.S) && j >= t.from &&
                                           j + 31 < t.end);
    }
    __device__ __forceinline__ static int64_t of_lane(int64_t x, int lane) {
        const uint32_t lo = __builtin_amdgcn_readlane((int)x, lane);
        return (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | lo;
    }
    // Instructions first, first + STEP, .. of tile e's keys to kdst and of its values to vdst (those
    // of the two that are asked for); pos: see look().
    template <int STEP, bool K, bool V, int N>
    __device__ __forceinline__ void issue(const SeqGeo& g, SharedTile& t, int e, int first,
                                          const int (&pos)[N], unsigned char* kdst,
                                          unsigned char* vdst) const {
        const int x = e - pass;
        const int64_t a0 = of_lane(at0, x), a1 = of_lane(at1, x);
        // (one branch for all loads: a choice for each of them took as long again)
        if (fast >> x & 1) {
            if constexpr (K) load<STEP, true>(g, t, 0, first, kb + a0, kb + a1, true, true, kdst);
            if constexpr (V) load<STEP, true>(g, t, 0, first, vb + a0, vb + a1, true, true, vdst);
        } else {
            const int j0 = t.tile(e);
            const bool b0 = ok0 >> x & 1, b1 = ok1 >> x & 1;
            if (GROUP && t.gaps) t.look(g, j0, pos);
            if constexpr (K) load<STEP, false>(g, t, j0, first, kb + a0, kb + a1, b0, b1, kdst);
            if constexpr (V) load<STEP, false>(g, t, j0, first, vb + a0, vb + a1, b0, b1, vdst);
        }
    }
    template <int STEP, bool FAST>
    __device__ __forceinline__ void load(const SeqGeo& g, const SharedTile& t, int j0, int first,
                                         const unsigned char* b0, const unsigned char* b1, bool ok0,
                                         bool ok1, unsigned char* dst) const {
#pragma unroll
        for (int u = 0; u < (R::kInstr + STEP - 1) / STEP; ++u) {
            const int n = first + u * STEP, r0 = n * R::kRpi;
            const unsigned char* base = (r0 >= 16 ? b1 : b0) + (r0 & 15) * (int)g.kt;
            const uint32_t off = rows.off(n, lane_rows);
            if constexpr (FAST) {
                seq_load(base, off, dst + n * 1024);
            } else {
                const bool see = (r0 >= 16 ? ok1 : ok0) && t.sees(g, j0 + r0 + rows.rowl);
                seq_load(see ? base + off : reinterpret_cast<const unsigned char*>(&kZeroRow),
                         dst + n * 1024);
            }
        }
    }
};

// Bits e of the keys base + e that a row at position pos sees.  (Rows of a group stand far apart: a
// distance is cut off where no key is seen any more, so that the window's end stays in 32 bits.)
__device__ __forceinline__ unsigned visible_keys(const SeqGeo& g, const SharedTile& t, int pos,
                                                 int base) {
    return seen_keys(max(pos - base, -64), g.W, g.S - base) & below(t.end - base) &
           ~below(t.from - base);
}

// The operand of this lane's row of q.
template <typename T, int D>
__device__ __forceinline__ void load_query(const SeqGeo& g, const SharedTile& t, int kvh, int tok,
                                           int head, const T* qg, int lane,
                                           typename Tr<T>::x8 (&qf)[D / 16]) {
    const unsigned char* qp = reinterpret_cast<const unsigned char*>(qg) +
                              ((int64_t)kvh * g.G + head) * g.qh + (int64_t)(t.qtok + tok) * g.qt;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
        qf[x] = ld_x8<T>(reinterpret_cast<const T*>(qp) + x * 16 + 8 * (lane >> 5));
}

// Many rows: four waves of 32 rows each share the staged key tiles (as the wide form of
// na_seq_fwd.hip).  Bound by a wave's chain through a stage: at D = 128 two waves a SIMD have 1.5 us
// of products, exponentials and LDS reads for two key tiles and 0.4 to 0.6 us of issuing the next
// ones' loads; the matrix cores are busy 32 % of the cycles.  (Issuing them inside the fold, behind
// its key reads, spills: chunks behind a prompt 317 us instead of 237, kernel times of first passes.)
template <typename T, int D, bool GROUP>
__device__ __forceinline__ void shared_wide(const SharedGeo& s, int bid, const T* __restrict__ qg,
                                            const T* __restrict__ kg, const T* __restrict__ vg,
                                            unsigned char* smem) {
    using F = SeqFrags<T, D>;
    using Ring = SeqRing<T, D>;
    constexpr int SK = Ring::kTiles, NB = Ring::kStages;
    const SeqGeo& g = s.g;
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & 3);
    SharedJob<GROUP, 7> job;
    if (!job.locate(s, bid, lane)) return;
    SharedTile& t = job.t;

    // ---- this lane's row, and the positions of the wave's rows ----
    const int m = wave * 32 + (lane & 31);
    int tok, head, pos;
    seq_row(g, t, m, tok, head);
    SeqState<T, D> st;
    st.init();
    load_query<T, D>(g, t, job.kvh, tok, head, qg, lane, st.qf);  // (arrives while the rest is found)
    int tf, hh;
    seq_row(g, t, wave * 32, tf, hh);
    int wmin, wmax;
    int all[GROUP ? 4 : 1];  // positions of rows lane % 32 of every wave
    if constexpr (GROUP) {
        pos = position_of(g, t.r0, t.r1, t.qtok + tf, t.qtok + tok, lane);
        wmin = wave_min(pos);
        wmax = wave_max(pos);
        int* rows = reinterpret_cast<int*>(smem);  // (before the stages use the LDS)
        if (lane < 32) rows[m] = pos;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) all[w] = rows[w * 32 + (lane & 31)];
        t.span(g, wave_min(min(min(all[0], all[1]), min(all[2], all[3]))),
               wave_max(max(max(all[0], all[1]), max(all[2], all[3]))), job.to);
        __syncthreads();
    } else {
        pos = t.pos0 + tok;
        wmin = wave_min(pos);
        wmax = wave_max(pos);
    }
    int e0, e1;
    job.keys(s, e0, e1);

    // Instructions of K and V by wave: those from kInstr on are V's, where the waves divide K's
    // evenly in equal shares of both, otherwise (D = 32 in 16 bits) two waves' of each.
    using R = SeqRows<T, D>;
    constexpr bool kEven = R::kInstr % 4 == 0;
    constexpr int kCount = 2 * R::kInstr / 4;
    static_assert(kEven || R::kInstr == 2, "equal shares");
    SharedStage<T, D, GROUP> ld;
    ld.init(g, job.kvh, lane, kg, vg);
    ld.look_up(g, t, e0, e1, lane, wmin, wmax);
    auto issue_stage = [&](int e, int buf) __attribute__((always_inline)) {
        if (e >= e1) return;
        if (e - ld.pass > kWave - SK)  // (uniform; from the stage on that is worked on)
            ld.look_up(g, t, e - (NB - 1) * SK, e1, lane, wmin, wmax);
#pragma unroll
        for (int i = 0; i < SK; ++i) {  // (a tile behind the last one: zeros)
            unsigned char* dst = smem + buf * Ring::kStage + i * 2 * F::kTile;
            if constexpr (kEven) {
                ld.template issue<4, true, true>(g, t, e + i, wave, all, dst, dst + F::kTile);
            } else if (wave < 2) {
                ld.template issue<2, true, false>(g, t, e + i, wave, all, dst, dst);
            } else {
                ld.template issue<2, false, true>(g, t, e + i, wave - 2, all, dst, dst + F::kTile);
            }
        }
    };
#pragma unroll
    for (int b = 0; b < NB - 1; ++b) issue_stage(e0 + b * SK, b);

    const bool live = wave * 32 < t.rows;
    const int64_t hq = (int64_t)job.kvh * g.G + head;
    F f;
    f.init(lane);
#pragma unroll
    for (int x = 0; x < F::kKS; ++x) settle(st.qf[x]);
    auto seen = [&](int base) __attribute__((always_inline)) {
        return visible_keys(g, t, pos, base);
    };

    // One stage, in buffer BUF (see na_seq_fwd.hip).
    auto stage = [&](int e, auto BUF) __attribute__((always_inline)) {
        constexpr int kBuf = decltype(BUF)::value;
        if (NB > 2 && e + (NB - 2) * SK < e1)
            wait_vmem_but<(NB - 2) * SK * kCount>();
        else
            wait_vmem();
        lds_barrier();
        issue_stage(e + (NB - 1) * SK, (kBuf + NB - 1) % NB);
        const unsigned char* base = smem + kBuf * Ring::kStage;
        const unsigned char* tile[SK];
        int j0[SK];
        bool on[SK];
        constexpr uint64_t kAll = (1ull << SK) - 1;
        const bool out = (~ld.out >> (e - ld.pass) & kAll) == 0;
        const bool full = (~ld.full >> (e - ld.pass) & kAll) == 0;
#pragma unroll
        for (int i = 0; i < SK; ++i) {
            tile[i] = base + i * 2 * F::kTile;
            j0[i] = t.tile(e + i);
            on[i] = i == 0 || e + i < e1;
        }
        if (live && !out) st.template fold<SK>(f, tile, lane, g.c, full, j0, on, seen);
    };
    for (int e = e0; e < e1;) {
        stage(e, std::integral_constant<int, 0>{});
        if ((e += SK) >= e1) break;
        stage(e, std::integral_constant<int, 1>{});
        if ((e += SK) >= e1) break;
        if constexpr (NB > 2) {
            stage(e, std::integral_constant<int, 2>{});
            e += SK;
        }
    }

    // ---- this split's part of the rows ----
    if constexpr (!GROUP) {
        if (lane < 32) no_shared_part(s, job, m, tok, head);
    }
    const float l = col_sum<32>(st.l);
    if (m >= t.rows) return;
    const bool some = l > 0.f;
    const float inv = some ? 1.f / l : 0.f;
    const int h = lane >> 5;
    const int64_t row = part_row(s, job.part, t.qtok + tok, hq);
    if (h == 0) s.part_lse[row] = or_nan(logsumexp2(st.mref, l), is_nan(bits_of(l)));
    if (!some) return;
    float* po = s.part + row * D;
#pragma unroll
    for (int db = 0; db < F::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            st16<f32x4>(po + db * 32 + i * 8 + h * 4,
                        f32x4{st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                              st.o[db][4 * i + 3]} * inv);
}

// LDS of the narrow form: a key and a value tile for each of four waves; then the join, as many
// columns at a time as fit there.
template <typename T, int D>
struct SharedNarrow {
    static constexpr int W = 4;
    static constexpr int kTile = SeqFrags<T, D>::kTile;
    static constexpr int kStages = W * 2 * kTile;
    static constexpr int kCols = D == 32 ? 32 : D / 2;      // columns joined at a time
    static constexpr int kRow = (kCols + 4) * 4;            // (padded: LDS banks)
    static constexpr int kJoin = W * 32 * kRow;
    static constexpr int kStat = kStages > kJoin ? kStages : kJoin;  // offset of the statistics
    static constexpr int kLds = kStat + W * 32 * 8;
};

// Few rows (one block of 32): the waves take every fourth key tile each and join.  A wave has one
// buffer for keys and one for values: the next tile's keys load as soon as this one's are in
// registers, its values likewise, so more waves fit a CU than with two buffers each.
template <typename T, int D, bool GROUP>
__device__ __forceinline__ void shared_narrow(const SharedGeo& s, int bid, const T* __restrict__ qg,
                                              const T* __restrict__ kg, const T* __restrict__ vg,
                                              unsigned char* smem) {
    using F = SeqFrags<T, D>;
    using R = SeqRows<T, D>;
    using N = SharedNarrow<T, D>;
    constexpr int W = N::W;
    const SeqGeo& g = s.g;
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & (W - 1));
    SharedJob<GROUP, 5> job;
    if (!job.locate(s, bid, lane)) return;
    SharedTile& t = job.t;
    int tok, head, pos;
    seq_row(g, t, lane & 31, tok, head);
    SeqState<T, D> st;
    st.init();
    load_query<T, D>(g, t, job.kvh, tok, head, qg, lane, st.qf);  // (arrives while the rest is found)
    if constexpr (GROUP) {
        int tf, hh;
        seq_row(g, t, 0, tf, hh);
        pos = position_of(g, t.r0, t.r1, t.qtok + tf, t.qtok + tok, lane);
    } else {
        pos = t.pos0 + tok;
    }
    const int wmin = wave_min(pos), wmax = wave_max(pos);
    if constexpr (GROUP) t.span(g, wmin, wmax, job.to);
    int e0, e1;
    job.keys(s, e0, e1);

    SharedStage<T, D, GROUP> ld;
    ld.init(g, job.kvh, lane, kg, vg);
    const int all[1] = {pos};
    F f;
    f.init(lane);
    auto seen = [&](int base) __attribute__((always_inline)) {
        return visible_keys(g, t, pos, base);
    };
    unsigned char* buf = smem + wave * 2 * F::kTile;
    for (int pass = e0; pass < e1; pass += kWave) {
        const int end = min(pass + kWave, e1);
        int e = pass + wave;
        ld.look_up(g, t, pass, e1, lane, wmin, wmax);
#pragma unroll
        for (int x = 0; x < F::kKS; ++x) settle(st.qf[x]);
        if (e < end) {
            ld.template issue<1, true, true>(g, t, e, 0, all, buf, buf + F::kTile);
        }
        for (; e < end; e += W) {
            const bool more = e + W < end;
            wait_vmem_but<R::kInstr>();  // (all but the values')
            const unsigned char* ks[1] = {buf};
            const int j0 = t.tile(e);
            const bool full = ld.full >> (e - pass) & 1;
            const int js[1] = {j0};
            const bool on[1] = {true};
            st.template fold<1>(
                f, ks, lane, g.c, full, js, on, seen,
                [&]() __attribute__((always_inline)) {
                    wait_lds();
                    __builtin_amdgcn_sched_barrier(0);
                    if (more) ld.template issue<1, true, false>(g, t, e + W, 0, all, buf, buf);
                },
                [&]() __attribute__((always_inline)) {
                    if (more) wait_vmem_but<R::kInstr>();  // (all but the next keys')
                    else wait_vmem();
                },
                [&]() __attribute__((always_inline)) {
                    wait_lds();
                    __builtin_amdgcn_sched_barrier(0);
                    if (more) ld.template issue<1, false, true>(g, t, e + W, 0, all, buf, buf + F::kTile);
                });
        }
    }

    // ---- join the waves: every sum relative to the largest reference ----
    const float l = col_sum<32>(st.l);
    float* stat = reinterpret_cast<float*>(smem + N::kStat);  // [wave][32] of (reference, sum)
    if (lane < 32) {
        stat[(wave * 32 + lane) * 2] = st.mref;
        stat[(wave * 32 + lane) * 2 + 1] = l;
        if constexpr (!GROUP) {
            if (wave == 0) no_shared_part(s, job, lane, tok, head);
        }
    }
    __syncthreads();
    const int col = lane & 31, h = lane >> 5;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, stat[(w * 32 + col) * 2]);
    const float scale = st.mref == -INFINITY ? 0.f : fast_exp2(st.mref - top);
    constexpr int kBlocks = N::kCols / 32;  // column blocks joined at a time
#pragma unroll
    for (int c0 = 0; c0 < F::kDB; c0 += kBlocks) {
        float* mine = reinterpret_cast<float*>(smem + (wave * 32 + col) * N::kRow);
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x16& o = st.o[c0 + db];
                st16<f32x4>(mine + db * 32 + i * 8 + h * 4,
                            f32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]} * scale);
            }
        __syncthreads();
        // each thread: four columns of a row
        for (int x = threadIdx.x; x < t.rows * (N::kCols / 4); x += W * 64) {
            const int row = x / (N::kCols / 4), d = x % (N::kCols / 4) * 4;
            float mx = -INFINITY, sum = 0.f;
            bool nan = false;
            f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; ++w) mx = fmaxf(mx, stat[(w * 32 + row) * 2]);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float m = stat[(w * 32 + row) * 2], lw = stat[(w * 32 + row) * 2 + 1];
                nan = nan || is_nan(bits_of(lw));
                sum += m == -INFINITY ? 0.f : fast_exp2(m - mx) * lw;
                acc += *reinterpret_cast<const f32x4*>(smem + (w * 32 + row) * N::kRow + d * 4);
            }
            const bool some = sum > 0.f;
            int tk, hd;
            seq_row(g, t, row, tk, hd);
            const int64_t pr = part_row(s, job.part, t.qtok + tk, (int64_t)job.kvh * g.G + hd);
            if (some) st16(s.part + pr * D + c0 * 32 + d, acc * (1.f / sum));
            if (c0 == 0 && d == 0) s.part_lse[pr] = or_nan(logsumexp2(mx, sum), nan);
        }
        if (c0 + kBlocks < F::kDB) __syncthreads();
    }
}

// Both problems in one launch: the workgroups of the shared keys, then those of the requests' own.
template <typename T, int D, bool NARROW_SHARED, bool NARROW_OWN>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? (D == 128 ? 2 : 4) : 1)) void shared_kernel(
    SharedGeo s, const T* __restrict__ qg, const T* __restrict__ kg, const T* __restrict__ vg) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int bid = (int)blockIdx.x - s.shared_jobs;
    if (bid < 0) {
        if constexpr (NARROW_SHARED) shared_narrow<T, D, true>(s, blockIdx.x, qg, kg, vg, smem);
        else shared_wide<T, D, true>(s, blockIdx.x, qg, kg, vg, smem);
    } else {
        if constexpr (NARROW_OWN) shared_narrow<T, D, false>(s, bid, qg, kg, vg, smem);
        else shared_wide<T, D, false>(s, bid, qg, kg, vg, smem);
    }
}

// Joins the parts of each row in a fixed order.  One workgroup per 32 rows of a (row tile of the
// requests, key/value head); D / 4 threads a row, which read a part's logsumexp each, so that the
// means' loads depend on nothing (one thread reading all of them in turn: 25 us for 33 parts of 1024
// rows, this 6 to 7).
template <typename T, int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedGeo s, int lgM, T* __restrict__ og,
                                                          float* __restrict__ lseg) {
    constexpr int kThreads = D / 4;  // of a row: 8, 16 or 32 neighbouring lanes
    const SeqGeo& g = s.g;
    const int id = blockIdx.x >> (lgM - 5), r0 = (blockIdx.x & ((1 << (lgM - 5)) - 1)) * 32;
    const int tile = g.fd_kv.div(id);
    const int kvh = id - tile * g.Hkv;
    SeqTile t;
    if (!seq_locate(g, tile, lgM, threadIdx.x & 63, t)) return;
    const int parts = s.shared_side.nsplit + s.own_side.nsplit;
    const int64_t apart = (int64_t)g.n * g.Hkv * g.G;
    const int mine = threadIdx.x % kThreads;
    for (int row = r0 + threadIdx.x / kThreads; row < min(r0 + 32, t.rows); row += 256 / kThreads) {
        int tok, head;
        seq_row(g, t, row, tok, head);
        const int64_t hr = (int64_t)kvh * g.G + head;
        const int64_t at = part_row(s, 0, t.qtok + tok, hr);
        const float* lse = s.part_lse + at;
        const float* y = s.part + at * D + mine * 4;
        float mx = -INFINITY;
        int nan = 0;
        for (int p = mine; p < parts; p += kThreads) {
            const float e = lse[p * apart];
            nan |= is_nan(bits_of(e));
            mx = fmaxf(mx, e);
        }
#pragma unroll
        for (int d = kThreads / 2; d > 0; d >>= 1) {
            mx = fmaxf(mx, __shfl_xor(mx, d, kWave));
            nan |= __shfl_xor(nan, d, kWave);
        }
        float sum = 0.f;
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
        for (int p0 = 0; p0 < parts; p0 += kThreads) {
            // (a part that sees nothing has no mean: it may hold anything, and weighs -1.  One whose
            // weight vanishes has a mean, which may be infinite or NaN)
            const float e = p0 + mine < parts ? lse[(p0 + mine) * apart] : -INFINITY;
            const float w = e == -INFINITY ? -1.f : fast_exp2(e - mx);
            const int n = min(kThreads, parts - p0);
            for (int x0 = 0; x0 < n; x0 += 8) {
                f32x4 v[8];
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    v[x] = ld16<f32x4>(y + (int64_t)(p0 + min(x0 + x, n - 1)) * apart * D);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const float wx = x0 + x < n ? __shfl(w, (x0 + x) % kThreads, kThreads) : -1.f;
                    sum += fmaxf(wx, 0.f);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[c] = wx >= 0.f ? fmaf(v[x][c], wx, acc[c]) : acc[c];
                }
            }
        }
        const bool some = sum > 0.f;
        T* op = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(og) + hr * g.oh +
                                     (int64_t)(t.qtok + tok) * g.ot);
        acc *= some ? 1.f / sum : 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = or_nan(acc[c], nan);
        st_x4<T>(op + mine * 4, acc);
        if (mine == 0)
            lseg[hr * g.lh + (int64_t)(t.qtok + tok) * g.lt] =
                or_nan(logsumexp2(mx, sum) * kLn2, nan);
    }
}

// ---- host ----
template <typename T, int D, bool NARROW_SHARED, bool NARROW_OWN>
hipError_t launch_both(const SharedGeo& s, const T* q, const T* k, const T* v, hipStream_t st) {
    constexpr size_t wide = SeqRing<T, D>::kLds, narrow = SharedNarrow<T, D>::kLds;
    constexpr size_t lds = NARROW_SHARED && NARROW_OWN ? narrow
                           : NARROW_SHARED || NARROW_OWN ? std::max(wide, narrow) : wide;
    auto kern = shared_kernel<T, D, NARROW_SHARED, NARROW_OWN>;
    const hipError_t e = seq_allow_lds(kern, lds);
    if (e != hipSuccess) return e;
    const unsigned own = (unsigned)s.own_side.ntiles * s.g.Hkv * s.own_side.nsplit;
    hipLaunchKernelGGL(kern, dim3(s.shared_jobs + own), dim3(256), lds, st, s, q, k, v);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_shared(const SharedGeo& s, const void* q, const void* k, const void* v, void* out,
                         float* lse, hipStream_t st) {
    auto q_ = static_cast<const T*>(q);
    auto k_ = static_cast<const T*>(k);
    auto v_ = static_cast<const T*>(v);
    const bool narrow = s.own_side.narrow;
    const hipError_t e = narrow && s.shared_side.narrow ? launch_both<T, D, true, true>(s, q_, k_, v_, st)
                         : narrow                       ? launch_both<T, D, false, true>(s, q_, k_, v_, st)
                         : s.shared_side.narrow         ? launch_both<T, D, true, false>(s, q_, k_, v_, st)
                                                        : launch_both<T, D, false, false>(s, q_, k_, v_, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((shared_join_kernel<T, D>),
                       dim3((unsigned)s.g.ntiles * s.g.Hkv * (narrow ? 1 : 4)), dim3(256), 0, st, s,
                       narrow ? 5 : 7, static_cast<T*>(out), lse);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_shared_d(const SharedGeo& s, int D, const void* q, const void* k, const void* v,
                           void* out, float* lse, hipStream_t st) {
    switch (D) {
        case 32: return launch_shared<T, 32>(s, q, k, v, out, lse, st);
        case 64: return launch_shared<T, 64>(s, q, k, v, out, lse, st);
        case 128: return launch_shared<T, 128>(s, q, k, v, out, lse, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_shared_attention(const SharedGeo& s, int D, int dtype, const void* q,
                                   const void* k, const void* v, void* out, float* lse,
                                   hipStream_t st) {
    switch (dtype) {
        case 0: return launch_shared_d<float>(s, D, q, k, v, out, lse, st);
        case 1: return launch_shared_d<_Float16>(s, D, q, k, v, out, lse, st);
        case 2: return launch_shared_d<__bf16>(s, D, q, k, v, out, lse, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace na
