// na_seq_kernels.h -- what the sequence kernels share: attention of a causal 1-D sequence whose
// queries see the `W` nearest tokens up to themselves and the first `S` tokens, over
// contiguous (strided) rows or over the pages of a cache.
//
// Rows.  The G query heads that share a key/value head are rows of one problem: row m of a
// (sequence, key/value head) is token m / G, head m % G of the group.  A workgroup tile is M
// consecutive rows, so any G packs without waste, a staged key serves every head of its
// group, and a tile of a window problem spans M / G tokens, which keeps its halo small.
//
// Keys are visited in 32-row tiles, aligned to 32 positions: the tiles of the first S tokens
// that lie before the window, then the window's.
#pragma once

#include "na_stage.h"

namespace na {

// Largest split of the pages of a request over workgroups (joined by a second launch).
constexpr int kSeqMaxSplit = 64;
constexpr int kSeqMaxTiles = 1 << 24;  // row tiles of a launch, at most

struct SeqGeo {
    int n;          // tokens per sequence (contiguous form); all new tokens (paged form)
    int G, Hkv, B;  // query heads per key/value head, key/value heads, sequences or requests
    int W, S;       // window (itself included), first tokens that stay visible
    int ntiles;     // row tiles per (sequence, key/value head); paged: over all requests
    int nsplit;     // key splits of a row tile (paged form; 1: none)
    int chunk;      // key tiles of a split
    int lgps, pages, max_pages;  // paged form: log2 page size, pages of the pool, table columns
    // fd_tiles divides by the row tiles of a (sequence, key/value head); paged: by those of all
    // requests and heads
    FastDiv fd_G, fd_tiles, fd_kv, fd_slices;
    // byte strides of batch, head, token (paged form: head, token of q and out)
    int64_t qb, qh, qt, kb, kh, kt, vb, vh, vt, ob, oh, ot;
    int64_t lb, lh, lt;  // logsumexp, in elements
    float c;             // scale * log2(e)
    int runs;            // contiguous form: order of the workgroups (seq_job)
    const int32_t* lengths;  // contiguous form: valid tokens per sequence, or null
    const int32_t *context, *cu, *table;  // paged form
};

// 16 zero bytes: what is staged for a row that nothing may see (behind the sequence, before
// the window, on a page that does not exist), so that such memory is not read at all.
__device__ const i32x4 kZeroRow = {0, 0, 0, 0};

// c + a b on 32x32x16 steps (fp32: eight 32x32x2 steps; step j contracts slots j of both
// halves of the wave).  A: lane l holds row l % 32, slots 8 (l / 32) .. +7; B the same of
// column l % 32; C entry i: row 8 (i / 4) + 4 (l / 32) + i % 4, column l % 32.
template <typename T>
__device__ __forceinline__ f32x16 mma32(typename Tr<T>::x8 a, typename Tr<T>::x8 b, f32x16 c) {
    if constexpr (sizeof(T) == 2) {
        return Tr<T>::mma(a, b, c);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}

// row (of 0..7) of entry i of a 32x32 result, without the lane's 4 (l / 32)
__device__ __forceinline__ constexpr int entry_row(int i) { return 8 * (i >> 2) + (i & 3); }

// Bits e of a lane's mask over the entries of a 32x32 result (entry i is row entry_row(i)):
// below(x) has those with e < x (entries reach 27).
__device__ __forceinline__ unsigned below(int x) { return (1u << min(max(x, 0), 31)) - 1u; }
// y where the mask has the bit of entry i, else `other`: the bit is spread over a word that
// selects, two instructions.  (In assembly: the compiler makes a comparison and a select of it,
// with the wait states between them.)
__device__ __forceinline__ float keep(unsigned mask, int i, float y, float other) {
    int t = 0;
#if defined(__HIP_DEVICE_COMPILE__)
    asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(t) : "v"(mask), "i"(entry_row(i)));
#endif
    return __int_as_float((__float_as_int(y) & t) | (__float_as_int(other) & ~t));
}
// The entries of a tile of keys that a row at distance `dist` from its first one (of this
// lane's half) sees; first: how many of them are first tokens.
__device__ __forceinline__ unsigned seen_keys(int dist, int W, int first) {
    return (below(dist + 1) & ~below(dist - W + 1)) | below(min(first, dist + 1));
}

// Ends the compiler's wait for the loads behind x here: it does not know that a written-out
// wait covers them, and would wait again where x is used, in the loop, for every stage load
// then in flight.
template <typename V>
__device__ __forceinline__ void settle(V& x) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(V) == 16) {
        i32x4 u = __builtin_bit_cast(i32x4, x);
        asm volatile("" : "+v"(u));
        x = __builtin_bit_cast(V, u);
    } else if constexpr (sizeof(V) == 32) {
        f32x8 u = __builtin_bit_cast(f32x8, x);
        asm volatile("" : "+v"(u));
        x = __builtin_bit_cast(V, u);
    } else {
        asm volatile("" : "+v"(x));
    }
#endif
}

// LDS rows of the staged tiles: Rows<T, D>, with a swizzle of its own for rows of 256 bytes in
// 16-bit types.  The transposed reads below take two 16-lane groups at a time, and here those
// of a pair read four 16-byte segments of the same four rows (a 16x16 layout: two segments of
// eight rows), which must fall on 16 different ones: rows 0..3 differ in the upper two bits of
// the segment, rows 4 apart in bit 1, rows 8 apart in bit 0.  With Rows' swizzle a third of
// the LDS cycles at D = 128 were conflicts.
template <typename T, int D>
struct SeqLay : Rows<T, D> {
    using B = Rows<T, D>;
    static constexpr bool kOwn = sizeof(T) == 2 && B::kSegs == 16;
    __device__ __forceinline__ static constexpr int swz(int r) {
        return kOwn ? (r & 1) << 2 ^ (r & 2) << 2 ^ (r & 4) >> 1 ^ (r & 8) >> 3 : B::swz(r);
    }
    __device__ __forceinline__ static int off(int r, int s) {
        return r * B::kRowBytes + ((s ^ swz(r)) << 4);
    }
};

// Operands read from a staged tile of 32 rows.
template <typename T, int D>
struct SeqFrags {
    using L = SeqLay<T, D>;
    using x8 = typename Tr<T>::x8;
    static constexpr int kKS = D / 16;  // contraction steps along D
    static constexpr int kDB = D / 32;  // blocks of 32 columns
    static constexpr int kRowB = L::kRowBytes;
    static constexpr int kTile = 32 * kRowB;
    static constexpr int kStepB = 16 * (int)sizeof(T);  // bytes of a row per contraction step
    int ro, co;

    __device__ __forceinline__ void init(int lane) {
        const int r = lane & 31, h = lane >> 5;
        ro = L::off(r, sizeof(T) == 2 ? h : 2 * h);
        if constexpr (sizeof(T) == 2) {
            // 16-lane group (2 h + e) of the transposed read: rows 4 h + s, columns
            // e * 16 + 4 q .. +3
            const int e = (lane >> 4) & 1, i = lane & 15;
            co = L::off(4 * h + (i >> 2), e * 2 + ((i & 3) >> 1)) + (i & 1) * 8;
        } else {
            co = h;
        }
    }

    // The fragments of a whole tile, all reads issued before any is used (the compiler, sparing
    // registers, would put each right before its product and expose its latency every time).
    __device__ __forceinline__ void rows(const unsigned char* tile, x8 (&x)[kKS]) const {
#pragma unroll
        for (int st = 0; st < kKS; ++st) x[st] = row(tile, st);
        __builtin_amdgcn_sched_barrier(0);
    }
    // (transposed: of 16-row half bi)
    __device__ __forceinline__ void cols(const unsigned char* tile, int bi, int lane,
                                         x8 (&x)[kDB]) const {
#pragma unroll
        for (int db = 0; db < kDB; ++db) x[db] = col(tile, db, bi, lane);
        __builtin_amdgcn_sched_barrier(0);
    }

    // lane l: row l % 32, elements 16 st + 8 (l / 32) .. +7
    __device__ __forceinline__ x8 row(const unsigned char* tile, int st) const {
        return row_at(tile, ro, st);
    }
    // (o: ro, or a copy of it that the compiler cannot see through, so that the offsets of the
    // steps are formed where they are used instead of kept in registers over the tile loop)
    __device__ __forceinline__ static x8 row_at(const unsigned char* tile, int o, int st) {
        const unsigned char* p = tile + (o ^ (st * kStepB));
        if constexpr (sizeof(T) == 2) {
            return __builtin_bit_cast(x8, lds16(p));
        } else {
            const f32x4 a = __builtin_bit_cast(f32x4, lds16(p));
            const f32x4 b = __builtin_bit_cast(f32x4, lds16(tile + (o ^ (st * kStepB) ^ 16)));
            return x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }

    // Transposed: lane l holds column 32 db + l % 32; slots 0..3 rows 16 bi + 4 (l / 32) + j,
    // slots 4..7 the rows 8 further on: the rows of entries 8 bi .. 8 bi + 7 of a 32x32
    // result, so such a result feeds the next product without a shuffle.
    __device__ __forceinline__ x8 col(const unsigned char* tile, int db, int bi, int lane) const {
        return col_at(tile, co, db, bi, lane);
    }
    __device__ __forceinline__ static x8 col_at(const unsigned char* tile, int co, int db, int bi,
                                                int lane) {
        if constexpr (sizeof(T) == 2) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            // (rows 8 further on have another swizzle)
            constexpr int kSwz8 = L::swz(8) << 4;
            const unsigned char* p = tile + bi * 16 * kRowB;
            const i32x2 a = __builtin_bit_cast(
                i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (co ^ (db << 6)))));
            const i32x2 b = __builtin_bit_cast(
                i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                           (lds_s16x4*)(p + 8 * kRowB + (co ^ (db << 6) ^ kSwz8))));
            return __builtin_bit_cast(x8, i32x4{a[0], a[1], b[0], b[1]});
        } else {
            const int d = db * 32 + (lane & 31);
            x8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = bi * 16 + (j < 4 ? 0 : 8) + 4 * co + (j & 3);
                v[j] = *reinterpret_cast<const float*>(tile + L::off(r, d >> 2) + (d & 3) * 4);
            }
            return v;
        }
    }
};


// ---- staging: 32 rows straight to LDS, 1024 bytes per wave instruction ----
// Instruction t covers rows t * kRpi .. of the tile, all inside one 16-row block, so its
// source is a uniform base plus a lane offset that differs between instructions only by the
// swizzle of the first row.
template <typename T, int D>
struct SeqRows {
    using L = SeqLay<T, D>;
    static constexpr int kRowB = L::kRowBytes;
    static constexpr int kTile = 32 * kRowB;
    static constexpr int kInstr = kTile / 1024;
    static constexpr int kRpi = 64 / L::kSegs;
    int rowl;      // this lane's row of an instruction
    uint32_t seg;  // byte of its segment, swizzled by that row
    __device__ __forceinline__ void init(int lane) {
        rowl = lane / L::kSegs;
        seg = (uint32_t)((lane % L::kSegs) ^ L::swz(rowl)) << 4;
    }
    // lane offset of instruction t from its first row; lane_rows: rowl * row stride
    __device__ __forceinline__ uint32_t off(int t, uint32_t lane_rows) const {
        return (seg ^ ((uint32_t)L::swz((t * kRpi) & 15) << 4)) + lane_rows;
    }
};

// 16 bytes per lane to consecutive LDS positions from dst, from a uniform base + lane offset
// or from lane addresses, in inline assembly: the compiler tracks none of them (it would wait
// for every one before each transposed LDS read), so every wait is written out.  No output
// registers.  The move and four idle states keep the distances that the hardware needs
// between a scalar register's write and its use by a vector memory instruction.
__device__ __forceinline__ void seq_load(const unsigned char* base, uint32_t off,
                                         unsigned char* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = (unsigned)(size_t)(lds_void*)dst;
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(off), "s"(base), "s"(m0)
                 : "memory");
#endif
}
__device__ __forceinline__ void seq_load(const unsigned char* addr, unsigned char* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = (unsigned)(size_t)(lds_void*)dst;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(addr), "s"(m0)
                 : "memory");
#endif
}

// Waits until at most N of this wave's vector memory operations are outstanding.
template <int N>
__device__ __forceinline__ void wait_vmem_but() {
    static_assert(N < 64, "6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// This wave's LDS reads are done (what they read may be overwritten).
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// This wave's LDS reads are done, and so are all waves'.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// This wave's stage loads have landed and its LDS reads are done, and so for all waves.
__device__ __forceinline__ void stage_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The rows of one workgroup tile: which request or sequence, which tokens, what they see.
struct SeqTile {
    int b;        // sequence or request
    int row0;     // first row (of n * G)
    int rows;     // rows of the tile that exist
    int qtok;     // first token of the request in q (paged; contiguous: 0)
    int pos0;     // position of the request's token 0
    int valid;    // tokens [0, valid) attend and are attended (contiguous: the length)
    int pmin, pmax;  // first and last position of the tile's attending rows
    int lo;       // first position that a row's window reaches
    int nS, w0, nT;  // tiles of the first tokens, first window tile, tiles in all (0: none)
    __device__ __forceinline__ void span(const SeqGeo& g) {
        lo = max(pmin - g.W + 1, 0);
        w0 = lo >> 5;
        nS = min((g.S + 31) >> 5, w0);
        nT = nS + (pmax >> 5) - w0 + 1;
    }
    // first position of key tile e
    __device__ __forceinline__ int tile(int e) const { return (e < nS ? e : w0 + e - nS) << 5; }
    // whether some row may see position j
    __device__ __forceinline__ bool sees(const SeqGeo& g, int j) const {
        return (j >= lo || j < g.S) && j <= pmax;
    }
};

// Paged form: row tile `tile` of M = 2^lgM rows -> its request and rows.  False: no such tile.
//   With at most 64 requests the wide form takes them by descending length, and each from its
// last rows on, so that the long tiles start first and the short ones fill the gaps at the end
// (requests of 2 to 9 thousand tokens: see na_seq_fwd.hip).  Every lane holds a request and
// adds up the tiles of those before it.
//   Otherwise request r's tiles start at floor(cu[r] G / M) + r, which leaves each at least as
// many as it has and needs no sum; the lanes search 64 requests at a time.
__device__ __forceinline__ bool seq_locate(const SeqGeo& g, int tile, int lgM, int lane,
                                           SeqTile& t) {
    int r, at;
    if (lgM == 7 && g.B <= 64) {
        const int i = min(lane, g.B - 1);
        const int start = g.cu[i], end = g.cu[i + 1];
        const bool ok = lane < g.B && start >= 0 && start < end && end <= g.n;
        const int count = ok ? end - start : 0;
        const int nt = ok ? (int)(((uint32_t)count * (uint32_t)g.G + 127u) >> 7) : 0;
        const int key = max(g.context[i], 0) / 2 + count / 2;
        int before = 0;
        for (int j = 0; j < g.B; ++j) {
            const int kj = __builtin_amdgcn_readlane(key, j);
            const int nj = __builtin_amdgcn_readlane(nt, j);
            before += kj > key || (kj == key && j < lane) ? nj : 0;
        }
        const uint64_t here = __builtin_amdgcn_ballot_w64(tile >= before && tile - before < nt);
        if (here == 0) return false;
        r = __builtin_ctzll(here);
        at = __builtin_amdgcn_readlane(nt, r) - 1 - (tile - __builtin_amdgcn_readlane(before, r));
    } else {
        // (offsets outside the rows, which have none, stay in order and below 2^30 this way)
        auto first = [&](int x) { return (min(max(g.cu[x], 0), g.n) * g.G >> lgM) + x; };
        int lo = 0, span = g.B;  // the request is in [lo, lo + span)
        while (span > 1) {
            const int step = (span + 63) >> 6;
            const int x = lo + lane * step;
            const bool in = lane * step < span && first(min(x, g.B - 1)) <= tile;
            const int below = __builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
            lo += (below > 0 ? below - 1 : 0) * step;
            span = min(step, g.B - lo);
        }
        r = uniform(lo);
        at = tile - first(r);
    }
    const int start = g.cu[r], end = g.cu[r + 1];
    if (start < 0 || start >= end || end > g.n) return false;
    const int n = end - start;
    t.b = r;
    if (at < 0 || at >= kSeqMaxTiles) return false;
    t.row0 = at << lgM;
    if (t.row0 < 0 || t.row0 >= n * g.G) return false;
    t.rows = min(n * g.G - t.row0, 1 << lgM);
    t.qtok = start;
    t.pos0 = min(max(g.context[r], 0), g.max_pages << g.lgps);
    t.valid = n;
    t.pmin = t.pos0 + g.fd_G.div(t.row0);
    t.pmax = t.pos0 + g.fd_G.div(t.row0 + t.rows - 1);
    t.span(g);
    return true;
}

// Key splits of a row tile of nT key tiles: split s < seq_splits has tiles [s chunk, ..), the
// last one whatever is left (the host sizes chunk by a bound that it is told).
__device__ __forceinline__ int seq_splits(const SeqGeo& g, int nT) {
    return max(1, min(g.nsplit, (nT + g.chunk - 1) / g.chunk));
}

// Contiguous form: workgroup -> row tile and (sequence, key/value head).  Short windows: runs of
// neighbouring tiles on one XCD, which share what its L2 holds.  Long ones: the long tiles of
// every sequence first, so that the short ones fill the gaps at the end, and a sequence on one
// XCD where there are eight (16 heads on 4, 8192 tokens, full causal, bf16 D = 128 forward in
// runs 346 us).
__device__ __forceinline__ void seq_job(const SeqGeo& g, int bid, int jobs, int& tile,
                                        int& slice) {
    if (g.runs) {
        const int id = xcd_remap(bid, jobs);
        slice = g.fd_tiles.div(id);
        tile = id - slice * g.ntiles;
    } else {
        tile = g.fd_slices.div(bid);
        slice = bid - tile * g.B * g.Hkv;
    }
    tile = g.ntiles - 1 - tile;
}

// Contiguous form: row tile `tile` of (sequence, key/value head) `slice`.
__device__ __forceinline__ void seq_contiguous(const SeqGeo& g, int tile, int slice, SeqTile& t) {
    t.b = g.fd_kv.div(slice);
    t.row0 = tile * 128;
    t.rows = min(g.n * g.G - t.row0, 128);
    t.qtok = t.pos0 = 0;
    t.valid = g.lengths ? min(max(g.lengths[t.b], 0), g.n) : g.n;
    t.pmin = g.fd_G.div(t.row0);
    t.pmax = min(g.fd_G.div(t.row0 + t.rows - 1), t.valid - 1);
    t.nT = 0;
    if (t.pmin < t.valid) t.span(g);
}

// Stages key tile `e` of the workgroup's tile: instructions first, first + STEP, ... of the
// 2 kInstr of K and V (first < STEP).
template <typename T, int D, bool PAGED, int STEP>
struct SeqStage {
    using R = SeqRows<T, D>;
    static constexpr int kCount = 2 * R::kInstr / STEP;
    static_assert(2 * R::kInstr % STEP == 0, "equal shares");
    // instructions of V: those from kInstr on, which is known at compile time where the waves
    // divide K's evenly
    static constexpr bool kEven = R::kInstr % STEP == 0;
    const unsigned char *kb, *vb;  // the head's rows (paged: of page 0)
    R rows;
    uint32_t klane, vlane;  // rowl * token stride
    int kt, vt;             // token strides (below 2^26 bytes)

    __device__ __forceinline__ void init(const SeqGeo& g, const SeqTile& t, int kvh, int lane,
                                         const void* k, const void* v) {
        rows.init(lane);
        kb = static_cast<const unsigned char*>(k) + kvh * g.kh;
        vb = static_cast<const unsigned char*>(v) + kvh * g.vh;
        if (!PAGED) {
            kb += t.b * g.kb;
            vb += t.b * g.vb;
        }
        kt = (int)g.kt;
        vt = (int)g.vt;
        klane = rows.rowl * (uint32_t)kt;
        vlane = rows.rowl * (uint32_t)vt;
    }

    __device__ __forceinline__ void issue(const SeqGeo& g, const SeqTile& t, int e, int first,
                                          unsigned char* dst) const {
        const int j0 = t.tile(e);
        bool fast = j0 + 31 <= t.pmax && (j0 >= t.lo || j0 + 31 < g.S);
        // byte offset of the first row of the tile's two 16-row blocks, and whether they exist
        int64_t k0, k1, v0, v1;
        bool ok0 = true, ok1 = true;
        if constexpr (PAGED) {
            // (pages hold whole blocks; a page of 16 rows ends inside the tile.  K and V pages
            // are laid out alike, and a page's bytes fit 31 bits)
            const int32_t* row = g.table + (int64_t)t.b * g.max_pages;
            const int col = j0 >> g.lgps;
            int id0 = -1, id1 = -1;
            if (col < g.max_pages) id0 = row[col];
            if (g.lgps != 4)
                id1 = id0;
            else if (col + 1 < g.max_pages && j0 + 16 <= t.pmax)
                id1 = row[col + 1];
            const int in = g.lgps == 4 ? 0 : (j0 & ((1 << g.lgps) - 1)) * kt;
            ok0 = (unsigned)id0 < (unsigned)g.pages;
            ok1 = (unsigned)id1 < (unsigned)g.pages;
            k0 = (int64_t)(ok0 ? id0 : 0) * (int)g.kb + in;
            k1 = (int64_t)(ok1 ? id1 : 0) * (int)g.kb + in + (g.lgps == 4 ? 0 : 16 * kt);
            v0 = k0;
            v1 = k1;
            fast = fast && ok0 && ok1;
        } else {
            k0 = (int64_t)j0 * kt;
            v0 = (int64_t)j0 * vt;
            k1 = k0 + 16 * kt;
            v1 = v0 + 16 * vt;
        }
        if (fast)
            load<true>(kb + k0, kb + k1, vb + v0, vb + v1, first, dst, true, true, t, g, j0);
        else
            load<false>(kb + k0, kb + k1, vb + v0, vb + v1, first, dst, ok0, ok1, t, g, j0);
    }

    // The loads themselves, from the first rows of the blocks; FAST: every row exists and is
    // seen by some row.  (Everything by value: selects between captured references end up in
    // scratch memory.)
    template <bool FAST>
    __device__ __forceinline__ void load(const unsigned char* k0, const unsigned char* k1,
                                         const unsigned char* v0, const unsigned char* v1,
                                         int first, unsigned char* dst, bool ok0, bool ok1,
                                         const SeqTile& t, const SeqGeo& g, int j0) const {
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            const int x = first + u * STEP;
            const bool isv = kEven ? u * STEP >= R::kInstr : x >= R::kInstr;
            const int n = isv ? x - R::kInstr : x;
            const int r0 = n * R::kRpi;
            const bool blk = r0 >= 16;
            const unsigned char* kx = blk ? k1 : k0;
            const unsigned char* vx = blk ? v1 : v0;
            const unsigned char* base = (isv ? vx : kx) + (r0 & 15) * (isv ? vt : kt);
            const uint32_t off = rows.off(n, isv ? vlane : klane);
            if constexpr (FAST) {
                seq_load(base, off, dst + x * 1024);
            } else {
                const bool see = (blk ? ok1 : ok0) && t.sees(g, j0 + r0 + rows.rowl);
                seq_load(see ? base + off : reinterpret_cast<const unsigned char*>(&kZeroRow),
                         dst + x * 1024);
            }
        }
    }
};

// Row m of the tile: token (of the request) and head of the group.
__device__ __forceinline__ void seq_row(const SeqGeo& g, const SeqTile& t, int m, int& tok,
                                        int& head) {
    const int r = t.row0 + min(m, t.rows - 1);
    tok = g.fd_G.div(r);
    head = r - tok * g.G;
}

// The backward's geometry: the forward's, the gradients' byte strides, and the cut of dk, dv.
struct SeqBwd {
    SeqGeo g;
    int64_t gb, gh, gt;  // dout
    int64_t qb, qh, qt, kb, kh, kt, vb, vh, vt;  // dq, dk, dv
    float scale;
    int ktiles;   // tiles of 128 keys
    int hsplit;   // workgroups that share the heads of a group
    int blocks;   // blocks of 32 keys with first tokens that rows outside the window see
    int chunks;   // row chunks of such a block, a workgroup each
    int first_jobs;
    FastDiv fd_ktiles, fd_hsplit, fd_blocks, fd_chunks;
    float *lse2, *delta;       // [B, H, n] each
    float *part, *first_part;  // [part][slice][key][dk, dv][D]
};

// 4 bytes per lane from lane addresses to consecutive LDS positions from dst (as seq_load).
__device__ __forceinline__ void seq_load4(const unsigned char* addr, unsigned char* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
    const unsigned m0 = (unsigned)(size_t)(lds_void*)dst;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, off"
                 :
                 : "v"(addr), "s"(m0)
                 : "memory");
#endif
}

// More LDS than a launch may ask for by default.
template <typename K>
inline hipError_t seq_allow_lds(K kern, size_t lds) {
    return lds <= 65536 ? hipSuccess
                        : hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

// Launchers (host).  part: split results, see the workspace of na_cache_attention.
hipError_t launch_seq_forward(const SeqGeo& g, int D, int dtype, bool paged, bool narrow,
                              const void* q, const void* k, const void* v, void* out, float* lse,
                              float* part, hipStream_t s);
hipError_t launch_seq_backward(const SeqBwd& b, int D, int dtype, const void* q, const void* k,
                               const void* v, const void* out, const float* lse, const void* dout,
                               void* dq, void* dk, void* dv, hipStream_t s);
hipError_t launch_cache_tables(int R, int tokens, int lgps, int max_pages, int num_free,
                               const int32_t* context, const int32_t* fresh,
                               const int32_t* free_pages, const int32_t* head, int32_t* table,
                               int32_t* cu, int64_t* slots, int32_t* positions, int32_t* new_head,
                               hipStream_t s);
hipError_t launch_cache_write(int tokens, int Hkv, int row_bytes, int lgps, int64_t slots_end,
                              int64_t kt, int64_t kh, int64_t vt, int64_t vh, const void* k,
                              const void* v, const int64_t* slots, void* k_pages, void* v_pages,
                              hipStream_t s);

}  // namespace na
