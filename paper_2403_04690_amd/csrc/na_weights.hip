// na_weights.hip -- the attention weight that every key of a paged cache gathers from new tokens
// (gfx950):
//
//   w[r, c, j] += sum over the new tokens i of request r and the query heads h of key/value head c of
//                 exp(scale q_ih . k_jc - lse_ih),   j seen by i,
//
// from the logsumexp that the tokens' attention returned.  A key's sum is one workgroup's alone, or
// where few keys meet many rows that of a few, each with a share of the rows, whose sums a second
// launch adds up: the order of every sum is fixed.
//
//   S = Q K^T (32 rows x 32 keys a step) leaves a key in one lane column (two lanes), whose entries
// are rows: a lane adds up its own exponentials, and the two halves meet once at the end.
// Scores, exponentials and sums are fp32; nothing is rounded on the way.
#include <type_traits>

#include "na_launch.h"
#include "na_seq_kernels.h"
#include "na_shared.h"

namespace na {

namespace {

constexpr float kNever = INFINITY;  // logsumexp of a row that does not exist: its weights are 0
__device__ const float kNeverRow = INFINITY;

// Bits e of the rows row + e (row: of the request's rows, token row / G) that see key j.
__device__ __forceinline__ unsigned seen_rows(const SeqGeo& g, int pos0, int row, int j) {
    const int f = g.fd_G.div(row);
    const int o = row - f * g.G;  // heads of token f that lie before the row
    const int d = j - (pos0 + f);  // the first token that sees the key, from token f on
    const int64_t lo = (int64_t)min(d, 33) * g.G - o;
    const int64_t hi = min((int64_t)d + g.W, (int64_t)33) * g.G - o;
    const unsigned from = ~below((int)max(min(lo, (int64_t)32), (int64_t)0));
    return j < g.S ? from : from & below((int)max(min(hi, (int64_t)32), (int64_t)0));
}

// Request r's new tokens.  False: it has none.
__device__ __forceinline__ bool weights_request(const SeqGeo& g, int r, SeqTile& t) {
    const int start = g.cu[r], end = g.cu[r + 1];
    if (start < 0 || start >= end || end > g.n) return false;
    t.b = r;
    t.row0 = 0;
    t.rows = (end - start) * g.G;
    t.qtok = start;
    t.pos0 = min(max(g.context[r], 0), g.max_pages << g.lgps);
    t.valid = end - start;
    t.pmin = t.pos0;
    t.pmax = t.pos0 + t.valid - 1;
    t.span(g);
    return true;
}

// Bytes of key j's row from the head's rows of page 0, or -1: no such page.
__device__ __forceinline__ int64_t key_offset(const SeqGeo& g, int r, int j) {
    const int col = j >> g.lgps;
    const int id = col < g.max_pages ? g.table[(int64_t)r * g.max_pages + col] : -1;
    if ((unsigned)id >= (unsigned)g.pages) return -1;
    return (int64_t)id * (int)g.kb + (int64_t)(j & ((1 << g.lgps) - 1)) * (int)g.kt;
}

__device__ __forceinline__ int64_t weights_at(const WeightsGeo& w, int r, int kvh) {
    return ((int64_t)r * w.g.Hkv + kvh) * w.capacity;
}

// The rows of a block of 32 as an operand: lane l has row l % 32.
template <typename T, int D>
__device__ __forceinline__ void load_rows(const SeqGeo& g, const SeqTile& t, int kvh, int row0,
                                          const T* qg, int lane,
                                          typename Tr<T>::x8 (&qf)[D / 16]) {
    const int m = min(row0 + (lane & 31), t.rows - 1);
    const int tok = g.fd_G.div(m), head = m - tok * g.G;
    const unsigned char* qp = reinterpret_cast<const unsigned char*>(qg) +
                              ((int64_t)kvh * g.G + head) * g.qh +
                              (int64_t)(t.qtok + tok) * g.qt;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
        qf[x] = ld_x8<T>(reinterpret_cast<const T*>(qp) + x * 16 + 8 * (lane >> 5));
}

// Logsumexp of row m, base 2.
__device__ __forceinline__ float row_lse(const WeightsGeo& w, const SeqTile& t, int kvh, int m) {
    if (m >= t.rows) return kNever;
    const SeqGeo& g = w.g;
    const int tok = g.fd_G.div(m), head = m - tok * g.G;
    return w.lse[(int64_t)(t.qtok + tok) * g.lt + (int64_t)kvh * g.G + head] * kLog2e;
}

constexpr int kFewTiles = 64;  // key tiles whose sums are in LDS at a time

template <typename T, int D>
struct WeightsFew {
    static constexpr int kTile = SeqFrags<T, D>::kTile;
    static constexpr int kWaves = 4;
    static constexpr int kLds = kWaves * kTile + kFewTiles * 32 * 4;
};

// Few rows (one block of 32: single tokens): each wave takes every kWaves-th key tile of the split,
// from an LDS buffer of its own, which the next tile's loads may fill as soon as its operands are in
// registers.  Bound by reading the keys once.
//   One new token for each of 32 requests over 8k to 32k cached ones, 16 heads on 4, bf16 D = 128: 553 MB
// in 109 us (5.1 TB/s).  With two buffers a wave, and so half the waves, 131; with the pages looked up
// tile by tile 150; three waves of three buffers 176 so.  Keys before `first` are read and multiplied
// like the others, and left out when the sums are stored.
template <typename T, int D>
__global__ __launch_bounds__((WeightsFew<T, D>::kWaves * 64), 1) void weights_few_kernel(
    WeightsGeo w, const T* __restrict__ qg, const T* __restrict__ kg) {
    using F = SeqFrags<T, D>;
    using R = SeqRows<T, D>;
    using L = WeightsFew<T, D>;
    constexpr int W = L::kWaves;
    extern __shared__ __align__(16) unsigned char smem[];
    float* sums = reinterpret_cast<float*>(smem + W * F::kTile);
    const SeqGeo& g = w.g;
    const int lane = threadIdx.x & 63;
    const int wave = uniform(threadIdx.x >> 6);
    const int slice = g.fd_tiles.div(blockIdx.x);
    const int split = blockIdx.x - slice * g.nsplit;
    const int r = g.fd_kv.div(slice), kvh = slice - r * g.Hkv;
    SeqTile t;
    if (!weights_request(g, r, t)) return;
    const int splits = seq_splits(g, t.nT);
    if (split >= splits) return;
    const int e0 = split * g.chunk, e1 = split == splits - 1 ? t.nT : e0 + g.chunk;
    const int first = w.first ? max(w.first[r], 0) : 0;

    R rows;
    rows.init(lane);
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(kg) + kvh * g.kh;
    const uint32_t klane = rows.rowl * (uint32_t)g.kt;
    // The pages of the kFewTiles tiles from `pass` on, a lane each (pages hold whole blocks of 16
    // keys): looked up once, not with every tile in front of its loads.
    int page0 = -1, page1 = -1;
    auto look_up = [&](int pass) __attribute__((always_inline)) {
        const int32_t* row = g.table + (int64_t)r * g.max_pages;
        const int col0 = t.tile(pass + lane) >> g.lgps, col1 = (t.tile(pass + lane) + 16) >> g.lgps;
        page0 = pass + lane < e1 && col0 < g.max_pages ? row[col0] : -1;
        page1 = pass + lane < e1 && col1 < g.max_pages ? row[col1] : -1;
    };
    auto issue = [&](int pass, int e, unsigned char* dst) __attribute__((always_inline)) {
        const int j0 = t.tile(e);
        const int id0 = __builtin_amdgcn_readlane(page0, e - pass);
        const int id1 = __builtin_amdgcn_readlane(page1, e - pass);
        const bool ok0 = (unsigned)id0 < (unsigned)g.pages, ok1 = (unsigned)id1 < (unsigned)g.pages;
        const int in = (1 << g.lgps) - 1, kt = (int)g.kt;
        const unsigned char* b0 = kb + (int64_t)(ok0 ? id0 : 0) * (int)g.kb + (j0 & in) * kt;
        const unsigned char* b1 = kb + (int64_t)(ok1 ? id1 : 0) * (int)g.kb + ((j0 + 16) & in) * kt;
        auto load = [&](auto fast) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < R::kInstr; ++n) {
                const int r0 = n * R::kRpi;
                const unsigned char* base = (r0 >= 16 ? b1 : b0) + (r0 & 15) * kt;
                const uint32_t off = rows.off(n, klane);
                if constexpr (decltype(fast)::value) {
                    seq_load(base, off, dst + n * 1024);
                } else {
                    const bool see = (r0 >= 16 ? ok1 : ok0) && t.sees(g, j0 + r0 + rows.rowl);
                    seq_load(see ? base + off : reinterpret_cast<const unsigned char*>(&kZeroRow),
                             dst + n * 1024);
                }
            }
        };
        // (one branch for all loads, not a choice for each)
        if (ok0 && ok1 && t.whole(g, j0)) load(std::true_type{});
        else load(std::false_type{});
    };
    F f;
    f.init(lane);
    const int h = lane >> 5;
    typename Tr<T>::x8 qf[F::kKS];
    float lse[16];
    unsigned char* buf = smem + wave * F::kTile;

    // (one block of rows unless there are more than the caller's bound says)
    for (int row0 = 0; row0 < t.rows; row0 += 32) {
        load_rows<T, D>(g, t, kvh, row0, qg, lane, qf);
#pragma unroll
        for (int i = 0; i < 16; ++i) lse[i] = row_lse(w, t, kvh, row0 + entry_row(i) + 4 * h);
#pragma unroll
        for (int x = 0; x < F::kKS; ++x) settle(qf[x]);
#pragma unroll
        for (int i = 0; i < 16; ++i) settle(lse[i]);
        const int pa = t.pos0 + g.fd_G.div(row0);  // (rows in order of their positions)
        for (int pass = e0; pass < e1; pass += kFewTiles) {
            const int end = min(pass + kFewTiles, e1);
            int e = pass + wave;
            look_up(pass);
            if (e < end) issue(pass, e, buf);
            for (; e < end; e += W) {
                wait_vmem();
                typename Tr<T>::x8 kf[F::kKS];
                f.rows(buf, kf);
                wait_lds();
                __builtin_amdgcn_sched_barrier(0);
                if (e + W < end) issue(pass, e + W, buf);
                f32x16 s = f32x16{} * 0.f;
#pragma unroll
                for (int x = 0; x < F::kKS; ++x) s = mma32<T>(qf[x], kf[x], s);
                const int j0 = t.tile(e);
                const bool full = pa >= j0 + 31 && (t.pmax - j0 < g.W || j0 + 31 < g.S);
                const unsigned m = full ? ~0u : seen_rows(g, t.pos0, row0 + 4 * h, j0 + (lane & 31));
                float sum = 0.f;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    if (row0 + 8 * b >= t.rows) continue;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int i = 4 * b + x;
                        const float y = fmaf(s[i], g.c, -lse[i]);
                        sum += fast_exp2(full ? y : keep(m, i, y, -INFINITY));
                    }
                }
                sum = col_sum<32>(sum);
                if (h == 0) sums[(e - pass) * 32 + lane] = sum;
            }
            __syncthreads();
            float* out = w.weights + weights_at(w, r, kvh);
            for (int x = threadIdx.x; x < (end - pass) * 32; x += W * 64) {
                const int j = t.tile(pass + (x >> 5)) + (x & 31);
                if (j >= first && j < w.capacity && t.sees(g, j)) out[j] += sums[x];
            }
            __syncthreads();
        }
    }
}

// The rows that see any key of the tiles [pass, end), in stages of 64.
constexpr int kStageRows = 64;
__device__ __forceinline__ void weights_stages(const WeightsGeo& w, const SeqTile& t, int pass, int end,
                                               int first, int& b0, int& b1) {
    const SeqGeo& g = w.g;
    const int ja = t.tile(pass), jb = t.tile(end - 1) + 31;
    const int ta = max(ja - t.pos0, 0);
    const int tb = ja < g.S ? t.valid : (int)min((int64_t)t.valid, (int64_t)jb - t.pos0 + g.W);
    b0 = b1 = 0;
    if (ta >= tb || jb < first) return;
    b0 = ta * g.G / kStageRows;
    b1 = (tb * g.G + kStageRows - 1) / kStageRows;
}

// Key tiles of a wave in the form for many rows: two while their operands leave the loop over the
// rows enough of the 256 registers of two waves a SIMD.  (16 bits at D = 128 and fp32 at D = 64 take
// all of them, and 4 and 6 more values are spilled: stored once in front of the first pass over
// the rows and read again once a pass, none within it.)
template <typename T, int D>
struct WeightsMany {
    static constexpr int kTiles = sizeof(T) == 4 && D == 128 ? 1 : 2;
    static constexpr int kStages = 3;
    static constexpr int kBlocks = kStageRows / 32;
    static constexpr int kTile = SeqFrags<T, D>::kTile;
    // rows, and each wave's copy of their lse
    static constexpr int kStage = kBlocks * kTile + 4 * kBlocks * 128;
    static constexpr int kLds = kStages * kStage;
};

// Many rows (chunks of prompts): four waves of kTiles x 32 keys each, whose operands stay in registers,
// share stages of 64 rows.  Bound by the vector unit (42 % of the cycles: an exponential, its
// argument and the sum for each pair) and the matrix cores (27 %) in turn, with two waves a SIMD:
// chunks of 1432 to 1846 tokens over 2k to 7k cached ones, 4 requests, 16 heads on 4, bf16 D = 128 193
// to 196 us a call (0.68 PFLOP/s), kernels 191 and 5.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void weights_many_kernel(WeightsGeo w,
                                                             const T* __restrict__ qg,
                                                             const T* __restrict__ kg) {
    using F = SeqFrags<T, D>;
    using R = SeqRows<T, D>;
    using M = WeightsMany<T, D>;
    constexpr int KT = M::kTiles, NB = M::kStages, RB = M::kBlocks;
    constexpr int kShare = RB * R::kInstr / 4, kCount = kShare + 1;
    static_assert(RB * R::kInstr % 4 == 0 && RB == 2, "equal shares, a lane for each row's lse");
    extern __shared__ __align__(16) unsigned char smem[];
    const SeqGeo& g = w.g;
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & 3);
    // (neighbours on eight XCDs in turn: requests of any length load them alike, and with a power
    // of two of shares an XCD's L2 holds the rows of only some.  Shares of a fixed number of rows
    // instead, the same keys' on all XCDs: 270 us where these took 230, kernel times of first passes)
    const int id = blockIdx.x >> w.lgshares, share = blockIdx.x & (w.shares - 1);
    const int slice = g.fd_tiles.div(id);
    const int split = id - slice * g.nsplit;
    const int r = g.fd_kv.div(slice), kvh = slice - r * g.Hkv;
    SeqTile t;
    if (!weights_request(g, r, t)) return;
    const int splits = seq_splits(g, t.nT);
    if (split >= splits) return;
    const int c1 = split == splits - 1 ? t.nT : (split + 1) * g.chunk;
    const int first = w.first ? max(w.first[r], 0) : 0;
    const int h = lane >> 5;
    F f;
    f.init(lane);
    R rows;
    rows.init(lane);
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(kg) + kvh * g.kh;

    // This wave's share of the loads of a stage: where row m of a load lies, and m's head.  A stage
    // is 64 rows on from the one before it: dt tokens and dh heads.
    struct Place {
        const unsigned char* p;
        int head;
    };
    const int dt = g.fd_G.div(kStageRows), dh = kStageRows - dt * g.G;
    auto row_at = [&](int m) __attribute__((always_inline)) {
        m = min(m, t.rows - 1);
        const int tok = g.fd_G.div(m), head = m - tok * g.G;
        return Place{reinterpret_cast<const unsigned char*>(qg) + ((int64_t)kvh * g.G + head) * g.qh +
                         (int64_t)(t.qtok + tok) * g.qt, head};
    };
    auto lse_at = [&](int m) __attribute__((always_inline)) {
        m = min(m, t.rows - 1);
        const int tok = g.fd_G.div(m), head = m - tok * g.G;
        return Place{reinterpret_cast<const unsigned char*>(w.lse) +
                         4 * ((int64_t)(t.qtok + tok) * g.lt + (int64_t)kvh * g.G + head), head};
    };
    auto advance = [&](Place& x, int64_t token, int64_t head) __attribute__((always_inline)) {
        x.p += dt * token + dh * head;
        if (dh == 0) return;  // (uniform)
        x.head += dh;
        if (x.head >= g.G) {
            x.head -= g.G;
            x.p += token - g.G * head;
        }
    };
    Place qp[kShare], lp;
    auto begin = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kShare; ++u)
            qp[u] = row_at(b * kStageRows + (wave + 4 * u) * R::kRpi + rows.rowl);
        lp = lse_at(b * kStageRows + lane);
    };
    // Rows of stage b, and their logsumexps, into buffer `buf`; stages in order from begin's on.
    auto issue = [&](int b, int buf) __attribute__((always_inline)) {
        unsigned char* dst = smem + buf * M::kStage;
        if ((b + 1) * kStageRows > t.rows) begin(b);  // (the last stage: rows that exist)
#pragma unroll
        for (int u = 0; u < kShare; ++u) {
            const int n = wave + 4 * u;
            seq_load(qp[u].p + rows.off(n % R::kInstr, 0), dst + n * 1024);
            advance(qp[u], g.qt, g.qh);
        }
        seq_load4(b * kStageRows + lane < t.rows
                      ? lp.p
                      : reinterpret_cast<const unsigned char*>(&kNeverRow),
                  dst + RB * M::kTile + wave * 256);
        advance(lp, 4 * g.lt, 4);
    };

    for (int pass = split * g.chunk, next; pass < c1; pass = next) {
        next = pass + 4 * KT;
        // ---- the rows that see any of the workgroup's keys, or its share of them ----
        int b0, b1;
        weights_stages(w, t, pass, min(pass + 4 * KT, c1), first, b0, b1);
        const bool shared = w.shares > 1 && pass < g.nsplit * g.chunk;
        if (share > 0 && !shared) break;  // (keys behind the caller's bound: one workgroup's)
        if (shared) {
            const int each = (b1 - b0 + w.shares - 1) >> w.lgshares;
            b0 = min(b0 + share * each, b1);
            b1 = min(b0 + each, b1);
        }
        // ---- this wave's keys ----
        const int e = pass + wave * KT;
        typename Tr<T>::x8 kf[KT][F::kKS];
        int j0[KT];
        bool on[KT];
        float sum[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            on[k] = e + k < c1;
            j0[k] = t.tile(on[k] ? e + k : pass);
            // (keys that nobody gathers for)
            on[k] = on[k] && j0[k] + 31 >= first;
            sum[k] = 0.f;
            const int j = j0[k] + (lane & 31);
            const int64_t at = t.sees(g, j) ? key_offset(g, r, j) : -1;
#pragma unroll
            for (int x = 0; x < F::kKS; ++x) {
                kf[k][x] = zero_x8<T>();
                if (at >= 0)
                    kf[k][x] = ld_x8<T>(reinterpret_cast<const T*>(kb + at) + x * 16 + 8 * h);
            }
        }
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int x = 0; x < F::kKS; ++x) settle(kf[k][x]);
        lds_barrier();  // (the stages of the pass before are read)
        if (b0 < b1) begin(b0);
#pragma unroll
        for (int x = 0; x < NB - 1; ++x)
            if (b0 + x < b1) issue(b0 + x, x);
        int buf = 0;
        for (int b = b0; b < b1; ++b, buf = buf == NB - 1 ? 0 : buf + 1) {
            if (b + NB - 2 < b1)
                wait_vmem_but<(NB - 2) * kCount>();
            else
                wait_vmem();
            lds_barrier();  // for every wave; and the stage before is read
            if (b + NB - 1 < b1) issue(b + NB - 1, buf == 0 ? NB - 1 : buf - 1);
            const unsigned char* tile = smem + buf * M::kStage;
            const int pa = t.pos0 + g.fd_G.div(b * RB * 32);
            const int pb = t.pos0 + g.fd_G.div(min(b * RB * 32 + RB * 32 - 1, t.rows - 1));
            bool full = true, none = true;
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                full = full && on[k] && pa >= j0[k] + 31 && (pb - j0[k] < g.W || j0[k] + 31 < g.S);
                none = none && (!on[k] || pb < j0[k] || (pa - (j0[k] + 31) >= g.W && j0[k] >= g.S));
            }
            // All pairs of a stage in one run of code (masks only where some pair is not seen), so
            // that one tile's products run beside another's exponentials.
            auto step = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    typename Tr<T>::x8 qf[F::kKS];
#pragma unroll
                    for (int x = 0; x < F::kKS; ++x) qf[x] = f.row(tile + rb * M::kTile, x);
                    float lse[16];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const f32x4 v = *reinterpret_cast<const f32x4*>(
                            tile + RB * M::kTile + wave * 256 + (rb * 32 + 8 * x + 4 * h) * 4);
#pragma unroll
                        for (int y = 0; y < 4; ++y) lse[4 * x + y] = v[y] * kLog2e;
                    }
                    f32x16 s[KT];
#pragma unroll
                    for (int k = 0; k < KT; ++k) {
                        s[k] = f32x16{} * 0.f;
#pragma unroll
                        for (int x = 0; x < F::kKS; ++x) s[k] = mma32<T>(qf[x], kf[k][x], s[k]);
                    }
#pragma unroll
                    for (int k = 0; k < KT; ++k) {
                        float y[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = fmaf(s[k][i], g.c, -lse[i]);
                        if constexpr (decltype(masked)::value) {
                            const unsigned m = on[k] ? seen_rows(g, t.pos0, (b * RB + rb) * 32 + 4 * h,
                                                                 j0[k] + (lane & 31))
                                                     : 0u;
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[i] = keep(m, i, y[i], -INFINITY);
                        }
                        float part[2] = {0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < 16; ++i) part[i & 1] += fast_exp2(y[i]);
                        sum[k] += part[0] + part[1];
                    }
                }
            };
            if (full) step(std::false_type{});
            else if (!none) step(std::true_type{});
        }
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            const float total = col_sum<32>(sum[k]);
            const int j = j0[k] + lane;
            if (shared) {
                if (e + k < c1 && h == 0)
                    w.part[((int64_t)share * g.B * g.Hkv + slice) * w.part_keys + (e + k) * 32 + lane] =
                        total;
            } else if (on[k] && h == 0 && j >= first && j < w.capacity && t.sees(g, j))
                w.weights[weights_at(w, r, kvh) + j] += total;
        }
    }
}

// Adds up the row shares of each key: a workgroup for 256 keys.
__global__ __launch_bounds__(256) void weights_join_kernel(WeightsGeo w) {
    const SeqGeo& g = w.g;
    const int slice = w.fd_joins.div(blockIdx.x);
    const int e = (blockIdx.x - slice * w.joins) * 8 + (threadIdx.x >> 5);
    const int r = g.fd_kv.div(slice), kvh = slice - r * g.Hkv;
    SeqTile t;
    if (!weights_request(g, r, t) || e >= min(t.nT, g.nsplit * g.chunk)) return;
    const int first = w.first ? max(w.first[r], 0) : 0;
    const int j = t.tile(e) + (threadIdx.x & 31);
    if (j < first || j >= w.capacity || !t.sees(g, j)) return;
    const float* part = w.part + slice * w.part_keys + e * 32 + (threadIdx.x & 31);
    float sum = 0.f;
#pragma unroll 8
    for (int x = 0; x < w.shares; ++x) sum += part[(int64_t)x * g.B * g.Hkv * w.part_keys];
    w.weights[weights_at(w, r, kvh) + j] += sum;
}

// ---- host ----
template <typename T, int D>
hipError_t launch_weights(const WeightsGeo& w, const void* q, const void* k, hipStream_t st) {
    auto q_ = static_cast<const T*>(q);
    auto k_ = static_cast<const T*>(k);
    const unsigned slices = (unsigned)w.g.B * w.g.Hkv, grid = slices * w.g.nsplit * w.shares;
    hipError_t e;
    if (w.form == 0) {
        constexpr size_t lds = WeightsFew<T, D>::kLds;
        auto kern = weights_few_kernel<T, D>;
        if ((e = seq_allow_lds(kern, lds)) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3(grid), dim3(WeightsFew<T, D>::kWaves * 64), lds, st, w, q_, k_);
    } else {
        constexpr size_t lds = WeightsMany<T, D>::kLds;
        auto kern = weights_many_kernel<T, D>;
        if ((e = seq_allow_lds(kern, lds)) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, w, q_, k_);
        if (w.shares > 1) {
            if ((e = hipGetLastError()) != hipSuccess) return e;
            hipLaunchKernelGGL(weights_join_kernel, dim3(slices * w.joins), dim3(256), 0, st, w);
        }
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_weights_d(const WeightsGeo& w, int D, const void* q, const void* k,
                            hipStream_t st) {
    switch (D) {
        case 32: return launch_weights<T, 32>(w, q, k, st);
        case 64: return launch_weights<T, 64>(w, q, k, st);
        case 128: return launch_weights<T, 128>(w, q, k, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_weights(const WeightsGeo& w, int D, int dtype, const void* q, const void* k,
                                hipStream_t st) {
    switch (dtype) {
        case 0: return launch_weights_d<float>(w, D, q, k, st);
        case 1: return launch_weights_d<_Float16>(w, D, q, k, st);
        case 2: return launch_weights_d<__bf16>(w, D, q, k, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace na
