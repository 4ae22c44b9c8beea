// na_seq_fwd.hip -- forward of attention over a sliding window and the first tokens, for
// contiguous sequences and for new tokens against a paged cache (gfx950).
//
//   out_i = sum_j exp(s_ij - lse_i) v_j,  s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij
//   over the j <= i with i - j < W or j < S.
//
// One pass over the keys with the running maximum and sum of an online softmax, in base 2.
//   S^T = K Q^T (32 keys x 32 rows a step) leaves a row's scores in one lane column (two
//   lanes), so the maximum needs one lane swap and P^T feeds O^T = V^T P^T from registers.
// Sums, maxima and accumulators are fp32.  P is rounded once to the type of V for its matrix
// product (16-bit types); the sum that divides it and the logsumexp take P unrounded.
//
// Two forms:
//   wide    four waves of 32 rows each share the staged key tiles: many rows
//   narrow  one block of 32 rows (new tokens x heads of a group); the four waves take
//           every fourth key tile each, from LDS buffers of their own without barriers, and
//           join their sums at the end: single tokens, where reading the cache is the work
#include <cmath>
#include <type_traits>

#include "na_launch.h"
#include "na_seq_state.h"

namespace na {

// Bound by the matrix cores and the vector unit in turn (the cache and the windows come from L2): at
// D = 64 the cores are busy 34 % of the cycles and the vector unit 60 %, so little of one overlaps
// the other; at D = 128, with two waves a SIMD, 26 to 33 % and 28 %, the rest waits.
//   16 heads on 4, 8192 tokens, bf16 D = 128: window 512 and 4 first tokens 55 to 62 us, full causal
// 284 to 297 us (0.93 to 0.97 PFLOP/s); 16 heads, 32768 tokens, window 1023, fp16 D = 64 203 to 208
// us (0.67); chunks of 512 to 2048 tokens over 2k to 8k cached ones, 4 requests, bf16 D = 128 317
// to 341 us (0.80).
template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? (D == 128 ? 2 : 4) : 1)) void seq_wide_kernel(
    SeqGeo g, const T* __restrict__ qg, const T* __restrict__ kg, const T* __restrict__ vg,
    T* __restrict__ og, float* __restrict__ lseg, float* __restrict__ part) {
    using F = SeqFrags<T, D>;
    using Ring = SeqRing<T, D>;
    constexpr int SK = Ring::kTiles, NB = Ring::kStages;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & 3);

    // ---- workgroup -> (split, row tile, key/value head, sequence) ----
    SeqTile t;
    int split = 0, kvh, tile;
    if constexpr (PAGED) {
        split = g.fd_tiles.div(blockIdx.x);
        const int id = blockIdx.x - split * g.ntiles * g.Hkv;
        tile = g.fd_kv.div(id);
        kvh = id - tile * g.Hkv;
        if (g.B > 64) tile = g.ntiles - 1 - tile;  // (long tiles of a request first, at least)
        if (!seq_locate(g, tile, 7, lane, t)) return;
    } else {
        int slice;
        seq_job(g, blockIdx.x, gridDim.x, tile, slice);
        seq_contiguous(g, tile, slice, t);
        kvh = slice - t.b * g.Hkv;
    }
    int e0 = 0, e1 = t.nT, splits = 1;
    if constexpr (PAGED) {
        splits = seq_splits(g, t.nT);
        if (split >= splits) return;
        e0 = split * g.chunk;
        e1 = split == splits - 1 ? t.nT : e0 + g.chunk;
    }

    SeqStage<T, D, PAGED, 4> ld;
    ld.init(g, t, kvh, lane, kg, vg);
    auto issue_stage = [&](int e, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SK; ++i)  // (a tile behind the last one: zeros)
            if (e < e1) ld.issue(g, t, e + i, wave, smem + buf * Ring::kStage + i * 2 * F::kTile);
    };
#pragma unroll
    for (int b = 0; b < NB - 1; ++b) issue_stage(e0 + b * SK, b);

    // ---- this lane's row, and the positions of the wave's rows ----
    const int m = wave * 32 + (lane & 31);
    int tok, head;
    seq_row(g, t, m, tok, head);
    const int pos = t.pos0 + tok;
    const bool live = wave * 32 < t.rows;
    int tf, tl, hh;
    seq_row(g, t, wave * 32, tf, hh);
    seq_row(g, t, wave * 32 + 31, tl, hh);
    const int wmin = t.pos0 + tf;
    const int wmax = min(t.pos0 + tl, PAGED ? t.pmax : t.valid - 1);
    const int64_t hq = (int64_t)kvh * g.G + head;
    SeqState<T, D> st;
    st.init();
    {
        const unsigned char* qp = reinterpret_cast<const unsigned char*>(qg) +
                                  (PAGED ? 0 : t.b * g.qb) + hq * g.qh +
                                  // (rows behind the length hold anything: not theirs)
                                  (int64_t)(t.qtok + max(min(tok, t.valid - 1), 0)) * g.qt;
#pragma unroll
        for (int s = 0; s < F::kKS; ++s)
            st.qf[s] = ld_x8<T>(reinterpret_cast<const T*>(qp) + s * 16 + 8 * (lane >> 5));
    }
    F f;
    f.init(lane);
#pragma unroll
    for (int s = 0; s < F::kKS; ++s) settle(st.qf[s]);

    auto seen = [&](int base) __attribute__((always_inline)) {
        return seen_keys(pos - base, g.W, g.S - base);
    };

    // One stage, in buffer BUF (a constant, so that LDS addresses are the lane's offsets plus
    // immediates).  Its loads have landed when no more than the later stages' are outstanding.
    auto stage = [&](int e, auto BUF) __attribute__((always_inline)) {
        constexpr int kBuf = decltype(BUF)::value;
        if (NB > 2 && e + (NB - 2) * SK < e1)  // NB - 2 stages behind it
            wait_vmem_but<(NB - 2) * SK * decltype(ld)::kCount>();
        else
            wait_vmem();
        lds_barrier();  // for every wave; and the stage before is read
        issue_stage(e + (NB - 1) * SK, (kBuf + NB - 1) % NB);
        const unsigned char* base = smem + kBuf * Ring::kStage;
        const unsigned char* tile[SK];
        int j0[SK];
        bool on[SK], out = true, full = true;
#pragma unroll
        for (int i = 0; i < SK; ++i) {
            tile[i] = base + i * 2 * F::kTile;
            j0[i] = t.tile(e + i);
            on[i] = i == 0 || e + i < e1;
            // outside every window of the wave's rows, and no first tokens
            out = out && (!on[i] || j0[i] > wmax || (wmin - (j0[i] + 31) >= g.W && j0[i] >= g.S));
            full = full && on[i] && j0[i] + 31 <= wmin && (wmax - j0[i] < g.W || j0[i] + 31 < g.S);
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

    // ---- epilogue ----
    const float l = col_sum<32>(st.l);
    if (m >= t.rows) return;
    const bool some = l > 0.f && (PAGED || tok < t.valid);
    const float inv = some ? 1.f / l : 0.f;
    const float lse2 = some ? st.mref + __log2f(l) : -INFINITY;
    const int h = lane >> 5;
    if (PAGED && splits > 1) {
        const int64_t row = ((int64_t)(tile * g.Hkv + kvh) * g.nsplit + split) * 128 + m;
        float* po = part + row * D;
#pragma unroll
        for (int db = 0; db < F::kDB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                st16<f32x4>(po + db * 32 + i * 8 + h * 4,
                            f32x4{st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                                  st.o[db][4 * i + 3]} * inv);
        if (h == 0) part[(int64_t)g.ntiles * g.Hkv * g.nsplit * 128 * D + row] = lse2;
        return;
    }
    T* op = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(og) + (PAGED ? 0 : t.b * g.ob) +
                                 hq * g.oh + (int64_t)(t.qtok + tok) * g.ot);
#pragma unroll
    for (int db = 0; db < F::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            st_x4<T>(op + db * 32 + i * 8 + h * 4,
                     f32x4{st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                           st.o[db][4 * i + 3]} * inv);
    if (h == 0)
        lseg[(PAGED ? 0 : t.b * g.lb) + hq * g.lh + (int64_t)(t.qtok + tok) * g.lt] =
            some ? lse2 * kLn2 : -INFINITY;
}

// Bound by reading the cache once: one new token for each of 32 requests over 8k to 32k cached
// ones, 16 heads on 4, fp16 D = 128, 1.07 GB in 211 us (5.1 TB/s).  Each wave stages whole tiles
// for itself, so no wave waits for another, and a split's key tiles are spread over the four.
template <typename T, int D>
__global__ __launch_bounds__((seq_narrow_waves<T, D>() * 64), 1) void seq_narrow_kernel(
    SeqGeo g, const T* __restrict__ qg, const T* __restrict__ kg, const T* __restrict__ vg,
    T* __restrict__ og, float* __restrict__ lseg, float* __restrict__ part) {
    using F = SeqFrags<T, D>;
    using N = SeqNarrow<T, D>;
    constexpr int W = N::W;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & (W - 1));

    SeqTile t;
    const int split = g.fd_tiles.div(blockIdx.x);
    const int id = blockIdx.x - split * g.ntiles * g.Hkv;
    const int tile = g.fd_kv.div(id);
    const int kvh = id - tile * g.Hkv;
    if (!seq_locate(g, tile, 5, lane, t)) return;
    const int splits = seq_splits(g, t.nT);
    if (split >= splits) return;
    const int e0 = split * g.chunk;
    const int e1 = split == splits - 1 ? t.nT : e0 + g.chunk;

    SeqStage<T, D, true, 1> ld;
    ld.init(g, t, kvh, lane, kg, vg);
    unsigned char* buf0 = smem + wave * 4 * F::kTile;
    int e = e0 + wave;
    if (e < e1) ld.issue(g, t, e, 0, buf0);

    int tok, head;
    seq_row(g, t, lane & 31, tok, head);
    const int pos = t.pos0 + tok;
    const int64_t hq = (int64_t)kvh * g.G + head;
    SeqState<T, D> st;
    st.init();
    {
        const unsigned char* qp = reinterpret_cast<const unsigned char*>(qg) + hq * g.qh +
                                  (int64_t)(t.qtok + tok) * g.qt;
#pragma unroll
        for (int s = 0; s < F::kKS; ++s)
            st.qf[s] = ld_x8<T>(reinterpret_cast<const T*>(qp) + s * 16 + 8 * (lane >> 5));
    }
    F f;
    f.init(lane);
#pragma unroll
    for (int s = 0; s < F::kKS; ++s) settle(st.qf[s]);
    auto seen = [&](int base) __attribute__((always_inline)) {
        return seen_keys(pos - base, g.W, g.S - base);
    };
    wait_vmem();  // (the first tile too: from here on only stage loads are outstanding)
    for (int buf = 0; e < e1; e += W, buf ^= 1) {
        if (e + W < e1) {
            ld.issue(g, t, e + W, 0, buf0 + (buf ^ 1) * 2 * F::kTile);
            wait_vmem_but<2 * SeqRows<T, D>::kInstr>();
        } else {
            wait_vmem();
        }
        const unsigned char* ks[1] = {buf0 + buf * 2 * F::kTile};
        const int j0 = t.tile(e);
        const bool full = j0 + 31 <= t.pmin && (t.pmax - j0 < g.W || j0 + 31 < g.S);
        const int js[1] = {j0};
        const bool on[1] = {true};
        st.template fold<1>(f, ks, lane, g.c, full, js, on, seen);
        wait_lds();  // before the next loads into this buffer
    }

    // ---- join the waves: every sum relative to the largest reference ----
    const float l = col_sum<32>(st.l);
    float* stat = reinterpret_cast<float*>(smem + N::kStat);  // [wave][32] of (reference, sum)
    if (lane < 32) {
        stat[(wave * 32 + lane) * 2] = st.mref;
        stat[(wave * 32 + lane) * 2 + 1] = l;
    }
    __syncthreads();
    const int col = lane & 31, h = lane >> 5;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, stat[(w * 32 + col) * 2]);
    const float scale = st.mref == -INFINITY ? 0.f : fast_exp2(st.mref - top);
    {
        float* mine = reinterpret_cast<float*>(smem + (wave * 32 + col) * N::kRow);
#pragma unroll
        for (int db = 0; db < F::kDB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                st16<f32x4>(mine + db * 32 + i * 8 + h * 4,
                            f32x4{st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                                  st.o[db][4 * i + 3]} * scale);
    }
    __syncthreads();
    // each thread: four columns of a row
    for (int x = threadIdx.x; x < t.rows * (D / 4); x += W * 64) {
        const int row = x / (D / 4), d = x % (D / 4) * 4;
        float mx = -INFINITY, sum = 0.f;
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) mx = fmaxf(mx, stat[(w * 32 + row) * 2]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float m = stat[(w * 32 + row) * 2];
            sum += m == -INFINITY ? 0.f : fast_exp2(m - mx) * stat[(w * 32 + row) * 2 + 1];
            acc += *reinterpret_cast<const f32x4*>(smem + (w * 32 + row) * N::kRow + d * 4);
        }
        const bool some = sum > 0.f;
        acc *= some ? 1.f / sum : 0.f;
        const float lse2 = some ? mx + __log2f(sum) : -INFINITY;
        if (splits > 1) {
            const int64_t pr = ((int64_t)(tile * g.Hkv + kvh) * g.nsplit + split) * 32 + row;
            st16<f32x4>(part + pr * D + d, acc);
            if (d == 0) part[(int64_t)g.ntiles * g.Hkv * g.nsplit * 32 * D + pr] = lse2;
        } else {
            int tk, hd;
            seq_row(g, t, row, tk, hd);
            const int64_t hr = (int64_t)kvh * g.G + hd;
            T* op = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(og) + hr * g.oh +
                                         (int64_t)(t.qtok + tk) * g.ot);
            st_x4<T>(op + d, acc);
            if (d == 0)
                lseg[hr * g.lh + (int64_t)(t.qtok + tk) * g.lt] = some ? lse2 * kLn2 : -INFINITY;
        }
    }
}

// Joins the splits of each row: out = sum_s 2^(lse_s - lse) out_s, in a fixed order.  One
// workgroup per 32 rows of a (row tile, key/value head); D / 4 threads a row.  4 to 5 us, most
// of it the launch and one chain of loads.
template <typename T, int D>
__global__ __launch_bounds__(256) void seq_join_kernel(SeqGeo g, int lgM, T* __restrict__ og,
                                                       float* __restrict__ lseg,
                                                       const float* __restrict__ part) {
    const int id = blockIdx.x >> (lgM - 5), r0 = (blockIdx.x & ((1 << (lgM - 5)) - 1)) * 32;
    int tile = g.fd_kv.div(id);
    const int kvh = id - tile * g.Hkv;
    const int64_t row0 = (int64_t)(tile * g.Hkv + kvh) * g.nsplit << lgM;
    SeqTile t;
    if (!seq_locate(g, tile, lgM, threadIdx.x & 63, t)) return;
    const int splits = seq_splits(g, t.nT);
    if (splits == 1) return;  // written by the only split
    const float* pl = part + ((int64_t)g.ntiles * g.Hkv * g.nsplit << lgM) * D + row0;
    const int end = min(32, t.rows - r0) * (D / 4);
    for (int x = threadIdx.x; x < end; x += 256) {
        const int row = r0 + x / (D / 4), d = x % (D / 4) * 4;
        float mx = -INFINITY, sum = 0.f;
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float e = pl[(s << lgM) + row];
            const f32x4 y = ld16<f32x4>(part + (row0 + (s << lgM) + row) * D + d);
            const float top = fmaxf(mx, e);
            const float a = mx == -INFINITY ? 0.f : fast_exp2(mx - top);
            const float w = e == -INFINITY ? 0.f : fast_exp2(e - top);
            sum = sum * a + w;
            acc = acc * a + y * w;
            mx = top;
        }
        const bool some = sum > 0.f;
        int tk, hd;
        seq_row(g, t, row, tk, hd);
        const int64_t hr = (int64_t)kvh * g.G + hd;
        T* op = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(og) + hr * g.oh +
                                     (int64_t)(t.qtok + tk) * g.ot);
        st_x4<T>(op + d, acc * (some ? 1.f / sum : 0.f));
        if (d == 0)
            lseg[hr * g.lh + (int64_t)(t.qtok + tk) * g.lt] =
                some ? (mx + __log2f(sum)) * kLn2 : -INFINITY;
    }
}

// ---- host ----
template <typename T, int D>
static hipError_t launch_fwd(const SeqGeo& g, bool paged, bool narrow, const T* q, const T* k,
                             const T* v, T* out, float* lse, float* part, hipStream_t s) {
    const unsigned tiles = (unsigned)g.ntiles * g.Hkv * (paged ? 1 : g.B);
    hipError_t e;
    if (narrow) {
        using N = SeqNarrow<T, D>;
        auto kern = seq_narrow_kernel<T, D>;
        if ((e = seq_allow_lds(kern, N::kLds)) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3(tiles * g.nsplit), dim3(N::W * 64), N::kLds, s, g, q, k, v,
                           out, lse, part);
    } else {
        constexpr size_t lds = SeqRing<T, D>::kLds;
        auto kern = paged ? seq_wide_kernel<T, D, true> : seq_wide_kernel<T, D, false>;
        if ((e = seq_allow_lds(kern, lds)) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3(tiles * g.nsplit), dim3(256), lds, s, g, q, k, v, out, lse,
                           part);
    }
    if ((e = hipGetLastError()) != hipSuccess || g.nsplit == 1) return e;
    hipLaunchKernelGGL((seq_join_kernel<T, D>), dim3(tiles * (narrow ? 1 : 4)), dim3(256), 0, s, g,
                       narrow ? 5 : 7, out, lse, part);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_fwd_d(const SeqGeo& g, int D, bool paged, bool narrow, const void* q,
                               const void* k, const void* v, void* out, float* lse, float* part,
                               hipStream_t s) {
    auto q_ = static_cast<const T*>(q);
    auto k_ = static_cast<const T*>(k);
    auto v_ = static_cast<const T*>(v);
    auto o_ = static_cast<T*>(out);
    switch (D) {
        case 32: return launch_fwd<T, 32>(g, paged, narrow, q_, k_, v_, o_, lse, part, s);
        case 64: return launch_fwd<T, 64>(g, paged, narrow, q_, k_, v_, o_, lse, part, s);
        case 128: return launch_fwd<T, 128>(g, paged, narrow, q_, k_, v_, o_, lse, part, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_seq_forward(const SeqGeo& g, int D, int dtype, bool paged, bool narrow,
                              const void* q, const void* k, const void* v, void* out, float* lse,
                              float* part, hipStream_t s) {
    switch (dtype) {
        case 0: return launch_fwd_d<float>(g, D, paged, narrow, q, k, v, out, lse, part, s);
        case 1: return launch_fwd_d<_Float16>(g, D, paged, narrow, q, k, v, out, lse, part, s);
        case 2: return launch_fwd_d<__bf16>(g, D, paged, narrow, q, k, v, out, lse, part, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace na
