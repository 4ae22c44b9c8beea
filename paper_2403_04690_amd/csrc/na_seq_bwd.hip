// na_seq_bwd.hip -- gradient of the attention of na_seq_fwd.hip over contiguous sequences
// (gfx950).
//
//   P_ij = exp(s_ij - lse_i), delta_i = dout_i . out_i, dA_ij = P_ij (dout_i . v_j - delta_i)
//   dq_i = scale sum_j dA_ij k_j
//   dk_j = scale sum_i dA_ij q_i,  dv_j = sum_i P_ij dout_i   over the rows of every head that
//                                                             shares the key head
//
// P is recomputed from the logsumexp; no weight reaches global memory; no atomics, every sum
// in a fixed order.  Three launches (two without first tokens and without split heads):
//   dq      row-major like the forward: 128 rows a workgroup, over the keys they see; it forms
//           delta, and leaves delta and the logsumexp in base 2 per row for the next launch
//   dk, dv  key-major: 128 keys a workgroup over the rows whose window holds them.  Rows run
//           head by head, so that staged rows are consecutive tokens.  Few key tiles (short
//           sequences, many heads a group) split the heads over workgroups.  The first tokens
//           are attended by every later row: those pairs (outside the window) are cut over
//           rows into workgroups of their own, in the same launch, behind the others
//   join    sums the fp32 parts that split heads and first tokens leave
// P and dA are rounded once to the tensors' type for their matrix products (16-bit types);
// everything else is fp32.  fp16 has too few exponents for both as they are: over thousands of
// keys P falls below its normal range, and dA goes with the size of dout, which small or large
// loss scales take below it or above its largest number.  So in fp16
//   P  enters dv times 2^15 (P <= 1), which the logsumexp that the dq launch leaves contains
//   dA is scaled by a power of two of its own per row (dq) or key (dk), a column of the products
//      and so a lane: lowered, with the accumulators, when a tile brings a value above 2^15, to
//      where the largest is at 2^11 to 2^12 (DaScale)
// and both are undone, exactly, in the fp32 sums.  Without, dv over 128k keys was off by twice what
// its roundings are, and dq with output gradients of 2^-14 by seven times; it costs 5 to 6 % of
// the gradient (16 heads on 4, 8192 tokens, D = 128: window 512 198 us without and 204 with, full
// causal 5.4 and 10.7 % above bf16; short sequences 31 and 33 us).
#include <type_traits>

#include "na_launch.h"
#include "na_seq_kernels.h"

namespace na {

// fp16 only; the other types have fp32's exponents.
template <typename T>
constexpr bool kHalf = std::is_same<T, _Float16>::value;
constexpr float kPExp = 15.f;  // base-2 exponent that P has in the dk, dv launch

// The power of two that a lane's dA is scaled by.  It starts so high that whatever is not lost in
// fp16's gradients anyway is in fp16's normal range (dout, v and P of 2^-24: 2^-72 in all), and
// the largest (dout, v of 2^16, D = 128, P of 2^kPExp: 2^56) still far from fp32's end.
struct DaScale {
    static constexpr float kStart = 0x1p+58f, kMost = 0x1p+15f;
    float by;
    __device__ __forceinline__ void init() { by = kStart; }
    // exactly 1 / by
    __device__ __forceinline__ float undo() const {
        return __int_as_float((254 << 23) - __float_as_int(by));
    }
    // x: the scaled values of a tile, two lanes a column; acc: what they are added to.  Returns
    // what `by` was multiplied with.
    template <int N>
    __device__ __forceinline__ float fit(float (&x)[16], f32x16 (&acc)[N]) {
        float top = fabsf(x[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
        if (!__builtin_amdgcn_ballot_w64(top > kMost)) return 1.f;
        top = col_max<32>(top);
        const float f = top > kMost ? ldexpf(1.f, 12 - __builtin_amdgcn_frexp_expf(top)) : 1.f;
        by *= f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= f;
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n] *= f;
        return f;
    }
};

// ---- dq: 32 rows a wave ----
template <typename T, int D>
struct DqState {
    using F = SeqFrags<T, D>;
    using x8 = typename Tr<T>::x8;
    x8 qf[F::kKS], gf[F::kKS];
    f32x16 dq[F::kDB];
    float lse2, delta;
    DaScale scale;  // (fp16) and delta under it
    float sdelta;

    // P and dout . v of a tile of keys; full, j0, pos: as in the forward.
    __device__ __forceinline__ void weights(const F& f, const unsigned char* kt,
                                            const unsigned char* vt, int lane, float c, bool full,
                                            int j0, int pos, int W, int S, f32x16& s, f32x16& dp) {
        x8 kf[F::kKS], vf[F::kKS];
        s = dp = f32x16{} * 0.f;
        f.rows(kt, kf);
        if constexpr (sizeof(T) == 2) f.rows(vt, vf);
#pragma unroll
        for (int st = 0; st < F::kKS; ++st) s = mma32<T>(kf[st], qf[st], s);
        if constexpr (sizeof(T) == 4) f.rows(vt, vf);
#pragma unroll
        for (int st = 0; st < F::kKS; ++st) dp = mma32<T>(vf[st], gf[st], dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fast_exp2(fmaf(s[i], c, -lse2));
        if (!full) {
            const int base = j0 + 4 * (lane >> 5);
            const unsigned m = seen_keys(pos - base, W, S - base);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = keep(m, i, s[i], 0.f);
        }
    }

    __device__ __forceinline__ void tile(const F& f, const unsigned char* kt,
                                         const unsigned char* vt, int lane, float c, bool full,
                                         int j0, int pos, int W, int S) {
        f32x16 s, dp;
        weights(f, kt, vt, lane, c, full, j0, pos, W, S, s, dp);
        x8 kc[2][F::kDB];
        f.cols(kt, 0, lane, kc[0]);
        if constexpr (sizeof(T) == 2) f.cols(kt, 1, lane, kc[1]);
        x8 pf[2];
        float x[16];
        if constexpr (kHalf<T>) {
            // (scaling by a power of two and the difference: one rounding, in one instruction)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = s[i] * fmaf(dp[i], scale.by, -sdelta);
            sdelta *= scale.fit(x, dq);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = s[i] * (dp[i] - delta);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) pf[i >> 3][i & 7] = Tr<T>::cvt(x[i]);
#pragma unroll
        for (int db = 0; db < F::kDB; ++db) dq[db] = mma32<T>(kc[0][db], pf[0], dq[db]);
        if constexpr (sizeof(T) == 4) f.cols(kt, 1, lane, kc[1]);
#pragma unroll
        for (int db = 0; db < F::kDB; ++db) dq[db] = mma32<T>(kc[1][db], pf[1], dq[db]);
    }
};

// Rows of fewer keys than this form delta themselves (see seq_dq_kernel).
constexpr int kFewKeys = 128;

// (a ring of three stages of a key tile, as the forward's)
//   delta_i = dout_i . out_i takes out as the forward rounded it.  Where a row has few keys, out
// is as large as a value, and that rounding is most of what dq is off by besides its own and
// dA's: in 16-bit types the row tiles with such rows (the first tokens', or all of a short
// window) pass over their keys twice, and first sum delta_i = sum_j P_ij dout_i . v_j
// unrounded.  (Error of dq, in errors of one rounding of it: 1.45 to 1.65 without, 1.40 to 1.47
// with.  Gradients of 16 heads on 4, 8192 tokens, bf16 D = 128: window 120, every tile twice,
// 86 and 96 us; window 512, the first ones only, 206 and 207.)
template <typename T, int D>
__global__ __launch_bounds__(256, (sizeof(T) == 4 ? 1 : D == 128 ? 2 : 3)) void seq_dq_kernel(
    SeqBwd b, const T* __restrict__ qg, const T* __restrict__ kg, const T* __restrict__ vg,
    const T* __restrict__ og, const float* __restrict__ lseg, const T* __restrict__ dog,
    T* __restrict__ dqg) {
    using F = SeqFrags<T, D>;
    constexpr int kBuf = 2 * F::kTile;
    extern __shared__ __align__(16) unsigned char smem[];
    const SeqGeo& g = b.g;
    const int lane = threadIdx.x & 63;
    const int wave = uniform((threadIdx.x >> 6) & 3);

    SeqTile t;
    int tile, slice;
    seq_job(g, blockIdx.x, gridDim.x, tile, slice);
    seq_contiguous(g, tile, slice, t);
    const int kvh = slice - t.b * g.Hkv;

    SeqStage<T, D, false, 4> ld;
    ld.init(g, t, kvh, lane, kg, vg);
    if (t.nT > 0) ld.issue(g, t, 0, wave, smem);
    if (t.nT > 1) ld.issue(g, t, 1, wave, smem + kBuf);

    const int m = wave * 32 + (lane & 31), h = lane >> 5;
    int tok, head;
    seq_row(g, t, m, tok, head);
    const bool live = wave * 32 < t.rows;
    int tf, tl, hh;
    seq_row(g, t, wave * 32, tf, hh);
    seq_row(g, t, wave * 32 + 31, tl, hh);
    const int wmin = tf, wmax = min(tl, t.valid - 1);
    const int64_t hq = (int64_t)kvh * g.G + head;
    const int64_t from = max(min(tok, t.valid - 1), 0);  // (rows behind the length: not theirs)
    DqState<T, D> st;
    {
        const T* qp = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(qg) +
                                                 t.b * g.qb + hq * g.qh + from * g.qt) + 8 * h;
        const T* op = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(og) +
                                                 t.b * g.ob + hq * g.oh + from * g.ot) + 8 * h;
        const T* gp = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(dog) +
                                                 t.b * b.gb + hq * b.gh + from * b.gt) + 8 * h;
        float d = 0.f;
#pragma unroll
        for (int s = 0; s < F::kKS; ++s) {
            st.qf[s] = ld_x8<T>(qp + s * 16);
            st.gf[s] = ld_x8<T>(gp + s * 16);
            d = dot8<T>(st.gf[s], ld_x8<T>(op + s * 16), d);
        }
        st.delta = col_sum<32>(d);
        st.lse2 = lseg[t.b * g.lb + hq * g.lh + from] * kLog2e;
    }
    F f;
    f.init(lane);
#pragma unroll
    for (int s = 0; s < F::kKS; ++s) {
        settle(st.qf[s]);
        settle(st.gf[s]);
    }
    settle(st.lse2);
    settle(st.delta);

    float own = 0.f;  // this lane's share of delta
    auto stage = [&](int e, auto BUF, auto FIRST) __attribute__((always_inline)) {
        constexpr int kAt = decltype(BUF)::value;
        if (e + 1 < t.nT)
            wait_vmem_but<decltype(ld)::kCount>();
        else
            wait_vmem();
        lds_barrier();
        if (e + 2 < t.nT) ld.issue(g, t, e + 2, wave, smem + (kAt + 2) % 3 * kBuf);
        const int j0 = t.tile(e);
        const bool out = j0 > wmax || (wmin - (j0 + 31) >= g.W && j0 >= g.S);
        const bool full = j0 + 31 <= wmin && (wmax - j0 < g.W || j0 + 31 < g.S);
        const unsigned char* kt = smem + kAt * kBuf;
        if (!live || out) return;
        if constexpr (decltype(FIRST)::value) {
            f32x16 s, dp;
            st.weights(f, kt, kt + F::kTile, lane, g.c, full, j0, tok, g.W, g.S, s, dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) own = fmaf(s[i], dp[i], own);
        } else {
            st.tile(f, kt, kt + F::kTile, lane, g.c, full, j0, tok, g.W, g.S);
        }
    };
    auto pass = [&](auto FIRST) __attribute__((always_inline)) {
        wait_vmem();  // (the row's own loads and stores too: from here on only stage loads count)
        for (int e = 0; e < t.nT; e += 3) {
            stage(e, std::integral_constant<int, 0>{}, FIRST);
            if (e + 1 < t.nT) stage(e + 1, std::integral_constant<int, 1>{}, FIRST);
            if (e + 2 < t.nT) stage(e + 2, std::integral_constant<int, 2>{}, FIRST);
        }
    };
    if constexpr (sizeof(T) == 2) {
        if (t.nT > 0 && min(t.pmin + 1, min(g.W, kFewKeys) + min(g.S, kFewKeys)) < kFewKeys) {
            pass(std::true_type{});
            st.delta = col_sum<32>(own);
            lds_barrier();  // (the last stages are read)
            ld.issue(g, t, 0, wave, smem);
            if (t.nT > 1) ld.issue(g, t, 1, wave, smem + kBuf);
        }
    }
    if (m < t.rows && h == 0) {
        const int64_t at = t.b * g.lb + hq * g.lh + tok;
        b.lse2[at] = kHalf<T> ? st.lse2 - kPExp : st.lse2;
        b.delta[at] = st.delta;
    }
    float scale = b.scale;
    if constexpr (kHalf<T>) {
        st.scale.init();
        st.sdelta = st.delta * st.scale.by;
    }
#pragma unroll
    for (int db = 0; db < F::kDB; ++db) st.dq[db] = f32x16{} * 0.f;
    pass(std::false_type{});

    if (m >= t.rows) return;
    const bool some = tok < t.valid;
    if constexpr (kHalf<T>) scale *= st.scale.undo();
    T* dp = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(dqg) + t.b * b.qb + hq * b.qh +
                                 (int64_t)tok * b.qt);
#pragma unroll
    for (int db = 0; db < F::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = some ? st.dq[db][4 * i + r] * scale : 0.f;
            st_x4<T>(dp + db * 32 + i * 8 + h * 4, x);
        }
}

// ---- dk, dv: 32 keys a wave ----
// A workgroup has 4 blocks of 32 keys and RS groups of four waves, one wave a block: the groups
// take the row tiles in turn and add up their sums at the end, so that few key tiles still fill
// the SIMDs (RS = 1 or 2).
// A staged tile: 32 rows of q, the same of dout, then their lse2 and delta (256 bytes).
// 16-bit types at D = 128 read the keys and values from LDS for each product: with their
// fragments in registers beside 128 accumulators, tens of registers spill, and every reload
// in the loop waits for the stage loads in flight too.
template <typename T, int D, int RS>
struct KvCfg {
    static constexpr int kRows = SeqFrags<T, D>::kTile;
    static constexpr int kBytes = 2 * kRows + 256;
    static constexpr bool kOwnLds = sizeof(T) == 2 && D == 128;
    static constexpr int kPer = D == 128 ? 1 : 2;  // tiles of a group per stage
    static constexpr int kBufs = 2 * kPer * RS;
    static constexpr int kOwn = kBufs * kBytes;  // LDS offset of the keys and values
    // a workgroup of first tokens: a buffer for each wave, and one block's keys and values
    static constexpr int kFirst = 4 * RS;
    static constexpr int kFirstOwn = kFirst * kBytes;
    static constexpr int kMain = kOwn + (kOwnLds ? 8 * kRows : 0);
    static constexpr int kFirstLds = kFirstOwn + (kOwnLds ? 2 * kRows : 0);
    static constexpr int kLds = kMain > kFirstLds ? kMain : kFirstLds;
    static_assert(kLds <= 160 * 1024, "LDS of a CU");
};

// OUT: kDk | kDv.  fp32 at D = 128 holds only one gradient's accumulators beside its
// fragments, and forms dv and dk in two launches.
enum { kDk = 1, kDv = 2 };
template <typename T, int D, int OUT, bool LDS>
struct KvState {
    using F = SeqFrags<T, D>;
    using x8 = typename Tr<T>::x8;
    static constexpr bool kKf = !LDS, kVf = (OUT & kDk) && !LDS;
    x8 kf[kKf ? F::kKS : 1], vf[kVf ? F::kKS : 1];
    f32x16 dk[OUT & kDk ? F::kDB : 1], dv[OUT & kDv ? F::kDB : 1];
    DaScale scale;  // (fp16)

    // Keys of this wave: lane l has key l % 32.
    __device__ __forceinline__ void init(const unsigned char* kp, const unsigned char* vp, int h) {
#pragma unroll
        for (int s = 0; s < F::kKS; ++s) {
            if constexpr (kKf) kf[s] = ld_x8<T>(reinterpret_cast<const T*>(kp) + s * 16 + 8 * h);
            if constexpr (kVf) vf[s] = ld_x8<T>(reinterpret_cast<const T*>(vp) + s * 16 + 8 * h);
        }
#pragma unroll
        for (int db = 0; db < F::kDB; ++db) {
            if constexpr (OUT & kDk) dk[db] = f32x16{} * 0.f;
            if constexpr (OUT & kDv) dv[db] = f32x16{} * 0.f;
        }
        if constexpr (kHalf<T>) scale.init();
    }
    // The sums without the powers of two of P and dA; before they meet other waves'.
    __device__ __forceinline__ void finish() {
        if constexpr (kHalf<T>) {
            constexpr float p = 1.f / (1 << 15);
            static_assert(kPExp == 15.f, "p is its inverse");
            const float a = scale.undo() * p;
#pragma unroll
            for (int db = 0; db < F::kDB; ++db) {
                if constexpr (OUT & kDk) dk[db] *= a;
                if constexpr (OUT & kDv) dv[db] *= p;
            }
        }
    }
    __device__ __forceinline__ void settle_keys() {
#pragma unroll
        for (int s = 0; s < F::kKS; ++s) {
            if constexpr (kKf) settle(kf[s]);
            if constexpr (kVf) settle(vf[s]);
        }
    }

    // Rows i0 .. i0 + 31.  Unless `full` (uniform), row i0 + 4 h + e sees this lane's key when
    // (unsigned)(dist + e) < len.  (One body with a branch around the mask alone: two bodies
    // meeting again in the accumulators spill them at D = 128.)  own: the wave's keys, then
    // its values (LDS).
    __device__ __forceinline__ void tile(const F& f, const unsigned char* qt, const unsigned char* own,
                                         int lane, float c, bool full, int dist, int len) {
        const unsigned char* gt = qt + F::kTile;
        const float* stat = reinterpret_cast<const float*>(gt + F::kTile) + 4 * (lane >> 5);
        const int ro = opaque(f.ro), co = opaque(f.co);
        constexpr int kKS = F::kKS, kDB = F::kDB;
        f32x16 s = f32x16{} * 0.f, dp = f32x16{} * 0.f;
#pragma unroll
        for (int st = 0; st < kKS; ++st)
            s = mma32<T>(F::row_at(qt, ro, st), LDS ? F::row_at(own, ro, st) : kf[kKf ? st : 0], s);
        if constexpr (OUT & kDk)
#pragma unroll
            for (int st = 0; st < kKS; ++st)
                dp = mma32<T>(F::row_at(gt, ro, st),
                              LDS ? F::row_at(own + F::kTile, ro, st) : vf[kVf ? st : 0], dp);
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const f32x4 lse2 = *reinterpret_cast<const f32x4*>(stat + 8 * i4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 4 * i4 + r;
                s[i] = fast_exp2(fmaf(s[i], c, -lse2[r]));
            }
        }
        if (!full) {
            const unsigned m = below(len - dist) & ~below(-dist);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = keep(m, i, s[i], 0.f);
        }
        x8 pf[2], df[2];
        if constexpr (OUT & kDv) {
#pragma unroll
            for (int i = 0; i < 16; ++i) pf[i >> 3][i & 7] = Tr<T>::cvt(s[i]);
#pragma unroll
            for (int bi = 0; bi < 2; ++bi)
#pragma unroll
                for (int db = 0; db < kDB; ++db)
                    dv[db] = mma32<T>(F::col_at(gt, co, db, bi, lane), pf[bi], dv[db]);
        }
        if constexpr (OUT & kDk) {
            float x[16];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const f32x4 delta = *reinterpret_cast<const f32x4*>(stat + 32 + 8 * i4);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 4 * i4 + r;
                    x[i] = s[i] * (dp[i] - delta[r]);
                    if constexpr (kHalf<T>) x[i] *= scale.by;
                }
            }
            if constexpr (kHalf<T>) scale.fit(x, dk);
#pragma unroll
            for (int i = 0; i < 16; ++i) df[i >> 3][i & 7] = Tr<T>::cvt(x[i]);
#pragma unroll
            for (int bi = 0; bi < 2; ++bi)
#pragma unroll
                for (int db = 0; db < kDB; ++db)
                    dk[db] = mma32<T>(F::col_at(qt, co, db, bi, lane), df[bi], dk[db]);
        }
    }

    // Adds the accumulators of waves [half, 2 half) to those of waves [0, half), through LDS,
    // one gradient at a time; every wave of the workgroup calls it.
    __device__ __forceinline__ void add_waves(unsigned char* lds, int wave, int half, int lane) {
        if constexpr (OUT & kDk) add_one(dk, lds, wave, half, lane);
        if constexpr (OUT & kDv) add_one(dv, lds, wave, half, lane);
    }
    __device__ __forceinline__ static void add_one(f32x16* acc, unsigned char* lds, int wave,
                                                   int half, int lane) {
        f32x4* at = reinterpret_cast<f32x4*>(lds) + (wave % half) * (F::kDB * 4 * kWave) + lane;
        __syncthreads();  // (what was there is read)
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int x = 0; x < F::kDB * 4; ++x)
                at[x * kWave] = f32x4{acc[x >> 2][4 * (x & 3)], acc[x >> 2][4 * (x & 3) + 1],
                                      acc[x >> 2][4 * (x & 3) + 2], acc[x >> 2][4 * (x & 3) + 3]};
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int x = 0; x < F::kDB * 4; ++x) {
                const f32x4 y = at[x * kWave];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[x >> 2][4 * (x & 3) + r] += y[r];
            }
    }
};

// Stages rows [i0, i0 + 32) of one head: q, dout, statistics; rows from `valid` on as zeros
// (their statistics are those of the last row; such pairs are masked).  Instructions first,
// first + STEP, .. of the tile.
template <typename T, int D, int STEP>
struct KvStage {
    using R = SeqRows<T, D>;
    static constexpr int kCount = 2 * R::kInstr / STEP;
    __device__ __forceinline__ static void issue(const SeqBwd& b, const unsigned char* q,
                                          const unsigned char* dout, const float* lse2,
                                          const float* delta, int i0, int valid, int first,
                                          int lane, unsigned char* dst) {
        const bool fast = i0 + 32 <= valid;
        // (formed for each tile: kept, these would be registers that the accumulators need)
        lane = opaque(lane);
        R rows;
        rows.init(lane);
        const uint32_t qlane = rows.rowl * (uint32_t)b.g.qt, glane = rows.rowl * (uint32_t)b.gt;
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            const int x = first + u * STEP;
            const bool isg = x >= R::kInstr;
            const int n = isg ? x - R::kInstr : x;
            const int r0 = n * R::kRpi;
            const unsigned char* base = (isg ? dout : q) + (int64_t)(i0 + r0) * (isg ? b.gt : b.g.qt);
            const uint32_t off = rows.off(n, isg ? glane : qlane);
            if (fast)
                seq_load(base, off, dst + x * 1024);
            else
                seq_load(i0 + r0 + rows.rowl < valid
                             ? base + off
                             : reinterpret_cast<const unsigned char*>(&kZeroRow),
                         dst + x * 1024);
        }
        if (first == 0) {
            const int row = min(i0 + (lane & 31), valid - 1);
            seq_load4(reinterpret_cast<const unsigned char*>((lane < 32 ? lse2 : delta) + row),
                      dst + 2 * R::kTile);
        }
    }
};

// Four values at a time of the 32 keys' gradients of a wave: put(column, values) for each.
template <int D, typename Put>
__device__ __forceinline__ void each_four(const f32x16* acc, int h, float scale, Put put) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = acc[db][4 * i + r] * scale;
            put(db * 32 + i * 8 + h * 4, x);
        }
}
// into fp32 parts ([key][dk, dv][D])
template <int D, int OUT, typename S>
__device__ __forceinline__ void store_part(const S& st, float* p, int h, float scale) {
    auto put = [&](int d, f32x4 x) { st16<f32x4>(p + d, x); };
    if constexpr (OUT & kDk) each_four<D>(st.dk, h, scale, put);
    p += D;
    if constexpr (OUT & kDv) each_four<D>(st.dv, h, 1.f, put);
}

//   Five products a pair from one pass over the rows: the matrix cores are busy 26 % of the cycles,
// the vector unit 22 %, LDS 24 %, in turn, with two waves a SIMD.  16 heads on 4, 8192 tokens,
// window 512, 4 first tokens, bf16 D = 128: 125 to 129 us (dq, three products a pair: 84 to 86);
// full causal: dq, dk and dv together 1000 to 1050 us, 0.65 to 0.69 PFLOP/s of the five counted.
template <typename T, int D, int OUT, int RS>
__global__ __launch_bounds__((256 * RS), (sizeof(T) == 4 ? 1 : D == 32 ? 3 : 2)) void
seq_dkv_kernel(SeqBwd b, const T* __restrict__ qg, const T* __restrict__ kg,
               const T* __restrict__ vg, const T* __restrict__ dog, T* __restrict__ dkg,
               T* __restrict__ dvg) {
    using C = KvCfg<T, D, RS>;
    extern __shared__ __align__(16) unsigned char smem[];
    const SeqGeo& g = b.g;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = uniform((threadIdx.x >> 6) & (4 * RS - 1));
    KvState<T, D, OUT, C::kOwnLds> st;
    SeqFrags<T, D> f;
    f.init(lane);

    const int jobs = gridDim.x - b.first_jobs;
    const bool first_role = (int)blockIdx.x >= jobs;
    int slice, k0, part;  // part: chunk of rows (first tokens), or of heads
    if (first_role) {
        const int id = b.fd_chunks.div(blockIdx.x - jobs);
        part = blockIdx.x - jobs - id * b.chunks;
        slice = b.fd_blocks.div(id);
        k0 = (id - slice * b.blocks) * 32;
    } else {
        // (the orders of seq_job; the first keys have the most rows)
        int tile;
        if (g.runs) {
            const int job = xcd_remap(blockIdx.x, jobs);
            const int id = b.fd_hsplit.div(job);
            part = job - id * b.hsplit;
            slice = b.fd_ktiles.div(id);
            tile = id - slice * b.ktiles;
        } else {
            const int id = g.fd_slices.div(blockIdx.x);
            slice = blockIdx.x - id * g.B * g.Hkv;
            tile = b.fd_hsplit.div(id);
            part = id - tile * b.hsplit;
        }
        k0 = tile * 128;
    }
    const int sb = g.fd_kv.div(slice), kvh = slice - sb * g.Hkv;
    const int valid = g.lengths ? min(max(g.lengths[sb], 0), g.n) : g.n;
    const unsigned char* qs = reinterpret_cast<const unsigned char*>(qg) + sb * g.qb +
                              (int64_t)kvh * g.G * g.qh;
    const unsigned char* gs = reinterpret_cast<const unsigned char*>(dog) + sb * b.gb +
                              (int64_t)kvh * g.G * b.gh;
    const int64_t stat = sb * g.lb + (int64_t)kvh * g.G * g.lh;

    const int w0 = first_role ? k0 : k0 + (wave & 3) * 32;  // this wave's first key
    const int key = w0 + (lane & 31);
    // (keys behind the length: the last one's rows, and no row sees them)
    const unsigned char* krow = reinterpret_cast<const unsigned char*>(kg) + sb * g.kb + kvh * g.kh;
    const unsigned char* vrow = reinterpret_cast<const unsigned char*>(vg) + sb * g.vb + kvh * g.vh;
    const int last_key = max(valid - 1, 0);
    unsigned char* own = smem + (first_role ? C::kFirstOwn : C::kOwn + (wave & 3) * 2 * C::kRows);
    if constexpr (C::kOwnLds) {
        if (wave < (first_role ? 1 : 4)) {
            SeqRows<T, D> rows;
            rows.init(lane);
#pragma unroll
            for (int n = 0; n < SeqRows<T, D>::kInstr; ++n) {
                const int r = min(w0 + n * SeqRows<T, D>::kRpi + rows.rowl, last_key);
                const uint32_t off = rows.off(n, 0u);
                seq_load(krow + r * g.kt + off, own + n * 1024);
                seq_load(vrow + r * g.vt + off, own + C::kRows + n * 1024);
            }
        }
    }
    {
        const int from = min(key, last_key);
        st.init(krow + from * g.kt, vrow + from * g.vt, h);
    }

    if (first_role) {
        // rows W or more behind the key: tiles of every head in turn, this chunk's share of
        // them, one wave a tile
        const int t0 = (int)min(((int64_t)k0 + g.W) >> 5, (int64_t)1 << 26);
        const int nt = max(0, ((valid - 1) >> 5) - t0 + 1);
        const int all = nt * g.G, per = (all + b.chunks - 1) / b.chunks;
        const int end = min(all, (part + 1) * per);
        using Ld = KvStage<T, D, 1>;
        unsigned char* buf = smem + wave * C::kBytes;
        const int len = key < g.S && valid - key > g.W ? valid - key - g.W : 0;
        st.settle_keys();
        stage_barrier();
        for (int e = part * per + wave; e < end; e += C::kFirst) {
            const int hd = e / nt, i0 = (t0 + e - hd * nt) * 32;
            Ld::issue(b, qs + hd * g.qh, gs + hd * b.gh, b.lse2 + stat + hd * g.lh,
                      b.delta + stat + hd * g.lh, i0, valid, 0, lane, buf);
            wait_vmem();
            const bool full = i0 - (k0 + 31) >= g.W && i0 + 32 <= valid && k0 + 31 < g.S;
            st.tile(f, buf, own, lane, g.c, full, i0 + 4 * h - key - g.W, len);
            wait_lds();
        }
        st.finish();
#pragma unroll
        for (int half = C::kFirst / 2; half >= 1; half /= 2) st.add_waves(smem, wave, half, lane);
        if (wave == 0) {
            const int64_t row = ((int64_t)part * g.B * g.Hkv + slice) * (b.blocks * 32) + key;
            store_part<D, OUT>(st, b.first_part + row * 2 * D, h, b.scale);
        }
        return;
    }

    // ---- rows whose window holds the tile's keys, head by head ----
    const int h0 = (int)((int64_t)g.G * part / b.hsplit);
    const int h1 = (int)((int64_t)g.G * (part + 1) / b.hsplit);
    const int klast = min(k0 + 127, valid - 1);
    const int64_t reach = (int64_t)klast + g.W - 1;
    const int last = (int)min((int64_t)valid - 1, reach);
    const int nt = k0 < valid ? (last >> 5) - (k0 >> 5) + 1 : 0;
    const int all = nt * (h1 - h0);
    const int group = RS == 1 ? 0 : wave >> 2;
    using Ld = KvStage<T, D, 4>;
    // this group's tiles: group, group + RS, .. of the list; the tile to stage and the one to use
    struct Iter {
        int e, hd, i;
    } in, at;
    in.e = group;
    in.hd = h0;
    in.i = group;
    auto wrap = [&](Iter& x) __attribute__((always_inline)) {
        while (x.i >= nt && x.e < all) {
            x.i -= nt;
            ++x.hd;
        }
    };
    wrap(in);
    at = in;
    auto next = [&](Iter& x) __attribute__((always_inline)) {
        x.e += RS;
        x.i += RS;
        wrap(x);
    };
    unsigned char* mine = smem + group * C::kPer * C::kBytes;
    constexpr int kStage = RS * C::kPer * C::kBytes;
    auto issue_stage = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C::kPer; ++i)
            if (in.e < all) {
                Ld::issue(b, qs + in.hd * g.qh, gs + in.hd * b.gh, b.lse2 + stat + in.hd * g.lh,
                         b.delta + stat + in.hd * g.lh, k0 + in.i * 32, valid, wave & 3, lane,
                         mine + buf * kStage + i * C::kBytes);
                next(in);
            }
    };
    issue_stage(0);
    const int len = valid > key ? min(g.W, valid - key) : 0;
    st.settle_keys();
    stage_barrier();
    constexpr int kStep = RS * C::kPer;
    for (int e = 0, buf = 0; e < all; e += kStep, buf ^= 1) {
        if (e + kStep < all) issue_stage(buf ^ 1);
#pragma unroll
        for (int i = 0; i < C::kPer; ++i) {
            if (at.e < all) {
                const int i0 = k0 + at.i * 32;
                next(at);
                // some row sees some key of the wave; all see all
                const bool some = i0 + 31 >= w0 && i0 - (w0 + 31) < g.W && w0 < valid;
                const bool full = i0 >= w0 + 31 && i0 + 31 - w0 < g.W && i0 + 32 <= valid;
                if (some)
                    st.tile(f, mine + buf * kStage + i * C::kBytes, own, lane, g.c, full,
                            i0 + 4 * h - key, len);
            }
        }
        if (e + kStep < all) stage_barrier();
    }
    st.finish();
    if constexpr (RS == 2) {
        st.add_waves(smem, wave, 4, lane);
        if (wave >= 4) return;
    }

    if (key >= g.n) return;
    if (b.hsplit > 1 || w0 < b.blocks * 32) {
        // (with one part only the first tokens' blocks have parts)
        const int keys = b.hsplit > 1 ? g.n : b.blocks * 32;
        const int64_t row = ((int64_t)part * g.B * g.Hkv + slice) * keys + key;
        store_part<D, OUT>(st, b.part + row * 2 * D, h, b.scale);
        return;
    }
    T* dk = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(dkg) + sb * b.kb + kvh * b.kh +
                                 (int64_t)key * b.kt);
    T* dv = reinterpret_cast<T*>(reinterpret_cast<unsigned char*>(dvg) + sb * b.vb + kvh * b.vh +
                                 (int64_t)key * b.vt);
    if constexpr (OUT & kDk)
        each_four<D>(st.dk, h, b.scale, [&](int d, f32x4 x) { st_x4<T>(dk + d, x); });
    if constexpr (OUT & kDv)
        each_four<D>(st.dv, h, 1.f, [&](int d, f32x4 x) { st_x4<T>(dv + d, x); });
}

// Sums the parts of each key (heads, then first tokens' chunks) and rounds once: four lanes per
// four columns of dk or dv, each with every fourth part, so that the loads of tens of parts are
// in flight together; a fixed order.  6 to 7 us.
template <typename T, int D>
__global__ __launch_bounds__(256) void seq_dkv_join_kernel(SeqBwd b, int first_parts,
                                                           T* __restrict__ dkg,
                                                           T* __restrict__ dvg) {
    const SeqGeo& g = b.g;
    const int keys = b.hsplit > 1 ? g.n : min(g.n, b.blocks * 32);
    const int stride = b.hsplit > 1 ? g.n : b.blocks * 32;  // keys of a slice's parts
    constexpr int kPer = 2 * D / 4;
    const int64_t slices = (int64_t)g.B * g.Hkv, total = slices * keys * kPer;
    const int q = threadIdx.x & 3;
    // (whole quads of lanes leave the loop together)
    for (int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 2; x < total;
         x += (int64_t)gridDim.x * 64) {
        const int64_t row = x / kPer;
        const int d = (int)(x % kPer) * 4;
        const int slice = (int)(row / keys), key = (int)(row % keys);
        f32x4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = q; p < b.hsplit; p += 4)
            sum += ld16<f32x4>(b.part + ((p * slices + slice) * stride + key) * 2 * D + d);
        if (key < b.blocks * 32)
#pragma unroll 8
            for (int p = q; p < first_parts; p += 4)
                sum += ld16<f32x4>(b.first_part +
                                   ((p * slices + slice) * (b.blocks * 32) + key) * 2 * D + d);
#pragma unroll
        for (int m = 1; m <= 2; m *= 2)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] += __shfl_xor(sum[r], m, kWave);
        if (q != 0) continue;
        const int sb = g.fd_kv.div(slice), kvh = slice - sb * g.Hkv;
        unsigned char* to =
            d < D ? reinterpret_cast<unsigned char*>(dkg) + sb * b.kb + kvh * b.kh + key * b.kt
                  : reinterpret_cast<unsigned char*>(dvg) + sb * b.vb + kvh * b.vh + key * b.vt;
        st_x4<T>(reinterpret_cast<T*>(to) + (d < D ? d : d - D), sum);
    }
}

// ---- host ----
template <typename T, int D>
static hipError_t launch_bwd(const SeqBwd& b, const T* q, const T* k, const T* v, const T* out,
                             const float* lse, const T* dout, T* dq, T* dk, T* dv, hipStream_t s) {
    const SeqGeo& g = b.g;
    const unsigned slices = (unsigned)g.B * g.Hkv;
    hipError_t e;
    constexpr size_t qlds = 3 * 2 * SeqFrags<T, D>::kTile;
    auto kq = seq_dq_kernel<T, D>;
    if ((e = seq_allow_lds(kq, qlds)) != hipSuccess) return e;
    hipLaunchKernelGGL(kq, dim3(slices * g.ntiles), dim3(256), qlds, s, b, q, k, v, out, lse, dout,
                       dq);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const unsigned jobs = slices * b.ktiles * b.hsplit;
    auto launch_dkv = [&](auto kern, int lds, int threads) {
        hipError_t r = seq_allow_lds(kern, lds);
        if (r != hipSuccess) return r;
        hipLaunchKernelGGL(kern, dim3(b.first_jobs + jobs), dim3(threads), lds, s, b, q, k, v, dout,
                           dk, dv);
        return hipGetLastError();
    };
    if constexpr (sizeof(T) == 4 && D == 128) {
        e = launch_dkv(seq_dkv_kernel<T, D, kDk, 1>, KvCfg<T, D, 1>::kLds, 256);
        if (e == hipSuccess) e = launch_dkv(seq_dkv_kernel<T, D, kDv, 1>, KvCfg<T, D, 1>::kLds, 256);
    } else if constexpr (sizeof(T) == 4) {
        e = launch_dkv(seq_dkv_kernel<T, D, kDk | kDv, 1>, KvCfg<T, D, 1>::kLds, 256);
    } else if (D == 128 || jobs < 512) {
        // (D = 128: one workgroup of eight waves a CU either way, by registers and LDS; below,
        // fewer than two workgroups a CU)
        e = launch_dkv(seq_dkv_kernel<T, D, kDk | kDv, 2>, KvCfg<T, D, 2>::kLds, 512);
    } else if constexpr (D < 128) {
        e = launch_dkv(seq_dkv_kernel<T, D, kDk | kDv, 1>, KvCfg<T, D, 1>::kLds, 256);
    }
    if (e != hipSuccess || (b.hsplit == 1 && b.blocks == 0)) return e;
    const int64_t units = (int64_t)slices * (b.hsplit > 1 ? g.n : b.blocks * 32) * (D / 2);
    const unsigned grid = (unsigned)std::min<int64_t>((units + 63) / 64, 1 << 16);
    hipLaunchKernelGGL((seq_dkv_join_kernel<T, D>), dim3(grid), dim3(256), 0, s, b,
                       b.chunks, dk, dv);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_bwd_d(const SeqBwd& b, int D, const void* q, const void* k, const void* v,
                               const void* out, const float* lse, const void* dout, void* dq,
                               void* dk, void* dv, hipStream_t s) {
    auto c = [](const void* p) { return static_cast<const T*>(p); };
    auto m = [](void* p) { return static_cast<T*>(p); };
    switch (D) {
        case 32: return launch_bwd<T, 32>(b, c(q), c(k), c(v), c(out), lse, c(dout), m(dq), m(dk), m(dv), s);
        case 64: return launch_bwd<T, 64>(b, c(q), c(k), c(v), c(out), lse, c(dout), m(dq), m(dk), m(dv), s);
        case 128: return launch_bwd<T, 128>(b, c(q), c(k), c(v), c(out), lse, c(dout), m(dq), m(dk), m(dv), s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_seq_backward(const SeqBwd& b, int D, int dtype, const void* q, const void* k,
                               const void* v, const void* out, const float* lse, const void* dout,
                               void* dq, void* dk, void* dv, hipStream_t s) {
    switch (dtype) {
        case 0: return launch_bwd_d<float>(b, D, q, k, v, out, lse, dout, dq, dk, dv, s);
        case 1: return launch_bwd_d<_Float16>(b, D, q, k, v, out, lse, dout, dq, dk, dv, s);
        case 2: return launch_bwd_d<__bf16>(b, D, q, k, v, out, lse, dout, dq, dk, dv, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace na
