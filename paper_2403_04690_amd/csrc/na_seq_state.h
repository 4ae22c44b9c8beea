// na_seq_state.h -- the running softmax of the sequence kernels' forward passes, and the LDS layouts
// of their two forms (see na_seq_fwd.hip).
#pragma once

#include <type_traits>

#include "na_seq_kernels.h"

namespace na {

constexpr float kSeqLazy = 8.f;  // base-2 headroom before the running maximum is raised

// How far (base 2) below a row's maximum the reference of its scores is put when it is raised.  In
// fp16 the weights then reach up to 2^15, and are in the normal range down to 2^-21 of the largest
// instead of 2^-14: beside a first token that takes most of the weight, thousands of keys have less
// than that, and may be all of the output.  (A first token of score 12 above 65k others, its value
// 0: off by twice the bound of the roundings with 0 here.)
template <typename T>
constexpr float kSeqBelow = std::is_same<T, _Float16>::value ? 7.f : 0.f;

// Running state of 32 rows: lane l holds row l % 32, and of the keys those of its half.
template <typename T, int D>
struct SeqState {
    using F = SeqFrags<T, D>;
    using x8 = typename Tr<T>::x8;
    x8 qf[F::kKS];
    f32x16 o[F::kDB];
    float mref, thr, l;

    __device__ __forceinline__ void init() {
        mref = -INFINITY;
        thr = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < F::kDB; ++db) o[db] = f32x16{} * 0.f;
    }

    // Folds N tiles of 32 keys into the state: K and V of tile n at tile[n] and tile[n] + kTile,
    // from position j0[n].  Unless `full` (uniform), some pair is not seen, and of a tile that
    // is not `on` none; seen(base): bit e says whether this lane's row sees key base + e, of the
    // keys base + entry_row(i).
    //   With two tiles the matrix cores and the vector unit can work side by side within a wave:
    // the second tile's scores beside the scaling of the first's, the first's values beside
    // the second's exponentials.  (Asking for that order instruction by instruction, with
    // scheduling groups, was 1 to 8 % slower than leaving it to the compiler.)
    //   (One body with a branch around the mask alone: two bodies that meet again in the
    // accumulators cost registers.)
    //   The weights are rounded to the values' type for the matrix cores, once; their sum takes them as
    // they are.  Each is off by half a step at most, on its own, so out moves by at most that times sum
    // p |v|: as much as its own rounding in the mean of independent keys (bf16 errors of 2.3e-3
    // instead of 1.7e-3 of the result).  In two halves they would take half as many products again.
    //   after_k and after_v run when this wave has read the tiles' keys and their values, before_v
    // in front of the values' reads.
    struct Nothing {
        __device__ __forceinline__ void operator()() const {}
    };
    template <int N, typename Seen, typename AfterK = Nothing, typename BeforeV = Nothing,
              typename AfterV = Nothing>
    __device__ __forceinline__ void fold(const F& f, const unsigned char* (&tile)[N],
                                         int lane, float c, bool full, const int (&j0)[N],
                                         const bool (&on)[N], Seen seen, AfterK after_k = {},
                                         BeforeV before_v = {}, AfterV after_v = {}) {
        f32x16 s[N];
        x8 kf[N][F::kKS];
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int st = 0; st < F::kKS; ++st) kf[n][st] = f.row(tile[n], st);
        }
        after_k();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n] = f32x16{} * 0.f;
#pragma unroll
            for (int st = 0; st < F::kKS; ++st) s[n] = mma32<T>(kf[n][st], qf[st], s[n]);
        }
        const float negm = mref == -INFINITY ? 0.f : -mref;
        float y[N][16];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) y[n][i] = fmaf(s[n][i], c, negm);
        if (!full) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int base = j0[n] + 4 * (lane >> 5);  // entry i is key base + entry_row(i)
                const unsigned m = on[n] ? seen(base) : 0u;
#pragma unroll
                for (int i = 0; i < 16; ++i) y[n][i] = keep(m, i, y[n][i], -INFINITY);
            }
        }
        float top = y[0][0];
#pragma unroll
        for (int i = 1; i < 16 * N; ++i) top = fmaxf(top, y[i >> 4][i & 15]);
        // raise the reference on a row's first key, or when it grows by more than kSeqLazy
        if (__builtin_amdgcn_ballot_w64(top > thr)) {
            const float ymax = col_max<32>(top);
            const bool raise = ymax > thr;
            const float up = raise ? ymax - kSeqBelow<T> : 0.f;
            const float alpha = thr == -INFINITY ? 0.f : fast_exp2(-up);
            mref = raise ? up - negm : mref;
            thr = mref != -INFINITY ? kSeqLazy + kSeqBelow<T> : -INFINITY;
            l *= alpha;
#pragma unroll
            for (int db = 0; db < F::kDB; ++db) o[db] *= alpha;
#pragma unroll
            for (int i = 0; i < 16 * N; ++i) y[i >> 4][i & 15] -= up;
        }
        x8 vf[N][2][F::kDB], pf[N][2];
        float sum[2];
        before_v();
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int bi = 0; bi < 2; ++bi)
#pragma unroll
                for (int db = 0; db < F::kDB; ++db)
                    vf[n][bi][db] = f.col(tile[n] + F::kTile, db, bi, lane);
        after_v();
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = fast_exp2(y[n][i]);
                sum[i & 1] = n == 0 && i < 2 ? p : sum[i & 1] + p;
                pf[n][i >> 3][i & 7] = Tr<T>::cvt(p);
            }
#pragma unroll
            for (int bi = 0; bi < 2; ++bi)
#pragma unroll
                for (int db = 0; db < F::kDB; ++db)
                    o[db] = mma32<T>(vf[n][bi][db], pf[n][bi], o[db]);
        }
        l += sum[0] + sum[1];
    }
};

// The wide form's ring of stages: tiles per stage, and stages (one read, the others in flight).
// At D = 128 registers allow two waves a SIMD, too few to hide one wave's exponentials behind
// another's products, so a stage has two tiles whose steps can overlap (16-bit types); below,
// four waves do that and three single stages take less LDS.
template <typename T, int D>
struct SeqRing {
    static constexpr int kTiles = D == 128 && sizeof(T) == 2 ? 2 : 1;
    static constexpr int kStages = kTiles == 2 ? 2 : 3;
    static constexpr int kStage = kTiles * 2 * SeqFrags<T, D>::kTile;
    static constexpr int kLds = kStages * kStage;
};

// Waves of the narrow form: the buffers of each (two key tiles) fit four to a CU's LDS, fp32
// at D = 128 two.
template <typename T, int D>
constexpr int seq_narrow_waves() {
    return sizeof(T) == 4 && D == 128 ? 2 : 4;
}

template <typename T, int D>
struct SeqNarrow {
    static constexpr int W = seq_narrow_waves<T, D>();
    static constexpr int kTile = SeqFrags<T, D>::kTile;
    static constexpr int kStages = W * 4 * kTile;
    static constexpr int kRow = (D + 4) * 4;           // a joined row (padded: LDS banks)
    static constexpr int kJoin = W * 32 * kRow;
    static constexpr int kStat = kStages > kJoin ? kStages : kJoin;  // offset of the statistics
    static constexpr int kLds = kStat + W * 32 * 8;
};

}  // namespace na
