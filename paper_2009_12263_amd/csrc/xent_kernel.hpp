// The products of the linear cross entropy (xent.hip): the matrix kernels of gemm_kernel.hpp with what becomes of a tile of
// results written here (TileCfg::OWN_STORE).  Rows are tokens (or words, XENT_ROUND), columns are words (values): a lane holds a row's results in
// runs of RUN consecutive columns, so the sums over a row are formed in the lane and one exchange with the other half of the
// wave, and 16-bit results leave in pieces of 16 bytes (32x32x16 instructions: 8).
//   XENT_STATS  a tile of logits becomes, for each of its rows and each wave's columns, their maximum and the sum of exponentials
//               relative to it, and the logit of the row's target if it is there.  Nothing else is stored.
//   XENT_DZ     a tile of logits becomes dz (16 bits).
//   XENT_ROUND  a tile of dw: multiplied by a factor in memory and rounded to 16 bits.
// Beside a K loop these epilogues are small: per 128x128 results of a wave 256 exponentials per lane, 1.6 % of the time of the matrix
// instructions at K = 4096.  Written as separate passes over logits in memory they cost 8 bytes per logit.
#pragma once
#include "kernel_table.hpp"
#include "row_ops.hpp"

namespace fg {

struct XentStat { float m, s; };            // maximum, and sum of exp(z - m)

constexpr float kLog2e = 1.44269504088896340736f;
// What exponentials are relative to where the maximum is none (no logit, or none above minus infinity).
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }

struct XentParams : GemmParams {            // alpha: the scale of the logits; D, ldd: dz or dw, rows contiguous
    XentStat *stats;                        // XENT_STATS: [run of columns][stats_stride rows]
    float *z_target;
    const void *targets;                    // of the rows
    const float *lse, *dloss, *factor;
    int64_t stats_stride;
    int32_t wide, vocab, v0, dloss_inc;     // targets are 64-bit; words there are; the word of column 0
};

enum XentKind { XENT_STATS = 0, XENT_DZ = 1, XENT_ROUND = 2 };

// x with the other half of the wave's
template <class Op>
__device__ __forceinline__ float with_other_half(float x, Op op) {
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned s0 = s[0], s1 = s[1];
    return op(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
}

template <class Base, int KIND>
struct XentCfg : Base {
    static constexpr bool OWN_STORE = true;
    using Params = XentParams;
    using T = typename std::conditional<Base::BF16, bf16_t, f16_t>::type;
    static constexpr int RUN = Base::ACC_LH;                            // consecutive columns of a lane: the other half of the wave has the next ones
    static constexpr int RUNS = 16 / RUN;                               // in a block; they begin 2 RUN columns apart
    static_assert(Base::acc_col(RUN) == 2 * RUN && Base::acc_col(RUN - 1) == RUN - 1, "");

    template <class Blocks>
    __device__ static __forceinline__ void store(const Params &p, const Blocks &blocks, int m_base, int n_base, int lane) {
        if constexpr (Base::WIDE) own_acc();
        const int lm = lane & 31, lh = lane >> 5;
        const int n_first = n_base + RUN * lh;                          // the lane's first column
        const bool edge = n_base + Base::WTN > p.N;
        static_for<Base::TI>([&](auto i) {
            const int row = m_base + 32 * (int)decltype(i)::value + lm;
            const bool there = row < p.M;
            if constexpr (KIND == XENT_STATS) {
                float z[Base::TJ][16], m = -__builtin_inff(), s = 0.f;
                static_for<Base::TJ>([&](auto j) {
                    const floatx16 a = blocks(i, j);
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[j][r] = a[r] * p.alpha;
                });
                if (edge) {
#pragma unroll
                    for (int j = 0; j < Base::TJ; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (n_first + 32 * j + Base::acc_col(r) >= p.N) z[j][r] = -__builtin_inff();
                }
#pragma unroll
                for (int j = 0; j < Base::TJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) m = __builtin_fmaxf(m, z[j][r]);
                m = with_other_half(m, [](float x, float y) { return __builtin_fmaxf(x, y); });
                const float base = base_of(m) * kLog2e;
#pragma unroll
                for (int j = 0; j < Base::TJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][r], kLog2e, -base));
                s = with_other_half(s, [](float x, float y) { return x + y; });
                if (there && lh == 0) p.stats[(int64_t)(n_base / Base::WTN) * p.stats_stride + row] = {m, s};
                const int target = there ? load_index(p.targets, p.wide, row, p.vocab) - p.v0 : -1, at = target - n_first;
                if (__ballot(target >= n_base && target < n_base + Base::WTN)) {
                    float hit = 0.f;
                    bool is = false;
#pragma unroll
                    for (int j = 0; j < Base::TJ; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const bool same = at == 32 * j + Base::acc_col(r);
                            hit = same ? z[j][r] : hit;
                            is |= same;
                        }
                    if (is && target >= 0) p.z_target[row] = hit;
                }
            } else {
                float factor = 0.f, lse2 = 0.f;
                int at = -1;
                bool live = there, hits = false;
                if constexpr (KIND == XENT_DZ) {
                    const int target = there ? load_index(p.targets, p.wide, row, p.vocab) : -1;
                    live = target >= 0;
                    if (live) {
                        factor = p.dloss[(int64_t)row * p.dloss_inc] * p.factor[0];
                        lse2 = p.lse[row] * kLog2e;
                    }
                    const int col = target - p.v0;
                    at = live ? col - n_first : -1;
                    hits = __ballot(live && col >= n_base && col < n_base + Base::WTN) != 0;
                } else {
                    factor = p.factor[1];
                }
                T *out = (T *)p.D + (int64_t)row * p.ldd + n_first;
                const float zs = p.alpha * kLog2e;
                static_for<Base::TJ>([&](auto j) {
                    const floatx16 a = blocks(i, j);
#pragma unroll
                    for (int h = 0; h < RUNS; ++h) {
                        const int c0 = 32 * (int)decltype(j)::value + 2 * RUN * h;         // (from n_first)
                        typename RowPiece<T, RUN>::vec v;
#pragma unroll
                        for (int e = 0; e < RUN; ++e) {
                            float d = a[RUN * h + e];
                            if constexpr (KIND == XENT_DZ) {
                                d = __builtin_amdgcn_exp2f(__builtin_fmaf(d, zs, -lse2));
                                if (hits) d -= at == c0 + e ? 1.f : 0.f;
                                d = live && !(edge && n_first + c0 + e >= p.N) ? d * factor : 0.f;
                            } else {
                                d *= factor;
                            }
                            v[e] = (T)d;
                        }
                        // rows of dz are as long as ldd, with zeros behind the last word; columns of dw are whole runs
                        const bool inside = !edge || n_first + c0 < (KIND == XENT_DZ ? (int)p.ldd : p.N);
                        if (there && inside) *(typename RowPiece<T, RUN>::unaligned *)(out + c0) = v;
                    }
                });
            }
            if constexpr (Base::WIDE) {
                __builtin_amdgcn_sched_barrier(0);
                own_acc();
            }
        });
    }
};

// The five tiles a plan can name: 256x256, 256x128, 128x128 with four buffers, 64x64 and 64x128 with two groups of waves (kernel_table.hpp).
enum { XENT_TILES = 5 };
const KernelEntry *kernel_table_xent(int kind, bool bf16);

#define FG_XENT_TABLE(FUNC, KIND, AKC, BKC, BF, NAME)                                                                      \
    const KernelEntry *FUNC() {                                                                                            \
        using A = XentCfg<FG_CFG_K32(256, 256, 64, 2, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using B = XentCfg<FG_CFG_K32(256, 128, 64, 3, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using C = XentCfg<FG_CFG_K32(128, 128, 64, 4, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using D = XentCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 64, 4, true), KIND>;                                       \
        using E = XentCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), KIND>;                                      \
        static const KernelEntry t[XENT_TILES] = {                                                                         \
            {(const void *)gemm_kernel<A>, NAME "_256x256x64", 256, 256, A::NTHREADS, A::LDS_BYTES},                       \
            {(const void *)gemm_kernel<B>, NAME "_256x128x64", 256, 128, B::NTHREADS, B::LDS_BYTES},                       \
            {(const void *)gemm_kernel<C>, NAME "_128x128x64_deep", 128, 128, C::NTHREADS, C::LDS_BYTES},                  \
            {(const void *)gemm_kernel<D>, NAME "_64x64x64", 64, 64, D::NTHREADS, D::LDS_BYTES, 2},                        \
            {(const void *)gemm_kernel<E>, NAME "_64x128x64", 64, 128, E::NTHREADS, E::LDS_BYTES, 2},                      \
        };                                                                                                                 \
        return t;                                                                                                          \
    }
// columns of a wave, on each tile: those of one run of XentParams::stats
constexpr int kXentWaveColumns[XENT_TILES] = {128, 64, 64, 32, 64};

}  // namespace fg
