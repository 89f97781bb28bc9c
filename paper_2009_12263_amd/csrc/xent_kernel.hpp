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
        // What the lane's rows need from memory is requested for all of them at once: a lone wave would wait for each.
        constexpr int COUNT = Base::TI, ROWS = 32;
        int target[COUNT];
        float lse[COUNT], dloss[COUNT];
        if constexpr (KIND != XENT_ROUND) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int row = m_base + ROWS * i + lane % ROWS, at = row < p.M ? row : p.M - 1;
                const int word = load_index(p.targets, p.wide, at, p.vocab);
                target[i] = row < p.M ? word : -1;
                if constexpr (KIND == XENT_DZ) {
                    lse[i] = p.lse[at];
                    dloss[i] = p.dloss[(int64_t)at * p.dloss_inc];
                }
            }
        }
        const int n_first = n_base + RUN * (lane >> 5);                  // the lane's first column
        const bool edge = n_base + Base::WTN > p.N;
        static_for<COUNT>([&](auto i) {
            const int row = m_base + ROWS * (int)decltype(i)::value + lane % ROWS;
            if constexpr (KIND == XENT_STATS) stats_of_rows<decltype(i)::value>(p, blocks, row, target[i], n_base, n_first, edge, lane);
            else if constexpr (KIND == XENT_DZ) dz_of_rows<decltype(i)::value>(p, blocks, row, target[i], lse[i], dloss[i], n_base, n_first, edge);
            else rounded_rows<decltype(i)::value>(p, blocks, row, n_first, edge);
            if constexpr (Base::WIDE) {
                __builtin_amdgcn_sched_barrier(0);
                own_acc();
            }
        });
    }

    template <int I, class Blocks>
    __device__ static __forceinline__ void stats_of_rows(const Params &p, const Blocks &blocks, int row, int word, int n_base, int n_first, bool edge, int lane) {
        constexpr int COUNT = 16 * Base::TJ, CHAINS = 4;                                         // (sums in four chains: a lone wave waits for each addition)
        constexpr auto col = [](int e) { return 32 * (e / 16) + Base::acc_col(e % 16); };
        float z[COUNT], top[CHAINS], sum[CHAINS] = {};
        static_for<Base::TJ>([&](auto j) {
            const floatx16 a = blocks(ic<I>{}, j);
#pragma unroll
            for (int r = 0; r < 16; ++r) z[16 * (int)decltype(j)::value + r] = a[r] * p.alpha;
        });
        if (edge) {
#pragma unroll
            for (int e = 0; e < COUNT; ++e) z[e] = col(e) < p.N - n_first ? z[e] : -__builtin_inff();
        }
#pragma unroll
        for (int e = 0; e < COUNT; ++e) top[e % CHAINS] = e < CHAINS ? z[e] : __builtin_fmaxf(top[e % CHAINS], z[e]);
        const float m = with_other_half(__builtin_fmaxf(__builtin_fmaxf(top[0], top[1]), __builtin_fmaxf(top[2], top[3])), [](float x, float y) { return __builtin_fmaxf(x, y); });
        const float base = base_of(m) * kLog2e;
#pragma unroll
        for (int e = 0; e < COUNT; ++e) sum[e % CHAINS] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[e], kLog2e, -base));
        const float s = with_other_half((sum[0] + sum[1]) + (sum[2] + sum[3]), [](float x, float y) { return x + y; });
        if (row < p.M && lane < 32) p.stats[(int64_t)(n_base / Base::WTN) * p.stats_stride + row] = {m, s};
        const int target = word - p.v0;
        const bool live = word >= 0 && target < p.N;
        if (__ballot(live && target >= n_base && target < n_base + Base::WTN)) {
            const int at = target - n_first;
            float hit = 0.f;
            bool is = false;
#pragma unroll
            for (int e = 0; e < COUNT; ++e) {
                const bool same = at == col(e);
                hit = same ? z[e] : hit;
                is |= same;
            }
            if (is && live) p.z_target[row] = hit;
        }
    }

    // Rows that are left out are zeros whatever their logits are, NaN and infinities too.
    template <int I, class Blocks>
    __device__ static __forceinline__ void dz_of_rows(const Params &p, const Blocks &blocks, int row, int word, float row_lse, float dloss, int n_base, int n_first, bool edge) {
        const bool there = row < p.M, live = word >= 0;
        const int col = word - p.v0;
        const float factor = dloss * p.factor[0], lse = row_lse * kLog2e;
        const float scale = p.alpha * kLog2e;
        const Kept kept = {live ? ~0u : 0u};
        const bool hits = __ballot(live && col >= n_base && col < n_base + Base::WTN) != 0;
        T *out = (T *)p.D + (int64_t)row * p.ldd + n_first;
        if (!edge && !hits) {
            runs<I>(blocks, out, there, [&](float a, int) { return __builtin_amdgcn_exp2f(__builtin_fmaf(a, scale, -lse)) * factor; }, [](int) { return true; }, kept);
        } else {
            // with the target's column, and columns past the last word: zeros, to the end of the row
            const int at = live ? col - n_first : -1, left = p.N - n_first, room = (int)p.ldd - n_first;
            runs<I>(blocks, out, there, [&](float a, int c) {
                const float d = (__builtin_amdgcn_exp2f(__builtin_fmaf(a, scale, -lse)) - (at == c ? 1.f : 0.f)) * factor;
                return c < left ? d : 0.f;
            }, [&](int c) { return c < room; }, kept);
        }
    }

    template <int I, class Blocks>
    __device__ static __forceinline__ void rounded_rows(const Params &p, const Blocks &blocks, int row, int n_first, bool edge) {
        const float factor = p.factor[1];
        const int left = edge ? p.N - n_first : Base::WTN;
        T *out = (T *)p.D + (int64_t)row * p.ldd + n_first;
        runs<I>(blocks, out, row < p.M, [&](float a, int) { return a * factor; }, [&](int c) { return c + RUN <= left; });
        // the row's last columns, if they are no whole run
        if (edge && p.N % RUN != 0 && row < p.M) {
            static_for<Base::TJ>([&](auto j) {
                const floatx16 a = blocks(ic<I>{}, j);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = 32 * (int)decltype(j)::value + Base::acc_col(r), c0 = c - r % RUN;
                    if (c0 < left && c0 + RUN > left && c < left) out[c] = (T)(a[r] * factor);
                }
            });
        }
    }

    // What is stored of a row: all bits or none.  (Two values at a time; chosen value by value, dz of 1960 x 13248 x 280 took 45 us instead of 38.)
    struct Kept { uint32_t bits; };
    struct All {};
    // Stores value(result, column), rounded, where the row is there and the run's first column is `inside`.
    template <int I, class Blocks, class Value, class Inside, class Which = All>
    __device__ static __forceinline__ void runs(const Blocks &blocks, T *out, bool there, Value &&value, Inside &&inside, Which which = {}) {
        typedef uint32_t words __attribute__((ext_vector_type(RUN / 2)));
        typedef float floats __attribute__((ext_vector_type(RUN)));
        using Vec = typename RowPiece<T, RUN>::vec;
        typedef __attribute__((address_space(1))) typename RowPiece<T, RUN>::unaligned *Global;
        static_for<Base::TJ>([&](auto j) {
            const floatx16 a = blocks(ic<I>{}, j);
#pragma unroll
            for (int h = 0; h < RUNS; ++h) {
                const int c0 = 32 * (int)decltype(j)::value + 2 * RUN * h;
                floats v;
#pragma unroll
                for (int e = 0; e < RUN; ++e) v[e] = value(a[RUN * h + e], c0 + e);
                Vec r = __builtin_convertvector(v, Vec);
                if constexpr (std::is_same<Which, Kept>::value) r = __builtin_bit_cast(Vec, __builtin_bit_cast(words, r) & which.bits);
                if (there && inside(c0)) *(Global)(out + c0) = r;
            }
        });
    }
};

// The five tiles a plan can name: 256x256, 256x128, 128x128 with four buffers, 64x64 and 64x128 with two groups of waves (kernel_table.hpp).
enum { XENT_TILES = 5 };
// Columns of a wave on each: those of one run of XentParams::stats, whose space the host counts by them.
constexpr int kXentWaveColumns[XENT_TILES] = {128, 64, 64, 32, 64};
const KernelEntry *kernel_table_xent(int kind, bool bf16);

#define FG_XENT_TABLE(FUNC, KIND, AKC, BKC, BF, NAME)                                                                      \
    const KernelEntry *FUNC() {                                                                                            \
        using A = XentCfg<FG_CFG_K32(256, 256, 64, 2, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using B = XentCfg<FG_CFG_K32(256, 128, 64, 3, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using C = XentCfg<FG_CFG_K32(128, 128, 64, 4, 2, 2, AKC, BKC, BF, false), KIND>;                                   \
        using D = XentCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 64, 4, true), KIND>;                                       \
        using E = XentCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), KIND>;                                      \
        static_assert(A::WTN == kXentWaveColumns[0] && B::WTN == kXentWaveColumns[1] && C::WTN == kXentWaveColumns[2] &&   \
                      D::WTN == kXentWaveColumns[3] && E::WTN == kXentWaveColumns[4], "");                                 \
        static const KernelEntry t[XENT_TILES] = {                                                                         \
            {(const void *)gemm_kernel<A>, NAME "_256x256x64", 256, 256, A::NTHREADS, A::LDS_BYTES},                       \
            {(const void *)gemm_kernel<B>, NAME "_256x128x64", 256, 128, B::NTHREADS, B::LDS_BYTES},                       \
            {(const void *)gemm_kernel<C>, NAME "_128x128x64_deep", 128, 128, C::NTHREADS, C::LDS_BYTES},                  \
            {(const void *)gemm_kernel<D>, NAME "_64x64x64", 64, 64, D::NTHREADS, D::LDS_BYTES, 2},                        \
            {(const void *)gemm_kernel<E>, NAME "_64x128x64", 64, 128, E::NTHREADS, E::LDS_BYTES, 2},                      \
        };                                                                                                                 \
        return t;                                                                                                          \
    }

}  // namespace fg
