// The products of the gated feed-forward block (gated.hip): the matrix kernels of gemm_kernel.hpp with what becomes of a tile of results written
// here (TileCfg::OWN_STORE).  Rows are tokens (or the rows of a weight, GATED_ROUND); a lane holds a row's results in runs of RUN
// consecutive columns, so that 16-bit results leave in pieces of 16 bytes (32x32x16 instructions: 8).
//   GATED_UP     X W_in^T.  Blocks of 32 columns are rows of G and of U in turn (TileCfg::PAIRED), so a lane holds g and u of the same columns: h = act(g) u in
//                16 bits is stored, and g and u in FP32 if they are wanted.
//   GATED_DOWN   dY W_out = dh.  With g and u from memory: dg, du and h in 16 bits.
//   GATED_ROUND  results rounded to 16 bits.
#pragma once
#include "kernel_table.hpp"
#include "row_ops.hpp"

namespace fg {

// act(g) = g q(g) with q = 1 / (1 + exp(-g (k0 + k1 g^2))): silu has k0 = 1, k1 = 0; in gelu (1 + tanh v) / 2 = 1 / (1 + exp(-2 v)).  relu and none have q of 0 or 1.
// One code for all: four copies of an epilogue would leave the instruction cache.
struct Activation {
    float k0, k1;
    int32_t relu, none;
    __host__ __device__ static Activation of(int act) {
        const float c = 2.f * 0.79788456080286535588f;                  // 2 sqrt(2 / pi)
        return {act == FG_ACT_GELU_TANH ? c : 1.f, act == FG_ACT_GELU_TANH ? 0.044715f * c : 0.f, act == FG_ACT_RELU, act == FG_ACT_NONE};
    }
    // act(g), and its derivative q + g q (1 - q) (k0 + 3 k1 g^2).  (Beyond 1000 q is 0 or 1: the bound keeps g^2 a number.)
    template <bool D>
    __device__ __forceinline__ float operator()(float g, float *d) const {
        const float x = __builtin_amdgcn_fmed3f(g, -1000.f, 1000.f), x2 = x * x, slope = __builtin_fmaf(k1, x2, k0);
        float q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * (x * slope)));
        q = relu ? (g > 0.f ? 1.f : 0.f) : none ? 1.f : q;
        if constexpr (D) *d = __builtin_fmaf(x * q * (1.f - q), __builtin_fmaf(3.f * k1, x2, k0), q);
        return relu ? (g > 0.f ? g : 0.f) : g * q;
    }
};

struct GatedParams : GemmParams {           // D, ldd: h, dgu or the rounded results, rows contiguous
    float *keep;                            // GATED_UP: g and u, rows of 2 hidden, or null
    const float *gu;                        // GATED_DOWN
    int64_t ldgu;                           // of both
    void *h;                                // GATED_DOWN
    int64_t ldh;
    // GATED_UP: block b of 32 columns of G is rows 32 b .. of W_in and its U `pair` rows on, b pair_step / 32 rows further for each b
    int64_t pair, pair_step;
    int32_t hidden;
    Activation act;
};

enum GatedKind { GATED_UP = 0, GATED_DOWN = 1, GATED_ROUND_KK = 2, GATED_ROUND_KN = 3, GATED_ROUND_NN = 4 };       // (round: A, B contiguous along K or not)

template <class Base, int KIND>
struct GatedCfg : Base {
    static constexpr bool OWN_STORE = true, PAIRED = KIND == GATED_UP;
    using Params = GatedParams;
    using T = typename std::conditional<Base::BF16, bf16_t, f16_t>::type;
    static constexpr int RUN = Base::ACC_LH, RUNS = 16 / RUN;           // consecutive columns of a lane; such runs in a block, 2 RUN columns apart
    static_assert(Base::acc_col(RUN) == 2 * RUN && Base::acc_col(RUN - 1) == RUN - 1, "");
    static_assert(!PAIRED || Base::TJ % 2 == 0, "a wave has blocks of G and U");
    typedef float floats __attribute__((ext_vector_type(RUN)));
    typedef float four __attribute__((ext_vector_type(4)));
    typedef four four_anywhere __attribute__((aligned(4)));
    using Vec = typename RowPiece<T, RUN>::vec;
    typedef __attribute__((address_space(1))) typename RowPiece<T, RUN>::unaligned *Global;
    typedef __attribute__((address_space(1))) four_anywhere *GlobalFloats;
    typedef const __attribute__((address_space(1))) four_anywhere *ConstFloats;

    template <class Blocks>
    __device__ static __forceinline__ void store(const Params &p, const Blocks &blocks, int m_base, int n_base, int lane) {
        if constexpr (Base::WIDE) own_acc();
        if constexpr (KIND == GATED_UP) up(p, blocks, m_base + lane % 32, n_base / 2 + RUN * (lane >> 5), n_base / 2 + Base::WTN / 2 > p.hidden);
        else if constexpr (KIND == GATED_DOWN) down(p, blocks, m_base + lane % 32, n_base + RUN * (lane >> 5), n_base + Base::WTN > p.hidden);
        else round(p, blocks, m_base + lane % 32, n_base + RUN * (lane >> 5), n_base + Base::WTN > p.N);
    }
    __device__ static __forceinline__ void step() {
        if constexpr (Base::WIDE) {
            __builtin_amdgcn_sched_barrier(0);
            own_acc();
        }
    }
    // the run's columns that are there, `left` of them; whole runs in one piece
    __device__ static __forceinline__ void put(T *to, floats v, int left) {
        const Vec r = __builtin_convertvector(v, Vec);
        if (left >= RUN) *(Global)to = r;
        else {
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                if (e < left) to[e] = r[e];
        }
    }
    __device__ static __forceinline__ void put(float *to, floats v, int left) {
        if (left >= RUN) {
#pragma unroll
            for (int q = 0; q < RUN / 4; ++q) *((GlobalFloats)to + q) = four{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        } else {
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                if (e < left) to[e] = v[e];
        }
    }

    // first: the lane's first column of h; the blocks of G and U lie side by side
    template <class Blocks>
    __device__ static __forceinline__ void up(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        const Activation act = p.act;
        static_for<Base::TI>([&](auto i) {
            const int row = row0 + 32 * (int)decltype(i)::value;
            T *h = (T *)p.D + (int64_t)row * p.ldd + first;
            float *g_out = p.keep + (int64_t)row * p.ldgu + first, *u_out = g_out + p.hidden;
            static_for<Base::TJ / 2>([&](auto jj) {
                constexpr int J = decltype(jj)::value;
                const floatx16 g = blocks(i, ic<2 * J>{}), u = blocks(i, ic<2 * J + 1>{});
#pragma unroll
                for (int r = 0; r < RUNS; ++r) {
                    const int c = 32 * J + 2 * RUN * r;
                    floats gv, uv, v;
#pragma unroll
                    for (int e = 0; e < RUN; ++e) {
                        gv[e] = g[RUN * r + e];
                        uv[e] = u[RUN * r + e];
                        v[e] = act.template operator()<false>(gv[e], nullptr) * uv[e];
                    }
                    if (row < p.M) {
                        if (!edge) {
                            put(h + c, v, RUN);
                            if (p.keep) {
                                put(g_out + c, gv, RUN);
                                put(u_out + c, uv, RUN);
                            }
                        } else {
                            // zeros behind the last column, to the end of h's row
                            const int left = p.hidden - first - c;
#pragma unroll
                            for (int e = 0; e < RUN; ++e) v[e] = e < left ? v[e] : 0.f;
                            if (first + c < p.ldd) put(h + c, v, RUN);
                            if (p.keep) {
                                put(g_out + c, gv, left);
                                put(u_out + c, uv, left);
                            }
                        }
                    }
                }
                step();
            });
        });
    }

    // What a lane needs from memory for a block: g and u of its columns.  Blocks are requested AHEAD of their turn: a lone wave waits for each otherwise.
    static constexpr int AHEAD = Base::WIDE && Base::TI * Base::TJ >= 4 ? 3 : 1;
    struct Pair { floats g[RUNS], u[RUNS]; };
    __device__ static __forceinline__ void fetch(const Params &p, const float *gu, int first, int j, bool edge, Pair &out) {
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            const int c = 32 * j + 2 * RUN * r, left = p.hidden - first - c;
            const float *g = gu + c, *u = g + p.hidden;
            if (!edge || left >= RUN) {
#pragma unroll
                for (int q = 0; q < RUN / 4; ++q) {
                    const four a = *((ConstFloats)g + q), b = *((ConstFloats)u + q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { out.g[r][4 * q + e] = a[e]; out.u[r][4 * q + e] = b[e]; }
                }
            } else {
#pragma unroll
                for (int e = 0; e < RUN; ++e) { out.g[r][e] = e < left ? g[e] : 0.f; out.u[r][e] = e < left ? u[e] : 0.f; }
            }
        }
    }
    template <class Blocks>
    __device__ static __forceinline__ void down(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        const Activation act = p.act;
        constexpr int COUNT = Base::TI * Base::TJ;
        Pair ahead[AHEAD];
        auto gu_of = [&](int i) { const int row = row0 + 32 * i; return p.gu + (int64_t)(row < p.M ? row : p.M - 1) * p.ldgu + first; };
        static_for<(AHEAD < COUNT ? AHEAD : COUNT)>([&](auto b) { fetch(p, gu_of(decltype(b)::value / Base::TJ), first, decltype(b)::value % Base::TJ, edge, ahead[decltype(b)::value]); });
        static_for<COUNT>([&](auto b) {
            constexpr int B = decltype(b)::value, I = B / Base::TJ, J = B % Base::TJ;
            const int row = row0 + 32 * I;
            const floatx16 dh = blocks(ic<I>{}, ic<J>{});
            const Pair in = ahead[B % AHEAD];
            T *dg = (T *)p.D + (int64_t)row * p.ldd + first, *du = dg + p.hidden, *h = (T *)p.h + (int64_t)row * p.ldh + first;
#pragma unroll
            for (int r = 0; r < RUNS; ++r) {
                const int c = 32 * J + 2 * RUN * r;
                floats vg, vu, vh;
#pragma unroll
                for (int e = 0; e < RUN; ++e) {
                    const float x = dh[RUN * r + e];
                    float d;
                    const float a = act.template operator()<true>(in.g[r][e], &d);
                    vg[e] = x * in.u[r][e] * d;
                    vu[e] = x * a;
                    vh[e] = a * in.u[r][e];
                }
                if (row < p.M) {
                    if (!edge) {
                        put(dg + c, vg, RUN);
                        put(du + c, vu, RUN);
                        put(h + c, vh, RUN);
                    } else {
                        const int left = p.hidden - first - c;
#pragma unroll
                        for (int e = 0; e < RUN; ++e) vh[e] = e < left ? vh[e] : 0.f;
                        put(dg + c, vg, left);
                        put(du + c, vu, left);
                        if (first + c < p.ldh) put(h + c, vh, RUN);
                        // the run with the last column: zeros behind du, to the end of its row
                        if (left > 0 && left <= RUN)
                            for (int z = 2 * p.hidden; z < (int)p.ldd; ++z) ((T *)p.D)[(int64_t)row * p.ldd + z] = (T)0.f;
                    }
                }
            }
            if constexpr (B + AHEAD < COUNT) fetch(p, gu_of((B + AHEAD) / Base::TJ), first, (B + AHEAD) % Base::TJ, edge, ahead[B % AHEAD]);
            step();
        });
    }

    template <class Blocks>
    __device__ static __forceinline__ void round(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        static_for<Base::TI>([&](auto i) {
            const int row = row0 + 32 * (int)decltype(i)::value;
            T *out = (T *)p.D + (int64_t)row * p.ldd + first;
            static_for<Base::TJ>([&](auto j) {
                const floatx16 a = blocks(i, j);
#pragma unroll
                for (int r = 0; r < RUNS; ++r) {
                    const int c = 32 * (int)decltype(j)::value + 2 * RUN * r;
                    floats v;
#pragma unroll
                    for (int e = 0; e < RUN; ++e) v[e] = a[RUN * r + e];
                    if (row < p.M) put(out + c, v, edge ? p.N - first - c : RUN);
                }
            });
            step();
        });
    }
};

// The tiles of a plan: 256x256, 256x128, 128x128 with four buffers, 64x64 and 64x128 with two groups of waves.  On the 64x64 tile a wave has one block
// of columns, not one of G and one of U: GATED_UP has the 64x128 tile in its place.
template <class Cfg> KernelEntry gated_entry(const char *name, int kg = 0) {
    return {(const void *)gemm_kernel<Cfg>, name, Cfg::BM, Cfg::BN, Cfg::NTHREADS, Cfg::LDS_BYTES, kg};
}
template <int KIND, bool AKC, bool BKC, bool BF> const KernelEntry *gated_table(const char *const (&names)[GATED_TILES]) {
    using D = typename std::conditional<KIND == GATED_UP, FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), FG_CFG_KG(AKC, BKC, BF, false, false, 64, 4, true)>::type;
    static const KernelEntry t[GATED_TILES] = {
        gated_entry<GatedCfg<FG_CFG_K32(256, 256, 64, 2, 2, 2, AKC, BKC, BF, false), KIND>>(names[0]),
        gated_entry<GatedCfg<FG_CFG_K32(256, 128, 64, 3, 2, 2, AKC, BKC, BF, false), KIND>>(names[1]),
        gated_entry<GatedCfg<FG_CFG_K32(128, 128, 64, 4, 2, 2, AKC, BKC, BF, false), KIND>>(names[2]),
        gated_entry<GatedCfg<D, KIND>>(names[3], 2),
        gated_entry<GatedCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), KIND>>(names[4], 2),
    };
    return t;
}
#define FG_GATED_TABLE(FUNC, KIND, AKC, BKC, BF, NAME)                                                                                       \
    const KernelEntry *FUNC() {                                                                                                              \
        static const char *const names[GATED_TILES] = {NAME "_256x256x64", NAME "_256x128x64", NAME "_128x128x64_deep",                      \
                                                       (KIND) == GATED_UP ? NAME "_64x128x64" : NAME "_64x64x64", NAME "_64x128x64"};        \
        return gated_table<KIND, AKC, BKC, BF>(names);                                                                                       \
    }

}  // namespace fg
