// The products of the gated feed-forward block (gated.hip): the matrix kernels of gemm_kernel.hpp with what becomes of a tile of results written
// here (TileCfg::OWN_STORE).  Rows are tokens (or the rows of a weight, GATED_ROUND); 16-bit results leave in pieces of 16 bytes.
//   GATED_UP     X W_in^T.  Blocks of 32 columns are rows of G and of U in turn (TileCfg::PAIRED), so a lane holds g and u of the same columns: h = act(g) u in
//                16 bits is stored, and g and u in FP32 if they are wanted.
//   GATED_DOWN   dY W_out = dh.  With g and u from memory: dg, du and h in 16 bits.
//   GATED_ROUND  results rounded to 16 bits.
// What the first two cost beside their products is memory: with g and u kept, UP writes 10 bytes for each value of h and DOWN reads 8 and writes 6, and with one wave
// per SIMD nothing else runs on a unit meanwhile.  8192 tokens of 1024 x 2560, binary16, with one code for all activations: UP 128 us (its product alone takes 61, its bytes 44), DOWN 130; without the loads
// of g and u 89, without the stores of dg and du 109, without the activations 120, with none of them 61.  (Activations of their own code and, for DOWN, two workgroups a
// unit, see GatedPair: 126 and 123.)  Loads and stores with the streaming policy: 3 % slower; 3 to 10 units ahead in place of 6: within 1 %; workgroups that begin
// half a tile apart: none the faster.
// (FP32 products and passes over them in place of all three, 8192 x 4096 x 10240, forward and backward: 5034 us, 4609 so.)
#pragma once
#include "kernel_table.hpp"
#include "row_ops.hpp"

namespace fg {

// act(g) = g q(g) with q = 1 / (1 + exp(-g (k0 + k1 g^2))): silu has k0 = 1, k1 = 0; in gelu (1 + tanh v) / 2 = 1 / (1 + exp(-2 v)).
// KIND: each has code of its own, half as many instructions as one for all (with nothing kept 8192 tokens of 1024 x 2560 114 us so, 97 without an activation);
// FG_ACT_RELU is relu or none.  All kernels share it, so what a NaN or an infinity of g becomes does not depend on which of them a size takes.
struct Activation {
    float k0, k1;                           // of gelu, times -log2 e
    int32_t kind;
    __host__ __device__ static Activation of(int act) {
        const float c = 2.f * 0.79788456080286535588f, minus_log2e = -1.44269504088896340736f;         // (2 sqrt(2 / pi))
        return {c * minus_log2e, 0.044715f * c * minus_log2e, act};
    }
    template <class F> __device__ __forceinline__ void pick(F &&f) const {
        if (kind == FG_ACT_SILU) f(std::integral_constant<int, FG_ACT_SILU>{});
        else if (kind == FG_ACT_GELU_TANH) f(std::integral_constant<int, FG_ACT_GELU_TANH>{});
        else f(std::integral_constant<int, FG_ACT_RELU>{});
    }
    // act(g), and its derivative q + g q (1 - q) (k0 + 3 k1 g^2).  (Of gelu's g bounded, by operations that keep a NaN: far out q (1 - q) is zero, and stays zero times a
    // finite slope.)
    template <bool D, int KIND>
    __device__ __forceinline__ float at(float g, float *d) const {
        constexpr float kMinusLn2 = -0.69314718055994530942f;
        if constexpr (KIND == FG_ACT_SILU) {
            const float q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * g)), a = g * q;
            if constexpr (D) *d = __builtin_fmaf(a, 1.f - q, q);
            return a;
        } else if constexpr (KIND == FG_ACT_GELU_TANH) {
            const float x = D ? __builtin_elementwise_minimum(__builtin_elementwise_maximum(g, -1000.f), 1000.f) : g, x2 = x * x;
            const float q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * __builtin_fmaf(k1, x2, k0)));
            if constexpr (D) *d = __builtin_fmaf(x * q * (1.f - q), kMinusLn2 * __builtin_fmaf(3.f * k1, x2, k0), q);
            return g * q;
        } else {
            const bool off = kind == FG_ACT_RELU && g <= 0.f;           // (not of a NaN)
            if constexpr (D) *d = off ? 0.f : kind == FG_ACT_RELU && g != g ? g : 1.f;
            return off ? 0.f : g;
        }
    }
};

// A second product of a launch (GATED_ROUND_NN).
struct SecondProduct {
    const _Float16 *A, *B;
    float *D;
    int64_t a_ks, b_ks, a_span, b_span, ldd;
    int32_t M, N, tiles_m, tiles_n;
    Division by_group;
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
    SecondProduct second;
    __device__ __forceinline__ void to_second() {
        A = second.A; B = second.B; D = second.D;
        a_ks = second.a_ks; b_ks = second.b_ks; a_span = second.a_span; b_span = second.b_span; ldd = second.ldd;
        M = second.M; N = second.N; tiles_m = second.tiles_m; tiles_n = second.tiles_n;
        by_group = second.by_group;
    }
};

enum GatedKind { GATED_UP = 0, GATED_DOWN = 1, GATED_ROUND_KK = 2, GATED_ROUND_KN = 3, GATED_ROUND_NN = 4 };       // (round: A, B contiguous along K or not)

template <class Base, int KIND>
struct GatedCfg : Base {
    static constexpr bool OWN_STORE = true, PAIRED = KIND == GATED_UP, GROUPED = KIND == GATED_ROUND_NN;
    using Params = GatedParams;
    using T = typename std::conditional<Base::BF16, bf16_t, f16_t>::type;
    static_assert(!PAIRED || Base::TJ % 2 == 0, "a wave has blocks of G and U");
    // A lane takes a wave's results in units of eight consecutive columns.  From 16x16 results (TileCfg::M16) a unit is ROWS = 16 rows of 32 columns: a load or a store
    // of 16 bytes a lane covers 64 bytes of each of 16 rows (the epilogues of the other products have 32 bytes of 32 rows at a time; with FP32
    // operands of the result's shape each line was then asked for four times).
    static constexpr int ROWS = Base::M16 ? 16 : 32, WIDTH = Base::M16 ? 32 : 16, UI = Base::WTM / ROWS, UJ = Base::WTN / WIDTH;
    typedef float eight __attribute__((ext_vector_type(8)));
    typedef float four __attribute__((ext_vector_type(4)));
    typedef four four_anywhere __attribute__((aligned(4)));
    using Vec = typename RowPiece<T, 8>::vec;
    typedef __attribute__((address_space(1))) typename RowPiece<T, 8>::unaligned *Global;
    typedef __attribute__((address_space(1))) four_anywhere *GlobalFloats;
    typedef const __attribute__((address_space(1))) four_anywhere *ConstFloats;

    // Unit (i, j): the lane's row is ROWS i + lane % ROWS, its first column WIDTH j + 8 (lane / ROWS).
    template <int I, int J, class Blocks>
    __device__ static __forceinline__ eight unit(const Blocks &blocks) {
        eight out;
        if constexpr (Base::M16) {
            // Quarter q of the wave has columns 4 q .. of both 16x16 results a and b; exchanged between halves and then between quarters it has a's or b's 8 (q % 2) ..
            const floatx4 a = acc_sum<Base, I, 2 * J>(), b = acc_sum<Base, I, 2 * J + 1>();
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = a[r], y = b[r];
                const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, y), false, false);
                const unsigned h0 = h[0], h1 = h[1];
                const auto q = __builtin_amdgcn_permlane16_swap(h0, h1, false, false);
                const unsigned q0 = q[0], q1 = q[1];
                out[r] = __builtin_bit_cast(float, q0);
                out[4 + r] = __builtin_bit_cast(float, q1);
            }
        } else {
            // Half a wave has columns 8 h .. + 3 and the other + 4 .. + 7: exchanged, each has eight of two such runs.
            const floatx16 a = blocks(ic<I>{}, ic<J / 2>{});
            static_assert(Base::M16 || (Base::ACC_LH == 4 && Base::acc_col(4) == 8), "");
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = a[8 * (J % 2) + r], y = a[8 * (J % 2) + 4 + r];
                const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, y), false, false);
                const unsigned h0 = h[0], h1 = h[1];
                out[r] = __builtin_bit_cast(float, h0);
                out[4 + r] = __builtin_bit_cast(float, h1);
            }
        }
        return out;
    }

    template <class Blocks>
    __device__ static __forceinline__ void store(const Params &p, const Blocks &blocks, int m_base, int n_base, int lane) {
        if constexpr (Base::WIDE) own_acc<Base::WAVES>();
        const int row0 = m_base + lane % ROWS, shift = 8 * (lane / ROWS);
        if constexpr (KIND == GATED_UP || KIND == GATED_DOWN)
            p.act.pick([&](auto act) {
                constexpr int ACT = decltype(act)::value;
                if constexpr (KIND == GATED_UP) up<ACT>(p, blocks, row0, n_base / 2 + shift, n_base / 2 + Base::WTN / 2 > p.hidden);
                else down<ACT>(p, blocks, row0, n_base + shift, n_base + Base::WTN > p.hidden);
            });
        else round(p, blocks, row0, n_base + shift, n_base + Base::WTN > p.N);
    }
    __device__ static __forceinline__ void step() {
        if constexpr (Base::WIDE) {
            __builtin_amdgcn_sched_barrier(0);
            own_acc<Base::WAVES>();
        }
    }
    // the columns that are there, `left` of them
    __device__ static __forceinline__ void put(T *to, eight v, int left) {
        const Vec r = __builtin_convertvector(v, Vec);
        if (left >= 8) *(Global)to = r;
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) to[e] = r[e];
        }
    }
    __device__ static __forceinline__ void put(float *to, eight v, int left) {
        if (left >= 8) {
            *(GlobalFloats)to = four{v[0], v[1], v[2], v[3]};
            *((GlobalFloats)to + 1) = four{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) to[e] = v[e];
        }
    }

    // first: the lane's first column of h; the blocks of G and U, 32 columns each, lie side by side
    template <int ACT, class Blocks>
    __device__ static __forceinline__ void up(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        const Activation act = p.act;
        constexpr int PER = 32 / WIDTH;                                 // units of a block
        static_for<UI>([&](auto i) {
            constexpr int I = decltype(i)::value;
            const int row = row0 + ROWS * I;
            T *h = (T *)p.D + (int64_t)row * p.ldd + first;
            float *g_out = p.keep + (int64_t)row * p.ldgu + first, *u_out = g_out + p.hidden;
            static_for<UJ / 2>([&](auto jj) {
                constexpr int JJ = decltype(jj)::value, J = JJ / PER * 2 * PER + JJ % PER, c = WIDTH * JJ;
                const eight g = unit<I, J>(blocks), u = unit<I, J + PER>(blocks);
                eight v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = act.template at<false, ACT>(g[e], nullptr) * u[e];
                if (row < p.M) {
                    if (!edge) {
                        put(h + c, v, 8);
                        if (p.keep) {
                            put(g_out + c, g, 8);
                            put(u_out + c, u, 8);
                        }
                    } else {
                        // zeros behind the last column, to the end of h's row
                        const int left = p.hidden - first - c;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0.f;
                        if (first + c < p.ldd) put(h + c, v, 8);
                        if (p.keep) {
                            put(g_out + c, g, left);
                            put(u_out + c, u, left);
                        }
                    }
                }
                step();
            });
        });
    }

    // What a lane needs from memory for a unit: g and u of its columns.  Units are requested AHEAD of their turn: a lone wave waits for each otherwise.
    static constexpr int AHEAD = Base::WIDE && Base::WAVES == 1 ? 6 : 2;
    struct Pair { eight g, u; };
    __device__ static __forceinline__ eight eight_of(const float *at, int left, bool edge) {
        eight out;
        if (!edge || left >= 8) {
            const four a = *(ConstFloats)at, b = *((ConstFloats)at + 1);
            out = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = e < left ? at[e] : 0.f;
        }
        return out;
    }
    template <int ACT, class Blocks>
    __device__ static __forceinline__ void down(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        const Activation act = p.act;
        constexpr int COUNT = UI * UJ;
        Pair ahead[AHEAD];
        auto fetch = [&](auto b) {
            constexpr int B = decltype(b)::value;
            const int row = row0 + ROWS * (B / UJ), c = WIDTH * (B % UJ);
            const float *g = p.gu + (int64_t)(row < p.M ? row : p.M - 1) * p.ldgu + first + c;
            ahead[B % AHEAD] = {eight_of(g, p.hidden - first - c, edge), eight_of(g + p.hidden, p.hidden - first - c, edge)};
        };
        static_for<(AHEAD < COUNT ? AHEAD : COUNT)>(fetch);
        static_for<COUNT>([&](auto b) {
            constexpr int B = decltype(b)::value, I = B / UJ, J = B % UJ, c = WIDTH * J;
            const int row = row0 + ROWS * I;
            const eight dh = unit<I, J>(blocks);
            const Pair in = ahead[B % AHEAD];
            T *dg = (T *)p.D + (int64_t)row * p.ldd + first, *du = dg + p.hidden, *h = (T *)p.h + (int64_t)row * p.ldh + first;
            eight vg, vu, vh;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float d;
                const float a = act.template at<true, ACT>(in.g[e], &d);
                vg[e] = dh[e] * in.u[e] * d;
                vu[e] = dh[e] * a;
                vh[e] = a * in.u[e];
            }
            if (row < p.M) {
                if (!edge) {
                    put(dg + c, vg, 8);
                    put(du + c, vu, 8);
                    put(h + c, vh, 8);
                } else {
                    const int left = p.hidden - first - c;
#pragma unroll
                    for (int e = 0; e < 8; ++e) vh[e] = e < left ? vh[e] : 0.f;
                    put(dg + c, vg, left);
                    put(du + c, vu, left);
                    if (first + c < p.ldh) put(h + c, vh, 8);
                    // with the last column: zeros behind du, to the end of its row
                    if (left > 0 && left <= 8)
                        for (int z = 2 * p.hidden; z < (int)p.ldd; ++z) ((T *)p.D)[(int64_t)row * p.ldd + z] = (T)0.f;
                }
            }
            if constexpr (B + AHEAD < COUNT) fetch(ic<B + AHEAD>{});
            step();
        });
    }

    template <class Blocks>
    __device__ static __forceinline__ void round(const Params &p, const Blocks &blocks, int row0, int first, bool edge) {
        static_for<UI>([&](auto i) {
            const int row = row0 + ROWS * (int)decltype(i)::value;
            T *out = (T *)p.D + (int64_t)row * p.ldd + first;
            static_for<UJ>([&](auto j) {
                constexpr int c = WIDTH * (int)decltype(j)::value;
                const eight v = unit<decltype(i)::value, decltype(j)::value>(blocks);
                if (row < p.M) put(out + c, v, edge ? p.N - first - c : 8);
            });
            step();
        });
    }
};

// Beside the tiles of a plan GATED_UP and GATED_DOWN have one of 128x128 for two workgroups a unit: 80 KB of LDS (rings of three and two buffers) and half of the
// registers each, so that one stores, or waits for g and u, while the other multiplies.  Its K loop reaches 0.7 of the 256x256 tile's rate, which short sums are
// worth (gated_tile in gated.hip).
// The tiles of a plan: 256x256, 256x128, 128x128 with four buffers, 64x64 and 64x128 with two groups of waves.  On the 64x64 tile a wave has one block
// of columns, not one of G and one of U: GATED_UP has the 64x128 tile in its place.
template <class Cfg> KernelEntry gated_entry(const char *name, int kg = 0) {
    return {(const void *)gemm_kernel<Cfg>, name, Cfg::BM, Cfg::BN, Cfg::NTHREADS, Cfg::LDS_BYTES, kg};
}
template <bool AKC, bool BKC, bool BF> using GatedPair = TileCfg<128, 128, 64, 2, 2, 2, AKC, BKC, false, 0, 0, true, BF, false, false, false, false, true, 1, false, 2, true>;
template <int KIND, bool AKC, bool BKC, bool BF> KernelEntry pair_entry(const char *name) {
    if constexpr (KIND == GATED_UP || KIND == GATED_DOWN) return gated_entry<GatedCfg<GatedPair<AKC, BKC, BF>, KIND>>(name);
    else return FG_EMPTY_ENTRY;
}
template <int KIND, bool AKC, bool BKC, bool BF> const KernelEntry *gated_table(const char *const (&names)[GATED_TILES]) {
    using D = typename std::conditional<KIND == GATED_UP, FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), FG_CFG_KG(AKC, BKC, BF, false, false, 64, 4, true)>::type;
    static const KernelEntry t[GATED_TILES] = {
        gated_entry<GatedCfg<FG_CFG_K32(256, 256, 64, 2, 2, 2, AKC, BKC, BF, false), KIND>>(names[0]),
        gated_entry<GatedCfg<FG_CFG_K32(256, 128, 64, 3, 2, 2, AKC, BKC, BF, false), KIND>>(names[1]),
        gated_entry<GatedCfg<FG_CFG_K32(128, 128, 64, 4, 2, 2, AKC, BKC, BF, false), KIND>>(names[2]),
        gated_entry<GatedCfg<D, KIND>>(names[3], 2),
        gated_entry<GatedCfg<FG_CFG_KG(AKC, BKC, BF, false, false, 128, 3, true), KIND>>(names[4], 2),
        pair_entry<KIND, AKC, BKC, BF>(names[5]),
    };
    return t;
}
#define FG_GATED_TABLE(FUNC, KIND, AKC, BKC, BF, NAME)                                                                                       \
    const KernelEntry *FUNC() {                                                                                                              \
        static const char *const names[GATED_TILES] = {NAME "_256x256x64", NAME "_256x128x64", NAME "_128x128x64_deep",                      \
                                                       (KIND) == GATED_UP ? NAME "_64x128x64" : NAME "_64x64x64", NAME "_64x128x64", NAME "_128x128x64_pair"};        \
        return gated_table<KIND, AKC, BKC, BF>(names);                                                                                       \
    }

}  // namespace fg
