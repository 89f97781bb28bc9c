// The gradient of a weight from few tokens, for the operators that have one (xent.hip, gated.hip): dw = dz^T x, times a factor in memory if there is one.
//
// Where the tokens fit KS steps of 32 k of the matrix units all of it is writing dw.  A wave takes 16 J words (rows of dw) and 128 columns
// with one read of both operands.  A lane reads J words and 8 columns of 8 tokens' rows and turns the values over in registers (one byte permutation each
// pair): vectors of 8 tokens, of which the j-th of dz and the i-th of x serve the product of words J m + j with columns 8 n + i.  A lane's
// results of i = 0 .. 7 are then 16 bytes of a row of dw, and those of 16 lanes two lines.  Bound by the writes (65536 words x 2048: 16 tokens 41 us or 6.5 TB/s, 64 tokens
// 56); the tiled kernels, whose one wave a SIMD does not write while it multiplies, take 84 and 88 (50001 x 1001, 33 tokens: 25 and 81).  With 128 tokens the operands fill
// the registers: 103 us and 103.
#pragma once
#include "gemm_kernel.hpp"
#include "row_ops.hpp"

#include "few_items.hpp"

namespace fg {

constexpr int64_t kFewTokens = 64;          // whose dw is written so

template <class T>
__device__ __forceinline__ floatx4 mfma_16x16x32(typename RowPiece<T>::vec a, typename RowPiece<T>::vec b, floatx4 c) {
    if constexpr (std::is_same<T, bf16_t>::value) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// dz: rows of `have` values (a multiple of 8), ld_dz apart, 16-byte aligned, of which the first `words` count; x: rows of dim values; out: words x dim.
template <class T> struct DwOfFew {
    const T *dz, *x;
    T *out;
    int64_t ld_dz, have, ldx, ldo, words, dim, items;           // items: of the launch, set by it
    int32_t dz_again, x_again;              // a token from this one on has the row of the one so many before it (0: each has its own)
};
// One or two such products of the same tokens in a launch.  factor[1]: what results are multiplied by.
template <class T> struct DwsOfFew { DwOfFew<T> at[2]; };
template <class T, int KS, int J>
__global__ __launch_bounds__(256, 2) void dw_of_few(const DwsOfFew<T> products, const float *factor, int tokens) {
    typedef typename RowPiece<T>::vec vec;
    const int lane = threadIdx.x & 63, at = lane & 15, quarter = lane >> 4;
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    FewItem item;
    if (!few_item(wave, products.at[0].items, products.at[0].dim, products.at[1].items, products.at[1].dim, 16 * J, item)) return;
    const DwOfFew<T> q = products.at[item.second ? 1 : 0];
    const T *dz = q.dz, *x = q.x;
    T *out = q.out;
    const int64_t ld_dz = q.ld_dz, have = q.have, ldx = q.ldx, ldo = q.ldo;
    const int words = (int)q.words, dim = (int)q.dim;
    typedef typename RowPiece<T, J>::vec words_vec;
    const int64_t word0 = item.word;
    const int p = item.strip * 16 + at, pieces = (dim + 7) / 8, there = min(p, pieces - 1);
    const bool in = word0 + at * J < have;
    vec a[KS][J], b[KS][8];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        words_vec w[8] = {};
        vec v[8] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int t = s * 32 + quarter * 8 + e;
            if (t < tokens) {
                const int of_dz = q.dz_again && t >= q.dz_again ? t - q.dz_again : t, of_x = q.x_again && t >= q.x_again ? t - q.x_again : t;
                if (in) w[e] = *(const words_vec *)(dz + of_dz * ld_dz + word0 + at * J);
                v[e] = load_raw<T, 8>(x + of_x * ldx, there, dim);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int j = 0; j < J; ++j) a[s][j][e] = w[e][j];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[s][i][e] = v[e][i];
        }
    }
    const float f = factor ? factor[1] : 1.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        floatx4 sum[8] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = mfma_16x16x32<T>(a[s][j], b[s][i], sum[i]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t word = word0 + (quarter * 4 + r) * J + j;
            if (word >= words || p >= pieces) continue;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = sum[i][r] * f;
            store_piece(out + word * ldo, p, dim, v);
        }
    }
}

// tokens <= kFewTokens; either product may have no words
template <class T>
void launch_dw_of_few(Launches &enqueue, DwOfFew<T> first, DwOfFew<T> second, const float *factor, int64_t tokens) {
    auto items = [](const DwOfFew<T> &q, int64_t each) { return few_items(q.words, q.dim, each); };
    auto few = [&](auto steps, auto run) {
        constexpr int KS = decltype(steps)::value, J = decltype(run)::value;
        first.items = items(first, 16 * J);
        second.items = items(second, 16 * J);
        enqueue(dw_of_few<T, KS, J>, dim3((unsigned)((first.items + second.items + 3) / 4)), dim3(256), DwsOfFew<T>{{first, second}}, factor, (int)tokens);
    };
    using std::integral_constant;
    // Fewer waves than there are SIMDs: 64 words each instead of 128 (2496 words x 1000: 16 tokens 5.0 us and 6.7, 64 tokens 5.9 and 8.0;
    // 65536 x 2048: 53 and 41, 73 and 56).
    const bool small = items(first, 128) + items(second, 128) < 1024;
    if (tokens <= 32) small ? few(integral_constant<int, 1>{}, integral_constant<int, 4>{}) : few(integral_constant<int, 1>{}, integral_constant<int, 8>{});
    else small ? few(integral_constant<int, 2>{}, integral_constant<int, 4>{}) : few(integral_constant<int, 2>{}, integral_constant<int, 8>{});
}

}  // namespace fg
