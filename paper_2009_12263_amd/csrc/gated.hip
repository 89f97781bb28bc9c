// Gated feed-forward block and its gradient.
//
//   [G U] = X W_in^T,   H = act(G) U,   Y = H W_out^T
//   dH = dY W_out,   dG = dH U act'(G),   dU = dH act(G),   dX = [dG dU] W_in,   dW_in = [dG dU]^T X,   dW_out = dY^T H
//
// 6 T D H operations forward (T tokens of D values, H hidden ones) and 12 T D H backward, on the matrix units, whose epilogues are the activation, its
// gradient and the rounding (gated_kernel.hpp).  8192 x 4096 x 10240 bfloat16, forward and backward: 4.44 to 4.54 ms, 1360 to 1390 TFLOP/s.
// A product that the planner splits along K (few tiles, a long K) goes through FP32 sums instead, and
// a pass over them is the epilogue.
//
// H, dG and dU are rounded to the operands' 16 bits, the only roundings but those of the results: an error of half a step each, so that
// results are 1.4 times as far from 64 bits as rounding alone makes them.  G and U are kept in FP32: in 16 bits theirs came on top (dX 1.9 times).
// Of few results (parts_of) the error of single values shows in the norm, 1.6 times that of rounding alone (2 tokens of 224 values), and the matrix units have time:
// there H, dG and dU are two 16-bit numbers each, a value and what its rounding left, in rows of their own of the same products.
//
// Of few tokens the forward products are all reading of weights: gated_few.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "cache_policy.hpp"
#include "few_tokens.hpp"
#include "gated_kernel.hpp"
#include "shared_rows.hpp"

namespace fg {
namespace {

// Copies of a call's operands for the tiled kernels, all in one launch: rows of `cols` values become rows of ldo (a multiple of 8), with zeros behind them.
// pair > 0 (W_in for GATED_UP): 32 rows of G, the 32 of U that lie `pair` rows on, and so on, zeros behind the last row of either.
struct PadArg {
    const void *in;
    void *out;
    int64_t ld, ldo, rows, pair;
    int32_t cols;
    int32_t first;                          // number of its first workgroup
};
constexpr int kMostPads = 6, kPadPieces = 1024;             // pieces of eight values of a workgroup
struct PadArgs {
    PadArg at[kMostPads];
    int32_t count;
};
template <class T>
__global__ __launch_bounds__(256) void gated_pad(const PadArgs a) {
    int which = 0;
#pragma unroll
    for (int i = 1; i < kMostPads; ++i) which = i < a.count && a.at[i].first <= (int)blockIdx.x ? i : which;
    const PadArg p = a.at[which];
    const int pieces = (int)(p.ldo / 8);
    const int64_t begin = (int64_t)((int)blockIdx.x - p.first) * kPadPieces, all = p.rows * pieces;
    typename RowPiece<T>::vec v[kPadPieces / 256] = {};
    T *to[kPadPieces / 256] = {};
#pragma unroll
    for (int t = 0; t < kPadPieces / 256; ++t) {
        const int64_t i = begin + t * 256 + threadIdx.x;
        if (i >= all) continue;
        const int64_t row = i / pieces;
        const int c = (int)(i - row * pieces) * 8;
        to[t] = (T *)p.out + row * p.ldo + c;
        int64_t from = row;
        if (p.pair) {
            from = row / 64 * 32 + row % 32;
            if (from >= p.pair) continue;
            from += row / 32 % 2 ? p.pair : 0;
        }
        const T *in = (const T *)p.in + from * p.ld;
        if (c + 8 <= p.cols) v[t] = load_raw<T, 8>(in, c / 8, p.cols);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[t][e] = c + e < p.cols ? in[c + e] : (T)0.f;
    }
#pragma unroll
    for (int t = 0; t < kPadPieces / 256; ++t)
        if (to[t]) *(typename RowPiece<T>::vec *)to[t] = v[t];
}

// Piece p of eight values of FP32 rows; zeros from `cols` on.
__device__ __forceinline__ void load_eight(const float *row, int c0, int cols, float (&v)[8]) {
    typedef float four __attribute__((ext_vector_type(4)));
    typedef four anywhere __attribute__((aligned(4)));
    if (c0 + 8 <= cols) {
        const four a = *(const anywhere *)(row + c0), b = *(const anywhere *)(row + c0 + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c0 + e < cols ? row[c0 + e] : 0.f;
    }
}
// Eight values of a 16-bit row, those before `cols`; with `rest` also what their rounding leaves.
template <class T>
__device__ __forceinline__ void store_eight(T *row, int c0, int cols, const float (&v)[8], T *rest) {
    typedef typename RowPiece<T, 8>::vec vec;
    typedef typename RowPiece<T, 8>::unaligned anywhere;
    vec hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = (T)v[e];
        const float off = v[e] - (float)hi[e];
        lo[e] = __builtin_fabsf(off) < __builtin_inff() ? (T)off : (T)0.f;           // (of an infinity nothing is left)
    }
    if (c0 + 8 <= cols) {
        *(anywhere *)(row + c0) = hi;
        if (rest) *(anywhere *)(rest + c0) = lo;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + e < cols) {
                row[c0 + e] = hi[e];
                if (rest) rest[c0 + e] = lo[e];
            }
    }
}
// The sums of values and of what their rounding left.  (Of an infinite weight the first is infinite, and the second, of zeros and of either sign, must not make a NaN of it.)
__device__ __forceinline__ float both_parts(float sum, float rest) { return __builtin_fabsf(sum) < __builtin_inff() ? sum + rest : sum; }
// f(row, first column) for pieces of eight columns
template <class F> __device__ __forceinline__ void each_piece(int64_t rows, int cols, F &&f) {
    const int pieces = (cols + 7) / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        f(row, (int)(i - row * pieces) * 8);
    }
}

// h = act(g) u, rounded, with zeros to the end of its rows, PARTS: and what its rounding leaves `rows` rows further on; g and u are copied to `keep` where it is given
template <class T, bool PARTS>
__global__ __launch_bounds__(256) void gated_product(const float *gu, int64_t ldgu, T *h, int64_t ldh, int64_t rows, int hidden, Activation act, float *keep, int64_t ldkeep) {
    each_piece(rows, hidden, [&](int64_t row, int c) {
        float g[8], u[8], v[8];
        load_eight(gu + row * ldgu, c, hidden, g);
        load_eight(gu + row * ldgu + hidden, c, hidden, u);
        act.pick([&](auto kind) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < hidden ? act.template at<false, decltype(kind)::value>(g[e], nullptr) * u[e] : 0.f;
        });
        store_eight<T>(h + row * ldh, c, (int)ldh, v, PARTS ? h + (rows + row) * ldh : nullptr);
        if (keep) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < hidden) {
                    keep[row * ldkeep + c + e] = g[e];
                    keep[row * ldkeep + hidden + c + e] = u[e];
                }
        }
    });
}
// dg and du behind each other, and h, with zeros to the end of their rows; PARTS: what their rounding leaves `rows` rows further on
template <class T, bool PARTS>
__global__ __launch_bounds__(256) void gated_product_grad(const float *gu, int64_t ldgu, const float *dh, int64_t lddh, T *h, int64_t ldh, T *dgu, int64_t ldd,
                                                          int64_t rows, int hidden, Activation act) {
    each_piece(rows, hidden, [&](int64_t row, int c) {
        float g[8], u[8], x[8], vg[8], vu[8], vh[8];
        load_eight(gu + row * ldgu, c, hidden, g);
        load_eight(gu + row * ldgu + hidden, c, hidden, u);
        load_eight(dh + row * lddh, c, hidden, x);
        act.pick([&](auto kind) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float d;
                const float a = act.template at<true, decltype(kind)::value>(g[e], &d);
                vg[e] = x[e] * u[e] * d;
                vu[e] = x[e] * a;
                vh[e] = c + e < hidden ? a * u[e] : 0.f;
            }
        });
        T *to = dgu + row * ldd, *rest = PARTS ? to + rows * ldd : nullptr;
        store_eight<T>(to, c, hidden, vg, rest);
        store_eight<T>(to + hidden, c, hidden, vu, PARTS ? rest + hidden : nullptr);
        store_eight<T>(h + row * ldh, c, (int)ldh, vh, PARTS ? h + (rows + row) * ldh : nullptr);
        if (c + 8 >= hidden)
            for (int z = 2 * hidden; z < (int)ldd; ++z) {
                to[z] = (T)0.f;
                if (PARTS) rest[z] = (T)0.f;
            }
    });
}
// Rounded; PARTS: the sums of row r and row rows + r.  No `in`: zeros.
template <class T, bool PARTS>
__global__ __launch_bounds__(256) void gated_round(const float *in, int64_t ldi, T *out, int64_t ldo, int64_t rows, int cols) {
    each_piece(rows, cols, [&](int64_t row, int c) {
        float v[8] = {}, w[8];
        if (in) load_eight(in + row * ldi, c, cols, v);
        if constexpr (PARTS) {
            load_eight(in + (rows + row) * ldi, c, cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = both_parts(v[e], w[e]);
        }
        store_eight<T>(out + row * ldo, c, cols, v, nullptr);
    });
}
// ---- few tokens -------------------------------------------------------------------------------------------------
// Sums over k of w[n][k] x[r][k] for up to 16 NB rows r of x, NB = 1, 2 or 4: reading w.  A workgroup takes 16 rows of w (UP: and as many of U), its waves 64 k each in
// turn: a lane reads its row's 16 bytes straight into the operand of a 16x16x32 matrix instruction, a wave two whole lines of each row.  The waves' sums are added
// up through LDS in their order.
// UP: h = act(g) u of the sums, in 16 bits, and what its rounding leaves `lo` rows further on (lo > 0); g and u are kept in FP32 where that is wanted.  x is row-major; h
// is written as the other form reads its x: operands of matrix instructions, those of 32 k and 16 rows one after the other.
// Otherwise: rounded; with lo > 0 the sums of rows r and lo + r.
// Bound by reading w with one token (4096 x 10240: 252 MB in 50 us); with more, x costs as well, which each workgroup reads from the L2: every row of it is a
// line of its own (16 tokens 61 us); of more rows (are_few) the tiled kernels share x through LDS.
struct FewArgs {
    const void *x, *w;
    void *out;
    float *keep;
    int64_t ldx, ldw, ldo, ldkeep;
    int32_t rows, lo, n, k;             // of x; see above; rows of w (UP: of G), and their values
    Activation act;
};
// Where h's value of row r and column c is, and the values of all of it.
constexpr int few_blocks(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }          // of 16 rows
__device__ __forceinline__ int64_t few_place(int blocks, int r, int c) { return ((int64_t)(c >> 5) * blocks + (r >> 4)) * 512 + ((c >> 3) & 3) * 128 + (r & 15) * 8 + (c & 7); }
constexpr int64_t few_values(int64_t rows, int64_t k) { return (k + 31) / 32 * 512 * few_blocks(rows); }
constexpr int few_threads(int blocks) { return blocks == 4 ? 512 : 1024; }             // of a workgroup, at most: operands of 64 rows take 142 registers

// Eight values of 16 bits from memory.  ODD: they may begin between two 32-bit words, where a load of 16 bytes takes several times as long; then the words that they lie in
// are read, and shifted once they are there (8 tokens of 1023 x 8191: 23 and 30 us the two forms, 15 and 16 so; of 1024 x 8192 9 and 13).
template <class T, bool ODD> struct FewPiece {
    typedef typename RowPiece<T>::vec vec;
    vec v;
    __device__ __forceinline__ void fetch(const T *p) { v = *(const typename RowPiece<T>::unaligned *)p; }
    __device__ __forceinline__ vec get(const T *) const { return v; }
};
template <class T> struct FewPiece<T, true> {
    typedef typename RowPiece<T>::vec vec;
    typedef uint32_t words __attribute__((ext_vector_type(4))), words_anywhere __attribute__((ext_vector_type(4), aligned(4)));
    words v;
    uint32_t last;                      // the word of the last value: the one behind v, or its end
    __device__ __forceinline__ void fetch(const T *p) {
        v = *(const words_anywhere *)((uintptr_t)p & ~(uintptr_t)3);
        last = *(const uint32_t *)(((uintptr_t)p + 14) & ~(uintptr_t)3);
    }
    __device__ __forceinline__ vec get(const T *row) const {            // row: where p was, but for whole words
        const uint32_t by = (uint32_t)(uintptr_t)row & 2;
        words r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_alignbyte(i < 3 ? v[i + 1] : last, v[i], by);
        return __builtin_bit_cast(vec, r);
    }
};

template <class T, int NB, bool UP, bool ODD>
__global__ __launch_bounds__(few_threads(NB)) void gated_few(const FewArgs a) {
    typedef typename RowPiece<T>::vec vec;
    typedef typename RowPiece<T>::unaligned anywhere;
    constexpr int G = UP ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) char few_parts[];
    floatx4 *part = (floatx4 *)few_parts;               // [wave][G][NB][lane]
    const int lane = threadIdx.x & 63, at = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, row = min(n0 + at, a.n - 1);
    const T *w[G], *x[NB];
#pragma unroll
    for (int g = 0; g < G; ++g) w[g] = (const T *)a.w + ((int64_t)row + (g ? a.n : 0)) * a.ldw + quarter * 8;
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = UP ? (const T *)a.x + (int64_t)min(b * 16 + at, a.rows - 1) * a.ldx + quarter * 8 : (const T *)a.x + b * 512 + lane * 8;
    auto x_at = [&](int b, int k) { return UP ? x[b] + k : x[b] + (int64_t)(k >> 5) * (NB * 512); };
    floatx4 sum[G][NB] = {};
    // Workgroups begin at places of their own and walk K in a circle: side by side from its start they read, of rows that often lie a power of two
    // apart, the same few address bits, and those choose the memory channel (16 tokens, 4096 x 10240: 46.6 and 38.0 us the two forms, 39.7 and 34.2 so).
    const int k_whole = a.k / 64 * 64, turns = a.k / 64;
    const int begin = turns > 0 ? (int)(blockIdx.x * 5u % (unsigned)turns) : 0;
    auto several = [&](int turn, auto count) {
        constexpr int S = 2 * decltype(count)::value;
        FewPiece<T, ODD> wv[S][G];
        FewPiece<T, ODD && UP> xv[S][NB];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            int t = turn + s / 2 * waves + begin;
            t = t >= turns ? t - turns : t;
            const int k = t * 64 + s % 2 * 32;
#pragma unroll
            for (int g = 0; g < G; ++g) wv[s][g].fetch(w[g] + k);
#pragma unroll
            for (int b = 0; b < NB; ++b) xv[s][b].fetch(x_at(b, k));
        }
        __builtin_amdgcn_sched_barrier(0);              // (all requests go out before the first is used)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int b = 0; b < NB; ++b) sum[g][b] = mfma_16x16x32<T>(wv[s][g].get(w[g]), xv[s][b].get(x[b]), sum[g][b]);
    };
    int turn = wave;
    for (; turn + waves < turns; turn += 2 * waves) several(turn, std::integral_constant<int, 2>{});
    if (turn < turns) several(turn, std::integral_constant<int, 1>{});
    if (k_whole < a.k && wave == turns % waves) {                   // the last values: element by element at the end of a row
        for (int last = k_whole; last < a.k; last += 32) {
            const int left = a.k - last - quarter * 8;
            auto piece = [&](const T *p, bool whole) {
                vec v = {};
                if (whole && left > 0) {
                    v = *(const anywhere *)p;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : (T)0.f;
                } else if (left >= 8) v = *(const anywhere *)p;
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) v[e] = p[e];
                return v;
            };
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const vec v = piece(w[g] + last, false);
#pragma unroll
                for (int b = 0; b < NB; ++b) sum[g][b] = mfma_16x16x32<T>(v, piece(x_at(b, last), !UP), sum[g][b]);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int b = 0; b < NB; ++b) part[((wave * G + g) * NB + b) * 64 + lane] = sum[g][b];
    __syncthreads();
    // A thread has row r of x and four columns.
    auto total = [&](int g, int r, int q) {
        const int slot = (g * NB + (r >> 4)) * 64 + q * 16 + (r & 15);
        floatx4 s = part[slot];
        for (int v = 1; v < waves; ++v) s += part[v * (G * NB * 64) + slot];
        return s;
    };
    const int rows = UP || a.lo == 0 ? a.rows : a.lo;
    for (int i = threadIdx.x; i < rows * 4; i += blockDim.x) {
        const int r = i >> 2, q = i & 3, c = n0 + 4 * q, left = a.n - c;
        if (left <= 0) continue;
        floatx4 v = total(0, r, q);
        if constexpr (UP) {
            const floatx4 u = total(1, r, q);
            if (a.keep) {
                float *g_out = a.keep + (int64_t)r * a.ldkeep + c, *u_out = g_out + a.n;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) { g_out[e] = v[e]; u_out[e] = u[e]; }
            }
            a.act.pick([&](auto kind) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = a.act.template at<false, decltype(kind)::value>(v[e], nullptr) * u[e];
            });
            // (both forms have as many blocks of rows of h: with lo > 0 it has 2 lo rows)
            auto place = [&](int row) { return (T *)a.out + few_place(few_blocks(a.lo ? 2 * a.lo : a.rows), row, c); };
            T *out = place(r), *rest = place(r + a.lo);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) {
                    out[e] = (T)v[e];
                    const float off = v[e] - (float)(T)v[e];
                    if (a.lo) rest[e] = __builtin_fabsf(off) < __builtin_inff() ? (T)off : (T)0.f;
                }
        } else {
            if (a.lo) {
                const floatx4 rest = total(0, a.lo + r, q);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = both_parts(v[e], rest[e]);
            }
            T *out = (T *)a.out + (int64_t)r * a.ldo + c;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) out[e] = (T)v[e];
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
constexpr int64_t kLargestWidth = kResultLd - 8;            // of dim and of 2 hidden: rows of FP32 results and of copies stay below the kernels' leading dimensions

template <class F> void with_half(int dtype, F &&f) {
    if (dtype == FG_F16) f(f16_t{});
    else f(bf16_t{});
}
fg_matrix rows_of(const void *p, int32_t dtype, int64_t ld, int32_t layout = FG_ROW) { return {const_cast<void *>(p), nullptr, dtype, layout, ld}; }
fg_matrix turned(fg_matrix m) { m.layout = FG_COL; return m; }
bool as_it_is(int64_t cols, const fg_matrix *m) { return cols % 8 == 0 && aligned_to(m->re, 16) && m->ld % 8 == 0 && m->ld < kKContiguousLd; }

// Whether gated_few takes so many rows; copies: the tiled kernels would need copies of weights.  Up to 16 rows it is the fastest (one token of 4096 x 10240 52 us, the tiled
// kernels 68; 16 63 and 61).  Up to 32 where the weights are small and launches count (32 tokens of 1024 x 2560 20.1 us, by four launches of tiled kernels and sums 22.1; of
// 2048 x 5120 34.7 and 27.1) or would be copied (32 of 2047 x 5119 44 and 50, of 4094 x 10238 113 and 159, 20 of 3754 x 1634 20 and 41).  Up to 64 where neither sum is long,
// for which its workgroups are too few (48 of 1024 x 2560 17 and 23, 64 of 2048 x 1500 21 and 30, of 512 x 1536 12 and 17, 50 of 999 x 3001 28 and 33; 64 of 768 x 4096 21 and
// 19, of 512 x 8192 28 and 20, 40 of 4096 x 1000 28 and 23, 64 of 2048 x 5120 39 and 27).
bool are_few(int64_t rows, int64_t D, int64_t H, bool copies) {
    if (rows <= 16) return true;
    if (rows <= 32) return copies || D * H <= (1 << 22);
    return rows <= 64 && D <= 2048 && H <= 3500 && D * H <= (3 << 20);
}

// Rows for each token of H, dG and dU: two where results are few.
int64_t parts_of(int64_t T, int64_t D, int64_t H) { return T * std::min(D, H) < 16384 ? 2 : 1; }

// Whether a product goes through FP32 sums: the planner splits its K.
bool by_sums(int64_t M, int64_t N, int64_t K) { return gemm_stored_scratch(M, N, K) > 0; }
// A lane of GATED_UP reaches U from G's rows with a 32-bit offset.
bool in_reach(int64_t H, const fg_matrix *W_in) { return (H + 128) * W_in->ld * 2 < (1ll << 31); }

// Where the parts of a workspace are.
struct Space {
    int64_t bytes = 0, scratch = 0, scratch_bytes = 0;
    int64_t take(int64_t n) { const int64_t at = bytes; bytes += up(n, 256); return at; }
    void partial(int64_t M, int64_t N, int64_t K) { scratch_bytes = std::max(scratch_bytes, gemm_stored_scratch(M, N, K)); }
};
struct ForwardSpace : Space {
    int64_t parts;
    bool few, up_by_sums, down_by_sums;
    int64_t x = 0, w_in = 0, w_out = 0, gu = 0, h, sums = 0;
    ForwardSpace(int64_t T, int64_t D, int64_t H, bool copy_x, bool copy_in, bool copy_out, bool own_gu) {
        const int64_t dp = up(D, 8), hp = up(H, 8);
        parts = parts_of(T, D, H);
        few = are_few(parts * T, D, H, copy_in || copy_out);            // (x is read where it is)
        up_by_sums = !few && (parts == 2 || by_sums(T, 2 * H, dp));
        down_by_sums = !few && (parts == 2 || by_sums(T, D, hp));
        h = take((few ? few_values(parts * T, H) : parts * T * hp) * 2);
        if (few) return;
        if (copy_x) x = take(T * dp * 2);
        if (copy_in) w_in = take(2 * up(H, 32) * dp * 2);
        if (copy_out) w_out = take(D * hp * 2);
        if (up_by_sums && own_gu) gu = take(T * up(2 * H, 4) * 4);
        if (down_by_sums) sums = take(parts * T * up(D, 4) * 4);
        if (up_by_sums) partial(T, 2 * H, dp);
        if (down_by_sums) partial(parts * T, D, hp);
        scratch = take(scratch_bytes);
    }
};
struct GradSpace : Space {
    int64_t parts, times;           // times: how often dY and X are needed, one copy behind the other
    // few: dw_of_few writes the weights' gradients (one token of 2232 x 4832 16 us, by the tiled kernels 41; 64 of 2048 x 5120 13 and 21; 60 of 333 x 777 7.4 and 6.6)
    bool few, down_by_sums, x_by_sums, in_by_sums, out_by_sums;
    int64_t dy = 0, x = 0, w_in = 0, w_out = 0, dh = 0, h, dgu, sums = 0;
    GradSpace(int64_t T, int64_t D, int64_t H, bool copy_dy, bool copy_x, bool copy_in, bool copy_out) {
        const int64_t dp = up(D, 8), hp = up(H, 8), gp = up(2 * H, 8);
        parts = parts_of(T, D, H);
        const int64_t tp = up(parts * T, 8);
        down_by_sums = parts == 2 || by_sums(T, H, dp);
        x_by_sums = parts == 2 || by_sums(T, D, gp);
        few = parts * T <= kFewTokens;
        in_by_sums = !few && by_sums(2 * H, D, tp);
        out_by_sums = !few && by_sums(D, H, tp);
        times = few ? 1 : parts;
        if (copy_dy || times == 2) dy = take(times * T * dp * 2);
        if ((copy_x || times == 2) && !few) x = take(times * T * dp * 2);
        if (copy_in) w_in = take(2 * H * dp * 2);
        if (copy_out) w_out = take(D * hp * 2);
        h = take(parts * T * hp * 2);
        dgu = take(parts * T * gp * 2);
        if (down_by_sums) { dh = take(T * up(H, 4) * 4); partial(T, H, dp); }
        int64_t most = 0;
        if (x_by_sums) { most = std::max(most, parts * T * up(D, 4)); partial(parts * T, D, gp); }
        if (in_by_sums) { most = std::max(most, 2 * H * up(D, 4)); partial(2 * H, D, tp); }
        if (out_by_sums) { most = std::max(most, D * up(H, 4)); partial(D, H, tp); }
        sums = take(most * 4);
        scratch = take(scratch_bytes);
    }
};

// Sizes that are not negative, with fewer than 2^25 tiles of 64 x 64 results in each product.
constexpr int64_t kMostTokens = 1 << 30;
bool in_range(int64_t T, int64_t D, int64_t H) { return T <= kMostTokens && D < kLargestWidth && H < (kLargestWidth + 1) / 2; }
bool few_tiles(int64_t T, int64_t D, int64_t H) {
    auto tiles = [](int64_t m, int64_t n) { return ((m + 63) / 64) * ((n + 63) / 64); };
    return tiles(T, std::max(2 * H, D)) < (1ll << 25) && tiles(2 * H, D) < (1ll << 25);
}

fg_status check_gated(int64_t T, int64_t D, int64_t H, const fg_matrix *X, const fg_matrix *W_in, const fg_matrix *W_out, int32_t act) {
    if (T < 0 || D < 0 || H < 0) return fail(FG_ERR_SHAPE, "negative size: %lld tokens, %lld values, %lld hidden", (long long)T, (long long)D, (long long)H);
    if (!in_range(T, D, H))
        return fail(FG_ERR_UNSUPPORTED, "more than 2^30 tokens, or dim or 2 hidden of 2^21 - 8 and more, are not supported");
    if (!few_tiles(T, D, H)) return fail(FG_ERR_UNSUPPORTED, "products of more than 2^25 tiles are not supported");
    if (fg_status st = check_rows("X", X, T, D)) return st;
    if (fg_status st = check_rows("W_in", W_in, 2 * H, D)) return st;
    if (fg_status st = check_rows("W_out", W_out, D, H)) return st;
    if (X->dtype == FG_F32 || X->dtype != W_in->dtype || X->dtype != W_out->dtype) return fail(FG_ERR_UNSUPPORTED, "X, W_in and W_out must all be FG_F16 or all FG_BF16");
    if (act != FG_ACT_NONE && act != FG_ACT_RELU && act != FG_ACT_SILU && act != FG_ACT_GELU_TANH) return fail(FG_ERR_LAYOUT, "unknown activation %d", act);
    return FG_OK;
}
fg_status check_like(const char *name, const fg_matrix *m, int64_t rows, int64_t cols, int dtype) {
    if (fg_status st = check_rows(name, m, rows, cols)) return st;
    if (m->dtype != dtype) return fail(FG_ERR_UNSUPPORTED, "%s must be %s", name, dtype == FG_F32 ? "FG_F32" : "of the element type of X");
    return FG_OK;
}

// An operand or a result (null: not wanted) of checked rows.
struct Rows {
    const char *name;
    const fg_matrix *m;
    int64_t rows, cols;
    RowSpan span() const { return {(uintptr_t)m->re, rows, m->ld * element_bytes(m->dtype), cols * element_bytes(m->dtype)}; }
};
// Results are written while operands are still to be read.
fg_status check_elsewhere(const Rows &out, const Rows &in) {
    if (out.m && in.m && share_bytes(out.span(), in.span())) return fail(FG_ERR_LAYOUT, "%s must be in other memory than %s", out.name, in.name);
    return FG_OK;
}

unsigned groups_for(int64_t rows, int64_t cols) { return (unsigned)std::min<int64_t>((rows * ((cols + 7) / 8) + 255) / 256, 8192); }

// Which tile of kernel_table_gated serves a product.  Two workgroups a unit where the epilogue's memory weighs against the sums and the GPU is filled: G and U up to K = 512
// (3000 tokens of 400 x 1500 37 -> 27 us, 2000 of 128 x 5000 37 -> 31; 4096 of 768 x 2048 40 -> 54), dh up to 1024 (3000 of 400 x 1500 39 -> 30, 8192 of 1024 x 2560 129 -> 125,
// 1003 of 1001 x 2729 24 -> 23; 1500 of 2048 x 8000 97 -> 94, but the products beside it, at the power limit, lose as much; with K = 4096 671 -> 925; 96 tiles 15.6 -> 17.9).
int gated_tile(int kind, int64_t M, int64_t N, int64_t K) {
    const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128);
    if ((kind == GATED_UP && K <= 512 && tiles >= 256) || (kind == GATED_DOWN && K <= 1024 && tiles >= 150)) return 5;
    switch (plan_tile(M, N, K)) {
        case TILE_256x256: case TILE_256x256_K32: return 0;
        case TILE_256x128: case TILE_256x128_PASS: return 1;
        case TILE_64x64: case TILE_64x64_KG2: case TILE_64x64_KG2_DEEP: return 3;
        case TILE_64x128_KG2: return 4;
        default: return 2;
    }
}

// Which tile both weights' gradients share in one launch; -1: they are faster one by one.  A round of tiles takes the time of one, K steps of 1.1, 0.75 or 0.5 us (256x256,
// 256x128, 128x128; partly filled rounds measured) and 3 us besides; a product that is split along K takes its share of the GPU and 12 us for two launches.  (8192 tokens, 5120 x 1024 and
// 1024 x 2560: 160 and 80 tiles, 104 and 75 us one by one.)
int tile_of_both(const GradSpace &s, int64_t M1, int64_t N1, int64_t M2, int64_t N2, int64_t K) {
    const int bm[] = {256, 256, 128}, bn[] = {256, 128, 128};
    const double step[] = {1.1, 0.75, 0.5}, steps = (double)((K + 63) / 64);
    auto tiles = [&](int t, int64_t m, int64_t n) { return ((m + bm[t] - 1) / bm[t]) * ((n + bn[t] - 1) / bn[t]); };
    auto time = [&](int t, int64_t n) { return (double)((n + 255) / 256) * (steps * step[t] + 3); };
    double one[2] = {1e30, 1e30}, both = 1e30;
    int best = 0;
    for (int t = 0; t < 3; ++t) {
        const int64_t n1 = tiles(t, M1, N1), n2 = tiles(t, M2, N2);
        one[0] = std::min(one[0], time(t, n1));
        one[1] = std::min(one[1], time(t, n2));
        if (time(t, n1 + n2) < both) { both = time(t, n1 + n2); best = t; }
    }
    auto split = [&](int64_t m, int64_t n) { return (double)tiles(2, m, n) * steps * 0.6 / 256 + 12; };
    if (s.in_by_sums) one[0] = std::min(one[0], split(M1, N1));
    if (s.out_by_sums) one[1] = std::min(one[1], split(M2, N2));
    return both < one[0] + one[1] ? best : -1;
}

// A call's operands and launches.
struct Call {
    Launches enqueue;
    char *space;
    int dtype;
    PadArgs pads = {};
    // m, or a copy at `at` whose rows are aligned and padded (`times`: so many, one behind the other), made by copies()
    fg_matrix aligned(const fg_matrix *m, int64_t rows, int64_t cols, bool copy, int64_t at, int64_t times = 1) {
        if (!copy && times == 1) return *m;
        const int64_t ld = fg::up(cols, 8);
        for (int64_t k = 0; k < times; ++k) add({m->re, space + at + k * rows * ld * 2, m->ld, ld, rows, 0, (int32_t)cols, 0});
        return rows_of(space + at, dtype, ld);
    }
    int64_t pad_groups = 0;
    void add(PadArg p) {
        p.first = (int32_t)pad_groups;
        pads.at[pads.count++] = p;
        pad_groups += (p.rows * (p.ldo / 8) + kPadPieces - 1) / kPadPieces;
    }
    void copies() {
        if (pads.count == 0) return;
        with_half(dtype, [&](auto t) { enqueue(gated_pad<decltype(t)>, dim3((unsigned)pad_groups), dim3(256), pads); });
        pads.count = 0;
        pad_groups = 0;
    }
    fg_status by_sums(const Space &s, int64_t M, int64_t N, int64_t K, int64_t k_rows, const fg_matrix &a, const fg_matrix &b, const fg_matrix &d, RoundedResult *rounded = nullptr) {
        if (fg_status st = enqueue.status("gated_pad")) return st;
        return gemm_stored(M, N, K, k_rows, 1.f, &a, &b, 0.f, nullptr, &d, (float *)(space + s.scratch), s.scratch_bytes, enqueue.stream, rounded);
    }
    template <bool PARTS> void round(const fg_matrix &in, const fg_matrix *out, int64_t rows, int64_t cols) {
        with_half(dtype, [&](auto t) {
            using T = decltype(t);
            enqueue(gated_round<T, PARTS>, dim3(groups_for(rows, cols)), dim3(256), (const float *)in.re, in.ld, (T *)out->re, out->ld, rows, (int)cols);
        });
    }
    // The products of both weights' gradients, [dG dU]^T X and dY^T H, which have the same K, in one launch on the same tile.
    fg_status both_weights(int tile, int64_t K, const fg_matrix &dgu, const fg_matrix &x, const fg_matrix *d_in, int64_t M1, int64_t N1, const fg_matrix &dy, const fg_matrix &h,
                           const fg_matrix *d_out, int64_t M2, int64_t N2) {
        const KernelEntry &k = kernel_table_gated(GATED_ROUND_NN, dtype == FG_BF16)[tile];
        GatedParams p;
        memset(&p, 0, sizeof p);
        auto span = [&](int64_t n, int64_t ld) { return fg::up((K - 1) * ld + n, 8); };
        p.M = (int32_t)M1; p.N = (int32_t)N1; p.K = (int32_t)K;
        p.tiles_m = (int32_t)((M1 + k.bm - 1) / k.bm); p.tiles_n = (int32_t)((N1 + k.bn - 1) / k.bn);
        p.A = (const _Float16 *)dgu.re; p.B = (const _Float16 *)x.re; p.D = (float *)d_in->re; p.ldd = d_in->ld;
        p.a_rs = p.b_rs = 1;
        p.a_ks = dgu.ld; p.b_ks = x.ld;
        p.a_span = span(M1, dgu.ld); p.b_span = span(N1, x.ld);
        p.alpha = 1.f;
        SecondProduct &q = p.second;
        q.M = (int32_t)M2; q.N = (int32_t)N2;
        q.tiles_m = (int32_t)((M2 + k.bm - 1) / k.bm); q.tiles_n = (int32_t)((N2 + k.bn - 1) / k.bn);
        q.A = (const _Float16 *)dy.re; q.B = (const _Float16 *)h.re; q.D = (float *)d_out->re; q.ldd = d_out->ld;
        q.a_ks = dy.ld; q.b_ks = h.ld;
        q.a_span = span(M2, dy.ld); q.b_span = span(N2, h.ld);
        q.by_group = tile_group(q.tiles_m, q.tiles_n);
        return launch_product(k, p, enqueue.stream, q.tiles_m * q.tiles_n);
    }
    // A product of the tiled kernels; k_rows: those that an operand has which is not K-contiguous (others count as zero).  f sets the parameters of its epilogue.
    template <class F> fg_status product(int kind, int64_t M, int64_t N, int64_t K, int64_t k_rows, const fg_matrix &a, const fg_matrix &b, F &&f) {
        if (fg_status st = enqueue.status("gated_pad")) return st;
        const bool a_kc = kind != GATED_ROUND_NN, b_kc = kind == GATED_UP || kind == GATED_ROUND_KK;
        const KernelEntry &k = kernel_table_gated(kind, dtype == FG_BF16)[gated_tile(kind, M, N, K)];
        GatedParams p;
        memset(&p, 0, sizeof p);
        p.M = (int32_t)M; p.N = (int32_t)N; p.K = (int32_t)K;
        p.tiles_m = (int32_t)((M + k.bm - 1) / k.bm); p.tiles_n = (int32_t)((N + k.bn - 1) / k.bn);
        p.A = (const _Float16 *)a.re; p.B = (const _Float16 *)b.re;
        p.a_rs = a_kc ? a.ld : 1; p.a_ks = a_kc ? 1 : a.ld;
        p.b_rs = b_kc ? b.ld : 1; p.b_ks = b_kc ? 1 : b.ld;
        p.a_span = fg::up(a_kc ? (M - 1) * a.ld + K : (k_rows - 1) * a.ld + M, 8);
        p.b_span = fg::up(b_kc ? (N - 1) * b.ld + K : (k_rows - 1) * b.ld + N, 8);
        p.alpha = 1.f;
        p.rotate = (p.tiles_m == 1 && b_kc) || (p.tiles_n == 1 && a_kc);
        p.once = p.tiles_m == 1 && streams_once((uintptr_t)b.re, b.ld, N * K * 2) ? 1 : p.tiles_n == 1 && streams_once((uintptr_t)a.re, a.ld, M * K * 2) ? 2 : 0;
        f(p);
        return launch_product(k, p, enqueue.stream);
    }
    // out = a b, rounded, by the tiled kernels or through sums at s.sums; kind: GATED_ROUND_..
    fg_status rounded(const Space &s, int64_t sums, bool through_sums, int kind, int64_t M, int64_t N, int64_t K, int64_t k_rows, const fg_matrix &a, const fg_matrix &b, const fg_matrix *out) {
        if (!through_sums)
            return product(kind, M, N, K, k_rows, a, b, [&](GatedParams &p) { p.D = (float *)out->re; p.ldd = out->ld; });
        const fg_matrix d = rows_of(space + sums, FG_F32, fg::up(N, 4));
        RoundedResult rounded = {out, false};
        if (fg_status st = by_sums(s, M, N, K, kind == GATED_ROUND_KK ? 0 : k_rows, kind == GATED_ROUND_NN ? turned(a) : a, kind == GATED_ROUND_KK ? turned(b) : b, d, &rounded)) return st;
        if (!rounded.done) round<false>(d, out, M, N);
        return enqueue.status("gated_round");
    }
    template <bool UP> void few(const FewArgs &a) {
        with_half(dtype, [&](auto t) {
            using T = decltype(t);
            auto launch = [&](auto nb, auto odd) {
                constexpr int NB = decltype(nb)::value;
                constexpr bool ODD = decltype(odd)::value;
                // Waves to fill the GPU (16 a unit), as long as each has eight turns (one token of 1024 x 2560: four waves for G and U 10.9 us, sixteen 11.5).
                const int tiles = (a.n + 15) / 16, steps = (a.k + 63) / 64;
                int waves = 1;
                while (waves < few_threads(NB) / 64 && tiles * waves < 4096 && steps >= 8 * waves) waves *= 2;
                enqueue.with_lds(waves * (UP ? 2 : 1) * NB * 1024, gated_few<T, NB, UP, ODD>, dim3((unsigned)tiles), dim3(64 * waves), a);
            };
            const bool odd = !aligned_to(a.w, 4) || a.ldw % 2 != 0 || (UP && (!aligned_to(a.x, 4) || a.ldx % 2 != 0));
            auto either = [&](auto nb) { odd ? launch(nb, std::true_type{}) : launch(nb, std::false_type{}); };
            switch (few_blocks(a.rows)) {
                case 1: either(std::integral_constant<int, 1>{}); break;
                case 2: either(std::integral_constant<int, 2>{}); break;
                default: either(std::integral_constant<int, 4>{});
            }
        });
    }
};

}  // namespace

#define FG_GATED(NAME) const KernelEntry *kernel_table_gated_##NAME##_f16(); const KernelEntry *kernel_table_gated_##NAME##_bf16();
FG_GATED(up) FG_GATED(down) FG_GATED(round_kk) FG_GATED(round_kn) FG_GATED(round_nn)
#undef FG_GATED
const KernelEntry *kernel_table_gated(int kind, bool bf16) {
    switch (kind) {
        case GATED_UP: return bf16 ? kernel_table_gated_up_bf16() : kernel_table_gated_up_f16();
        case GATED_DOWN: return bf16 ? kernel_table_gated_down_bf16() : kernel_table_gated_down_f16();
        case GATED_ROUND_KK: return bf16 ? kernel_table_gated_round_kk_bf16() : kernel_table_gated_round_kk_f16();
        case GATED_ROUND_KN: return bf16 ? kernel_table_gated_round_kn_bf16() : kernel_table_gated_round_kn_f16();
        default: return bf16 ? kernel_table_gated_round_nn_bf16() : kernel_table_gated_round_nn_f16();
    }
}

hipError_t load_gated_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)gated_round<f16_t, false>);
}

}  // namespace fg

using namespace fg;

extern "C" {

int64_t fg_gated_ffn_workspace(int64_t tokens, int64_t dim, int64_t hidden) {
    if (tokens <= 0 || dim <= 0 || hidden <= 0 || !in_range(tokens, dim, hidden) || !few_tiles(tokens, dim, hidden)) return 0;
    // (the kernel for few tokens makes no copies)
    return std::max(ForwardSpace(tokens, dim, hidden, true, true, true, true).bytes, ForwardSpace(tokens, dim, hidden, true, false, false, true).bytes);
}

fg_status fg_gated_ffn(int64_t tokens, int64_t dim, int64_t hidden, const fg_matrix *X, const fg_matrix *W_in, const fg_matrix *W_out, int32_t act,
                       const fg_matrix *Y, const fg_matrix *GU, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_gated(tokens, dim, hidden, X, W_in, W_out, act)) return st;
    if (fg_status st = check_like("Y", Y, tokens, dim, X->dtype)) return st;
    if (GU) if (fg_status st = check_like("GU", GU, tokens, 2 * hidden, FG_F32)) return st;
    if (tokens == 0) return FG_OK;
    Call call = {Launches(hip_stream), (char *)workspace, X->dtype};
    if (dim == 0) {                         // G and U are empty sums
        if (GU && hidden > 0)
            call.enqueue(gated_round<float, false>, dim3(groups_for(tokens, 2 * hidden)), dim3(256), (const float *)nullptr, (int64_t)0, (float *)GU->re, GU->ld, tokens, (int)(2 * hidden));
        return call.enqueue.status("gated_round");
    }
    const Rows operands[] = {{"X", X, tokens, dim}, {"W_in", W_in, 2 * hidden, dim}, {"W_out", W_out, dim, hidden}}, y = {"Y", Y, tokens, dim}, kept = {"GU", GU, tokens, 2 * hidden};
    for (const Rows &in : operands)
        if (fg_status st = check_elsewhere(y, in)) return st;
    if (hidden == 0) {
        call.round<false>(rows_of(nullptr, FG_F32, 0), Y, tokens, dim);
        return call.enqueue.status("gated_round");
    }
    for (const Rows &in : operands)
        if (fg_status st = check_elsewhere(kept, in)) return st;
    if (fg_status st = check_elsewhere(kept, y)) return st;
    const bool copy_x = !as_it_is(dim, X), copy_out = !as_it_is(hidden, W_out), copy_in = !as_it_is(dim, W_in) || !in_reach(hidden, W_in);
    const bool own_gu = !GU || !aligned_to(GU->re, 16) || GU->ld % 4 != 0 || GU->ld >= kResultLd;        // (so that results do not depend on where GU is)
    const ForwardSpace at(tokens, dim, hidden, copy_x, copy_in, copy_out, own_gu);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    const int64_t dp = up(dim, 8), hp = up(hidden, 8);
    const fg_matrix h = rows_of(call.space + at.h, X->dtype, hp);
    float *keep = GU ? (float *)GU->re : nullptr;
    const int64_t ldkeep = GU ? GU->ld : 0;
    const Activation activation = Activation::of(act);
    if (at.few) {
        const int32_t lo = at.parts == 2 ? (int32_t)tokens : 0;
        call.few<true>({X->re, W_in->re, h.re, keep, X->ld, W_in->ld, hp, ldkeep, (int32_t)tokens, lo, (int32_t)hidden, (int32_t)dim, activation});
        call.few<false>({h.re, W_out->re, Y->re, nullptr, hp, W_out->ld, Y->ld, 0, (int32_t)tokens + lo, lo, (int32_t)dim, (int32_t)hidden, activation});
        return call.enqueue.status("gated_few");
    }
    const fg_matrix x = call.aligned(X, tokens, dim, copy_x, at.x), w_out = call.aligned(W_out, dim, hidden, copy_out, at.w_out);
    if (at.up_by_sums) {
        const fg_matrix w_in = call.aligned(W_in, 2 * hidden, dim, copy_in, at.w_in), gu = !own_gu ? *GU : rows_of(call.space + at.gu, FG_F32, up(2 * hidden, 4));
        call.copies();
        if (fg_status st = call.by_sums(at, tokens, 2 * hidden, dp, 0, x, turned(w_in), gu)) return st;
        with_half(X->dtype, [&](auto t) {
            using T = decltype(t);
            auto pass = [&](auto kernel) {
                call.enqueue(kernel, dim3(groups_for(tokens, hidden)), dim3(256), (const float *)gu.re, gu.ld, (T *)h.re, hp, tokens, (int)hidden, activation,
                             own_gu ? keep : nullptr, ldkeep);
            };
            if (at.parts == 2) pass(gated_product<T, true>);
            else pass(gated_product<T, false>);
        });
    } else {
        fg_matrix w_in = *W_in;
        int64_t pair = hidden, pair_step = 32;
        if (copy_in) {
            w_in = rows_of(call.space + at.w_in, X->dtype, dp);
            pair = 32;
            pair_step = 64;
            call.add({W_in->re, w_in.re, W_in->ld, dp, 2 * up(hidden, 32), hidden, (int32_t)dim, 0});
        }
        call.copies();
        const int64_t columns = 2 * up(hidden, 32);
        if (fg_status st = call.product(GATED_UP, tokens, columns, dp, 0, x, w_in, [&](GatedParams &p) {
                p.b_span = up(((copy_in ? columns : 2 * hidden) - 1) * w_in.ld + dp, 8);
                p.D = (float *)h.re; p.ldd = hp;
                p.keep = keep; p.ldgu = ldkeep;
                p.pair = pair; p.pair_step = pair_step;
                p.hidden = (int32_t)hidden; p.act = activation;
            })) return st;
    }
    if (at.parts == 2) {
        const fg_matrix sums = rows_of(call.space + at.sums, FG_F32, up(dim, 4));
        if (fg_status st = call.by_sums(at, 2 * tokens, dim, hp, 0, h, turned(w_out), sums)) return st;
        call.round<true>(sums, Y, tokens, dim);
        return call.enqueue.status("gated_round");
    }
    return call.rounded(at, at.sums, at.down_by_sums, GATED_ROUND_KK, tokens, dim, hp, 0, h, w_out, Y);
}

int64_t fg_gated_ffn_grad_workspace(int64_t tokens, int64_t dim, int64_t hidden) {
    if (tokens <= 0 || dim <= 0 || hidden <= 0 || !in_range(tokens, dim, hidden) || !few_tiles(tokens, dim, hidden)) return 0;
    return GradSpace(tokens, dim, hidden, true, true, true, true).bytes;
}

fg_status fg_gated_ffn_grad(int64_t tokens, int64_t dim, int64_t hidden, const fg_matrix *dY, const fg_matrix *X, const fg_matrix *W_in,
                            const fg_matrix *W_out, int32_t act, const fg_matrix *GU, const fg_matrix *dX, const fg_matrix *dW_in, const fg_matrix *dW_out,
                            void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_gated(tokens, dim, hidden, X, W_in, W_out, act)) return st;
    if (fg_status st = check_like("dY", dY, tokens, dim, X->dtype)) return st;
    if (fg_status st = check_like("GU", GU, tokens, 2 * hidden, FG_F32)) return st;
    if (dX) if (fg_status st = check_like("dX", dX, tokens, dim, X->dtype)) return st;
    if (dW_in) if (fg_status st = check_like("dW_in", dW_in, 2 * hidden, dim, X->dtype)) return st;
    if (dW_out) if (fg_status st = check_like("dW_out", dW_out, dim, hidden, X->dtype)) return st;
    if (dim == 0) return FG_OK;
    const Rows operands[] = {{"dY", dY, tokens, dim}, {"X", X, tokens, dim}, {"W_in", W_in, 2 * hidden, dim}, {"W_out", W_out, dim, hidden}},
               results[] = {{"dX", dX, tokens, dim}, {"dW_in", dW_in, 2 * hidden, dim}, {"dW_out", dW_out, dim, hidden}}, kept = {"GU", GU, tokens, 2 * hidden};
    for (const Rows &out : results)
        for (const Rows &in : operands)
            if (fg_status st = check_elsewhere(out, in)) return st;
    Call call = {Launches(hip_stream), (char *)workspace, X->dtype};
    if (tokens == 0 || hidden == 0) {
        const fg_matrix none = rows_of(nullptr, FG_F32, 0);
        if (dX && tokens > 0) call.round<false>(none, dX, tokens, dim);
        if (dW_in && hidden > 0) call.round<false>(none, dW_in, 2 * hidden, dim);
        if (dW_out && hidden > 0) call.round<false>(none, dW_out, dim, hidden);
        return call.enqueue.status("gated_round");
    }
    if (!dX && !dW_in && !dW_out) return FG_OK;
    for (const Rows &out : results)
        if (fg_status st = check_elsewhere(out, kept)) return st;
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (fg_status st = check_elsewhere(results[i], results[j])) return st;
    const bool copy_dy = !as_it_is(dim, dY), copy_x = !as_it_is(dim, X), copy_in = !as_it_is(dim, W_in), copy_out = !as_it_is(hidden, W_out);
    const GradSpace at(tokens, dim, hidden, copy_dy, copy_x, copy_in, copy_out);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    const int64_t dp = up(dim, 8), hp = up(hidden, 8), gp = up(2 * hidden, 8), rows = at.parts * tokens, tp = up(rows, 8);
    const fg_matrix dy = call.aligned(dY, tokens, dim, copy_dy, at.dy, at.times), w_out = call.aligned(W_out, dim, hidden, copy_out, at.w_out),
                    w_in = dX ? call.aligned(W_in, 2 * hidden, dim, copy_in, at.w_in) : *W_in, x = dW_in && !at.few ? call.aligned(X, tokens, dim, copy_x, at.x, at.times) : *X;
    call.copies();
    const fg_matrix h = rows_of(call.space + at.h, X->dtype, hp), dgu = rows_of(call.space + at.dgu, X->dtype, gp);
    const Activation activation = Activation::of(act);
    if (at.down_by_sums) {
        const fg_matrix dh = rows_of(call.space + at.dh, FG_F32, up(hidden, 4));
        if (fg_status st = call.by_sums(at, tokens, hidden, dp, dim, dy, w_out, dh)) return st;
        with_half(X->dtype, [&](auto t) {
            using T = decltype(t);
            auto pass = [&](auto kernel) {
                call.enqueue(kernel, dim3(groups_for(tokens, hidden)), dim3(256), (const float *)GU->re, GU->ld, (const float *)dh.re, dh.ld, (T *)h.re, hp, (T *)dgu.re, gp,
                             tokens, (int)hidden, activation);
            };
            if (at.parts == 2) pass(gated_product_grad<T, true>);
            else pass(gated_product_grad<T, false>);
        });
        if (fg_status st = call.enqueue.status("gated_product_grad")) return st;
    } else if (fg_status st = call.product(GATED_DOWN, tokens, hidden, dp, dim, dy, w_out, [&](GatedParams &p) {
                   p.D = (float *)dgu.re; p.ldd = gp;
                   p.h = h.re; p.ldh = hp;
                   p.gu = (const float *)GU->re; p.ldgu = GU->ld;
                   p.hidden = (int32_t)hidden; p.act = activation;
               })) return st;
    if (dX) {
        if (at.parts == 2) {
            const fg_matrix sums = rows_of(call.space + at.sums, FG_F32, up(dim, 4));
            if (fg_status st = call.by_sums(at, rows, dim, gp, 2 * hidden, dgu, w_in, sums)) return st;
            call.round<true>(sums, dX, tokens, dim);
        } else if (fg_status st = call.rounded(at, at.sums, at.x_by_sums, GATED_ROUND_KN, tokens, dim, gp, 2 * hidden, dgu, w_in, dX)) return st;
    }
    if (at.few) {
        with_half(X->dtype, [&](auto t) {
            using T = decltype(t);
            const int32_t again = at.parts == 2 ? (int32_t)tokens : 0;          // (both parts of a token have its row of x and dy)
            DwOfFew<T> in = {(const T *)dgu.re, (const T *)X->re, nullptr, gp, gp, X->ld, 0, 0, dim, 0, 0, again},
                       out = {(const T *)dy.re, (const T *)h.re, nullptr, dy.ld, dp, hp, 0, 0, hidden, 0, again, 0};
            if (dW_in) { in.out = (T *)dW_in->re; in.ldo = dW_in->ld; in.words = 2 * hidden; }
            if (dW_out) { out.out = (T *)dW_out->re; out.ldo = dW_out->ld; out.words = dim; }
            if (dW_in || dW_out) launch_dw_of_few<T>(call.enqueue, in, out, nullptr, rows);
        });
        return call.enqueue.status("dw_of_few");
    }
    const int tile = dW_in && dW_out ? tile_of_both(at, 2 * hidden, dim, dim, hidden, rows) : -1;
    if (tile >= 0) return call.both_weights(tile, rows, dgu, x, dW_in, 2 * hidden, dim, dy, h, dW_out, dim, hidden);
    if (dW_in)
        if (fg_status st = call.rounded(at, at.sums, at.in_by_sums, GATED_ROUND_NN, 2 * hidden, dim, at.in_by_sums ? tp : rows, rows, dgu, x, dW_in)) return st;
    if (dW_out)
        if (fg_status st = call.rounded(at, at.sums, at.out_by_sums, GATED_ROUND_NN, dim, hidden, at.out_by_sums ? tp : rows, rows, dy, h, dW_out)) return st;
    return call.enqueue.status("gated_ffn_grad");
}

}  // extern "C"
