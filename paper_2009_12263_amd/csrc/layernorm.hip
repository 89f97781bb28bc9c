// Layer norm of the rows of a matrix, and its gradient.
//
//   mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),  xh = (x - mean) rstd,  y = xh gamma + beta
//   g = dy gamma,  dx = rstd (g - sum g / n - xh sum (g xh) / n),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Bound by memory: x is read and y written once; x and dy are read and dx written once.  A row is held in the registers of W
// waves (up to kPieces pieces of 16 bytes per lane), so nothing is read twice and the variance is summed from the
// differences to the mean, without the cancellation of a mean of squares.  A lane keeps the same columns in every row that
// its workgroup takes: gamma and beta stay in registers, and so do the sums of dgamma and dbeta over those rows; each wave group
// writes its sums once, and a second pass adds them in a fixed order, so that results do not depend on scheduling.  All
// arithmetic is FP32; each result is rounded once, when it is stored.
#include "row_ops.hpp"

#include <algorithm>
#include <type_traits>

namespace fg {
namespace {

constexpr int kPieces = 2;                  // of 16 bytes per lane and row
constexpr int kMaxWaves = 16;
// Waves per SIMD that the registers of the gradient's kernels leave room for: with four, workgroups of eight and sixteen waves fill a unit; smaller ones
// do as well with three, and with fewer sums to add up (16384 x 2048 bfloat16 50.4 us with four, 45.2 with three).
constexpr int grad_waves(int w) { return w <= 4 ? 3 : 4; }

struct LayerNormArgs {
    const void *x, *dy;
    void *out;                              // y, or dx
    const void *gamma, *beta;
    float *mean, *rstd;
    float *partial;                         // per workgroup: dgamma's sums over its rows, then dbeta's (cols each)
    int64_t ldx, lddy, ldo, rows;
    int32_t cols;
    float eps, width;                       // width: cols, to divide by
    int64_t row0;                           // kernels with a workgroup for each row: the first one's
};

// Workgroups of one wave a row hold four rows, those of the gradient with two waves a row two: the sums of a workgroup's rows are added up before they
// are written (16384 x 1024 bfloat16, gradient: 40.9 us with sums of each wave, 24.1 so).
template <int W> constexpr int kRowsPerGroup = W == 1 ? 4 : 1;
template <int W> constexpr int kGradRows = W == 1 ? 4 : W == 2 ? 2 : 1;

template <class T, class P, int W, int R_>
struct RowLane {
    static constexpr int N = RowPiece<T>::N, NT = 64 * W, R = R_;
    using Raw = typename RowPiece<T>::vec;
    using Param = typename RowPiece<P, N>::vec;
    int lane, cols, pieces;
    int sub;                                // which of the workgroup's rows
    __device__ RowLane(int n) : lane(threadIdx.x % NT), cols(n), pieces((n + N - 1) / N), sub(R == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT)) {}
    __device__ __forceinline__ int64_t first_row() const { return (int64_t)blockIdx.x * R + sub; }
    // f(c, piece) for the pieces of this lane
    template <class F> __device__ __forceinline__ void each(F &&f) const {
#pragma unroll
        for (int c = 0; c < kPieces; ++c)
            if (lane + c * NT < pieces) f(c, lane + c * NT);
    }
    // f(e, own) for the elements of a piece; `own` is a constant but in a row's last piece, which can hold its neighbour's elements too
    template <class F> __device__ __forceinline__ void elements(int piece, F &&f) const {
        if ((piece + 1) * N <= cols) {
#pragma unroll
            for (int e = 0; e < N; ++e) f(e, true);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) f(e, own_element<N>(piece, cols, e));
        }
    }
    __device__ __forceinline__ void load(const T *row, Raw (&out)[kPieces]) const {
        each([&](int c, int p) { out[c] = load_raw<T, N>(row, p, cols); });
    }
    __device__ __forceinline__ void params(const void *p, Param (&out)[kPieces], float otherwise) const {
        each([&](int c, int piece) { out[c] = p ? load_raw<P, N>((const P *)p, piece, cols) : (Param)(P)otherwise; });
    }
};

// A workgroup requests its next row before it works on the one that it has: rows are on their way all the time.  (One row at a time: 16384x4096
// bfloat16 97 us.)
template <class T, class P, int W>
__global__ __launch_bounds__(64 * W * kRowsPerGroup<W>) void layernorm(const LayerNormArgs a) {
    using Lane = RowLane<T, P, W, kRowsPerGroup<W>>;
    constexpr int N = Lane::N;
    __shared__ float slots[2][W];
    const Lane l(a.cols);
    const int64_t step = (int64_t)gridDim.x * Lane::R;
    typename Lane::Param gamma[kPieces], beta[kPieces];
    typename Lane::Raw ahead[kPieces];
    if (l.first_row() < a.rows) l.load((const T *)a.x + l.first_row() * a.ldx, ahead);
    l.params(a.gamma, gamma, 1.f);
    l.params(a.beta, beta, 0.f);
    for (int64_t row = l.first_row(); row < a.rows; row += step) {
        T *y = (T *)a.out + row * a.ldo;
        float v[kPieces][N], sum = 0.f, square = 0.f;
        l.each([&](int c, int) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[c][i] = (float)ahead[c][i];
        });
        if (row + step < a.rows) l.load((const T *)a.x + (row + step) * a.ldx, ahead);
        l.each([&](int c, int p) { l.elements(p, [&](int i, bool own) { sum += own ? v[c][i] : 0.f; }); });
        const float mean = group_sum<W>(sum, slots[0]) / a.width;
        l.each([&](int c, int p) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[c][i] -= mean;
            l.elements(p, [&](int i, bool own) { square += own ? v[c][i] * v[c][i] : 0.f; });
        });
        const float rstd = 1.f / __builtin_sqrtf(group_sum<W>(square, slots[1]) / a.width + a.eps);
        l.each([&](int c, int p) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[c][i] = v[c][i] * rstd * (float)gamma[c][i] + (float)beta[c][i];
            store_piece(y, p, a.cols, v[c]);
        });
        if (l.lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <class T, class P, int W, bool SUMS>
__global__ __launch_bounds__(64 * W * kGradRows<W>, grad_waves(W)) void layernorm_grad(const LayerNormArgs a) {
    using Lane = RowLane<T, P, W, kGradRows<W>>;
    constexpr int N = Lane::N, R = Lane::R;
    __shared__ float slots[4][R][W], pool[SUMS && R > 1 ? 2 : 1][SUMS && R > 1 ? 64 * W * kPieces * N : 1];
    // Large workgroups have no registers left for gamma: each lane keeps its part in LDS.  (A spilled register is reloaded in the order of the loads, behind
    // the next row: 16384 x 8192 binary16, FP32 parameters, 182 us with four spilled, 163 so.  Of the kernels of eight waves those of bfloat16 have two spilled all the
    // same: 16384 x 5120 118 to 122 us, binary16 102; 16384 x 8192 154 to 163, binary16 162 to 168.)
    constexpr bool LDS = W >= 8;
    __shared__ __attribute__((aligned(16))) float4 gamma_of[LDS ? kPieces : 1][LDS ? N / 4 : 1][LDS ? 64 * W : 1];
    const Lane l(a.cols);
    const int64_t step = (int64_t)gridDim.x * R;
    typename Lane::Param gamma[kPieces];
    typename Lane::Raw ahead_x[kPieces], ahead_dy[kPieces];
    float ahead_mean = 0.f, ahead_rstd = 0.f, sum_gamma[SUMS ? kPieces : 1][N] = {}, sum_beta[SUMS ? kPieces : 1][N] = {};
    auto load = [&](int64_t row) {
        ahead_mean = a.mean[row];
        ahead_rstd = a.rstd[row];
        l.load((const T *)a.x + row * a.ldx, ahead_x);
        l.load((const T *)a.dy + row * a.lddy, ahead_dy);
    };
    l.params(a.gamma, gamma, 1.f);
    if constexpr (LDS)
        l.each([&](int c, int) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) gamma_of[c][q][threadIdx.x] = make_float4((float)gamma[c][4 * q], (float)gamma[c][4 * q + 1], (float)gamma[c][4 * q + 2], (float)gamma[c][4 * q + 3]);
        });
    auto times_gamma = [&](int c, const float (&d)[N], float (&g)[N]) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            if constexpr (LDS) {
                const float4 v = gamma_of[c][q][threadIdx.x];
                g[4 * q] = d[4 * q] * v.x; g[4 * q + 1] = d[4 * q + 1] * v.y; g[4 * q + 2] = d[4 * q + 2] * v.z; g[4 * q + 3] = d[4 * q + 3] * v.w;
            } else {
#pragma unroll
                for (int i = 4 * q; i < 4 * q + 4; ++i) g[i] = d[i] * (float)gamma[c][i];
            }
        }
    };
    if (l.first_row() < a.rows) load(l.first_row());
    int turn = 0;
    // All rows of a workgroup go round together, for the barriers of their sums; those past the last row do nothing in between.
    for (int64_t row = l.first_row(); row - l.sub < a.rows; row += step) {
        const bool on = R == 1 || row < a.rows;
        const float mean = ahead_mean, rstd = ahead_rstd;
        typename Lane::Raw x[kPieces], dy[kPieces];
        float s1 = 0.f, s2 = 0.f;
        if (on) {
            l.each([&](int c, int) { x[c] = ahead_x[c]; dy[c] = ahead_dy[c]; });
            if (row + step < a.rows) load(row + step);
            l.each([&](int c, int p) {
                float d[N], g[N];
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = (float)dy[c][i];
                times_gamma(c, d, g);
                l.elements(p, [&](int i, bool own) {
                    const float xh = ((float)x[c][i] - mean) * rstd;
                    if constexpr (SUMS) {                               // (those of other pieces' elements are not stored)
                        sum_gamma[c][i] += d[i] * xh;
                        sum_beta[c][i] += d[i];
                    }
                    s1 += own ? g[i] : 0.f;
                    s2 += own ? g[i] * xh : 0.f;
                });
            });
        }
        const float c1 = group_sum<W>(s1, slots[turn][l.sub]) / a.width, c2 = group_sum<W>(s2, slots[turn + 1][l.sub]) / a.width;
        turn ^= 2;
        if (!on) continue;
        T *dx = (T *)a.out + row * a.ldo;
        l.each([&](int c, int p) {
            float d[N], o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = (float)dy[c][i];
            times_gamma(c, d, o);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float xh = ((float)x[c][i] - mean) * rstd;
                o[i] = rstd * (o[i] - c1 - xh * c2);
            }
            store_piece(dx, p, a.cols, o);
        });
    }
    if constexpr (SUMS) {
        float *to = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
        if constexpr (R == 1) {
            l.each([&](int c, int p) {
                store_piece(to, p, a.cols, sum_gamma[c]);
                store_piece(to + a.cols, p, a.cols, sum_beta[c]);
            });
        } else {
            for (int r = 0; r < R; ++r) {               // in the order of the rows
                if (l.sub == r)
                    l.each([&](int c, int p) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (own_element<N>(p, a.cols, i)) {
                                const int col = first_of_piece<N>(p, a.cols) + i;
                                pool[0][col] = (r ? pool[0][col] : 0.f) + sum_gamma[c][i];
                                pool[1][col] = (r ? pool[1][col] : 0.f) + sum_beta[c][i];
                            }
                    });
                __syncthreads();
            }
            for (int col = threadIdx.x; col < a.cols; col += 64 * W * R) {
                to[col] = pool[0][col];
                to[a.cols + col] = pool[1][col];
            }
        }
    }
}

// ---- rows that the registers do not hold --------------------------------------------------------
// One workgroup a row, which is read again for each sum (from the L2).
template <class T, class P>
__global__ __launch_bounds__(1024) void layernorm_wide(const LayerNormArgs a) {
    constexpr int N = RowPiece<T>::N;
    __shared__ float slots[2][16];
    const int n = a.cols, pieces = (n + N - 1) / N;
    const int64_t row = a.row0 + blockIdx.x;
    const T *x = (const T *)a.x + row * a.ldx;
    T *y = (T *)a.out + row * a.ldo;
    float v[N], sum = 0.f, square = 0.f;
    for (int p = threadIdx.x; p < pieces; p += 1024) {
        load_piece(x, p, n, v);
#pragma unroll
        for (int i = 0; i < N; ++i) sum += own_element<N>(p, n, i) ? v[i] : 0.f;
    }
    const float mean = group_sum<16>(sum, slots[0]) / a.width;
    for (int p = threadIdx.x; p < pieces; p += 1024) {
        load_piece(x, p, n, v);
#pragma unroll
        for (int i = 0; i < N; ++i) square += own_element<N>(p, n, i) ? (v[i] - mean) * (v[i] - mean) : 0.f;
    }
    const float rstd = 1.f / __builtin_sqrtf(group_sum<16>(square, slots[1]) / a.width + a.eps);
    const P *gamma = (const P *)a.gamma, *beta = (const P *)a.beta;
    for (int p = threadIdx.x; p < pieces; p += 1024) {
        load_piece(x, p, n, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int col = first_of_piece<N>(p, n) + i;
            v[i] = (v[i] - mean) * rstd * (gamma ? (float)gamma[col] : 1.f) + (beta ? (float)beta[col] : 0.f);
        }
        store_piece(y, p, n, v);
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

template <class T, class P>
__global__ __launch_bounds__(1024) void layernorm_grad_wide(const LayerNormArgs a) {
    constexpr int N = RowPiece<T>::N;
    __shared__ float slots[2][16];
    const int n = a.cols, pieces = (n + N - 1) / N;
    const int64_t row = a.row0 + blockIdx.x;
    const T *x = (const T *)a.x + row * a.ldx, *dy = (const T *)a.dy + row * a.lddy;
    T *dx = (T *)a.out + row * a.ldo;
    const P *gamma = (const P *)a.gamma;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float xh[N], g[N], s1 = 0.f, s2 = 0.f;
    auto load = [&](int p) {
        load_piece(x, p, n, xh);
        load_piece(dy, p, n, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            xh[i] = (xh[i] - mean) * rstd;
            if (gamma) g[i] *= (float)gamma[first_of_piece<N>(p, n) + i];
        }
    };
    for (int p = threadIdx.x; p < pieces; p += 1024) {
        load(p);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s1 += own_element<N>(p, n, i) ? g[i] : 0.f;
            s2 += own_element<N>(p, n, i) ? g[i] * xh[i] : 0.f;
        }
    }
    const float c1 = group_sum<16>(s1, slots[0]) / a.width, c2 = group_sum<16>(s2, slots[1]) / a.width;
    for (int p = threadIdx.x; p < pieces; p += 1024) {
        load(p);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = rstd * (g[i] - c1 - xh[i] * c2);
        store_piece(dx, p, n, g);
    }
}

// The columns' sums over every gridDim.y-th row, for such rows (before dx is written, which may be in place).
template <class T>
__global__ __launch_bounds__(256) void layernorm_column_sums(const LayerNormArgs a) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= a.cols) return;
    float sum_gamma = 0.f, sum_beta = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float d = (float)((const T *)a.dy)[row * a.lddy + col];
        sum_gamma += d * (((float)((const T *)a.x)[row * a.ldx + col] - a.mean[row]) * a.rstd[row]);
        sum_beta += d;
    }
    float *to = a.partial + (int64_t)blockIdx.y * 2 * a.cols;
    to[col] = sum_gamma;
    to[a.cols + col] = sum_beta;
}

// ---- second pass of the columns' sums ---------------------------------------------------------------
// A workgroup adds the `groups` sums of 32 of the 2 cols columns: 32 lanes along the columns, 32 runs of groups side by
// side, which are then added in order.
template <class P>
__global__ __launch_bounds__(1024) void layernorm_sums(const float *partial, int groups, int64_t cols, int64_t group0, P *dgamma, P *dbeta) {
    __shared__ float part[32][33];
    const int at = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t col = (group0 + blockIdx.x) * 32 + at;
    const int each = (groups + 31) / 32, first = run * each, last = min(first + each, groups);
    float sum = 0.f;
    if (col < 2 * cols) {
#pragma unroll 4
        for (int g = first; g < last; ++g) sum += partial[g * 2 * cols + col];
    }
    part[run][at] = sum;
    __syncthreads();
    if (run == 0 && col < 2 * cols) {
        for (int r = 1; r < 32; ++r) sum += part[r][at];
        if (col < cols) { if (dgamma) dgamma[col] = (P)sum; }
        else if (dbeta) dbeta[col - cols] = (P)sum;
    }
}

// ---- host ------------------------------------------------------------------------------------------
constexpr int kNumCU = 256;

// How many waves hold a row: as few as its pieces need; 0: too wide.
int waves_for(int64_t cols, int elem) {
    const int64_t pieces = (cols * elem + 15) / 16;
    for (int w = 1; w <= kMaxWaves; w *= 2)
        if (pieces <= (int64_t)64 * w * kPieces) return w;
    return 0;
}
// How many workgroups share the rows of a gradient: enough to fill the GPU, and no more sums than that for the second pass.
int64_t grad_groups(int64_t rows, int64_t cols, int elem) {
    const int w = waves_for(cols, elem);
    if (w == 0) return std::min<int64_t>(rows, 64);
    const int rows_each = w == 1 ? kGradRows<1> : w == 2 ? kGradRows<2> : 1;
    return std::min<int64_t>((rows + rows_each - 1) / rows_each, kNumCU * 4 * grad_waves(w) / (w * rows_each));
}

template <class F> fg_status with_type(int dtype, F &&f) {
    switch (dtype) {
        case FG_F16: return f(f16_t{});
        case FG_BF16: return f(bf16_t{});
        default: return f(float{});
    }
}
// f(element, parameter): the parameters are FP32 or of the elements' type
template <class F> fg_status with_types(int dtype, int param_dtype, F &&f) {
    return with_type(dtype, [&](auto t) { return param_dtype == FG_F32 ? f(t, float{}) : f(t, t); });
}
template <class F> void with_waves(int w, F &&f) {
    switch (w) {
        case 1: f(std::integral_constant<int, 1>{}); break;
        case 2: f(std::integral_constant<int, 2>{}); break;
        case 4: f(std::integral_constant<int, 4>{}); break;
        case 8: f(std::integral_constant<int, 8>{}); break;
        default: f(std::integral_constant<int, 16>{});
    }
}

// A result that lies where an operand does has its rows where the operand's are: a workgroup writes only rows that no other reads.
fg_status check_in_place(const char *name, const fg_matrix *in, const char *out_name, const fg_matrix *out, int64_t rows) {
    if (rows > 1 && in->re == out->re && in->ld != out->ld)
        return fail(FG_ERR_LAYOUT, "%s in the place of %s must have its leading dimension", out_name, name);
    return FG_OK;
}

fg_status check_layernorm(int64_t rows, int64_t cols, const fg_matrix *X, const char *name, const fg_matrix *Y, const void *gamma, int32_t param_dtype) {
    if (rows < 0 || cols < 0) return fail(FG_ERR_SHAPE, "negative size: %lld rows of %lld", (long long)rows, (long long)cols);
    if (rows > (1 << 30) || cols > (1 << 30)) return fail(FG_ERR_UNSUPPORTED, "sizes above 2^30 are not supported");
    if (fg_status st = check_rows("X", X, rows, cols)) return st;
    if (fg_status st = check_rows(name, Y, rows, cols)) return st;
    if (X->dtype != Y->dtype) return fail(FG_ERR_UNSUPPORTED, "X and %s must have the same element type", name);
    if (cols > 0) if (fg_status st = check_in_place("X", X, name, Y, rows)) return st;
    if (param_dtype != FG_F32 && param_dtype != X->dtype) return fail(FG_ERR_LAYOUT, "gamma and beta must be FG_F32 or of the type of X");
    if (!aligned_to(gamma, element_bytes(param_dtype))) return fail(FG_ERR_ALIGN, "gamma must be aligned to an element");
    return FG_OK;
}

}  // namespace

hipError_t load_layernorm_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)layernorm<float, float, 1>);
}

}  // namespace fg

using namespace fg;

extern "C" {

fg_status fg_layernorm(int64_t rows, int64_t cols, const fg_matrix *X, const void *gamma, const void *beta, int32_t param_dtype, float eps,
                       const fg_matrix *Y, float *mean, float *rstd, void *hip_stream) {
    if (fg_status st = check_layernorm(rows, cols, X, "Y", Y, gamma, param_dtype)) return st;
    if (!(eps >= 0.f)) return fail(FG_ERR_SHAPE, "eps must not be negative");
    if (!aligned_to(beta, element_bytes(param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return fail(FG_ERR_ALIGN, "beta, mean and rstd must be aligned to an element");
    if (rows == 0 || cols == 0) return FG_OK;
    LayerNormArgs a = {X->re, nullptr, Y->re, gamma, beta, mean, rstd, nullptr, X->ld, 0, Y->ld, rows, (int32_t)cols, eps, (float)cols, 0};
    Launches enqueue(hip_stream);
    const int w = waves_for(cols, element_bytes(X->dtype));
    return with_types(X->dtype, param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        if (w == 0) in_parts(rows, [&](int64_t first, dim3 grid) {
            a.row0 = first;
            enqueue(layernorm_wide<T, P>, grid, dim3(1024), a);
        });
        else with_waves(w, [&](auto tag) {
            constexpr int W = tag, R = kRowsPerGroup<W>;
            static const int per_cu = [] {              // workgroups that fit a unit
                int n = 0;
                return hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void *)layernorm<T, P, W>, 64 * W * R, 0) == hipSuccess && n > 0 ? n : 1;
            }();
            const unsigned grid = (unsigned)std::min<int64_t>((rows + R - 1) / R, kNumCU * per_cu);
            enqueue(layernorm<T, P, W>, dim3(grid), dim3(64 * W * R), a);
        });
        return enqueue.status("layernorm");
    });
}

int64_t fg_layernorm_grad_workspace(int64_t rows, int64_t cols, int32_t dtype) {
    if (rows <= 0 || cols <= 0 || !element_bytes(dtype)) return 0;
    return grad_groups(rows, cols, element_bytes(dtype)) * 2 * cols * 4;
}

fg_status fg_layernorm_grad(int64_t rows, int64_t cols, const fg_matrix *dY, const fg_matrix *X, const void *gamma, int32_t param_dtype,
                            const float *mean, const float *rstd, const fg_matrix *dX, void *dgamma, void *dbeta,
                            void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_layernorm(rows, cols, X, "dX", dX, gamma, param_dtype)) return st;
    if (fg_status st = check_rows("dY", dY, rows, cols, true)) return st;
    if (dY->dtype != X->dtype) return fail(FG_ERR_UNSUPPORTED, "X and dY must have the same element type");
    if (cols > 0) if (fg_status st = check_in_place("dY", dY, "dX", dX, rows)) return st;
    const unsigned es = element_bytes(param_dtype);
    if (!aligned_to(dgamma, es) || !aligned_to(dbeta, es) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return fail(FG_ERR_ALIGN, "mean, rstd, dgamma and dbeta must be aligned to an element");
    if (cols == 0) return FG_OK;
    const bool sums = dgamma || dbeta;
    if (rows > 0 && (!mean || !rstd)) return fail(FG_ERR_NULL, "mean and rstd of the forward pass are NULL");
    const int64_t need = sums ? fg_layernorm_grad_workspace(rows, cols, X->dtype) : 0;
    if (fg_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    LayerNormArgs a = {X->re, dY->re, dX->re, gamma, nullptr, const_cast<float *>(mean), const_cast<float *>(rstd), (float *)workspace,
                       X->ld, dY->ld, dX->ld, rows, (int32_t)cols, 0.f, (float)cols, 0};
    Launches enqueue(hip_stream);
    const int w = waves_for(cols, element_bytes(X->dtype));
    const int64_t groups = rows > 0 ? grad_groups(rows, cols, element_bytes(X->dtype)) : 0;      // no row: the sums are zero
    return with_types(X->dtype, param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        if (rows > 0 && w == 0) {
            if (sums) enqueue(layernorm_column_sums<T>, dim3((unsigned)((cols + 255) / 256), (unsigned)groups), dim3(256), a);
            in_parts(rows, [&](int64_t first, dim3 grid) {
                a.row0 = first;
                enqueue(layernorm_grad_wide<T, P>, grid, dim3(1024), a);
            });
        } else if (rows > 0) with_waves(w, [&](auto tag) {
            constexpr int W = tag;
            const dim3 grid((unsigned)groups), block(64 * W * kGradRows<W>);
            if (sums) enqueue(layernorm_grad<T, P, W, true>, grid, block, a);
            else enqueue(layernorm_grad<T, P, W, false>, grid, block, a);
        });
        if (fg_status st = enqueue.status("layernorm_grad")) return st;
        if (!sums) return FG_OK;
        in_parts((2 * cols + 31) / 32, [&](int64_t first, dim3 grid) {
            enqueue(layernorm_sums<P>, grid, dim3(1024), (const float *)workspace, (int)groups, cols, first, (P *)dgamma, (P *)dbeta);
        });
        return enqueue.status("layernorm_sums");
    });
}

}  // extern "C"
