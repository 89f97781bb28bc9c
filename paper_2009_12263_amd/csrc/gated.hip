// Gated feed-forward block and its gradient.
//
//   [G U] = X W_in^T,   H = act(G) U,   Y = H W_out^T
//   dH = dY W_out,   dG = dH U act'(G),   dU = dH act(G),   dX = [dG dU] W_in,   dW_in = [dG dU]^T X,   dW_out = dY^T H
//
// 6 T D H operations forward (T tokens of D values, H hidden ones), 12 T D H backward, on the matrix units.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "kernel_table.hpp"
#include "row_ops.hpp"

namespace fg {
namespace {

constexpr float kLog2eG = 1.44269504088896340736f;

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + __builtin_amdgcn_exp2f(-kLog2eG * x)); }
// act(g), and its derivative
template <int ACT>
__device__ __forceinline__ void activate(float g, float &a, float &d) {
    if constexpr (ACT == FG_ACT_NONE) { a = g; d = 1.f; }
    else if constexpr (ACT == FG_ACT_RELU) { a = g > 0.f ? g : 0.f; d = g > 0.f ? 1.f : 0.f; }
    else if constexpr (ACT == FG_ACT_SILU) { const float q = sigmoid(g); a = g * q; d = q * (1.f + g * (1.f - q)); }
    else {
        // (1 + tanh u) / 2 = sigmoid(2 u), u = c (g + 0.044715 g^3)
        const float c2 = 2.f * 0.79788456080286535588f, q = sigmoid(c2 * (g + 0.044715f * g * g * g));
        a = g * q;
        d = q + c2 * g * q * (1.f - q) * (1.f + 3.f * 0.044715f * g * g);
    }
}
template <class F> void with_act(int act, F &&f) {
    switch (act) {
        case FG_ACT_NONE: f(std::integral_constant<int, FG_ACT_NONE>{}); break;
        case FG_ACT_RELU: f(std::integral_constant<int, FG_ACT_RELU>{}); break;
        case FG_ACT_SILU: f(std::integral_constant<int, FG_ACT_SILU>{}); break;
        default: f(std::integral_constant<int, FG_ACT_GELU_TANH>{});
    }
}

// Copies rows of `cols` values to rows of ldo (a multiple of 8), with zeros behind them.
template <class T>
__global__ __launch_bounds__(256) void gated_pad(const T *in, int64_t ld, T *out, int64_t ldo, int64_t rows, int cols) {
    const int pieces = (int)(ldo / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int p = (int)(i - row * pieces);
        const T *from = in + row * ld;
        typename RowPiece<T>::vec v;
        if ((p + 1) * 8 <= cols) v = load_raw<T, 8>(from, p, cols);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p * 8 + e < cols ? from[p * 8 + e] : (T)0.f;
        *(typename RowPiece<T>::vec *)(out + row * ldo + p * 8) = v;
    }
}

// h = act(g) u, rounded, in rows of ldh with zeros behind them; g and u are copied to `keep` where it is given
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_product(const float *gu, int64_t ldgu, T *h, int64_t ldh, int64_t rows, int hidden, float *keep, int64_t ldkeep) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * ldh; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / ldh;
        const int c = (int)(i - row * ldh);
        float a = 0.f, d = 0.f;
        if (c < hidden) {
            const float g = gu[row * ldgu + c], u = gu[row * ldgu + hidden + c];
            activate<ACT>(g, a, d);
            a *= u;
            if (keep) {
                keep[row * ldkeep + c] = g;
                keep[row * ldkeep + hidden + c] = u;
            }
        }
        h[i] = (T)a;
    }
}
// h as above, dg and du behind each other in rows of ldd with zeros behind them
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_product_grad(const float *gu, int64_t ldgu, const float *dh, int64_t lddh, T *h, int64_t ldh, T *dgu, int64_t ldd,
                                                          int64_t rows, int hidden) {
    const int64_t wide = ldd > ldh ? ldd : ldh;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * wide; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / wide;
        const int c = (int)(i - row * wide);
        if (c < hidden) {
            float a, d;
            activate<ACT>(gu[row * ldgu + c], a, d);
            const float u = gu[row * ldgu + hidden + c], x = dh[row * lddh + c];
            dgu[row * ldd + c] = (T)(x * u * d);
            dgu[row * ldd + hidden + c] = (T)(x * a);
            h[row * ldh + c] = (T)(a * u);
        } else {
            if (c < ldh) h[row * ldh + c] = (T)0.f;
            if (c >= 2 * hidden && c < ldd) dgu[row * ldd + c] = (T)0.f;
        }
    }
}
template <class T>
__global__ __launch_bounds__(256) void gated_round(const float *in, int64_t ldi, T *out, int64_t ldo, int64_t rows, int cols) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / cols;
        const int c = (int)(i - row * cols);
        out[row * ldo + c] = in ? (T)in[row * ldi + c] : (T)0.f;
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

// Where the parts of a workspace are.
struct Space {
    int64_t bytes = 0;
    int64_t take(int64_t n) { const int64_t at = bytes; bytes += up(n, 256); return at; }
};
struct ForwardSpace : Space {
    int64_t x, w_in, w_out, gu, h, sums, scratch, scratch_bytes;
    ForwardSpace(int64_t T, int64_t D, int64_t H, bool copy_x, bool copy_in, bool copy_out, bool has_gu) {
        const int64_t dp = up(D, 8), hp = up(H, 8);
        x = copy_x ? take(T * dp * 2) : 0;
        w_in = copy_in ? take(2 * H * dp * 2) : 0;
        w_out = copy_out ? take(D * hp * 2) : 0;
        gu = has_gu ? 0 : take(T * up(2 * H, 4) * 4);
        h = take(T * hp * 2);
        sums = take(T * up(D, 4) * 4);
        scratch_bytes = std::max(gemm_stored_scratch(T, 2 * H, dp), gemm_stored_scratch(T, D, hp));
        scratch = take(scratch_bytes);
    }
};
struct GradSpace : Space {
    int64_t dy, x, w_in, w_out, dh, h, dgu, sums, scratch, scratch_bytes;
    GradSpace(int64_t T, int64_t D, int64_t H, bool copy_dy, bool copy_x, bool copy_in, bool copy_out) {
        const int64_t dp = up(D, 8), hp = up(H, 8), gp = up(2 * H, 8), tp = up(T, 8);
        dy = copy_dy ? take(T * dp * 2) : 0;
        x = copy_x ? take(T * dp * 2) : 0;
        w_in = copy_in ? take(2 * H * dp * 2) : 0;
        w_out = copy_out ? take(D * hp * 2) : 0;
        dh = take(T * up(H, 4) * 4);
        h = take(T * hp * 2);
        dgu = take(T * gp * 2);
        sums = take(std::max({T, 2 * H}) * up(D, 4) * 4 > D * up(H, 4) * 4 ? std::max({T, 2 * H}) * up(D, 4) * 4 : D * up(H, 4) * 4);
        scratch_bytes = std::max({gemm_stored_scratch(T, H, dp), gemm_stored_scratch(T, D, gp), gemm_stored_scratch(2 * H, D, tp), gemm_stored_scratch(D, H, tp)});
        scratch = take(scratch_bytes);
    }
};

fg_status check_gated(int64_t T, int64_t D, int64_t H, const fg_matrix *X, const fg_matrix *W_in, const fg_matrix *W_out, int32_t act) {
    if (T < 0 || D < 0 || H < 0) return fail(FG_ERR_SHAPE, "negative size: %lld tokens, %lld values, %lld hidden", (long long)T, (long long)D, (long long)H);
    if (T > (1 << 30) || D >= kLargestWidth || 2 * H >= kLargestWidth)
        return fail(FG_ERR_UNSUPPORTED, "more than 2^30 tokens, or dim or 2 hidden of 2^21 - 8 and more, are not supported");
    auto tiles = [](int64_t m, int64_t n) { return ((m + 63) / 64) * ((n + 63) / 64); };
    if (tiles(T, std::max(2 * H, D)) >= (1ll << 25) || tiles(2 * H, D) >= (1ll << 25)) return fail(FG_ERR_UNSUPPORTED, "products of more than 2^25 tiles are not supported");
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

unsigned groups_for(int64_t values, int each) { return (unsigned)std::min<int64_t>((values + 256 * each - 1) / (256 * each), 8192); }

// A call's operands and launches.
struct Call {
    Launches enqueue;
    char *space;
    int dtype;
    int64_t scratch, scratch_bytes;
    // m, or a copy at `at` whose rows are aligned and padded
    fg_matrix aligned(const fg_matrix *m, int64_t rows, int64_t cols, bool copy, int64_t at) {
        if (!copy) return *m;
        const int64_t ld = up(cols, 8);
        with_half(dtype, [&](auto t) {
            using T = decltype(t);
            enqueue(gated_pad<T>, dim3(groups_for(rows * ld, 8)), dim3(256), (const T *)m->re, m->ld, (T *)(space + at), ld, rows, (int)cols);
        });
        return rows_of(space + at, dtype, ld);
    }
    fg_status product(int64_t M, int64_t N, int64_t K, int64_t k_rows, const fg_matrix &a, const fg_matrix &b, const fg_matrix &d) {
        return gemm_stored(M, N, K, k_rows, 1.f, &a, &b, 0.f, nullptr, &d, (float *)(space + scratch), scratch_bytes, enqueue.stream);
    }
    void round(const fg_matrix &in, const fg_matrix *out, int64_t rows, int64_t cols) {
        with_half(dtype, [&](auto t) {
            using T = decltype(t);
            enqueue(gated_round<T>, dim3(groups_for(rows * cols, 1)), dim3(256), (const float *)in.re, in.ld, (T *)out->re, out->ld, rows, (int)cols);
        });
    }
};

}  // namespace

hipError_t load_gated_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)gated_round<f16_t>);
}

}  // namespace fg

using namespace fg;

extern "C" {

int64_t fg_gated_ffn_workspace(int64_t tokens, int64_t dim, int64_t hidden) {
    if (tokens <= 0 || dim <= 0 || hidden <= 0) return 0;
    return ForwardSpace(tokens, dim, hidden, true, true, true, false).bytes;
}

fg_status fg_gated_ffn(int64_t tokens, int64_t dim, int64_t hidden, const fg_matrix *X, const fg_matrix *W_in, const fg_matrix *W_out, int32_t act,
                       const fg_matrix *Y, const fg_matrix *GU, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_gated(tokens, dim, hidden, X, W_in, W_out, act)) return st;
    if (fg_status st = check_like("Y", Y, tokens, dim, X->dtype)) return st;
    if (GU) if (fg_status st = check_like("GU", GU, tokens, 2 * hidden, FG_F32)) return st;
    if (tokens == 0 || dim == 0) return FG_OK;
    Call call = {Launches(hip_stream), (char *)workspace, X->dtype, 0, 0};
    if (hidden == 0) {
        call.round(rows_of(nullptr, FG_F32, 0), Y, tokens, dim);
        return call.enqueue.status("gated_round");
    }
    const bool copy_x = !as_it_is(dim, X), copy_in = !as_it_is(dim, W_in), copy_out = !as_it_is(hidden, W_out);
    const bool own_gu = !GU || !aligned_to(GU->re, 16) || GU->ld % 4 != 0 || GU->ld >= kResultLd;        // (so that results do not depend on where GU is)
    const ForwardSpace at(tokens, dim, hidden, copy_x, copy_in, copy_out, !own_gu);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    call.scratch = at.scratch; call.scratch_bytes = at.scratch_bytes;
    const int64_t dp = up(dim, 8), hp = up(hidden, 8);
    const fg_matrix x = call.aligned(X, tokens, dim, copy_x, at.x), w_in = call.aligned(W_in, 2 * hidden, dim, copy_in, at.w_in),
                    w_out = call.aligned(W_out, dim, hidden, copy_out, at.w_out);
    const fg_matrix gu = !own_gu ? *GU : rows_of(call.space + at.gu, FG_F32, up(2 * hidden, 4)), h = rows_of(call.space + at.h, X->dtype, hp),
                    sums = rows_of(call.space + at.sums, FG_F32, up(dim, 4));
    if (fg_status st = call.product(tokens, 2 * hidden, dp, 0, x, turned(w_in), gu)) return st;
    with_half(X->dtype, [&](auto t) {
        using T = decltype(t);
        with_act(act, [&](auto a) {
            call.enqueue(gated_product<T, decltype(a)::value>, dim3(groups_for(tokens * hp, 1)), dim3(256), (const float *)gu.re, gu.ld, (T *)h.re, hp, tokens, (int)hidden,
                         own_gu && GU ? (float *)GU->re : nullptr, GU ? GU->ld : 0);
        });
    });
    if (fg_status st = call.product(tokens, dim, hp, 0, h, turned(w_out), sums)) return st;
    call.round(sums, Y, tokens, dim);
    return call.enqueue.status("gated_ffn");
}

int64_t fg_gated_ffn_grad_workspace(int64_t tokens, int64_t dim, int64_t hidden) {
    if (tokens <= 0 || dim <= 0 || hidden <= 0) return 0;
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
    Call call = {Launches(hip_stream), (char *)workspace, X->dtype, 0, 0};
    if (dim == 0) return FG_OK;
    if (tokens == 0 || hidden == 0) {
        const fg_matrix none = rows_of(nullptr, FG_F32, 0);
        if (dX && tokens > 0) call.round(none, dX, tokens, dim);
        if (dW_in && hidden > 0) call.round(none, dW_in, 2 * hidden, dim);
        if (dW_out && hidden > 0) call.round(none, dW_out, dim, hidden);
        return call.enqueue.status("gated_round");
    }
    if (!dX && !dW_in && !dW_out) return FG_OK;
    const bool copy_dy = !as_it_is(dim, dY), copy_x = !as_it_is(dim, X), copy_in = !as_it_is(dim, W_in), copy_out = !as_it_is(hidden, W_out);
    const GradSpace at(tokens, dim, hidden, copy_dy, copy_x, copy_in, copy_out);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    call.scratch = at.scratch; call.scratch_bytes = at.scratch_bytes;
    const int64_t dp = up(dim, 8), hp = up(hidden, 8), gp = up(2 * hidden, 8), tp = up(tokens, 8);
    const fg_matrix dy = call.aligned(dY, tokens, dim, copy_dy, at.dy), x = call.aligned(X, tokens, dim, copy_x, at.x),
                    w_in = call.aligned(W_in, 2 * hidden, dim, copy_in, at.w_in), w_out = call.aligned(W_out, dim, hidden, copy_out, at.w_out);
    const fg_matrix dh = rows_of(call.space + at.dh, FG_F32, up(hidden, 4)), h = rows_of(call.space + at.h, X->dtype, hp),
                    dgu = rows_of(call.space + at.dgu, X->dtype, gp);
    auto sums = [&](int64_t cols) { return rows_of(call.space + at.sums, FG_F32, up(cols, 4)); };
    if (fg_status st = call.product(tokens, hidden, dp, dim, dy, w_out, dh)) return st;
    with_half(X->dtype, [&](auto t) {
        using T = decltype(t);
        with_act(act, [&](auto a) {
            call.enqueue(gated_product_grad<T, decltype(a)::value>, dim3(groups_for(tokens * gp, 1)), dim3(256), (const float *)GU->re, GU->ld, (const float *)dh.re, dh.ld,
                         (T *)h.re, hp, (T *)dgu.re, gp, tokens, (int)hidden);
        });
    });
    if (fg_status st = call.enqueue.status("gated_product_grad")) return st;
    if (dX) {
        if (fg_status st = call.product(tokens, dim, gp, 2 * hidden, dgu, w_in, sums(dim))) return st;
        call.round(sums(dim), dX, tokens, dim);
    }
    if (dW_in) {
        if (fg_status st = call.product(2 * hidden, dim, tp, tokens, turned(dgu), x, sums(dim))) return st;
        call.round(sums(dim), dW_in, 2 * hidden, dim);
    }
    if (dW_out) {
        if (fg_status st = call.product(dim, hidden, tp, tokens, turned(dy), h, sums(hidden))) return st;
        call.round(sums(hidden), dW_out, dim, hidden);
    }
    return call.enqueue.status("gated_ffn_grad");
}

}  // extern "C"
