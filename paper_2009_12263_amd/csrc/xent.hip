// Softmax cross entropy of a linear layer over a vocabulary, and its gradient.
//
//   z[t][v] = scale x[t].w[v],   lse[t] = log sum over v of exp z[t][v],   loss[t] = lse[t] - z[t][target[t]]
//   dz[t][v] = (exp(z[t][v] - lse[t]) - [v = target[t]]) dloss[t],   dx[t] = scale dz[t].w,   dw[v] = scale sum over t of dz[t][v] x[t]
//
// The logits are as large as tokens x vocabulary and nobody wants them.  The vocabulary is walked in pieces: of a piece's logits, each token
// keeps the maximum and the sum of exponentials relative to it, and the logit of its target; the pairs (m, s) of all pieces are
// joined as sum s exp(m - max m).  The gradient forms a piece's logits again and turns them into dz, in 16 bits, which two products
// read: dw's rows of the piece, and the piece's part of dx, added up in FP32.
//
// The logits of a piece never leave the registers of the matrix kernels (xent_kernel.hpp).  Those take 16-byte aligned rows of a multiple of 8
// values; others are copied into the workspace first, padded with zeros, W a piece at a time (logits of such operands through
// memory, from the general matrix kernel to kernels on rows: 8192 tokens x 50000 words x 1001 with gradients 6516 us, 3122 so).
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "cache_policy.hpp"
#include "few_tokens.hpp"
#include "xent_kernel.hpp"

namespace fg {
namespace {

template <int W>
__device__ __forceinline__ float group_max(float v, float *slot) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = __builtin_fmaxf(v, slot[w]);
    return v;
}

// Piece p of eight of a row of `cols` values, zeros behind them.
template <class T>
__device__ __forceinline__ typename RowPiece<T>::vec padded_piece(const T *row, int p, int cols) {
    if ((p + 1) * 8 <= cols) return load_raw<T, 8>(row, p, cols);
    typename RowPiece<T>::vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p * 8 + e < cols ? row[p * 8 + e] : (T)0.f;
    return v;
}

// Copies rows of `cols` values to rows of ldo (a multiple of 8) that are aligned, with zeros behind them.
template <class T>
__global__ __launch_bounds__(256) void xent_pad(const T *in, int64_t ld, T *out, int64_t ldo, int64_t rows, int cols) {
    const int pieces = (int)(ldo / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int p = (int)(i - row * pieces);
        *(typename RowPiece<T>::vec *)(out + row * ldo + p * 8) = padded_piece(in + row * ld, p, cols);
    }
}

// ---- joining ----------------------------------------------------------------------------------------------
// A workgroup joins the statistics of 1024 / G tokens, G threads a token: each a G-th of the parts in turn, then by halves, always the same
// ones.  stats: `parts` runs of `stride` tokens.
template <int G>
__global__ __launch_bounds__(1024) void xent_join(const XentStat *stats, int parts, int64_t stride, int64_t tokens, const void *targets, bool wide, int vocab,
                                                  const float *z_target, float *loss, float *lse) {
    constexpr int TOKENS = 1024 / G;
    __shared__ XentStat part[G][TOKENS];
    const int at = threadIdx.x % TOKENS, g = threadIdx.x / TOKENS;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + at;
    XentStat sum = {-__builtin_inff(), 0.f};
    auto add = [&](XentStat o) {
        const float top = __builtin_fmaxf(sum.m, o.m), base = base_of(top);
        // (a part without anything has m = -inf and s = 0: exp of minus infinity, or of 0, times 0)
        sum.s = sum.s * __builtin_amdgcn_exp2f((sum.m - base) * kLog2e) + o.s * __builtin_amdgcn_exp2f((o.m - base) * kLog2e);
        sum.m = top;
    };
    if (t < tokens) {
#pragma unroll 4
        for (int p = g; p < parts; p += G) add(stats[p * stride + t]);
    }
    for (int half = G / 2; half > 0; half /= 2) {
        if (g >= half && g < 2 * half) part[g][at] = sum;
        __syncthreads();
        if (g < half) add(part[g + half][at]);
    }
    if (g != 0 || t >= tokens) return;
    const float total = base_of(sum.m) + __builtin_logf(sum.s);
    lse[t] = total;
    loss[t] = load_index(targets, wide, t, vocab) < 0 ? 0.f : total - z_target[t];
}

// ---- what the gradient's products begin with ---------------------------------------------------------------
// The first workgroup: the scaling of dz.  dz is kept as c dz, c = 2^k / max |dloss|.  With one dloss for all tokens (the mean of the losses) what is rounded is then exp(z - lse) - 1 or exp(z -
// lse) itself: relative to dloss, the same rounding of nearly -1 in every token would shift all of dx and dw one way (8192 tokens,
// bfloat16: error against 64 bits 2.6e-3 so, half of which is the rounding of the results).  Binary16: k = 14, so that |c dz|
// is at most 2^14 and what is 2^-38 of the largest is still a number.  With a dloss for each token the rounding of dz is one more beside that of the
// results (binary16, 2048 x 32768 x 1024: 2.8e-4 from 64 bits, with dz in FP32 2.1e-4): the matrix units take 16-bit operands.  factor[0] = c, factor[1] = scale / c.
//
// The others: x's rows for the products, aligned and padded like xent_pad's, with zeros for the tokens that are left out.  Their dz is zero, but a row of a
// token nobody asks for may hold anything, and in dw = dz^T x zero times infinity or NaN would reach every word.  (Beside the scaling's chain of latencies up
// to 64 tokens cost nothing, 4.1 us either way; looked up by dw_of_few instead, the targets took it from 41 to 47 us, with 64 tokens from 56 to 80.)
template <class T>
__global__ __launch_bounds__(1024) void xent_prepare(const float *dloss, int64_t dloss_inc, const void *targets, bool wide, int vocab, int64_t tokens, float scale,
                                                     float *factor, const T *x, int64_t ldx, T *out, int64_t ldo, int cols) {
    if (blockIdx.x > 0) {
        const int pieces = (int)(ldo / 8);
        for (int64_t i = (int64_t)(blockIdx.x - 1) * 1024 + threadIdx.x; i < tokens * pieces; i += (int64_t)(gridDim.x - 1) * 1024) {
            const int64_t t = i / pieces;
            const int p = (int)(i - t * pieces);
            typename RowPiece<T>::vec v = {};
            if (load_index(targets, wide, t, vocab) >= 0) v = padded_piece(x + t * ldx, p, cols);
            *(typename RowPiece<T>::vec *)(out + t * ldo + p * 8) = v;
        }
        return;
    }
    __shared__ float slots[16];
    float top = 0.f;
    for (int64_t t = threadIdx.x; t < tokens; t += 1024)
        if (load_index(targets, wide, t, vocab) >= 0) top = __builtin_fmaxf(top, __builtin_fabsf(dloss[t * dloss_inc]));
    top = group_max<16>(top, slots);
    if (threadIdx.x == 0) {
        const bool usable = top > 0.f && top < __builtin_inff();
        const float range = std::is_same<T, f16_t>::value ? 16384.f : 1.f, unit = usable ? __builtin_fmaxf(top, 1e-30f) : 1.f;
        factor[0] = usable ? range / unit : 1.f;
        factor[1] = usable ? scale * (unit / range) : scale;
    }
}

// rows x cols FP32 values times *factor (no `in`: zeros; no target: zeros in that row), rounded into `out`
template <class T>
__global__ __launch_bounds__(256) void xent_round(const float *in, int64_t ld, const float *factor, const void *targets, bool wide, int vocab, T *out, int64_t ldo,
                                                  int64_t rows, int cols) {
    const int pieces = (cols + 7) / 8;
    const float f = *factor;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int p = (int)(i - row * pieces);
        const bool live = in && load_index(targets, wide, row, vocab) >= 0;
        float v[8];
        if (live) load_piece(in + row * ld, p, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = live ? v[e] * f : 0.f;
        store_piece(out + row * ldo, p, cols, v);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = 256ll << 20;        // of dz: what the memory-side cache holds
constexpr int64_t kCopyBytes = 64ll << 20;          // of a piece of W that is copied
constexpr int64_t kTokenBlock = 16384;              // tokens whose statistics are kept at a time
constexpr int64_t kFewestWords = 256;               // of a piece; pieces begin at multiples of it
constexpr int64_t kMostWords = kKContiguousLd - kFewestWords;          // of a piece of dz, whose rows the product with dX reads along the words

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Words of a piece that cost `each` bytes a word, of `bytes` in all.
int64_t words_of(int64_t bytes, int64_t each, int64_t fewest, int64_t vocab) {
    return std::min(std::max(fewest, bytes / std::max<int64_t>(each, 1) / kFewestWords * kFewestWords), up(vocab, 8));
}

// Which tile of kernel_table_xent serves a product.
int xent_tile(int64_t M, int64_t N, int64_t K) {
    switch (plan_tile(M, N, K)) {
        case TILE_256x256: case TILE_256x256_K32: return 0;
        case TILE_256x128: case TILE_256x128_PASS: return 1;
        case TILE_64x64: case TILE_64x64_KG2: case TILE_64x64_KG2_DEEP: return 3;
        case TILE_64x128_KG2: return 4;
        default: return 2;
    }
}

// Which operands are copied.
struct Copies {
    bool x, w;
    Copies(bool x_, bool w_) : x(x_), w(w_) {}
    Copies(int64_t dim, const fg_matrix *X, const fg_matrix *W) {
        auto fits = [&](const fg_matrix *m) { return dim % 8 == 0 && aligned_to(m->re, 16) && m->ld % 8 == 0 && m->ld < kKContiguousLd; };
        x = !fits(X);
        w = !fits(W);
    }
};

// Workspaces.  Forward: the statistics of a block of tokens, the logits of their targets, and copies of operands.
struct StatsSpace {
    int64_t block, words, ld, stats, z_target, x, w, bytes;
    int tile;
    StatsSpace(int64_t words_, int64_t tokens, int64_t vocab, int64_t dim, Copies c) : block(std::min(tokens, kTokenBlock)), words(c.w ? words_ : up(vocab, 8)), ld(up(dim, 8)) {
        tile = xent_tile(block, std::min(words, vocab), dim);
        stats = 0;
        z_target = stats + up(up(vocab, 256) / kXentWaveColumns[tile] * block * (int64_t)sizeof(XentStat), 256);
        x = z_target + up(block * 4, 256);
        w = x + (c.x ? up(block * ld * 2, 256) : 0);
        bytes = w + (c.w ? words * ld * 2 : 0);
    }
    static int64_t preferred(int64_t, int64_t vocab, int64_t dim) { return words_of(kCopyBytes, up(dim, 8) * 2, kFewestWords, vocab); }
};
// Gradient: dz of a piece, the sums of dx, x without the rows of left-out tokens (xent_prepare), and a copy of w.  What the workspace has behind them serves a split of the product with dX.
struct GradSpace {
    int64_t words, ld, ld_dz, ld_dx, dz, dx, factor, x, w, bytes;
    GradSpace(int64_t words_, int64_t tokens, int64_t, int64_t dim, Copies c) : words(words_), ld(up(dim, 8)), ld_dz(up(words, 8)), ld_dx(up(dim, 4)) {
        dz = 0;
        dx = dz + up(tokens * ld_dz * 2, 256);
        factor = dx + up(tokens * ld_dx * 4, 256);
        x = factor + 256;
        w = x + up(tokens * ld * 2, 256);
        bytes = w + (c.w ? up(words * ld * 2, 256) : 0);
    }
    static int64_t preferred(int64_t tokens, int64_t vocab, int64_t) { return std::min(words_of(kPieceBytes, 2 * tokens, 2048, vocab), kMostWords); }
};
// The space of a call: pieces of the preferred size, or smaller ones that fit `bytes`.
template <class Space> Space space_within(int64_t bytes, int64_t tokens, int64_t vocab, int64_t dim, Copies c) {
    int64_t words = Space::preferred(tokens, vocab, dim);
    while (words > kFewestWords && Space(words, tokens, vocab, dim, c).bytes > bytes) words = std::max(kFewestWords, words / 2 / kFewestWords * kFewestWords);
    return Space(words, tokens, vocab, dim, c);
}
// What the queries give serves rows of any alignment: where dim lets the kernels take them as they are, each of the four combinations of copies, with W
// copied in the smallest pieces.  (No combination stands for another: the tile, and with it the statistics, follows the words of a piece.)
template <class Space> int64_t space_for(int64_t tokens, int64_t vocab, int64_t dim) {
    const int64_t words = Space::preferred(tokens, vocab, dim);
    if (dim % 8 != 0) return Space(words, tokens, vocab, dim, Copies(true, true)).bytes;
    int64_t bytes = 0;
    for (bool x : {false, true})
        for (bool w : {false, true}) bytes = std::max(bytes, Space(w ? std::min(kFewestWords, words) : words, tokens, vocab, dim, Copies(x, w)).bytes);
    return bytes;
}

// The partial products of dX's product, of the pieces that the preferred size gives.
int64_t grad_scratch(int64_t tokens, int64_t vocab, int64_t dim) {
    const int64_t words = GradSpace::preferred(tokens, vocab, dim), last = vocab % words;
    int64_t bytes = last > 0 ? gemm_stored_scratch(tokens, dim, up(last, 8)) : 0;
    if (vocab >= words) bytes = std::max(bytes, gemm_stored_scratch(tokens, dim, up(words, 8)));
    return bytes;
}

fg_status check_xent(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype) {
    if (tokens < 0 || vocab < 0 || dim < 0) return fail(FG_ERR_SHAPE, "negative size: %lld tokens, %lld words, %lld values", (long long)tokens, (long long)vocab, (long long)dim);
    if (vocab == 0) return fail(FG_ERR_SHAPE, "the vocabulary is empty");
    if (tokens > (1 << 30) || vocab > (1 << 30) || dim > (1 << 30)) return fail(FG_ERR_UNSUPPORTED, "sizes above 2^30 are not supported");
    if (dim >= (1 << 21)) return fail(FG_ERR_UNSUPPORTED, "rows of 2^21 values or more are not supported");
    if (fg_status st = check_rows("X", X, tokens, dim)) return st;
    if (fg_status st = check_rows("W", W, vocab, dim)) return st;
    if (X->dtype == FG_F32 || X->dtype != W->dtype) return fail(FG_ERR_UNSUPPORTED, "X and W must both be FG_F16 or both FG_BF16");
    return check_indices("targets", targets, index_dtype, tokens);
}

fg_matrix rows_of(const void *p, int32_t dtype, int64_t ld, int32_t layout = FG_ROW) { return {const_cast<void *>(p), nullptr, dtype, layout, ld}; }
const void *row_at(const fg_matrix *m, int64_t row) { return (const char *)m->re + row * m->ld * element_bytes(m->dtype); }

template <class F> void with_half(int dtype, F &&f) {
    if (dtype == FG_F16) f(f16_t{});
    else f(bf16_t{});
}

// The parameters of a product of the tiled kernels: M x N results, A and B both K-contiguous or both not.
XentParams product(const KernelEntry &k, bool kc, int64_t M, int64_t N, int64_t K, const void *A, int64_t lda, const void *B, int64_t ldb) {
    XentParams p;
    memset(&p, 0, sizeof p);
    p.M = (int32_t)M; p.N = (int32_t)N; p.K = (int32_t)K;
    p.tiles_m = (int32_t)((M + k.bm - 1) / k.bm); p.tiles_n = (int32_t)((N + k.bn - 1) / k.bn);
    p.A = (const _Float16 *)A; p.B = (const _Float16 *)B;
    p.a_rs = kc ? lda : 1; p.a_ks = kc ? 1 : lda;
    p.b_rs = kc ? ldb : 1; p.b_ks = kc ? 1 : ldb;
    p.a_span = up(kc ? (M - 1) * lda + K : (K - 1) * lda + M, 8);
    p.b_span = up(kc ? (N - 1) * ldb + K : (K - 1) * ldb + N, 8);
    p.rotate = kc && (p.tiles_m == 1 || p.tiles_n == 1);
    p.once = p.tiles_m == 1 && streams_once((uintptr_t)B, ldb, N * K * 2) ? 1 : p.tiles_n == 1 && streams_once((uintptr_t)A, lda, M * K * 2) ? 2 : 0;
    return p;
}

fg_status run_join(const XentStat *stats, int64_t parts, int64_t stride, int64_t tokens, const void *targets, bool wide, int64_t vocab, const float *z_target, float *loss,
                   float *lse, hipStream_t stream) {
    Launches enqueue(stream);
    auto launch = [&](auto tag) {
        constexpr int G = decltype(tag)::value, TOKENS = 1024 / G;
        enqueue(xent_join<G>, dim3((unsigned)((tokens + TOKENS - 1) / TOKENS)), dim3(1024), stats, (int)parts, stride, tokens, targets, wide, (int)vocab,
                           z_target, loss, lse);
    };
    // Enough workgroups to share the reads: 16 tokens of 2048 parts 20.2 us with 16 threads each, 6.0 with 256; 8192 of 1024 17.4 with 16.
    if (tokens <= 256) launch(std::integral_constant<int, 256>{});
    else if (tokens <= 4096) launch(std::integral_constant<int, 64>{});
    else launch(std::integral_constant<int, 16>{});
    return enqueue.status("xent_join");
}

// Rows row0 .. row0 + n - 1 of m as the matrix kernels take them: themselves, or copied to `to`.
fg_status aligned_rows(const fg_matrix *m, int64_t row0, int64_t n, int64_t dim, bool copy, void *to, int64_t ld, fg_matrix &out, hipStream_t stream) {
    out = rows_of(row_at(m, row0), m->dtype, m->ld);
    if (!copy || ld == 0) return FG_OK;
    Launches enqueue(stream);
    with_half(m->dtype, [&](auto t) {
        using T = decltype(t);
        const unsigned groups = (unsigned)std::min<int64_t>((n * (ld / 8) + 255) / 256, 8192);
        enqueue(xent_pad<T>, dim3(groups), dim3(256), (const T *)out.re, out.ld, (T *)to, ld, n, (int)dim);
    });
    out = rows_of(to, m->dtype, ld);
    return enqueue.status("xent_pad");
}

}  // namespace

const KernelEntry *kernel_table_xent_stats_f16();
const KernelEntry *kernel_table_xent_stats_bf16();
const KernelEntry *kernel_table_xent_dz_f16();
const KernelEntry *kernel_table_xent_dz_bf16();
const KernelEntry *kernel_table_xent_round_f16();
const KernelEntry *kernel_table_xent_round_bf16();
const KernelEntry *kernel_table_xent(int kind, bool bf16) {
    if (kind == XENT_STATS) return bf16 ? kernel_table_xent_stats_bf16() : kernel_table_xent_stats_f16();
    if (kind == XENT_DZ) return bf16 ? kernel_table_xent_dz_bf16() : kernel_table_xent_dz_f16();
    return bf16 ? kernel_table_xent_round_bf16() : kernel_table_xent_round_f16();
}


hipError_t load_xent_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)xent_join<16>);
}

}  // namespace fg

using namespace fg;

extern "C" {

int64_t fg_linear_xent_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens <= 0 || vocab <= 0 || dim < 0) return 0;
    return space_for<StatsSpace>(tokens, vocab, dim);
}

fg_status fg_linear_xent(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype,
                         float scale, float *loss, float *lse, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_xent(tokens, vocab, dim, X, W, targets, index_dtype)) return st;
    if (tokens == 0) return FG_OK;
    if (!loss || !lse) return fail(FG_ERR_NULL, "loss or lse is NULL");
    if (!aligned_to(loss, 4) || !aligned_to(lse, 4)) return fail(FG_ERR_ALIGN, "loss and lse must be aligned to an element");
    const Copies copies(dim, X, W);
    const auto at = space_within<StatsSpace>(workspace_bytes, tokens, vocab, dim, copies);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    char *space = (char *)workspace;
    const bool wide = index_dtype == FG_I64;
    const KernelEntry &k = kernel_table_xent(XENT_STATS, X->dtype == FG_BF16)[at.tile];
    for (int64_t t0 = 0; t0 < tokens; t0 += at.block) {
        const int64_t rows = std::min(at.block, tokens - t0);
        fg_matrix x, w;
        if (fg_status st = aligned_rows(X, t0, rows, dim, copies.x, space + at.x, at.ld, x, stream)) return st;
        XentStat *stats = (XentStat *)(space + at.stats);
        float *z_target = (float *)(space + at.z_target);
        const void *of_block = (const char *)targets + t0 * (wide ? 8 : 4);
        int64_t parts = 0;
        for (int64_t v0 = 0; v0 < vocab; v0 += at.words) {
            const int64_t n = std::min(at.words, vocab - v0);
            if (fg_status st = aligned_rows(W, v0, n, dim, copies.w, space + at.w, at.ld, w, stream)) return st;
            XentParams p = product(k, true, rows, n, at.ld, x.re, x.ld, w.re, w.ld);
            p.alpha = scale;
            p.stats = stats + parts * at.block;
            p.stats_stride = at.block;
            p.z_target = z_target;
            p.targets = of_block; p.wide = wide; p.vocab = (int32_t)vocab; p.v0 = (int32_t)v0;
            if (fg_status st = launch_product(k, p, stream)) return st;
            parts += up(n, k.bn) / kXentWaveColumns[at.tile];
        }
        if (fg_status st = run_join(stats, parts, at.block, rows, of_block, wide, vocab, z_target, loss + t0, lse + t0, stream)) return st;
    }
    return FG_OK;
}

int64_t fg_linear_xent_grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens < 0 || vocab <= 0 || dim <= 0) return 0;
    return space_for<GradSpace>(tokens, vocab, dim) + (tokens > 0 ? grad_scratch(tokens, vocab, dim) : 0);
}

fg_status fg_linear_xent_grad(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype,
                              float scale, const float *lse, const float *dloss, int64_t dloss_inc, const fg_matrix *dX, const fg_matrix *dW,
                              void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_xent(tokens, vocab, dim, X, W, targets, index_dtype)) return st;
    if (fg_status st = check_rows("dX", dX, tokens, dim)) return st;
    if (fg_status st = check_rows("dW", dW, vocab, dim)) return st;
    if (dX->dtype != X->dtype || dW->dtype != X->dtype) return fail(FG_ERR_UNSUPPORTED, "dX and dW must have the element type of X");
    if (up(dim, 4) >= kResultLd) return fail(FG_ERR_UNSUPPORTED, "gradients of rows of more than 2^21 - 4 values are not supported");
    if (dloss_inc != 0 && dloss_inc != 1) return fail(FG_ERR_SHAPE, "dloss_inc must be 0 or 1");
    if (dim == 0) return FG_OK;
    if (tokens > 0 && (!lse || !dloss)) return fail(FG_ERR_NULL, "lse or dloss is NULL");
    if (!aligned_to(lse, 4) || !aligned_to(dloss, 4)) return fail(FG_ERR_ALIGN, "lse and dloss must be aligned to an element");
    const Copies copies(dim, X, W);
    const auto at = space_within<GradSpace>(workspace_bytes, tokens, vocab, dim, copies);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    Launches enqueue(stream);
    char *space = (char *)workspace;
    const bool wide = index_dtype == FG_I64, bf16 = X->dtype == FG_BF16;
    float *sums = (float *)(space + at.dx), *factor = (float *)(space + at.factor);
    auto round = [&](const float *in, const fg_matrix *out, int64_t rows) {
        const unsigned groups = (unsigned)std::min<int64_t>((rows * ((dim + 7) / 8) + 255) / 256, 8192);
        with_half(X->dtype, [&](auto t) {
            using T = decltype(t);
            enqueue(xent_round<T>, dim3(groups), dim3(256), in, at.ld_dx, factor + 1, targets, wide, (int)vocab, (T *)out->re, out->ld, rows,
                               (int)dim);
        });
        return enqueue.status("xent_round");
    };
    const fg_matrix x = rows_of(space + at.x, X->dtype, at.ld);
    fg_matrix w;
    with_half(X->dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t groups = std::min<int64_t>((tokens * (at.ld / 8) + 1023) / 1024, 2048);
        enqueue(xent_prepare<T>, dim3((unsigned)(1 + groups)), dim3(1024), dloss, dloss_inc, targets, wide,
                           (int)vocab, tokens, scale, factor, (const T *)X->re, X->ld, (T *)(space + at.x), at.ld, (int)dim);
    });
    if (fg_status st = enqueue.status("xent_prepare")) return st;
    if (tokens == 0) return round(nullptr, dW, vocab);
    const fg_matrix dz = rows_of(space + at.dz, X->dtype, at.ld_dz), sum_dx = rows_of(sums, FG_F32, at.ld_dx);
    for (int64_t v0 = 0; v0 < vocab; v0 += at.words) {
        const int64_t n = std::min(at.words, vocab - v0);
        if (fg_status st = aligned_rows(W, v0, n, dim, copies.w, space + at.w, at.ld, w, stream)) return st;
        const KernelEntry &kz = kernel_table_xent(XENT_DZ, bf16)[xent_tile(tokens, n, dim)];
        XentParams p = product(kz, true, tokens, n, at.ld, x.re, x.ld, w.re, w.ld);
        p.alpha = scale;
        p.targets = targets; p.wide = wide; p.vocab = (int32_t)vocab; p.v0 = (int32_t)v0;
        p.lse = lse; p.dloss = dloss; p.dloss_inc = (int32_t)dloss_inc; p.factor = factor;
        p.D = (float *)dz.re; p.ldd = at.ld_dz;
        if (fg_status st = launch_product(kz, p, stream)) return st;
        if (tokens <= kFewTokens) {
            with_half(X->dtype, [&](auto t) {
                using T = decltype(t);
                launch_dw_of_few<T>(enqueue, {(const T *)dz.re, (const T *)x.re, (T *)row_at(dW, v0), at.ld_dz, at.ld_dz, x.ld, dW->ld, n, dim, 0, 0, 0}, {}, factor, tokens);
            });
            if (fg_status st = enqueue.status("dw_of_few")) return st;
        } else {
            // neither operand is K-contiguous: any number of tokens
            const KernelEntry &kw = kernel_table_xent(XENT_ROUND, bf16)[xent_tile(n, dim, tokens)];
            XentParams q = product(kw, false, n, dim, tokens, dz.re, at.ld_dz, x.re, x.ld);
            q.factor = factor;
            q.D = (float *)row_at(dW, v0); q.ldd = dW->ld;
            if (fg_status st = launch_product(kw, q, stream)) return st;
        }
        // dz has zeros from n on to the next multiple of 8
        if (fg_status st = gemm_stored(tokens, dim, up(n, 8), n, 1.f, &dz, &w, v0 == 0 ? 0.f : 1.f, &sum_dx, &sum_dx, (float *)(space + at.bytes),
                                        workspace_bytes - at.bytes, stream))
            return st;
    }
    return round(sums, dX, tokens);
}

}  // extern "C"
