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
// Operands that meet the alignment of the tiled kernels: a piece's logits never leave the registers (xent_kernel.hpp).  Others: they
// pass through the workspace, from fg_gemm to the kernels on rows below.
#include <algorithm>
#include <cstring>

#include "cache_policy.hpp"
#include "xent_kernel.hpp"

namespace fg {
namespace {

using Stat = XentStat;

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

// ---- pieces of the logits in memory ---------------------------------------------------------------------
// Statistics of token blockIdx.x over the n logits of a piece that begins at word v0; rows are long enough for whole pieces of 8.
__global__ __launch_bounds__(256) void xent_row_stats(const float *z, int64_t ld, int n, int v0, const void *targets, bool wide, int vocab, Stat *stats, float *z_target) {
    __shared__ float slots[2][4];
    const int64_t t = blockIdx.x;
    const float *row = z + t * ld;
    const int pieces = (n + 3) / 4;
    float m = -__builtin_inff(), s = 0.f, v[4];
    for (int p = threadIdx.x; p < pieces; p += 256) {
        load_piece(row, p, pieces * 4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __builtin_fmaxf(m, p * 4 + i < n ? v[i] : -__builtin_inff());
    }
    m = group_max<4>(m, slots[0]);
    const float base = base_of(m);
    for (int p = threadIdx.x; p < pieces; p += 256) {
        load_piece(row, p, pieces * 4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) s += p * 4 + i < n ? __builtin_amdgcn_exp2f((v[i] - base) * kLog2e) : 0.f;
    }
    s = group_sum<4>(s, slots[1]);
    if (threadIdx.x == 0) {
        stats[t] = {m, s};
        const int target = load_index(targets, wide, t, vocab) - v0;
        if (target >= 0 && target < n) z_target[t] = row[target];
    }
}

// dz of token blockIdx.x over a piece, with zeros from n on to the next multiple of 8.
template <class T>
__global__ __launch_bounds__(256) void xent_row_grad(const float *z, int64_t ldz, int n, int v0, const void *targets, bool wide, int vocab, const float *lse,
                                                     const float *dloss, int64_t dloss_inc, const float *factor, T *dz, int64_t ld) {
    const int64_t t = blockIdx.x;
    const float *row = z + t * ldz;
    const int target = load_index(targets, wide, t, vocab);
    const float g = target < 0 ? 0.f : dloss[t * dloss_inc] * factor[0], base = lse[t];
    for (int p = threadIdx.x; p < (n + 7) / 8; p += 256) {
        float v[8];
        load_piece(row, p, p * 8 + 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int col = p * 8 + i;
            const float d = __builtin_amdgcn_exp2f((v[i] - base) * kLog2e) - (v0 + col == target ? 1.f : 0.f);
            v[i] = target < 0 || col >= n ? 0.f : d * g;
        }
        store_piece(dz + t * ld, p, p * 8 + 8, v);
    }
}

// ---- joining ----------------------------------------------------------------------------------------------
// A workgroup joins the statistics of 1024 / G tokens, G threads a token: each a G-th of the parts in turn, then by halves, always the same
// ones.  stats: `parts` runs of `stride` tokens.
template <int G>
__global__ __launch_bounds__(1024) void xent_join(const Stat *stats, int parts, int64_t stride, int64_t tokens, const void *targets, bool wide, int vocab,
                                                  const float *z_target, float *loss, float *lse) {
    constexpr int TOKENS = 1024 / G;
    __shared__ Stat part[G][TOKENS];
    const int at = threadIdx.x % TOKENS, g = threadIdx.x / TOKENS;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + at;
    Stat sum = {-__builtin_inff(), 0.f};
    auto add = [&](Stat o) {
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

// ---- scaling of dz ------------------------------------------------------------------------------------------
// dz is kept as c dz, c = 2^k / max |dloss|.  With one dloss for all tokens (the mean of the losses) what is rounded is then exp(z - lse) - 1 or exp(z -
// lse) itself: relative to dloss, the same rounding of nearly -1 in every token would shift all of dx and dw one way (8192 tokens,
// bfloat16: error against 64 bits 2.6e-3 so, half of which is the rounding of the results).  Binary16: k = 14, so that |c dz|
// is at most 2^14 and what is 2^-38 of the largest is still a number.  factor[0] = c, factor[1] = scale / c.
__global__ __launch_bounds__(1024) void xent_factor(const float *dloss, int64_t dloss_inc, const void *targets, bool wide, int vocab, int64_t tokens, bool half,
                                                    float scale, float *factor) {
    __shared__ float slots[16];
    float top = 0.f;
    for (int64_t t = threadIdx.x; t < tokens; t += 1024)
        if (load_index(targets, wide, t, vocab) >= 0) top = __builtin_fmaxf(top, __builtin_fabsf(dloss[t * dloss_inc]));
    top = group_max<16>(top, slots);
    if (threadIdx.x == 0) {
        const bool usable = top > 0.f && top < __builtin_inff();
        const float range = half ? 16384.f : 1.f, unit = usable ? __builtin_fmaxf(top, 1e-30f) : 1.f;
        factor[0] = usable ? range / unit : 1.f;
        factor[1] = usable ? scale * (unit / range) : scale;
    }
}

// rows x cols FP32 values times *factor (no `in`: zeros), rounded into `out`
template <class T>
__global__ __launch_bounds__(256) void xent_round(const float *in, int64_t ld, const float *factor, T *out, int64_t ldo, int64_t rows, int cols) {
    const int pieces = (cols + 7) / 8;
    const float f = *factor;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int p = (int)(i - row * pieces);
        float v[8];
        if (in) load_piece(in + row * ld, p, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = in ? v[e] * f : 0.f;
        store_piece(out + row * ldo, p, cols, v);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = 256ll << 20;        // of logits (FP32) or dz: what the memory-side cache holds
constexpr int64_t kTokenBlock = 16384;              // tokens whose statistics are kept at a time
constexpr int64_t kFewestWords = 256;               // of a piece

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The most words of a piece; a word costs `bytes` per token.
int64_t preferred_words(int64_t tokens, int64_t vocab, int64_t bytes) {
    const int64_t words = std::max<int64_t>(2048, kPieceBytes / (bytes * std::max<int64_t>(tokens, 1)) / 256 * 256);
    return std::min({words, up(vocab, 8), (int64_t)1 << 20});            // (a row of logits is a leading dimension of fg_gemm's D)
}
// The most words, up to that many, of a piece whose space fits `bytes`.
template <class Space, class... Sizes>
int64_t words_within(int64_t words, int64_t bytes, Sizes... sizes) {
    while (words > kFewestWords && Space(words, sizes...).bytes > bytes) words = std::max(kFewestWords, words / 2 / 256 * 256);
    return words;
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

// Workspaces.  Forward: the statistics of a block of tokens and the logits of the targets; with logits in memory, a piece of them.
struct StatsSpace {
    int64_t parts, stats, z_target, bytes;
    StatsSpace(int64_t tokens, int64_t vocab, int64_t dim) {
        const int64_t block = std::min(tokens, kTokenBlock);
        parts = up(vocab, kernel_table_xent(XENT_STATS, false)[xent_tile(block, vocab, dim)].bn) / kXentWaveColumns[xent_tile(block, vocab, dim)];
        stats = 0;
        z_target = up(parts * block * (int64_t)sizeof(Stat), 256);
        bytes = z_target + up(tokens * 4, 256);
    }
};
struct RowsSpace {
    int64_t words, parts, z, stats, z_target, bytes;
    RowsSpace(int64_t words_, int64_t tokens, int64_t vocab) : words(words_) {
        parts = (vocab + words - 1) / words;
        z = 0;
        stats = z + up(tokens * words * 4, 256);
        z_target = stats + up(parts * tokens * (int64_t)sizeof(Stat), 256);
        bytes = z_target + up(tokens * 4, 256);
    }
};
// Gradient: dz of a piece, the sums of dx, and, with logits in memory, a piece of them and dw's rows of it.
struct GradSpace {
    int64_t words, ld_dz, ld, dz, dx, factor, z, dw, bytes;
    GradSpace(int64_t words_, int64_t tokens, int64_t dim, bool tiled) : words(words_) {
        ld_dz = up(words, 8);
        ld = up(dim, 4);
        dz = 0;
        dx = dz + up(tokens * ld_dz * 2, 256);
        factor = dx + up(tokens * ld * 4, 256);
        z = factor + 256;
        dw = z + (tiled ? 0 : up(tokens * words * 4, 256));
        bytes = dw + (tiled ? 0 : up(words * ld * 4, 256));
    }
};

fg_status check_xent(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype) {
    if (tokens < 0 || vocab < 0 || dim < 0) return fail(FG_ERR_SHAPE, "negative size: %lld tokens, %lld words, %lld values", (long long)tokens, (long long)vocab, (long long)dim);
    if (vocab == 0) return fail(FG_ERR_SHAPE, "the vocabulary is empty");
    if (tokens > (1 << 30) || vocab > (1 << 30) || dim > (1 << 30)) return fail(FG_ERR_UNSUPPORTED, "sizes above 2^30 are not supported");
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

bool tiled_dim(int64_t dim) { return dim > 0 && dim % 8 == 0; }
// Whether the tiled kernels take X and W: 16-byte aligned rows, within the reach of a lane's offsets.
bool tiled(int64_t dim, const fg_matrix *X, const fg_matrix *W) {
    auto fits = [](const fg_matrix *m) { return aligned_to(m->re, 16) && m->ld % 8 == 0 && m->ld < (1 << 22); };
    return tiled_dim(dim) && fits(X) && fits(W);
}

// Logits of words v0 .. v0 + n - 1 in memory.
fg_status piece_logits(int64_t tokens, int64_t dim, const fg_matrix *X, const fg_matrix *W, float scale, int64_t v0, int64_t n, float *z, int64_t ldz, void *stream) {
    const fg_matrix b = rows_of(row_at(W, v0), W->dtype, W->ld, FG_COL), d = rows_of(z, FG_F32, ldz);
    return fg_gemm(tokens, n, dim, scale, X, &b, 0.f, nullptr, &d, nullptr, stream);
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

fg_status run_join(const Stat *stats, int64_t parts, int64_t stride, int64_t tokens, const void *targets, bool wide, int64_t vocab, const float *z_target, float *loss,
                   float *lse, hipStream_t stream) {
    auto launch = [&](auto tag) {
        constexpr int G = decltype(tag)::value, TOKENS = 1024 / G;
        hipLaunchKernelGGL((xent_join<G>), dim3((unsigned)((tokens + TOKENS - 1) / TOKENS)), dim3(1024), 0, stream, stats, (int)parts, stride, tokens, targets, wide, (int)vocab,
                           z_target, loss, lse);
    };
    // Enough workgroups to share the reads: 16 tokens of 2048 parts 20.2 us with 16 threads each, 6.0 with 256; 8192 of 1024 17.4 with 16.
    if (tokens <= 256) launch(std::integral_constant<int, 256>{});
    else if (tokens <= 4096) launch(std::integral_constant<int, 64>{});
    else launch(std::integral_constant<int, 16>{});
    return check_launch("xent_join");
}

fg_status xent_tiled(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, bool wide, float scale, float *loss,
                     float *lse, char *w, hipStream_t stream) {
    const StatsSpace at(tokens, vocab, dim);
    const int64_t block = std::min(tokens, kTokenBlock);
    const KernelEntry &k = kernel_table_xent(XENT_STATS, X->dtype == FG_BF16)[xent_tile(block, vocab, dim)];
    for (int64_t t0 = 0; t0 < tokens; t0 += block) {
        const int64_t n = std::min(block, tokens - t0);
        XentParams p = product(k, true, n, vocab, dim, row_at(X, t0), X->ld, W->re, W->ld);
        p.alpha = scale;
        p.stats = (Stat *)(w + at.stats);
        p.stats_stride = block;
        p.z_target = (float *)(w + at.z_target);
        p.targets = (const char *)targets + t0 * (wide ? 8 : 4);
        p.wide = wide; p.vocab = (int32_t)vocab;
        if (fg_status st = launch_product(k, p, stream)) return st;
        if (fg_status st = run_join(p.stats, at.parts, block, n, p.targets, wide, vocab, p.z_target, loss + t0, lse + t0, stream)) return st;
    }
    return FG_OK;
}

fg_status xent_rows(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, bool wide, float scale, float *loss,
                    float *lse, char *w, const RowsSpace &at, hipStream_t stream) {
    float *z = (float *)(w + at.z), *z_target = (float *)(w + at.z_target);
    Stat *stats = (Stat *)(w + at.stats);
    for (int64_t part = 0; part < at.parts; ++part) {
        const int64_t v0 = part * at.words, n = std::min(at.words, vocab - v0);
        if (fg_status st = piece_logits(tokens, dim, X, W, scale, v0, n, z, at.words, stream)) return st;
        hipLaunchKernelGGL(xent_row_stats, dim3((unsigned)tokens), dim3(256), 0, stream, z, at.words, (int)n, (int)v0, targets, wide, (int)vocab, stats + part * tokens, z_target);
    }
    return run_join(stats, at.parts, tokens, tokens, targets, wide, vocab, z_target, loss, lse, stream);
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

}  // namespace fg

using namespace fg;

extern "C" {

// (What the query gives serves rows of any alignment: where dim lets the tiled kernels take them, with the smallest pieces.)
int64_t fg_linear_xent_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens <= 0 || vocab <= 0 || dim < 0) return 0;
    if (!tiled_dim(dim)) return RowsSpace(preferred_words(tokens, vocab, 4), tokens, vocab).bytes;
    return std::max(StatsSpace(tokens, vocab, dim).bytes, RowsSpace(std::min(kFewestWords, up(vocab, 8)), tokens, vocab).bytes);
}

fg_status fg_linear_xent(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype,
                         float scale, float *loss, float *lse, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_xent(tokens, vocab, dim, X, W, targets, index_dtype)) return st;
    if (tokens == 0) return FG_OK;
    if (!loss || !lse) return fail(FG_ERR_NULL, "loss or lse is NULL");
    if (!aligned_to(loss, 4) || !aligned_to(lse, 4)) return fail(FG_ERR_ALIGN, "loss and lse must be aligned to an element");
    const bool wide = index_dtype == FG_I64;
    if (tiled(dim, X, W)) {
        if (fg_status st = check_workspace(workspace, workspace_bytes, StatsSpace(tokens, vocab, dim).bytes)) return st;
        return xent_tiled(tokens, vocab, dim, X, W, targets, wide, scale, loss, lse, (char *)workspace, (hipStream_t)hip_stream);
    }
    const RowsSpace at(words_within<RowsSpace>(preferred_words(tokens, vocab, 4), workspace_bytes, tokens, vocab), tokens, vocab);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    return xent_rows(tokens, vocab, dim, X, W, targets, wide, scale, loss, lse, (char *)workspace, at, (hipStream_t)hip_stream);
}

int64_t fg_linear_xent_grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens < 0 || vocab <= 0 || dim <= 0) return 0;
    if (!tiled_dim(dim)) return GradSpace(preferred_words(tokens, vocab, 4), tokens, dim, false).bytes;
    return std::max(GradSpace(preferred_words(tokens, vocab, 2), tokens, dim, true).bytes, GradSpace(std::min(kFewestWords, up(vocab, 8)), tokens, dim, false).bytes);
}

fg_status fg_linear_xent_grad(int64_t tokens, int64_t vocab, int64_t dim, const fg_matrix *X, const fg_matrix *W, const void *targets, int32_t index_dtype,
                              float scale, const float *lse, const float *dloss, int64_t dloss_inc, const fg_matrix *dX, const fg_matrix *dW,
                              void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_xent(tokens, vocab, dim, X, W, targets, index_dtype)) return st;
    if (fg_status st = check_rows("dX", dX, tokens, dim)) return st;
    if (fg_status st = check_rows("dW", dW, vocab, dim)) return st;
    if (dX->dtype != X->dtype || dW->dtype != X->dtype) return fail(FG_ERR_UNSUPPORTED, "dX and dW must have the element type of X");
    if (dloss_inc != 0 && dloss_inc != 1) return fail(FG_ERR_SHAPE, "dloss_inc must be 0 or 1");
    if (dim == 0) return FG_OK;
    if (tokens > 0 && (!lse || !dloss)) return fail(FG_ERR_NULL, "lse or dloss is NULL");
    if (!aligned_to(lse, 4) || !aligned_to(dloss, 4)) return fail(FG_ERR_ALIGN, "lse and dloss must be aligned to an element");
    const bool in_tiles = tiled(dim, X, W), wide = index_dtype == FG_I64, bf16 = X->dtype == FG_BF16;
    const GradSpace at(words_within<GradSpace>(preferred_words(tokens, vocab, in_tiles ? 2 : 4), workspace_bytes, tokens, dim, in_tiles), tokens, dim, in_tiles);
    if (fg_status st = check_workspace(workspace, workspace_bytes, at.bytes)) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    char *w = (char *)workspace;
    float *z = (float *)(w + at.z), *dw = (float *)(w + at.dw), *dx = (float *)(w + at.dx), *factor = (float *)(w + at.factor);
    void *dz = w + at.dz;
    hipLaunchKernelGGL(xent_factor, dim3(1), dim3(1024), 0, stream, dloss, dloss_inc, targets, wide, (int)vocab, tokens, !bf16, scale, factor);
    const fg_matrix sum_dx = rows_of(dx, FG_F32, at.ld), part_dw = rows_of(dw, FG_F32, at.ld);
    auto round = [&](const float *in, const fg_matrix *out, int64_t row0, int64_t rows) {
        if (rows == 0) return;
        const unsigned groups = (unsigned)std::min<int64_t>((rows * ((dim + 7) / 8) + 255) / 256, 8192);
        with_half(X->dtype, [&](auto t) {
            using T = decltype(t);
            hipLaunchKernelGGL((xent_round<T>), dim3(groups), dim3(256), 0, stream, in, at.ld, factor + 1, (T *)row_at(out, row0), out->ld, rows, (int)dim);
        });
    };
    if (tokens == 0) round(nullptr, dW, 0, vocab);
    for (int64_t v0 = 0; v0 < vocab && tokens > 0; v0 += at.words) {
        const int64_t n = std::min(at.words, vocab - v0);
        const fg_matrix dz_r = rows_of(dz, X->dtype, at.ld_dz), w_piece = rows_of(row_at(W, v0), W->dtype, W->ld);
        if (in_tiles) {
            const KernelEntry &kz = kernel_table_xent(XENT_DZ, bf16)[xent_tile(tokens, n, dim)];
            XentParams p = product(kz, true, tokens, n, dim, X->re, X->ld, w_piece.re, W->ld);
            p.alpha = scale;
            p.targets = targets; p.wide = wide; p.vocab = (int32_t)vocab; p.v0 = (int32_t)v0;
            p.lse = lse; p.dloss = dloss; p.dloss_inc = (int32_t)dloss_inc; p.factor = factor;
            p.D = (float *)dz; p.ldd = at.ld_dz;
            if (fg_status st = launch_product(kz, p, stream)) return st;
            // neither operand is K-contiguous: any number of tokens
            const KernelEntry &kw = kernel_table_xent(XENT_ROUND, bf16)[xent_tile(n, dim, tokens)];
            XentParams q = product(kw, false, n, dim, tokens, dz, at.ld_dz, X->re, X->ld);
            q.factor = factor;
            q.D = (float *)row_at(dW, v0); q.ldd = dW->ld;
            if (fg_status st = launch_product(kw, q, stream)) return st;
            // dz has zeros from n on to the next multiple of 8
            if (fg_status st = gemm_stored(tokens, dim, up(n, 8), n, 1.f, &dz_r, &w_piece, v0 == 0 ? 0.f : 1.f, &sum_dx, &sum_dx, stream)) return st;
        } else {
            if (fg_status st = piece_logits(tokens, dim, X, W, scale, v0, n, z, at.words, stream)) return st;
            with_half(X->dtype, [&](auto t) {
                using T = decltype(t);
                hipLaunchKernelGGL((xent_row_grad<T>), dim3((unsigned)tokens), dim3(256), 0, stream, z, at.words, (int)n, (int)v0, targets, wide, (int)vocab, lse,
                                   dloss, dloss_inc, factor, (T *)dz, at.ld_dz);
            });
            const fg_matrix dz_t = rows_of(dz, X->dtype, at.ld_dz, FG_COL);
            if (fg_status st = fg_gemm(n, dim, tokens, 1.f, &dz_t, X, 0.f, nullptr, &part_dw, nullptr, stream)) return st;
            round(dw, dW, v0, n);
            if (fg_status st = fg_gemm(tokens, dim, n, 1.f, &dz_r, &w_piece, v0 == 0 ? 0.f : 1.f, &sum_dx, &sum_dx, nullptr, stream)) return st;
        }
    }
    round(dx, dX, 0, tokens);
    return check_launch("xent_grad");
}

}  // extern "C"
