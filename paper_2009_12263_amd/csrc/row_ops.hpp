// What the kernels that work on rows of a matrix share (layernorm.hip, embedding.hip, xent.hip): element types, 16-byte
// accesses to rows that need not be aligned to them, sums over a wave and over the waves of a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.hpp"
#include "status.hpp"

namespace fg {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

// N elements of T, sixteen bytes unless it is said otherwise.  The type is aligned to an element only: a row of odd length begins
// anywhere, and the memory system takes an access of 16 bytes at any element.
template <class T, int N_ = 16 / (int)sizeof(T)> struct RowPiece {
    static constexpr int N = N_;
    typedef T vec __attribute__((ext_vector_type(N_)));
    typedef vec unaligned __attribute__((aligned(sizeof(T))));
};

// A row of n elements is cut into pieces of N.  Where N does not divide n, the last piece is moved back to end with the row: it holds some of
// its neighbour's elements again, and every access is one of 16 bytes.  (Element by element under a mask, a wave waits for the elements of one
// row before it requests the next: sums of 9999 rows of 1001 FP32 33.1 us, 26.2 so.)  Rows shorter than a piece go element by element.
template <int N> __device__ __forceinline__ int first_of_piece(int p, int n) { return min(p * N, max(n - N, 0)); }
// Whether element e of piece p is the piece's own.
template <int N> __device__ __forceinline__ bool own_element(int p, int n, int e) { const int at = first_of_piece<N>(p, n) + e; return at >= p * N && at < n; }

// Piece p as it is stored (zeros past the end of a row that is shorter).
template <class T, int N>
__device__ __forceinline__ typename RowPiece<T, N>::vec load_raw(const T *row, int p, int n) {
    if (n >= N) return *(const typename RowPiece<T, N>::unaligned *)(row + first_of_piece<N>(p, n));
    typename RowPiece<T, N>::vec v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? row[e] : (T)0.f;
    return v;
}
// The same as FP32.
template <class T, int N>
__device__ __forceinline__ void load_piece(const T *row, int p, int n, float (&out)[N]) {
    const typename RowPiece<T, N>::vec v = load_raw<T, N>(row, p, n);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = (float)v[e];
}
// The piece's own elements, rounded to nearest even once.
template <class T, int N>
__device__ __forceinline__ void store_piece(T *row, int p, int n, const float (&in)[N]) {
    if ((p + 1) * N <= n) {
        typename RowPiece<T, N>::vec v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)in[e];
        *(typename RowPiece<T, N>::unaligned *)(row + p * N) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (own_element<N>(p, n, e)) row[first_of_piece<N>(p, n) + e] = (T)in[e];
    }
}

// Every lane gets op over the 64 lanes; the same bits in all of them (each step combines two values that both sides see).
template <class Op>
__device__ __forceinline__ float wave_reduce(float v, Op op) {
    auto turned = [](float x, auto ctrl) {         // the value of the lane so many further on in the row of 16
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v = op(v, turned(v, std::integral_constant<int, 0x128>{}));
    v = op(v, turned(v, std::integral_constant<int, 0x124>{}));
    v = op(v, turned(v, std::integral_constant<int, 0x122>{}));
    v = op(v, turned(v, std::integral_constant<int, 0x121>{}));
    {
        const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        const unsigned s0 = s[0], s1 = s[1];
        v = op(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
    }
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned s0 = s[0], s1 = s[1];
    return op(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return __builtin_fmaxf(a, b); }); }

// Sum over W waves of a workgroup (the first W, the next W, ...), in the order of the waves; every wave of the workgroup takes part.  `slot` (W floats of LDS for each W waves) must not be in use by a sum less than
// two barriers ago: callers alternate between two.
template <int W>
__device__ __forceinline__ float group_sum(float v, float *slot) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) slot[(threadIdx.x >> 6) % W] = v;
        __syncthreads();
        v = slot[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += slot[w];
    }
    return v;
}

// Row index `at` of a list of ids; -1 where it names none of the n rows.
__device__ __forceinline__ int load_index(const void *ids, bool wide, int64_t at, int n) {
    const int64_t id = wide ? ((const int64_t *)ids)[at] : (int64_t)((const int32_t *)ids)[at];
    return id >= 0 && id < n ? (int)id : -1;
}

// ---- host ---------------------------------------------------------------------------------------
inline int element_bytes(int dtype) { return dtype == FG_F32 ? 4 : dtype == FG_F16 || dtype == FG_BF16 ? 2 : 0; }

// A matrix whose rows are contiguous, of rows x cols elements of one of the three types.  `broadcast`: only read, and
// all its rows may be the same one (ld 0).
inline fg_status check_rows(const char *name, const fg_matrix *m, int64_t rows, int64_t cols, bool broadcast = false) {
    if (!m) return fail(FG_ERR_NULL, "%s is NULL", name);
    if (m->im || !element_bytes(m->dtype)) return fail(FG_ERR_LAYOUT, "%s must be a real FG_F16, FG_BF16 or FG_F32 matrix", name);
    if (m->layout != FG_ROW) return fail(FG_ERR_LAYOUT, "%s must be row-major (FG_ROW)", name);
    if (rows > 0 && cols > 0) {
        if (!m->re) return fail(FG_ERR_NULL, "%s->re is NULL", name);
        if (!aligned_to(m->re, element_bytes(m->dtype))) return fail(FG_ERR_ALIGN, "%s: element pointers must be aligned to an element", name);
        if (m->ld < cols && !(broadcast && m->ld == 0)) return fail(FG_ERR_SHAPE, "%s: ld=%lld is smaller than %lld", name, (long long)m->ld, (long long)cols);
    }
    return FG_OK;
}
// Token ids and targets: FG_I32 or FG_I64.
inline fg_status check_indices(const char *name, const void *p, int dtype, int64_t n) {
    if (dtype != FG_I32 && dtype != FG_I64) return fail(FG_ERR_LAYOUT, "%s must be FG_I32 or FG_I64", name);
    if (n > 0 && !p) return fail(FG_ERR_NULL, "%s is NULL", name);
    if (!aligned_to(p, dtype == FG_I64 ? 8 : 4)) return fail(FG_ERR_ALIGN, "%s must be aligned to an element", name);
    return FG_OK;
}
inline fg_status check_workspace(const void *workspace, int64_t bytes, int64_t need) {
    if (need > 0 && !workspace) return fail(FG_ERR_NULL, "the workspace is NULL");
    if (!aligned_to(workspace, 16)) return fail(FG_ERR_ALIGN, "the workspace must be 16-byte aligned");
    if (bytes < need) return fail(FG_ERR_SHAPE, "the workspace has %lld bytes, %lld are needed", (long long)bytes, (long long)need);
    return FG_OK;
}
// f(first, n) for groups first .. first + n - 1 of a launch's `groups` workgroups (up to 1024 threads): a launch holds fewer than 2^32 threads, so
// larger ones are made in parts.
template <class F> void in_parts(int64_t groups, F &&f) {
    constexpr int64_t kMost = 1 << 21;
    for (int64_t first = 0; first < groups; first += kMost) f(first, dim3((unsigned)(groups - first < kMost ? groups - first : kMost)));
}
}  // namespace fg
