// What the kernels that work on rows of a matrix share (layernorm.hip, embedding.hip, xent.hip): element types, 16-byte
// accesses to rows that need not be aligned to them, sums over a wave and over the waves of a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "status.hpp"

namespace fg {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

// Sixteen bytes of T.  The type is aligned to an element only: a row of odd length begins anywhere, and the memory system takes
// an access of 16 bytes at any element.
template <class T> struct Piece {
    static constexpr int N = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(N)));
    typedef vec unaligned __attribute__((aligned(sizeof(T))));
};

// Piece p of a row of n elements as FP32; past the end: `fill`.
template <class T>
__device__ __forceinline__ void load_piece(const T *row, int p, int n, float (&out)[Piece<T>::N], float fill = 0.f) {
    constexpr int N = Piece<T>::N;
    if ((p + 1) * N <= n) {
        const typename Piece<T>::vec v = *(const typename Piece<T>::unaligned *)(row + p * N);
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = p * N + e < n ? (float)row[p * N + e] : fill;
    }
}
// Rounded to nearest even once.
template <class T>
__device__ __forceinline__ void store_piece(T *row, int p, int n, const float (&in)[Piece<T>::N]) {
    constexpr int N = Piece<T>::N;
    if ((p + 1) * N <= n) {
        typename Piece<T>::vec v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)in[e];
        *(typename Piece<T>::unaligned *)(row + p * N) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (p * N + e < n) row[p * N + e] = (T)in[e];
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

// Sum over the W waves of a workgroup, in the order of the waves.  `slot` (W floats of LDS) must not be in use by a sum less than
// two barriers ago: callers alternate between two.
template <int W>
__device__ __forceinline__ float group_sum(float v, float *slot) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        v = slot[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += slot[w];
    }
    return v;
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
inline fg_status check_launch(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FG_OK : fail(FG_ERR_LAUNCH, "launch of %s failed: %s", what, hipGetErrorString(e));
}

}  // namespace fg
