// What follows a backward pass, over all tensors of a model at once: the norm of the gradients, and the AdamW step.
//
//   norm = scale sqrt(sum over all g^2),   factor = scale min(1, max_norm / norm)
//   g' = factor g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: each value of a tensor is read and written once (28 bytes a 16-bit parameter with an FP32 copy, gradient and FP32 moments,
// 10 with moments in eight bits and no copy).  A launch covers the tensors that a kernel's arguments hold; each workgroup takes a
// chunk of one, which its lanes find together.  Nothing is kept between calls: the tensors' addresses travel with the launch.
//
// Moments in eight bits (e4m3) have an FP32 scale for each 256 values, the largest of them / 448.  Of v the root is kept: its range
// of 2^17 is one of 2^34 of v.  A root that is not zero is held at least as the smallest such number: m / (root + eps) of a v that was rounded
// to zero would be m / eps.  The step itself uses m and v in FP32, as they are before they are rounded.
//
// Measured: 386 M values, bfloat16 with FP32 copies 2076 us (5.2 TB/s), in eight bits 764 to 781 (5.0), 75 M FP32 values 398 (5.3), 193 tensors of 1.6 M values in two launches 18 to 22; the
// norm of 386 M binary16 values 129 (6.0).
//
// The operations are written one by one, without fused ones: what eight bits hold changes by 1/16 where a sum falls on the other side of a border.
#include "row_ops.hpp"
#include "shared_spans.hpp"

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

namespace fg {
namespace {

constexpr int kThreads = 256;
constexpr int kStateBlock = 256;            // values that share a scale
constexpr int kLaneBlock = 16;              // of them in a lane: 16 lanes, a row of the wave, share one
// Values of a workgroup.  Small models: those that its threads take at once; four turns one after the other, each waiting for memory, took 10 us a launch of 48 short
// tensors, one 4.  Large ones: more, for the sake of what a workgroup does once.
constexpr int kChunk = 8192, kSmallChunk = 2048;
constexpr int64_t kSmallModel = 4096 * kSmallChunk;
constexpr float kTop = 448.f, kLeast = 0x1p-9f;         // of e4m3: the largest number, the smallest one above zero
constexpr float kNothing = 1e-30f;          // a block whose largest value is smaller is zero (its scale's reciprocal would overflow)

template <bool SMALL> struct TensorArg {
    void *p;
    const void *g;
    float *master;
    void *m, *v;
    int64_t n;
    int32_t kind;
};
template <> struct TensorArg<true> : TensorArg<false> { float *m_scale, *v_scale; };
// The same of a short tensor whose memory is near to the others': the arrays' distances from the lowest address, in steps of two bytes, 32 bits each and five more
// beside n and kind.  Twice as many fit a launch.
constexpr int kNearStep = 2, kNearBits = 23, kKindBits = 4, kFarBits = 5;          // kNearBits: of n
constexpr uint64_t kNear = (uint64_t)kNearStep << (32 + kFarBits);
template <bool SMALL> struct NearArg {
    static constexpr int kArrays = SMALL ? 7 : 5;           // p, g, master, m, v, m_scale, v_scale
    uint32_t low[kArrays], more[2];
    void set(int64_t n, int kind, uint64_t base, const void *const (&arrays)[kArrays]) {
        uint64_t rest = (uint64_t)n | (uint64_t)kind << kNearBits;
        for (int i = 0; i < kArrays; ++i) {
            const uint64_t at = arrays[i] && n > 0 ? ((uint64_t)arrays[i] - base) / kNearStep : 0;
            low[i] = (uint32_t)at;
            rest |= at >> 32 << (kNearBits + kKindBits + kFarBits * i);
        }
        more[0] = (uint32_t)rest;
        more[1] = (uint32_t)(rest >> 32);
    }
    __device__ __forceinline__ TensorArg<SMALL> whole(char *base) const {
        const uint64_t rest = more[0] | (uint64_t)more[1] << 32;
        auto there = [&](int i) { return base + (low[i] | (rest >> (kNearBits + kKindBits + kFarBits * i) & ((1 << kFarBits) - 1)) << 32) * kNearStep; };
        TensorArg<SMALL> t;
        t.p = there(0); t.g = there(1); t.master = (float *)there(2); t.m = there(3); t.v = there(4);
        if constexpr (SMALL) { t.m_scale = (float *)there(5); t.v_scale = (float *)there(6); }
        t.n = (int64_t)(rest & ((1 << kNearBits) - 1));
        t.kind = (int32_t)(rest >> kNearBits & ((1 << kKindBits) - 1));
        return t;
    }
};
static_assert(kNearBits + kKindBits + 7 * kFarBits <= 64 && kSmallModel <= 1 << kNearBits, "");

// Arguments are copied through the command path: few tensors have a short list of them.  A list has at most two for each lane of a wave, and as many as fit 4 KB.
template <class Arg, int CAP> struct List {
    int32_t first[CAP];                     // number of a tensor's first chunk in the launch; behind the last tensor the number of all
    Arg at[CAP];
};

struct StepArgs {
    double lr, beta1, beta2, eps, decay;
    const int64_t *step;
    const float *factor, *lr_factor;
    char *base;                             // of NearArg
    int32_t chunk;
};
// What a step needs of them, in FP32.
struct Rates {
    float beta1, other1, beta2, other2, eps, keep, rate, root, factor;
};

// Which tensor chunk c is in: the last one that does not begin behind it.  Each lane looks at one or two: a bisection, six reads of the arguments one after the other, took
// 8 us of a launch, whose workgroups all wait for them.
template <class L, int CAP = sizeof(L::first) / 4>
__device__ __forceinline__ int tensor_of(const L &list, int c) {
    static_assert(CAP <= 128, "");
    const int lane = threadIdx.x & 63;
    int before = __builtin_popcountll(__ballot(lane < CAP && list.first[lane < CAP ? lane : 0] <= c));
    if constexpr (CAP > 64) before += __builtin_popcountll(__ballot(64 + lane < CAP && list.first[64 + lane < CAP ? 64 + lane : 0] <= c));
    return before - 1;
}
template <bool SMALL> __device__ __forceinline__ TensorArg<SMALL> whole(const TensorArg<SMALL> &t, char *) { return t; }
template <bool SMALL> __device__ __forceinline__ TensorArg<SMALL> whole(const NearArg<SMALL> &t, char *base) { return t.whole(base); }

// x^t by squaring; 64-bit, for 1 - x^t of an x near 1.
__device__ __forceinline__ double power(double x, int64_t t) {
    double y = 1.0;
    for (; t > 0 && y != 0.0; t >>= 1, x *= x)
        if (t & 1) y *= x;
    return y;
}

// False where there is nothing to do: a factor that is no finite number (gradients that overflowed), or no step.
__device__ __forceinline__ bool rates_of(const StepArgs &s, Rates &r) {
    const int64_t t = *s.step;
    r.factor = s.factor ? *s.factor : 1.f;
    if (t < 1 || !(__builtin_fabsf(r.factor) < __builtin_inff())) return false;
    const double lr = s.lr_factor ? s.lr * (double)*s.lr_factor : s.lr;
    r.beta1 = (float)s.beta1; r.other1 = (float)(1.0 - s.beta1);
    r.beta2 = (float)s.beta2; r.other2 = (float)(1.0 - s.beta2);
    r.eps = (float)s.eps;
    r.keep = (float)(1.0 - lr * s.decay);
    r.rate = (float)(lr / (1.0 - power(s.beta1, t)));
    r.root = (float)(1.0 / __builtin_sqrt(1.0 - power(s.beta2, t)));
    return true;
}

// One value: m and v become the new ones, the new parameter and v's root are returned.
__device__ __forceinline__ float stepped(const Rates &r, float p, float g, float &m, float &v, float &root) {
#pragma clang fp contract(off)
    g = g * r.factor;
    m = m * r.beta1 + g * r.other1;
    v = v * r.beta2 + g * g * r.other2;
    root = __builtin_sqrtf(v);
    return p * r.keep - r.rate * (m / (root * r.root + r.eps));
}

// N values from `at` on, those past the end of n left as they are.
template <class T, int N>
__device__ __forceinline__ void load_values(const T *from, int64_t at, int64_t n, float (&out)[N]) {
    constexpr int E = 16 / (int)sizeof(T) < N ? 16 / (int)sizeof(T) : N;
    if (at + N <= n) {
#pragma unroll
        for (int h = 0; h < N / E; ++h) {
            const typename RowPiece<T, E>::vec v = *(const typename RowPiece<T, E>::unaligned *)(from + at + h * E);
#pragma unroll
            for (int e = 0; e < E; ++e) out[h * E + e] = (float)v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = at + e < n ? (float)from[at + e] : 0.f;
    }
}
template <class T, int N>
__device__ __forceinline__ void store_values(T *to, int64_t at, int64_t n, const float (&in)[N]) {
    constexpr int E = 16 / (int)sizeof(T) < N ? 16 / (int)sizeof(T) : N;
    if (at + N <= n) {
#pragma unroll
        for (int h = 0; h < N / E; ++h) {
            typename RowPiece<T, E>::vec v;
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (T)in[h * E + e];
            *(typename RowPiece<T, E>::unaligned *)(to + at + h * E) = v;
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e < n) to[at + e] = (T)in[e];
    }
}

// ---- moments in eight bits ----------------------------------------------------------------------------
typedef uint32_t codes16 __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void load_codes(const void *from, int64_t at, int64_t n, float scale, float (&out)[kLaneBlock]) {
    codes16 c = {};
    if (at + kLaneBlock <= n) c = *(const codes16 *)((const uint8_t *)from + at);
    else
        for (int e = 0; e < kLaneBlock; ++e)
            if (at + e < n) c[e / 4] |= (uint32_t)((const uint8_t *)from)[at + e] << (e % 4 * 8);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
        out[4 * w] = lo[0] * scale; out[4 * w + 1] = lo[1] * scale; out[4 * w + 2] = hi[0] * scale; out[4 * w + 3] = hi[1] * scale;
    }
}
__device__ __forceinline__ void store_codes(void *to, int64_t at, int64_t n, const float (&in)[kLaneBlock]) {
    codes16 c;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(in[4 * w], in[4 * w + 1], 0, false);
        c[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in[4 * w + 2], in[4 * w + 3], word, true);
    }
    if (at + kLaneBlock <= n) *(codes16 *)((uint8_t *)to + at) = c;
    else
        for (int e = 0; e < kLaneBlock; ++e)
            if (at + e < n) ((uint8_t *)to)[at + e] = (uint8_t)(c[e / 4] >> (e % 4 * 8));
}
// The largest of a row of 16 lanes, in all of them.
__device__ __forceinline__ float row_max(float v) {
    auto turned = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v = __builtin_fmaxf(v, turned(v, std::integral_constant<int, 0x128>{}));
    v = __builtin_fmaxf(v, turned(v, std::integral_constant<int, 0x124>{}));
    v = __builtin_fmaxf(v, turned(v, std::integral_constant<int, 0x122>{}));
    return __builtin_fmaxf(v, turned(v, std::integral_constant<int, 0x121>{}));
}
// A block's values relative to its scale, and the scale.  FLOOR: at least kLeast where they are not zero.
template <bool FLOOR>
__device__ __forceinline__ float relative(float (&x)[kLaneBlock]) {
#pragma clang fp contract(off)
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < kLaneBlock; ++e) top = __builtin_fmaxf(top, __builtin_fabsf(x[e]));
    top = row_max(top);
    const float by = top >= kNothing ? kTop * (1.f / top) : 0.f;
#pragma unroll
    for (int e = 0; e < kLaneBlock; ++e) {
        x[e] *= by;
        if (FLOOR) x[e] = x[e] > 0.f && x[e] < kLeast ? kLeast : x[e];
    }
    return top >= kNothing ? top * (1.f / kTop) : 0.f;
}

// ---- the step -----------------------------------------------------------------------------------------
// P: parameters, G: gradients, COPY: with an FP32 copy, which is what the step reads.
template <class P, class G, bool COPY, bool SMALL>
__device__ __forceinline__ void step_chunk(const TensorArg<SMALL> &t, const StepArgs &s, int64_t begin, int chunk) {
    constexpr int N = SMALL ? kLaneBlock : 8;
    const int64_t end = begin + chunk < t.n ? begin + chunk : t.n;
    Rates r;
    bool known = false;
    // (the lanes of a row are in the same block, and go round together)
    for (int64_t at = begin + threadIdx.x * N; SMALL ? at / kStateBlock * kStateBlock < end : at < end; at += kThreads * N) {
        float p[N], g[N], m[N], v[N], root[N];
        load_values<G, N>((const G *)t.g, at, t.n, g);
        if constexpr (COPY) load_values<float, N>(t.master, at, t.n, p);
        else load_values<P, N>((const P *)t.p, at, t.n, p);
        if constexpr (SMALL) {
            const int64_t block = at / kStateBlock;
            load_codes(t.m, at, t.n, t.m_scale[block], m);
            load_codes(t.v, at, t.n, t.v_scale[block], v);
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = v[e] * v[e];
        } else {
            load_values<float, N>((const float *)t.m, at, t.n, m);
            load_values<float, N>((const float *)t.v, at, t.n, v);
        }
        // (the rates wait for memory too, and take their time: behind the first values' requests)
        if (!known && !rates_of(s, r)) return;
        known = true;
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = stepped(r, p[e], g[e], m[e], v[e], root[e]);
        if constexpr (COPY) store_values<float, N>(t.master, at, t.n, p);
        store_values<P, N>((P *)t.p, at, t.n, p);
        if constexpr (SMALL) {
            const float sm = relative<false>(m), sv = relative<true>(root);
            store_codes(t.m, at, t.n, m);
            store_codes(t.v, at, t.n, root);
            if (at % kStateBlock == 0) {
                t.m_scale[at / kStateBlock] = sm;
                t.v_scale[at / kStateBlock] = sv;
            }
        } else {
            store_values<float, N>((float *)t.m, at, t.n, m);
            store_values<float, N>((float *)t.v, at, t.n, v);
        }
    }
}

// kind: the type of the parameters (FG_F16, FG_BF16, FG_F32), + 4 with FP32 gradients, + 8 with an FP32 copy of the parameters
constexpr int kWideGrad = 4, kCopy = 8;
static_assert(FG_F32 < kWideGrad && FG_BF16 < kWideGrad && kWideGrad + kCopy + FG_BF16 < 1 << kKindBits, "");

// Arg: TensorArg or NearArg
template <int CAP, bool SMALL, class Arg>
__global__ __launch_bounds__(kThreads) void adamw(const List<Arg, CAP> a, const StepArgs s) {
    const int which = tensor_of(a, (int)blockIdx.x);
    const TensorArg<SMALL> t = whole<SMALL>(a.at[which], s.base);
    const int64_t begin = ((int64_t)blockIdx.x - a.first[which]) * s.chunk;
    switch (t.kind) {
        case FG_F16: return step_chunk<f16_t, f16_t, false, SMALL>(t, s, begin, s.chunk);
        case FG_BF16: return step_chunk<bf16_t, bf16_t, false, SMALL>(t, s, begin, s.chunk);
        case FG_F32 + kWideGrad: return step_chunk<float, float, false, SMALL>(t, s, begin, s.chunk);
        case FG_F16 + kWideGrad: return step_chunk<f16_t, float, false, SMALL>(t, s, begin, s.chunk);
        case FG_BF16 + kWideGrad: return step_chunk<bf16_t, float, false, SMALL>(t, s, begin, s.chunk);
        case FG_F16 + kCopy: return step_chunk<f16_t, f16_t, true, SMALL>(t, s, begin, s.chunk);
        case FG_BF16 + kCopy: return step_chunk<bf16_t, bf16_t, true, SMALL>(t, s, begin, s.chunk);
        case FG_F16 + kCopy + kWideGrad: return step_chunk<f16_t, float, true, SMALL>(t, s, begin, s.chunk);
        case FG_BF16 + kCopy + kWideGrad: return step_chunk<bf16_t, float, true, SMALL>(t, s, begin, s.chunk);
    }
}

// ---- the norm -------------------------------------------------------------------------------------------
constexpr int kNormGroups = 2048;           // of a launch, at most
struct GradArg {
    const void *g;
    int64_t n;
    int32_t dtype;
};

template <class G>
__device__ __forceinline__ double squares_of(const GradArg &t, int64_t begin) {
    constexpr int N = 16 / (int)sizeof(G) * 2;
    const int64_t end = begin + kChunk < t.n ? begin + kChunk : t.n;
    double sum = 0.0;
    for (int64_t at = begin + threadIdx.x * N; at < end; at += kThreads * N) {
        float g[N];
        load_values<G, N>((const G *)t.g, at, t.n, g);
#pragma unroll
        for (int e = 0; e < N; ++e) sum += (double)g[e] * (double)g[e];
    }
    return sum;
}

// Sum over a workgroup of W waves, by halves; in the first thread.
template <int W>
__device__ __forceinline__ double group_total(double v, double *slots) {
    slots[threadIdx.x] = v;
    __syncthreads();
    for (int half = 32 * W; half > 0; half /= 2) {
        if ((int)threadIdx.x < half) slots[threadIdx.x] += slots[threadIdx.x + half];
        __syncthreads();
    }
    return slots[0];
}

// Sums in 64 bits: of 10^9 squares nothing is lost, and those of the largest and smallest FP32 values have room.
template <int CAP>
__global__ __launch_bounds__(kThreads) void grad_squares(const List<GradArg, CAP> a, int chunks, double *partial) {
    __shared__ double slots[kThreads];
    double sum = 0.0;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int which = tensor_of(a, c);
        const GradArg t = a.at[which];
        const int64_t begin = ((int64_t)c - a.first[which]) * kChunk;
        sum += t.dtype == FG_F16 ? squares_of<f16_t>(t, begin) : t.dtype == FG_BF16 ? squares_of<bf16_t>(t, begin) : squares_of<float>(t, begin);
    }
    sum = group_total<kThreads / 64>(sum, slots);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm(const double *partial, int64_t parts, double scale, double max_norm, float *norm, float *factor) {
    __shared__ double slots[1024];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < parts; i += 1024) sum += partial[i];
    sum = group_total<16>(sum, slots);
    if (threadIdx.x != 0) return;
    const double n = __builtin_sqrt(sum) * scale;
    *norm = (float)n;
    // (a norm that is no finite FP32 number gives a factor that is none)
    if (factor) *factor = !((float)n < __builtin_inff()) ? __builtin_nanf("") : (float)(n > max_norm ? max_norm / n * scale : scale);
}

// ---- host ------------------------------------------------------------------------------------------------
constexpr int kFewTensors = 6, kFewGrads = 16, kMoreGrads = 64, kMostGrads = 128;
template <bool SMALL> constexpr int kMostTensors = SMALL ? 48 : 64;
template <bool SMALL> constexpr int kMostNear = SMALL ? 100 : 120;
constexpr int64_t kMostChunks = 1 << 23;    // of a launch: fewer than 2^32 threads

int64_t chunks_of(int64_t n, int chunk) { return (n + chunk - 1) / chunk; }

fg_status check_tensor_count(int64_t count, const void *tensors) {
    if (count < 0) return fail(FG_ERR_SHAPE, "negative number of tensors: %lld", (long long)count);
    if (count > 0 && !tensors) return fail(FG_ERR_NULL, "the list of tensors is NULL");
    return FG_OK;
}
fg_status check_values(const char *name, int64_t i, const void *p, int dtype, int64_t n) {
    if (!element_bytes(dtype)) return fail(FG_ERR_LAYOUT, "tensor %lld: %s must be FG_F16, FG_BF16 or FG_F32", (long long)i, name);
    if (n > 0 && !p) return fail(FG_ERR_NULL, "tensor %lld: %s is NULL", (long long)i, name);
    if (!aligned_to(p, element_bytes(dtype))) return fail(FG_ERR_ALIGN, "tensor %lld: %s must be aligned to an element", (long long)i, name);
    return FG_OK;
}
fg_status check_length(int64_t i, int64_t n) {
    if (n < 0) return fail(FG_ERR_SHAPE, "tensor %lld: negative length %lld", (long long)i, (long long)n);
    if (n > kMostChunks * kChunk) return fail(FG_ERR_UNSUPPORTED, "tensor %lld: more than 2^36 values are not supported", (long long)i);
    return FG_OK;
}

fg_status check_adamw_tensor(int64_t i, const fg_adamw_tensor &t) {
    if (fg_status st = check_length(i, t.n)) return st;
    if (fg_status st = check_values("param", i, t.param, t.param_dtype, t.n)) return st;
    if (fg_status st = check_values("grad", i, t.grad, t.grad_dtype, t.n)) return st;
    if (t.grad_dtype != FG_F32 && t.grad_dtype != t.param_dtype) return fail(FG_ERR_LAYOUT, "tensor %lld: grad must be FG_F32 or of the type of param", (long long)i);
    if (t.master && t.param_dtype == FG_F32) return fail(FG_ERR_LAYOUT, "tensor %lld: FG_F32 parameters have no other FP32 copy", (long long)i);
    if (t.n > 0 && (!t.exp_avg || !t.exp_avg_sq)) return fail(FG_ERR_NULL, "tensor %lld: exp_avg or exp_avg_sq is NULL", (long long)i);
    if (!t.avg_scale != !t.sq_scale) return fail(FG_ERR_NULL, "tensor %lld: moments in eight bits need both scales", (long long)i);
    const unsigned align = t.avg_scale ? 16 : 4;
    if (!aligned_to(t.exp_avg, align) || !aligned_to(t.exp_avg_sq, align)) return fail(FG_ERR_ALIGN, "tensor %lld: moments must be aligned to %u bytes", (long long)i, align);
    if (!aligned_to(t.master, 4) || !aligned_to(t.avg_scale, 4) || !aligned_to(t.sq_scale, 4))
        return fail(FG_ERR_ALIGN, "tensor %lld: master, avg_scale and sq_scale must be aligned to an element", (long long)i);
    return FG_OK;
}

// The arrays of a tensor (end 0: it has none such); all but the first are written.
constexpr int kArrays = 7;
constexpr const char *kArrayNames[kArrays] = {"grad", "param", "master", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale"};
struct Arrays {
    uintptr_t begin[kArrays], end[kArrays];
    explicit Arrays(const fg_adamw_tensor &t) {
        const int64_t moment = t.n * (t.avg_scale ? 1 : 4), scales = (t.n + kStateBlock - 1) / kStateBlock * 4;
        const struct { const void *at; int64_t bytes; } arrays[kArrays] = {{t.grad, t.n * element_bytes(t.grad_dtype)}, {t.param, t.n * element_bytes(t.param_dtype)}, {t.master, t.n * 4},
                                                                           {t.exp_avg, moment}, {t.exp_avg_sq, moment}, {t.avg_scale, scales}, {t.sq_scale, scales}};
        for (int k = 0; k < kArrays; ++k) {
            begin[k] = (uintptr_t)arrays[k].at;
            end[k] = arrays[k].at && t.n > 0 ? begin[k] + (uintptr_t)arrays[k].bytes : 0;
        }
    }
};

// What one workgroup writes another would read or write at the same time.  (Host time of a call with 193 tensors: packed into one memory 17 us, of which this is less than one; allocated one
// by one 22; in shuffled order 23; each list in an order of its own 33.)
fg_status check_apart(int64_t count, const fg_adamw_tensor *tensors, const int64_t *step, const float *grad_factor, const float *lr_factor) {
    const struct { const char *name; uintptr_t at, bytes; } values[] = {{"step", (uintptr_t)step, 8}, {"grad_factor", (uintptr_t)grad_factor, 4}, {"lr_factor", (uintptr_t)lr_factor, 4}};
    constexpr int kValues = 3;
    // Each kind of array in the order of the tensors and away from the other kinds: nothing more to look at.
    uintptr_t begin[kArrays], end[kArrays] = {}, last = 0;
    for (uintptr_t &b : begin) b = UINTPTR_MAX;
    bool apart = true;
    int64_t falls = 0;
    for (int64_t i = 0; i < count; ++i) {
        const Arrays a(tensors[i]);
        if (tensors[i].n == 0) continue;
        falls += a.begin[1] < last;
        last = a.begin[1];
        for (int k = 0; k < kArrays; ++k) {
            if (!a.end[k]) continue;
            apart &= k == 0 || a.begin[k] >= end[k];
            begin[k] = std::min(begin[k], a.begin[k]);
            end[k] = std::max(end[k], a.end[k]);
        }
    }
    for (int k = 1; k < kArrays; ++k) {
        for (int j = 0; j < k; ++j) apart &= end[j] <= begin[k] || end[k] <= begin[j];
        for (const auto &v : values) apart &= !v.at || v.at + v.bytes <= begin[k] || end[k] <= v.at;
    }
    if (apart) return FG_OK;
    try {
        // Lists whose tensors are in another order than their memory are mostly all in the same one: that of the parameters.
        std::vector<std::pair<uintptr_t, int64_t>> order;
        if (falls > count / 8 && falls < count - count / 8) {
            for (int64_t i = 0; i < count; ++i) order.push_back({(uintptr_t)tensors[i].param, i});
            std::sort(order.begin(), order.end());
        }
        // of: kArrays i + k, array k of tensor i; -1 - j, a value
        std::vector<Arrays> arrays;
        arrays.reserve((size_t)count);
        for (int64_t i = 0; i < count; ++i) arrays.emplace_back(tensors[order.empty() ? i : order[(size_t)i].second]);
        auto array = [&](int k, int64_t i) {
            const Arrays &a = arrays[(size_t)i];
            return Span{a.begin[k], a.end[k], kArrays * (order.empty() ? i : order[(size_t)i].second) + k, k > 0};
        };
        auto any = [&](int k, int64_t i) {
            if (k < kArrays) return array(k, i);
            const auto &v = values[k - kArrays];
            return Span{v.at, i == 0 && v.at ? v.at + v.bytes : 0, kArrays - 1 - k, false};
        };
        Span x, y, first, second;
        if (!shared_spans(kArrays + kValues, count, any, x, y)) return FG_OK;
        for (int k = 1; k < kArrays; ++k)               // (the plainest words for it)
            if (shared_spans(1, count, [&](int, int64_t i) { return array(k, i); }, first, second))
                return fail(FG_ERR_LAYOUT, "tensors %lld and %lld have values of %s in common", (long long)(first.of / kArrays), (long long)(second.of / kArrays), kArrayNames[k]);
        for (int64_t i = 0; i < count; ++i)
            if (tensors[i].n > 0 && (tensors[i].exp_avg == tensors[i].exp_avg_sq || (tensors[i].avg_scale && tensors[i].avg_scale == tensors[i].sq_scale)))
                return fail(FG_ERR_LAYOUT, "tensor %lld: both moments are in the same memory", (long long)i);
        if (x.of < 0 || y.of < 0) {
            const Span &in = x.of < 0 ? y : x, &value = x.of < 0 ? x : y;
            return fail(FG_ERR_LAYOUT, "%s is in %s of tensor %lld", values[-1 - value.of].name, kArrayNames[in.of % kArrays], (long long)(in.of / kArrays));
        }
        return fail(FG_ERR_LAYOUT, "%s of tensor %lld and %s of tensor %lld have memory in common", kArrayNames[x.of % kArrays], (long long)(x.of / kArrays), kArrayNames[y.of % kArrays],
                    (long long)(y.of / kArrays));
    } catch (const std::bad_alloc &) {
        return fail(FG_ERR_UNSUPPORTED, "no host memory for a list of %lld tensors", (long long)count);
    }
}

// The lowest address of the tensors' memory; 0 where some begins too far from it for NearArg.
uintptr_t near_base(int64_t count, const fg_adamw_tensor *tensors) {
    uintptr_t low = UINTPTR_MAX, high = 0;
    for (int64_t i = 0; i < count; ++i) {
        const fg_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        for (const void *p : {(const void *)t.param, t.grad, (const void *)t.master, (const void *)t.exp_avg, (const void *)t.exp_avg_sq, (const void *)t.avg_scale, (const void *)t.sq_scale}) {
            if (!p) continue;
            low = std::min(low, (uintptr_t)p);
            high = std::max(high, (uintptr_t)p);
        }
    }
    return high - low < kNear ? low : 0;
}

// Hands out tensors to launches: f(first tensor, tensors, chunks) with as many as `most` and kMostChunks allow; tensors without values count as well.
template <class Length, class F> void in_launches(int64_t count, int most, int chunk, Length &&length, F &&f) {
    int64_t begin = 0, chunks = 0;
    for (int64_t i = 0; i < count; ++i) {
        const int64_t c = chunks_of(length(i), chunk);
        if (i > begin && (i - begin == most || chunks + c > kMostChunks)) {
            f(begin, (int)(i - begin), chunks);
            begin = i;
            chunks = 0;
        }
        chunks += c;
    }
    if (count > begin) f(begin, (int)(count - begin), chunks);
}
// The list of a launch's n tensors: fill(i, its arguments) sets one's arguments, length(i) its values.
template <class Arg, int CAP, class Length, class Fill> void make_list(List<Arg, CAP> &list, int n, int chunk, Length &&length, Fill &&fill) {
    int64_t first = 0;
    for (int i = 0; i < CAP; ++i) {
        list.first[i] = (int32_t)first;
        if (i >= n) continue;
        fill(i, list.at[i]);
        first += chunks_of(length(i), chunk);
    }
}

}  // namespace

hipError_t load_adamw_kernels() {
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)grad_norm);
}

}  // namespace fg

using namespace fg;

extern "C" {

fg_status fg_adamw(int64_t count, const fg_adamw_tensor *tensors, const int64_t *step, double lr, double beta1, double beta2, double eps,
                   double weight_decay, const float *grad_factor, const float *lr_factor, void *hip_stream) {
    if (fg_status st = check_tensor_count(count, tensors)) return st;
    if (!std::isfinite(lr) || !std::isfinite(weight_decay)) return fail(FG_ERR_SHAPE, "lr and weight_decay must be finite");
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1)) return fail(FG_ERR_SHAPE, "beta1 and beta2 must be at least 0 and below 1");
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(FG_ERR_SHAPE, "eps must not be negative");
    if (!step) return fail(FG_ERR_NULL, "step is NULL");
    if (!aligned_to(step, 8) || !aligned_to(grad_factor, 4) || !aligned_to(lr_factor, 4))
        return fail(FG_ERR_ALIGN, "step, grad_factor and lr_factor must be aligned to an element");
    bool some[2] = {};
    int64_t values = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (fg_status st = check_adamw_tensor(i, tensors[i])) return st;
        values = std::min(values + tensors[i].n, kSmallModel);
        if (tensors[i].n > 0) some[tensors[i].avg_scale != nullptr] = true;
    }
    if (some[0] && some[1]) return fail(FG_ERR_UNSUPPORTED, "moments in FP32 and in eight bits need calls of their own");
    if (!some[0] && !some[1]) return FG_OK;
    if (fg_status st = check_apart(count, tensors, step, grad_factor, lr_factor)) return st;
    const int chunk = values < kSmallModel ? kSmallChunk : kChunk;
    Launches enqueue(hip_stream);
    auto all = [&](auto small) {
        constexpr bool SMALL = decltype(small)::value;
        // A small model takes as long as its launches; one of more tensors than the long list has is handed over as NearArg where its memory allows it
        // (193 tensors of 1.6 M values: four launches 24.7 us, two 17.8; with moments in eight bits five 45 and two 19).
        const uintptr_t base = values < kSmallModel && count > kMostTensors<SMALL> ? near_base(count, tensors) : 0;
        auto launch = [&](auto cap, auto list_of, int64_t begin, int n, int64_t chunks) {
            constexpr int CAP = decltype(cap)::value;
            using Arg = decltype(list_of);
            List<Arg, CAP> a = {};
            static_assert(sizeof a + sizeof(StepArgs) <= 4096, "");
            make_list(a, n, chunk, [&](int i) { return tensors[begin + i].n; }, [&](int i, Arg &arg) {
                const fg_adamw_tensor &t = tensors[begin + i];
                const int kind = t.param_dtype + (t.grad_dtype == FG_F32 ? kWideGrad : 0) + (t.master ? kCopy : 0);
                if constexpr (!std::is_same<Arg, NearArg<SMALL>>::value) {
                    arg.p = t.param; arg.g = t.grad; arg.master = t.master; arg.m = t.exp_avg; arg.v = t.exp_avg_sq; arg.n = t.n; arg.kind = kind;
                    if constexpr (SMALL) { arg.m_scale = t.avg_scale; arg.v_scale = t.sq_scale; }
                } else if constexpr (SMALL) arg.set(t.n, kind, base, {t.param, t.grad, t.master, t.exp_avg, t.exp_avg_sq, t.avg_scale, t.sq_scale});
                else arg.set(t.n, kind, base, {t.param, t.grad, t.master, t.exp_avg, t.exp_avg_sq});
            });
            const StepArgs s = {lr, beta1, beta2, eps, weight_decay, step, grad_factor, lr_factor, (char *)base, chunk};
            enqueue(adamw<CAP, SMALL, Arg>, dim3((unsigned)chunks), dim3(kThreads), a, s);
        };
        in_launches(count, base ? kMostNear<SMALL> : kMostTensors<SMALL>, chunk, [&](int64_t i) { return tensors[i].n; }, [&](int64_t begin, int n, int64_t chunks) {
            using std::integral_constant;
            if (chunks == 0) return;
            if (n <= kFewTensors) launch(integral_constant<int, kFewTensors>{}, TensorArg<SMALL>{}, begin, n, chunks);
            else if (n <= kMostTensors<SMALL>) launch(integral_constant<int, kMostTensors<SMALL>>{}, TensorArg<SMALL>{}, begin, n, chunks);
            else launch(integral_constant<int, kMostNear<SMALL>>{}, NearArg<SMALL>{}, begin, n, chunks);
        });
    };
    if (some[1]) all(std::true_type{});
    else all(std::false_type{});
    return enqueue.status("adamw");
}

// (a launch more for each 2^36 values: more than four of those have no room on a GPU)
int64_t fg_grad_norm_workspace(int64_t count) { return count <= 0 ? 0 : ((count + kMostGrads - 1) / kMostGrads + 4) * kNormGroups * 8; }

fg_status fg_grad_norm(int64_t count, const fg_values *grads, float scale, float max_norm, float *norm, float *factor, void *workspace,
                       int64_t workspace_bytes, void *hip_stream) {
    if (fg_status st = check_tensor_count(count, grads)) return st;
    if (!norm) return fail(FG_ERR_NULL, "norm is NULL");
    if (!aligned_to(norm, 4) || !aligned_to(factor, 4)) return fail(FG_ERR_ALIGN, "norm and factor must be aligned to an element");
    if (!(scale > 0) || !std::isfinite(scale)) return fail(FG_ERR_SHAPE, "scale must be positive");
    if (!(max_norm > 0)) return fail(FG_ERR_SHAPE, "max_norm must be positive");
    for (int64_t i = 0; i < count; ++i) {
        if (fg_status st = check_length(i, grads[i].n)) return st;
        if (fg_status st = check_values("grad", i, grads[i].values, grads[i].dtype, grads[i].n)) return st;
    }
    int64_t parts = 0;
    auto launches = [&](auto &&f) { in_launches(count, kMostGrads, kChunk, [&](int64_t i) { return grads[i].n; }, f); };
    launches([&](int64_t, int, int64_t chunks) { parts += std::min<int64_t>(chunks, kNormGroups); });
    if (fg_status st = check_workspace(workspace, workspace_bytes, parts * 8)) return st;
    for (int64_t i = 0; i < count; ++i) {
        const uintptr_t begin = (uintptr_t)grads[i].values, end = begin + (uintptr_t)(grads[i].n * element_bytes(grads[i].dtype));
        for (const float *out : {norm, factor})
            if (out && (uintptr_t)out < end && begin < (uintptr_t)out + 4) return fail(FG_ERR_LAYOUT, "%s is in gradient %lld", out == norm ? "norm" : "factor", (long long)i);
    }
    if (norm == factor) return fail(FG_ERR_LAYOUT, "norm and factor are in the same memory");
    Launches enqueue(hip_stream);
    double *partial = (double *)workspace;
    launches([&](int64_t begin, int n, int64_t chunks) {
        if (chunks == 0) return;
        const unsigned groups = (unsigned)std::min<int64_t>(chunks, kNormGroups);
        auto launch = [&](auto cap) {
            constexpr int CAP = decltype(cap)::value;
            List<GradArg, CAP> a = {};
            static_assert(sizeof a <= 4000, "");
            make_list(a, n, kChunk, [&](int i) { return grads[begin + i].n; }, [&](int i, GradArg &arg) {
                arg = {grads[begin + i].values, grads[begin + i].n, grads[begin + i].dtype};
            });
            enqueue(grad_squares<CAP>, dim3(groups), dim3(kThreads), a, (int)chunks, partial);
        };
        if (n <= kFewGrads) launch(std::integral_constant<int, kFewGrads>{});
        else if (n <= kMoreGrads) launch(std::integral_constant<int, kMoreGrads>{});
        else launch(std::integral_constant<int, kMostGrads>{});
        partial += groups;
    });
    enqueue(grad_norm, dim3(1), dim3(1024), (const double *)workspace, parts, (double)scale, (double)max_norm, norm, factor);
    return enqueue.status("grad_norm");
}

}  // extern "C"
