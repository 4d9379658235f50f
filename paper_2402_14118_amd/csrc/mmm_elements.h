// Elements of the types the library takes, eight of a row at a time, and what is computed of one: activations and their slopes.
// Device code shared by the epilogue of the multiplication, its gradient and the norms.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mmm_internal.h"

// what a type is computed in
template <typename T> struct mmm_wide { typedef float type; };
template <> struct mmm_wide<double> { typedef double type; };

// N neighbours of a row that starts at any element
template <typename T, int N> struct mmm_row_piece {
    typedef T vec __attribute__((ext_vector_type(N)));
    typedef vec type __attribute__((aligned(sizeof(T)), may_alias));
};

constexpr int MMM_PIECE = 8;   // elements of a row per lane and access: 16 bytes of the 16-bit types

// the first `n` of eight elements of a row, as floats; the others are zero
template <typename T> __device__ __forceinline__ void mmm_load_piece(const T *at, int n, float (&out)[MMM_PIECE])
{
    if (n >= MMM_PIECE) {
        typedef typename mmm_row_piece<T, MMM_PIECE>::type piece;
        const piece v = *reinterpret_cast<const piece *>(at);
#pragma unroll
        for (int q = 0; q < MMM_PIECE; ++q) out[q] = (float)v[q];
    } else {
#pragma unroll
        for (int q = 0; q < MMM_PIECE; ++q) out[q] = q < n ? (float)at[q] : 0.f;
    }
}
// the same, left as they are
template <typename T> struct mmm_raw_piece { typedef T type __attribute__((ext_vector_type(MMM_PIECE))); };
template <typename T> __device__ __forceinline__ typename mmm_raw_piece<T>::type mmm_load_raw(const T *at, int n)
{
    typedef typename mmm_row_piece<T, MMM_PIECE>::type piece;
    typename mmm_raw_piece<T>::type v;
    if (n >= MMM_PIECE) {
        v = *reinterpret_cast<const piece *>(at);
    } else {
#pragma unroll
        for (int q = 0; q < MMM_PIECE; ++q) v[q] = q < n ? at[q] : (T)0.f;
    }
    return v;
}
// the first `n` of eight values to a row, rounded to nearest even once
template <typename T> __device__ __forceinline__ void mmm_store_piece(T *at, int n, const float (&in)[MMM_PIECE])
{
    if (n >= MMM_PIECE) {
        typedef typename mmm_row_piece<T, MMM_PIECE>::type piece;
        piece v;
#pragma unroll
        for (int q = 0; q < MMM_PIECE; ++q) v[q] = (T)in[q];
        *reinterpret_cast<piece *>(at) = v;
    } else {
#pragma unroll
        for (int q = 0; q < MMM_PIECE; ++q)
            if (q < n) at[q] = (T)in[q];
    }
}

// e^(v + less) for v from -120 to 88, `less` small: 2^y of the vector unit with what the product of v and log2 e is rounded by put back (v up to a
// hundred is rounded by a hundred times 2^-25, as much relative to the result).
__device__ __forceinline__ float mmm_exp(float v, float less = 0.f)
{
    constexpr float L = 1.44269502162933349609375f, MORE = 1.925963033500e-8f;   // log2 e in two parts
    const float y = v * L, rest = __builtin_fmaf(v, L, -y) + __builtin_fmaf(v, MORE, less * L);
    const float e = __builtin_amdgcn_exp2f(y);
    return __builtin_fmaf(e, rest * 0.693147180559945f, e);
}
// 1 / (1 + e^-v); 0 and 1 in the limits, and something between for NaN
__device__ __forceinline__ float mmm_sigmoid(float v)
{
    const float e = mmm_exp(fminf(fmaxf(-v, -87.f), 87.f));
    return v < -87.f ? 0.f : __builtin_amdgcn_rcpf(1.f + e);
}
__device__ __forceinline__ double mmm_sigmoid(double v) { return 1.0 / (1.0 + exp(-v)); }

// The normal distribution function, and e^(-z^2 / 2).  For u = |z|, x = u / sqrt 2: Phi(-u) = erfc(x) / 2 = e^(-x^2) (t Q(t)) with t = 1 / (1 + 0.3 x), where
// e^(x^2) erfc(x) / t is smooth: Q, of degree 8, was fitted to it for u up to 15 (least squares, weighted until the largest relative error was
// least: 2.0e-8).  Behind that the result is 0 in float.  One path for all lanes: the library's erfc takes both sides of its branches in a wave (777 x 3001 x
// 1992 half with GELU 17.5 us, with this 16.6; the gradient through GELU, 777 x 1992, 7.7 and 6.1).  Off by up to 8 times 2^-24 of it.
// FINE (results that stay floats): t Q(t) answers a rounding of t with up to 3.7 times as much.  What t is off by, relative to it, is worked out and taken off, and so is what
// the two products are rounded by: up to 5 times 2^-24, and the 2-norm of GELU's slope over N(-.5, 1) is off by 4.8e-8 instead of 8.7e-8 of it (1024 x 512 x 16384 floats 144.8 -> 147.0 us,
// 777 x 3001 x 1992 104.6 -> 105.0, gradients the same).
template <bool FINE> __device__ __forceinline__ float mmm_normal(float z, float &bell)
{
    constexpr float S = 0.212132034355964f;   // 0.3 / sqrt 2
    const float u = fminf(fabsf(z), 15.f), square = u * u;
    bell = mmm_exp(-0.5f * square, -0.5f * __builtin_fmaf(u, u, -square));
    const float one_and = __builtin_fmaf(u, S, 1.f), t = __builtin_amdgcn_rcpf(one_and);
    float q = -0.0647779107093811f;
    q = __builtin_fmaf(q, t, 0.24286802113056183f);
    q = __builtin_fmaf(q, t, -0.256333589553833f);
    q = __builtin_fmaf(q, t, 0.27410486340522766f);
    q = __builtin_fmaf(q, t, -0.047513507306575775f);
    q = __builtin_fmaf(q, t, 0.10755327343940735f);
    q = __builtin_fmaf(q, t, 0.07414324581623077f);
    q = __builtin_fmaf(q, t, 0.08536188304424286f);
    q = __builtin_fmaf(q, t, 0.08459370583295822f);   // (Q / 2)
    float tail;
    if constexpr (FINE) {
        // t (1 + off) is the reciprocal; (t Q)' t / (t Q) is a straight line within .07; products and what they leave
        const float more = __builtin_fmaf(u, S, -(one_and - 1.f)), off = __builtin_fmaf(-t, more, __builtin_fmaf(-t, one_and, 1.f));
        const float by = off * __builtin_fmaf(t, 3.9457922f, -0.23464205f);
        const float tq = t * q, tq_left = __builtin_fmaf(t, q, -tq), all = bell * tq, all_left = __builtin_fmaf(bell, tq, -all);
        tail = all + __builtin_fmaf(all, by, __builtin_fmaf(bell, tq_left, all_left));
    } else {
        tail = bell * t * q;
    }
    return z < 0.f ? tail : 1.f - tail;
}
template <bool FINE> __device__ __forceinline__ float mmm_normal(float z)
{
    float bell;
    return mmm_normal<FINE>(z, bell);
}
template <bool> __device__ __forceinline__ double mmm_normal(double z) { return 0.5 * erfc(z * -0.70710678118654752440); }

// act(z): GELU is z times the normal distribution function; its tanh form is z times a sigmoid: (1 + tanh u) / 2 = sigmoid(2 u).  An infinite -z is 0 in
// the limit, where z times 0 is NaN.  T: type of the operands.
template <typename T, typename E, int N> __device__ __forceinline__ void mmm_activate(E (&z)[N], int32_t act)
{
    if (act == MMM_ACT_RELU) {
#pragma unroll
        for (int q = 0; q < N; ++q) z[q] = z[q] < E(0) ? E(0) : z[q];
    } else if (act == MMM_ACT_GELU) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const E p = mmm_normal<sizeof(T) == 4>(z[q]);
            z[q] = p == E(0) ? E(0) : z[q] * p;
        }
    } else if (act != MMM_ACT_NONE) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const E p = mmm_sigmoid(act == MMM_ACT_SILU ? z[q] : E(1.5957691216057307117) * z[q] * (E(1) + E(0.044715) * z[q] * z[q]));   // 2 sqrt(2 / pi)
            z[q] = p == E(0) ? E(0) : z[q] * p;
        }
    }
}

// d[q] *= act'(z[q]); that of ReLU at 0 is 0, at NaN NaN.  The terms with z vanish in both limits.  T: type of the result.
template <typename T, int N> __device__ __forceinline__ void mmm_apply_slope(float (&d)[N], const float (&z)[N], int32_t act)
{
    if (act == MMM_ACT_RELU) {
#pragma unroll
        for (int q = 0; q < N; ++q) d[q] *= z[q] > 0.f ? 1.f : z[q] <= 0.f ? 0.f : z[q];
    } else if (act == MMM_ACT_GELU) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            float bell;
            const float p = mmm_normal<sizeof(T) == 4>(z[q], bell), more = z[q] * bell * 0.39894228040143267794f;   // 1 / sqrt(2 pi)
            d[q] *= fabsf(z[q]) > 15.f ? p : p + more;
        }
    } else if (act != MMM_ACT_NONE) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const bool silu = act == MMM_ACT_SILU;
            const float at = silu ? z[q] : 1.5957691216057307117f * z[q] * (1.f + 0.044715f * z[q] * z[q]);
            const float p = mmm_sigmoid(at), w = p * mmm_sigmoid(-at);   // p (1 - p)
            d[q] *= w == 0.f ? p : p + z[q] * w * (silu ? 1.f : 1.5957691216057307117f * (1.f + 0.134145f * z[q] * z[q]));
        }
    }
}

// N neighbours of a row of either type, as E
template <typename T, typename E, int N> __device__ __forceinline__ void mmm_load_as(const void *base, int64_t at, E (&out)[N])
{
    typedef typename mmm_row_piece<T, N>::type piece;
    const piece v = *reinterpret_cast<const piece *>(static_cast<const T *>(base) + at);
#pragma unroll
    for (int q = 0; q < N; ++q) out[q] = (E)v[q];
}
template <typename T, typename E, int N> __device__ __forceinline__ void mmm_store_as(void *base, int64_t at, const E (&in)[N])
{
    typedef typename mmm_row_piece<T, N>::type piece;
    piece v;
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = (T)in[q];
    *reinterpret_cast<piece *>(static_cast<T *>(base) + at) = v;
}

// The epilogue of N neighbours of rows of C, in steps: what is the same in every row; what is asked for of a row ahead of its sums; Z and act(Z); C.
// T: type of the inputs, E: of the sums.
template <typename T, typename E, int N> struct mmm_column_values {
    E bias[N];
    bool wide;   // C, residual and Z are of the type of the sums
    __device__ __forceinline__ void load(const mmm_epilogue_args &e, int64_t col)
    {
        wide = sizeof(T) == sizeof(E) || e.out_dtype == MMM_F32;
#pragma unroll
        for (int q = 0; q < N; ++q) bias[q] = E(0);
        if (e.bias != nullptr) mmm_load_as<T, E, N>(e.bias, col, bias);
    }
    // (element by element without a residual: nothing is read, and nothing is added)
    __device__ __forceinline__ void residual(const mmm_epilogue_args &e, int64_t row, int64_t col, E (&more)[N]) const
    {
        if (e.residual == nullptr) return;
        if (wide)
            mmm_load_as<E, E, N>(e.residual, row * e.ldr + col, more);
        else
            mmm_load_as<T, E, N>(e.residual, row * e.ldr + col, more);
    }
    __device__ __forceinline__ void store(void *base, int64_t ld, int64_t row, int64_t col, const E (&v)[N]) const
    {
        if (wide)
            mmm_store_as<E, E, N>(base, row * ld + col, v);
        else
            mmm_store_as<T, E, N>(base, row * ld + col, v);
    }
    __device__ __forceinline__ void activate(const mmm_epilogue_args &e, E (&z)[N], int64_t row, int64_t col) const
    {
        if (e.bias != nullptr)
#pragma unroll
            for (int q = 0; q < N; ++q) z[q] += bias[q];
        if (e.preact != nullptr) store(e.preact, e.ldp, row, col, z);
        mmm_activate<T>(z, e.activation);
    }
    __device__ __forceinline__ void finish(const mmm_epilogue_args &e, E (&z)[N], const E (&more)[N], void *C, int64_t ldc, int64_t row, int64_t col) const
    {
        if (e.residual != nullptr)
#pragma unroll
            for (int q = 0; q < N; ++q) z[q] += more[q];
        store(C, ldc, row, col, z);
    }
};
