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

__device__ __forceinline__ float mmm_exp(float v) { return expf(v); }
__device__ __forceinline__ double mmm_exp(double v) { return exp(v); }
__device__ __forceinline__ float mmm_erfc(float v) { return erfcf(v); }
__device__ __forceinline__ double mmm_erfc(double v) { return erfc(v); }

// 1 / (1 + exp(-v)): 0 and 1 where the exponential leaves the range
template <typename E> __device__ __forceinline__ E mmm_sigmoid(E v) { return E(1) / (E(1) + mmm_exp(-v)); }

// act(z).  GELU is z times the normal distribution function, written with erfc, which keeps its digits for negative z; its tanh
// form is z times a sigmoid: (1 + tanh u) / 2 = sigmoid(2 u).  An infinite -z is 0 in the limit, where z times 0 is NaN.
template <typename E, int N> __device__ __forceinline__ void mmm_activate(E (&z)[N], int32_t act)
{
    if (act == MMM_ACT_RELU) {
#pragma unroll
        for (int q = 0; q < N; ++q) z[q] = z[q] < E(0) ? E(0) : z[q];
    } else if (act != MMM_ACT_NONE) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            E p;
            if (act == MMM_ACT_GELU)
                p = E(0.5) * mmm_erfc(z[q] * E(-0.70710678118654752440));
            else if (act == MMM_ACT_GELU_TANH)
                p = mmm_sigmoid(E(1.5957691216057307117) * z[q] * (E(1) + E(0.044715) * z[q] * z[q]));   // 2 sqrt(2 / pi)
            else
                p = mmm_sigmoid(z[q]);
            z[q] = p == E(0) ? E(0) : z[q] * p;
        }
    }
}

// act'(z); that of ReLU at 0 is 0.  The terms with z vanish in both limits.
__device__ __forceinline__ float mmm_slope(float z, int32_t act)
{
    switch (act) {
    case MMM_ACT_RELU: return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    case MMM_ACT_GELU: {
        const float e = expf(-0.5f * z * z);
        return 0.5f * erfcf(z * -0.70710678118654752440f) + (e == 0.f ? 0.f : z * e * 0.39894228040143267794f);   // 1 / sqrt(2 pi)
    }
    case MMM_ACT_GELU_TANH: {
        const float p = mmm_sigmoid(1.5957691216057307117f * z * (1.f + 0.044715f * z * z));
        const float w = p * mmm_sigmoid(-1.5957691216057307117f * z * (1.f + 0.044715f * z * z));   // p (1 - p)
        return p + (w == 0.f ? 0.f : z * w * 1.5957691216057307117f * (1.f + 0.134145f * z * z));
    }
    case MMM_ACT_SILU: {
        const float p = mmm_sigmoid(z), w = p * mmm_sigmoid(-z);
        return p + (w == 0.f ? 0.f : z * w);
    }
    }
    return 1.f;
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

// The epilogue of N neighbours of rows of C: what is the same in every row, and what is done to one.  T: type of the inputs, E: of the sums.
template <typename T, typename E, int N> struct mmm_column_values {
    E bias[N];
    __device__ __forceinline__ void load(const mmm_epilogue_args &e, int64_t col)
    {
#pragma unroll
        for (int q = 0; q < N; ++q) bias[q] = E(0);
        if (e.bias != nullptr) mmm_load_as<T, E, N>(e.bias, col, bias);
    }
    __device__ __forceinline__ void finish(const mmm_epilogue_args &e, const E (&sum)[N], void *C, int64_t ldc, int64_t row, int64_t col) const
    {
        const bool wide = sizeof(T) == sizeof(E) || e.out_dtype == MMM_F32;
        auto load = [&](const void *base, int64_t ld, E (&out)[N]) __attribute__((always_inline)) {
            if (wide)
                mmm_load_as<E, E, N>(base, row * ld + col, out);
            else
                mmm_load_as<T, E, N>(base, row * ld + col, out);
        };
        auto store = [&](void *base, int64_t ld, const E (&in)[N]) __attribute__((always_inline)) {
            if (wide)
                mmm_store_as<E, E, N>(base, row * ld + col, in);
            else
                mmm_store_as<T, E, N>(base, row * ld + col, in);
        };
        E z[N], more[N];
        if (e.residual != nullptr) load(e.residual, e.ldr, more);
#pragma unroll
        for (int q = 0; q < N; ++q) z[q] = e.bias != nullptr ? sum[q] + bias[q] : sum[q];
        if (e.preact != nullptr) store(e.preact, e.ldp, z);
        mmm_activate(z, e.activation);
        if (e.residual != nullptr)
#pragma unroll
            for (int q = 0; q < N; ++q) z[q] += more[q];
        store(C, ldc, z);
    }
};
