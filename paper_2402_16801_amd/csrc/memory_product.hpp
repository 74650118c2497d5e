// Tiles of a matrix product on the matrix cores, and what is done with a result before it is stored (memory_product.hip).
//
// A product is C[m][n] = sum over k of Q[m][k] P[n][k].  The instruction's first operand is P, so that its result leaves neighbouring
// columns n in one lane; which row of P stands at which place of the instruction is free, and is chosen so that a lane holds
// 4 FP columns in a row (see Tile).
#pragma once

#include "memory_common.hpp"

namespace mem {

// Where row m of a matrix lies: rows are numbered as steps times environments.  n is 1 where one stride does.
struct Rows {
    int64_t step, env;
    uint32_t n;
    __device__ __forceinline__ int64_t at(uint32_t m) const { return n == 1 ? (int64_t)m * step : (int64_t)(m / n) * step + (int64_t)(m % n) * env; }
};

// ---- activations ---------------------------------------------------------------------------------
constexpr float GELU_2K = 1.5957691216057308f, GELU_C = 0.044715f;      // 2 sqrt(2 / pi)

template <int COUNT> __device__ __forceinline__ void activate(float (&v)[COUNT], int act)
{
    if (act == CRAFTAX_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];
    } else if (act == CRAFTAX_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) v[j] *= sigmoid(v[j]);
    } else if (act == CRAFTAX_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) v[j] *= sigmoid(GELU_2K * v[j] * __builtin_fmaf(GELU_C * v[j], v[j], 1.0f));
    }
}
// the derivative at p
__device__ __forceinline__ float slope_of(float p, int act)
{
    if (act == CRAFTAX_ACT_NONE) return 1.0f;
    if (act == CRAFTAX_ACT_RELU) return p > 0.0f ? 1.0f : (p <= 0.0f ? 0.0f : p);
    if (act == CRAFTAX_ACT_SILU) {
        const float g = sigmoid(p);
        return g * __builtin_fmaf(p, 1.0f - g, 1.0f);
    }
    // beyond 16 it is 0 or 1, and the square would leave the range of numbers
    p = p > 16.0f ? 16.0f : (p < -16.0f ? -16.0f : p);
    const float g = sigmoid(GELU_2K * p * __builtin_fmaf(GELU_C * p, p, 1.0f));
    return __builtin_fmaf(p * g * (1.0f - g) * GELU_2K, __builtin_fmaf(3.0f * GELU_C * p, p, 1.0f), g);
}

// ---- what is done with COUNT columns of a row -------------------------------------------------------
// out = residual + act(sum + bias), and pre = sum + bias
template <typename E, typename R> struct Finish {
    const float* bias;
    const R* residual;
    R* out;
    E* pre;
    Rows residual_rows, out_rows, pre_rows;
    int act, columns;
    template <typename P, int COUNT> static __device__ __forceinline__ void store(P* p, int count, const float (&v)[COUNT])
    {
        Pack<P, COUNT> q;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) q.v[j] = Elem<P>::down(v[j]);
        if (count >= COUNT) {
            *reinterpret_cast<Pack<P, COUNT>*>(p) = q;
        } else {
#pragma unroll
            for (int j = 0; j < COUNT; ++j)
                if (j < count) p[j] = q.v[j];
        }
    }
    template <typename P, int COUNT> static __device__ __forceinline__ void add(const P* p, int count, float (&v)[COUNT])
    {
        if (count >= COUNT) {
            const Pack<P, COUNT> q = *reinterpret_cast<const Pack<P, COUNT>*>(p);
#pragma unroll
            for (int j = 0; j < COUNT; ++j) v[j] += Elem<P>::up(q.v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < COUNT; ++j)
                if (j < count) v[j] += Elem<P>::up(p[j]);
        }
    }
    template <int COUNT> __device__ __forceinline__ void operator()(uint32_t m, int n, float (&v)[COUNT]) const
    {
        const int count = columns - n;
        if (count <= 0) return;
        if (bias) add(bias + n, count, v);
        if (pre) store(pre + pre_rows.at(m) + n, count, v);
        activate(v, act);
        if (residual) add(residual + residual_rows.at(m) + n, count, v);
        store(out + out_rows.at(m) + n, count, v);
    }
};

// ---- operands of the matrix instructions --------------------------------------------------------------
// A fragment is 16 rows by 64 bytes along k: lane l holds 16 bytes of row l % 16, from byte 16 (l / 16) on.
typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 BF8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));
typedef short S4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4v __attribute__((ext_vector_type(4)));

template <typename E> struct Frag;
template <> struct Frag<__bf16> {
    static __device__ __forceinline__ F4 times(U4v a, U4v b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(BF8, a), __builtin_bit_cast(BF8, b), c, 0, 0, 0); }
};
template <> struct Frag<_Float16> {
    static __device__ __forceinline__ F4 times(U4v a, U4v b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0); }
};
// 16 values along k in four instructions of four; lane group g has k = 4 g .. 4 g + 3 instead of g, 4 + g, ..: the order of k is free as
// long as both operands have the same
template <> struct Frag<float> {
    static __device__ __forceinline__ F4 times(U4v a, U4v b, F4 c)
    {
        const F4 x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k], y[k], c, 0, 0, 0);
        return c;
    }
};

// up to 16 bytes from p on, of which `count` values are there; the others are 0
template <typename E> __device__ __forceinline__ U4v load_some(const E* p, int count)
{
    constexpr int V = 16 / sizeof(E);
    if (count >= V) return __builtin_bit_cast(U4v, *reinterpret_cast<const Pack<E, V>*>(p));
    Pack<E, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = j < count ? p[j] : (E)0.0f;
    return __builtin_bit_cast(U4v, q);
}

}  // namespace mem
