// What the policy memory operators share: element types, vectors of activations, moves across lanes,
// sums of partial results, and the host's checks.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/craftax.h"
#include "memory_grid.hpp"

namespace mem {

constexpr int WAVE = 64;
constexpr int CHIP_SIMDS = 1024;      // 256 compute units of four

// ---- element types ----------------------------------------------------------------------------
// Arithmetic is in float; an activation is rounded once, to nearest even, when it is stored.
template <typename E> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Elem<__bf16> {
    static __device__ __forceinline__ float up(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 down(float v) { return (__bf16)v; }
};
template <> struct Elem<_Float16> {
    static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
};

// V elements in a row, loaded and stored at once; gfx950 takes 4-, 8- and 16-byte accesses at any
// address in global memory, so only elements are aligned.
template <typename E, int V> struct alignas(sizeof(E)) Pack { E v[V]; };

// a view on the device
template <typename P> struct Seq {
    P* data;
    int64_t step, env;
    __device__ __forceinline__ P* at(int t, int i) const { return data + (int64_t)t * step + (int64_t)i * env; }
};

// ---- elementary functions ------------------------------------------------------------------------
// One hardware exponential and reciprocal each (relative error about 2^-23).
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

__device__ __forceinline__ float sigmoid(float v)
{
    return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-v * LOG2E));
}

// max(v, 0) + log(1 + e) with e = exp(-|v|): log(1 + e) = 2 artanh(q) with q = e / (2 + e) <= 1/3, whose
// series q (2 + 2/3 q^2 + 2/5 q^4 + ...) is below 2^-24 of its sum after eight terms.  No digit of a
// small e is lost, as it would be in 1 + e.
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp2_fast(-__builtin_fabsf(v) * LOG2E);
    const float q = e * __builtin_amdgcn_rcpf(2.0f + e), s = q * q;
    float r = 2.0f / 15.0f;
#pragma unroll
    for (int k = 13; k >= 1; k -= 2) r = __builtin_fmaf(r, s, 2.0f / (float)k);
    return (v < 0.0f ? 0.0f : v) + q * r;
}

// v is computed, or has arrived from memory, here and not where it is used
__device__ __forceinline__ void pin(float& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void pin(uint32_t& v) { asm volatile("" : "+v"(v)); }
template <typename E> __device__ __forceinline__ void pin16(E& v)
{
    uint16_t bits = __builtin_bit_cast(uint16_t, v);
    asm volatile("" : "+v"(bits));
    v = __builtin_bit_cast(E, bits);
}
__device__ __forceinline__ void pin(__bf16& v) { pin16(v); }
__device__ __forceinline__ void pin(_Float16& v) { pin16(v); }
template <typename T, int N> __device__ __forceinline__ void pin(T (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) pin(v[k]);
}

template <typename T, int N, int M> __device__ __forceinline__ void pin(T (&v)[N][M])
{
#pragma unroll
    for (int k = 0; k < N; ++k) pin(v[k]);
}

// ---- moves across lanes ----------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_ROR8 = 0x128;

struct Pair { float a, b; };
// upper 32 lanes of a <-> lower 32 lanes of b
__device__ __forceinline__ Pair swap32(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// odd rows of 16 lanes of a <-> even rows of b
__device__ __forceinline__ Pair swap16(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// sum over the 64 lanes, in every lane (the order of the additions is fixed)
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp<DPP_XOR1>(v);
    v += dpp<DPP_XOR2>(v);
    v += dpp<DPP_HALF_MIRROR>(v);
    v += dpp<DPP_ROR8>(v);
    Pair p = swap16(v, v);
    v = p.a + p.b;
    p = swap32(v, v);
    return p.a + p.b;
}

// the block's number in a launch that lies over x and z (see spread), `wide` blocks in x: an argument, since the grid's own size arrives
// later than those
__device__ __forceinline__ int64_t spread_block(unsigned wide) { return (int64_t)((uint64_t)blockIdx.z * wide + blockIdx.x); }

// ---- sums of partial results -----------------------------------------------------------------------
// put(c, sum over rows of part[row][c]) for every column: a block takes 16 columns, 16 threads each add
// every 16th row, in a fixed order.
constexpr int SUM_COLUMNS = 16, SUM_ROWS = 16;
template <typename Put>
static __global__ __launch_bounds__(SUM_COLUMNS* SUM_ROWS) void k_sum_rows(const float* part, int rows, int64_t columns, unsigned wide, Put put)
{
    __shared__ float sums[SUM_ROWS][SUM_COLUMNS];
    const int x = threadIdx.x % SUM_COLUMNS, y = threadIdx.x / SUM_COLUMNS;
    const int64_t c = spread_block(wide) * SUM_COLUMNS + x;
    constexpr int GO = 8;
    float s = 0.0f;
    if (c < columns) {
        int r = y;
        for (; r + (GO - 1) * SUM_ROWS < rows; r += GO * SUM_ROWS) {
            float v[GO];
#pragma unroll
            for (int k = 0; k < GO; ++k) v[k] = part[(int64_t)(r + k * SUM_ROWS) * columns + c];
#pragma unroll
            for (int k = 0; k < GO; ++k) s += v[k];
        }
        for (; r < rows; r += SUM_ROWS) s += part[(int64_t)r * columns + c];
    }
    sums[y][x] = s;
    __syncthreads();
    if (y != 0 || c >= columns) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < SUM_ROWS; ++k) s += sums[k][x];
    put(c, s);
}

// ---- host ------------------------------------------------------------------------------------------
inline int refuse(int code, const char* text, const char** why)
{
    *why = text;
    return code;
}

inline size_t elem_bytes(uint32_t dtype) { return dtype == CRAFTAX_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t v) { return (v + 255) / 256 * 256; }

inline int launched(const char** why)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)CRAFTAX_OK : refuse(CRAFTAX_E_HIP, hipGetErrorString(e), why);
}

template <typename Put> inline void sum_rows(const float* part, int rows, int64_t columns, Put put, hipStream_t st)
{
    const Spread grid = spread(ceil_div(columns, SUM_COLUMNS), SUM_COLUMNS * SUM_ROWS);
    hipLaunchKernelGGL(k_sum_rows<Put>, dim3(grid.x, 1, grid.z), dim3(SUM_COLUMNS * SUM_ROWS), 0, st, part, rows, columns, grid.x, put);
}

template <typename E> Seq<E> seq(const craftax_view& v) { return {static_cast<E*>(v.data), v.step, v.env}; }
template <typename E> Seq<const E> seq_in(const craftax_view& v) { return {static_cast<const E*>(v.data), v.step, v.env}; }

// calls f with a value of the element type
template <typename F> inline void with_type(uint32_t dtype, F&& f)
{
    if (dtype == CRAFTAX_F32) f(float{});
    else if (dtype == CRAFTAX_BF16) f(__bf16{});
    else f(_Float16{});
}

}  // namespace mem
