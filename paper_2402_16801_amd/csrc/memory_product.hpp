// Tiles of a matrix product on the matrix cores, and what is done with a result before it is stored (memory_product.hip).
//
// A product is C[m][n] = sum over k of Q[m][k] P[n][k].  The instruction's first operand is P, so that its result leaves neighbouring
// columns n in one lane; which row of P stands at which place of the instruction is free, and is chosen so that a lane holds
// 4 FP columns in a row (see Tile).
#pragma once

#include "memory_common.hpp"

#include <type_traits>

namespace mem {

// Where row m of a matrix lies: rows are numbered as steps times environments.  n is 1 where one stride does.
struct Rows {
    int64_t step, env;
    uint32_t n;
    __device__ __forceinline__ int64_t at(uint32_t m) const { return n == 1 ? (int64_t)m * step : (int64_t)(m / n) * step + (int64_t)(m % n) * env; }
};

// ---- activations ---------------------------------------------------------------------------------
constexpr float GELU_2K = 1.5957691216057308f, GELU_C = 0.044715f;      // 2 sqrt(2 / pi)

// v sigmoid(2 k (v + c v^3)), with the constants of the exponential's base multiplied in
template <int ACT, int COUNT> __device__ __forceinline__ void activate(float (&v)[COUNT])
{
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
        if (ACT == CRAFTAX_ACT_RELU) v[j] = v[j] < 0.0f ? 0.0f : v[j];
        if (ACT == CRAFTAX_ACT_SILU) v[j] *= sigmoid(v[j]);
        if (ACT == CRAFTAX_ACT_GELU_TANH) {
            const float e = exp2_fast(v[j] * __builtin_fmaf(v[j] * v[j], -GELU_2K * GELU_C * LOG2E, -GELU_2K * LOG2E));
            v[j] *= __builtin_amdgcn_rcpf(1.0f + e);
        }
    }
}
// the same for an activation that is known when the kernel runs; ACT -1
template <int COUNT> __device__ __forceinline__ void activate(float (&v)[COUNT], int act)
{
    if (act == CRAFTAX_ACT_RELU) activate<CRAFTAX_ACT_RELU>(v);
    else if (act == CRAFTAX_ACT_SILU) activate<CRAFTAX_ACT_SILU>(v);
    else if (act == CRAFTAX_ACT_GELU_TANH) activate<CRAFTAX_ACT_GELU_TANH>(v);
}
// the derivative at p; beyond `END` it is 0 or 1, and infinities would come up against a 0
template <int ACT> __device__ __forceinline__ float slope_of(float p)
{
    constexpr float END = ACT == CRAFTAX_ACT_GELU_TANH ? 16.0f : 256.0f;
    if (ACT == CRAFTAX_ACT_RELU) return p > 0.0f ? 1.0f : (p <= 0.0f ? 0.0f : p);
    p = p > END ? END : (p < -END ? -END : p);
    if (ACT == CRAFTAX_ACT_SILU) {
        const float e = exp2_fast(-p * LOG2E), g = __builtin_amdgcn_rcpf(1.0f + e);
        return g * __builtin_fmaf(p, rest_of(g, e), 1.0f);
    }
    if (ACT == CRAFTAX_ACT_GELU_TANH) {
        const float square = p * p;
        const float e = exp2_fast(p * __builtin_fmaf(square, -GELU_2K * GELU_C * LOG2E, -GELU_2K * LOG2E));
        const float g = __builtin_amdgcn_rcpf(1.0f + e);
        return g * __builtin_fmaf(rest_of(g, e), p * __builtin_fmaf(square, 3.0f * GELU_C * GELU_2K, GELU_2K), 1.0f);
    }
    return 1.0f;
}

// Not of the header's activations: what float16 products of a gradient end with (see k_largest), a multiplication by a number that lies on the device.
constexpr int ACT_SCALED = CRAFTAX_ACT_GELU_TANH + 1;

// How many of COUNT neighbouring columns are there: all of them; all or none, where COUNT divides their number; any number.
enum Edge { INNER, VECTORS, VALUES };

// ---- what is done with COUNT columns of a row -------------------------------------------------------
// out = residual + act(sum + bias), and pre = sum + bias
template <typename E, typename R> struct Finish {
    const float* bias;
    const R* residual;
    R* out;
    E* pre;
    Rows residual_rows, out_rows, pre_rows;
    int act, columns;
    const float* factor;     // ACT_SCALED
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
    // What is added to COUNT columns, as it lies in memory.  Taken in front of the stores of other rows: the compiler has to suppose that
    // those change it, and would wait for a load in each row.
    template <int COUNT> struct Bias { float v[COUNT]; };
    template <Edge EDGE, int COUNT> __device__ __forceinline__ Bias<COUNT> take_bias(int n) const
    {
        Bias<COUNT> b = {};
        if (bias && (EDGE == INNER || columns > n)) add(bias + n, EDGE == VALUES ? columns - n : COUNT, b.v);
        return b;
    }
    // (At a ragged end the compiler makes one load of this, from memory or from a zeroed place in scratch: 12 to 68 bytes of it in nearly every kernel here,
    // written once a row and read by that load.  No register is spilled.)
    template <Edge EDGE, int COUNT> __device__ __forceinline__ Pack<R, COUNT> take_residual(uint32_t m, int n) const
    {
        Pack<R, COUNT> q = {};
        if (!residual || (EDGE != INNER && columns <= n)) return q;
        const R* p = residual + residual_rows.at(m) + n;
        if (EDGE != VALUES || columns - n >= COUNT) return *reinterpret_cast<const Pack<R, COUNT>*>(p);
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (j < columns - n) q.v[j] = p[j];
        return q;
    }
    // ACT: the activation, or -1 where it is only known when the kernel runs.
    template <Edge EDGE, int ACT, int COUNT> __device__ __forceinline__ void put(uint32_t m, int n, float (&v)[COUNT], const Pack<R, COUNT>& r) const
    {
        if (EDGE != INNER && columns <= n) return;
        const int count = EDGE == VALUES ? columns - n : COUNT;
        if (pre) store(pre + pre_rows.at(m) + n, count, v);
        if (std::is_same_v<E, _Float16> && (ACT == ACT_SCALED || (ACT < 0 && act == ACT_SCALED))) {
#pragma unroll
            for (int j = 0; j < COUNT; ++j) v[j] *= *factor;
        } else if constexpr (ACT < 0) {
            activate(v, act);
        } else {
            activate<ACT>(v);
        }
        if (residual) {
#pragma unroll
            for (int j = 0; j < COUNT; ++j) v[j] += Elem<R>::up(r.v[j]);
        }
        store(out + out_rows.at(m) + n, count, v);
    }
    template <int COUNT> __device__ __forceinline__ void operator()(uint32_t m, int n, float (&v)[COUNT]) const
    {
        const Bias<COUNT> b = take_bias<VALUES, COUNT>(n);
#pragma unroll
        for (int j = 0; j < COUNT; ++j) v[j] += b.v[j];
        put<VALUES, -1>(m, n, v, take_residual<VALUES, COUNT>(m, n));
    }
};

// ---- operands of the matrix instructions --------------------------------------------------------------
// A fragment is 16 rows by 64 bytes along k: lane l holds 16 bytes of row l % 16, from byte 16 (l / 16) on.
typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 BF2 __attribute__((ext_vector_type(2)));
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

// ODD: 16-bit rows that begin at any multiple of two bytes.  A load of 16 bytes that does not begin at a multiple of four takes several times as
// long, so five words are read from the one before on, and shifted (64 rows of 1,345 values onto 512: 12.0 us without, 1,344 values 6.0).  The fifth
// is the last that holds any of the 16 bytes.
template <bool ODD, typename E> __device__ __forceinline__ U4v load_chunk(const E* p)
{
    if constexpr (!ODD) {
        return __builtin_bit_cast(U4v, *reinterpret_cast<const Pack<E, 16 / sizeof(E)>*>(p));
    } else {
        const uint32_t off = (uint32_t)(uintptr_t)p & 2u;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(p) - off);
        const Pack<uint32_t, 4> q = *reinterpret_cast<const Pack<uint32_t, 4>*>(w);
        const uint32_t last = w[off ? 4 : 3];
        U4v out;
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = __builtin_amdgcn_alignbit(j < 3 ? q.v[j + 1] : last, q.v[j], off * 8);
        return out;
    }
}
// 16 bytes of a row from value k on; those at or behind `end`, of which there is one at least, are 0.  No branches: behind one every load would be waited for.
template <typename E> __device__ __forceinline__ U4v load_some(const E* row, int64_t k, int64_t end)
{
    constexpr int V = 16 / sizeof(E);
    Pack<E, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = row[k + j < end ? k + j : 0];
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = k + j < end ? q.v[j] : (E)0.0f;
    return __builtin_bit_cast(U4v, q);
}

// ---- tiles --------------------------------------------------------------------------------------------
constexpr int TILE_BYTES = 128;        // along k, of a tile that lies with k inside
template <typename E> constexpr int tile_k() { return TILE_BYTES / (int)sizeof(E); }

// A matrix operand: rows of k (INSIDE) or rows of the other index, one behind the other along k.
template <typename E> struct Operand {
    const E* data;
    Rows rows;
};

template <typename E, typename R> struct ProductParams {
    Operand<E> p, q;
    int64_t k;               // length of the sums
    uint32_t m;              // rows of the result
    int n;                   // columns of it
    uint32_t m_tiles, n_tiles;
    int64_t k_part;          // of a part of the sums, a multiple of the tile
    uint32_t tiles;          // numbers of tiles, a multiple of the dies
    float* part;             // [parts][m][n], or nullptr: one part, finished here
    unsigned wide;
    Finish<E, R> finish;
};

// The place of a 16-byte chunk in a tile: exchanged within the row by a number of the row, so that the chunks that are read at once lie in
// different banks.  INSIDE: rows of BYTES bytes along k; a fragment of P is read from rows 0..3, 4 FP .. 4 FP + 3, .. (see Stage::frag).
template <int FP, bool IS_P, int BYTES = TILE_BYTES> __device__ __forceinline__ int inside_key(int row)
{
    if (BYTES == 64) return IS_P ? ((row >> 1) & 1) | ((row / (4 * FP)) & 1) << 1 : (row >> 1) & 3;
    return IS_P ? (row & 3) | ((row / (4 * FP)) & 1) << 2 : row & 7;
}
template <typename E, int TILE> __device__ __forceinline__ int across_key(int k)
{
    return (sizeof(E) == 2 ? ((k & 3) << 1) | ((k >> 3) & 1) << 3 : ((k >> 2) & 3) << 2) & (TILE * (int)sizeof(E) / 16 - 1);
}
// The fragment of 16 columns from `col` on and 64 bytes along k from the half-th on, of a tile of rows along k of 16-bit values.  A group of 16
// lanes reads four rows of 16 values and gets them column by column.  (lds is restricted: the compiler has no types for these reads, supposes that they
// may be of what loads are writing to LDS, and would wait for those.)
template <typename E, int TILE> __device__ __forceinline__ U4v across_frag(const char* __restrict lds, int first, int half)
{
    const int lane = threadIdx.x & (WAVE - 1), i = lane & 15, g = lane >> 4;
    U4v out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int k = half * 32 + g * 8 + h * 4 + i / 4, col = first + i % 4 * 4;
        const char* at = lds + (k * (TILE / 8) + ((col / 8) ^ across_key<E, TILE>(k))) * 16 + col % 8 * 2;
        const S4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)(at));
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        out[2 * h] = (uint32_t)bits;
        out[2 * h + 1] = (uint32_t)(bits >> 32);
    }
    return out;
}

// Which tile has number t.  Consecutive blocks go to the eight dies in turn, so every die gets a piece of the tiles: by rows of tiles, whose tiles
// read the same rows of Q, and part by part of the sums.  Some of the last numbers have no tile.
constexpr uint32_t DIES = 8;
struct TilePlace {
    uint32_t m, n, part;
    bool on;
    template <typename P> __device__ __forceinline__ TilePlace(const P& p, uint32_t t)
    {
        const uint32_t at = t % DIES * (p.tiles / DIES) + t / DIES, in_part = p.m_tiles * p.n_tiles, in = at % in_part;
        part = at / in_part;
        m = in / p.n_tiles;
        n = in % p.n_tiles;
        on = t < p.tiles && (int64_t)part * p.k_part < p.k;
    }
};

namespace host {
// Tiles that come straight from memory to LDS (memory_product_direct.hip).  LARGE: 256 by 256, else 128 by 128.  For 16-bit types; every row
// of an operand begins at a multiple of 16 bytes, and so does what is left of one behind `k` (INSIDE) or behind the columns.
template <bool INSIDE, typename E, typename R> void launch_direct(const ProductParams<E, R>& p, int64_t tiles, bool large, hipStream_t st);
}  // namespace host

}  // namespace mem
