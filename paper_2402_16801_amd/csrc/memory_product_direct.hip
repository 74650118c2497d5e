// Large tiles of a matrix product of 16-bit types, straight from memory to LDS: 256 x 256 by eight wavefronts of 128 rows by 64 columns
// each, or 128 x 128 by four of 64 by 64, two tiles of 64 along k.
//
// What bounds them: a step of 64 along k of a 256 x 256 tile is 2,048 cycles of matrix instructions for a SIMD and 2,048 cycles of a compute unit's
// LDS at 128 bytes each (192 KiB of fragments read, 64 KiB written), and it takes about 4,000.  8,192 squared in bfloat16: 920 to 1,040 us, 1,060
// to 1,200 TFLOP/s, the library's product 1,400.  At the widths of a policy sums are short (512 is eight steps) and a tile's results, 128 KiB
// (256 with what an activation's backward pass needs), take memory as long as a third of its sums or longer; blocks go on to further tiles, whose
// first operands are under way while results are stored.  262,144 rows of 512 onto 1,024 with gelu, its argument kept: 468 us, 1.49 GB.
#include "memory_product.hpp"

#include <type_traits>

namespace mem {

// What lies behind the end of the sums or of the columns comes from here, 16 bytes at a time.
alignas(16) static __device__ const uint32_t g_zeros[4] = {0, 0, 0, 0};

// Fragment f of P, with k inside, stands for rows 32 (f / 2) + 8 (i / 4) + 4 (f % 2) + i % 4, so that a lane holds eight columns in a row of two
// fragments.
template <bool IS_P, int BYTES> __device__ __forceinline__ U4v inside_frag(const char* lds, int row, int f, int half)
{
    const int lane = threadIdx.x & (WAVE - 1), i = lane & 15, g = lane >> 4;
    const int r = row + (IS_P ? f / 2 * 32 + f % 2 * 4 + i / 4 * 8 + i % 4 : f * 16 + i);
    return *reinterpret_cast<const U4v*>(lds + r * BYTES + ((half * 4 + g) ^ inside_key<2, IS_P, BYTES>(r)) * 16);
}

// until LEFT memory operations of this wavefront are under way, and no LDS read
template <int LEFT> __device__ __forceinline__ void wait_loads()
{
    static_assert(LEFT < 64, "the counter has six bits");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | (LEFT >> 4) << 14);
}
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int BIASES = 4096;       // 16 KiB: two tiles of 128 x 128 have a compute unit's LDS for themselves

// A block of WP x WQ wavefronts computes tiles of 16 FP WP columns by 16 FQ WQ rows, one after the other: tile blockIdx.x, the one gridDim.x
// behind it, ..  A wavefront's load fills 1 KiB of LDS in the order of its lanes, so the chunks are exchanged by the addresses the lanes read from.
//
// Order of things: the sums of a step; a wait for the loads of the next step; a barrier, behind which nobody reads this step's stage; the loads
// that go there; and, behind a tile's last step, its results.  Results that are under way need not be waited for with the loads that were
// begun before them: at least STORES instructions store a whole tile.
template <typename E, typename R, int ACT, bool INSIDE, int FP, int FQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_product_direct(const ProductParams<E, R> p)
{
    static_assert(sizeof(E) == 2 && FP % 2 == 0, "16-bit types, fragments of P in pairs");
    constexpr int WAVES = WP * WQ, TP = 16 * FP * WP, TQ = 16 * FQ * WQ, K = 64, BYTES = 2 * K, STAGES = 2;
    constexpr int LOADS_P = TP / 8 / WAVES, LOADS = (TP + TQ) / 8 / WAVES;       // of a wavefront for a step
    constexpr int STORES = FP * FQ * 4 * (int)sizeof(R) / 16;
    static_assert(TP % (8 * WAVES) == 0 && TQ % (8 * WAVES) == 0, "a load of a wavefront is one operand's");
    constexpr int STAGE = (TP + TQ) * BYTES;
    // One array for all: of two the compiler supposes that reads may be of what loads write, and waits for these in every step.
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * STAGE + (INSIDE ? BIASES * 4 : 0)];
    float* biases = reinterpret_cast<float*>(lds + STAGES * STAGE);
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), wp = wave % WP * 16 * FP, wq = wave / WP * 16 * FQ;

    auto next = [&](uint32_t t) {            // the next number that has a tile
        while (t < p.tiles && !TilePlace(p, t).on) t += gridDim.x;
        return t;
    };
    uint32_t tile = next(blockIdx.x);
    if (tile >= p.tiles) return;
    auto whole_columns = [&](uint32_t t) {   // across: all columns of the tile are there
        const TilePlace place(p, t);
        return (place.n + 1) * TP <= (uint32_t)p.n && (place.m + 1) * TQ <= p.m;
    };

    // Loads.  INSIDE: load j of a wavefront is rows 8 (wave + WAVES j) .. + 7 of a tile, eight chunks of 16 bytes along k each.  Else it is 1 KiB of
    // rows along k.  Which chunk of a row a lane reads is the same for all its loads of an operand.
    constexpr int ROWS_P = INSIDE ? 8 : 1024 / (TP * 2), ROWS_Q = INSIDE ? 8 : 1024 / (TQ * 2);          // of a load
    static_assert(INSIDE || (WAVES * ROWS_P % 4 == 0 && WAVES * ROWS_Q % 4 == 0), "keys repeat with a wavefront's loads, but for bit 3 of the row");
    uint32_t coming = tile;                  // the tile whose operands are loaded, from k = `at` on, up to `end`
    int at = 0, end = 0;
    const char *base_p = nullptr, *base_q = nullptr;
    uint32_t from[LOADS];                    // bytes behind the base
    const int row_p = wave * ROWS_P + lane / (64 / ROWS_P), row_q = wave * ROWS_Q + lane / (64 / ROWS_Q);
    // INSIDE: a chunk's k within a step; else 0, or a number behind all sums where a lane's chunk is behind the columns
    int chunk_p = (lane % 8 ^ inside_key<2, true>(row_p)) * 8, chunk_q = (lane % 8 ^ inside_key<2, false>(row_q)) * 8;
    auto point = [&] {
        const TilePlace place(p, coming);
        const uint32_t m0 = place.m * TQ, n0 = place.n * TP;
        at = (int)((int64_t)place.part * p.k_part);
        end = p.k - at < p.k_part ? (int)p.k : at + (int)p.k_part;
        const int64_t step_p = p.p.rows.step * 2, step_q = p.q.rows.step * 2;
        if (INSIDE) {
            base_p = (const char*)p.p.data + (int64_t)n0 * step_p + (int64_t)at * 2;
            base_q = (const char*)p.q.data + (int64_t)m0 * step_q + (int64_t)at * 2;
        } else {
            base_p = (const char*)(p.p.data + n0) + (int64_t)at * step_p;
            base_q = (const char*)(p.q.data + m0) + (int64_t)at * step_q;
            chunk_p = chunk_q = 0;
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const bool is_p = j < LOADS_P;
            const int r = is_p ? row_p + j * WAVES * ROWS_P : row_q + (j - LOADS_P) * WAVES * ROWS_Q;
            const uint32_t step = (uint32_t)(is_p ? step_p : step_q), left = is_p ? (uint32_t)p.n - n0 : p.m - m0;
            if (INSIDE) {
                from[j] = ((uint32_t)r < left ? (uint32_t)r : left - 1) * step + (is_p ? chunk_p : chunk_q) * 2;
            } else {
                const int row_chunks = (is_p ? TP : TQ) / 8;
                const uint32_t column = (uint32_t)((lane % row_chunks) ^ (is_p ? across_key<E, TP>(r) : across_key<E, TQ>(r))) * 8;
                from[j] = (uint32_t)r * step + column * 2;
                if (column >= left) from[j] = ~0u;
            }
        }
    };
    auto load = [&](int stage) {
        if (coming >= p.tiles) return;
        auto one = [&](int j, const void* src) {
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             (__attribute__((address_space(3))) void*)(lds + stage * STAGE + (wave + j * WAVES) * 1024), 16, 0, 0);
        };
        const bool every = INSIDE ? at + K <= end : at + K <= end && whole_columns(coming);
        if (every) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) one(j, (j < LOADS_P ? base_p : base_q) + from[j]);
        } else {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int k = INSIDE ? (j < LOADS_P ? chunk_p : chunk_q) : j < LOADS_P ? row_p + j * WAVES * ROWS_P : row_q + (j - LOADS_P) * WAVES * ROWS_Q;
                const bool there = k < end - at && (INSIDE || from[j] != ~0u);
                one(j, there ? (const void*)((j < LOADS_P ? base_p : base_q) + from[j]) : (const void*)g_zeros);
            }
        }
        at += K;
        if (at < end) {
            base_p += INSIDE ? 2 * K : 2 * K * p.p.rows.step;
            base_q += INSIDE ? 2 * K : 2 * K * p.q.rows.step;
        } else {
            coming = next(coming + gridDim.x);
            if (coming < p.tiles) point();
        }
    };

    point();
#pragma unroll
    for (int s = 0; s < STAGES; ++s) load(s);
    // Sums begin with the bias, which is kept in LDS: read from memory for every tile, the wait for it would be for the stores of the tile before,
    // too.  More columns than there is room for get it added in the end.
    const bool early = INSIDE && p.finish.bias && !p.part && p.n_tiles * TP <= BIASES, late = INSIDE && p.finish.bias && !p.part && !early;
    if (early)
        for (int c = threadIdx.x; c < (int)p.n_tiles * TP; c += 64 * WAVES) biases[c] = c < p.n ? p.finish.bias[c] : 0.0f;
    wait_loads<0>();
    barrier();
    int turn = 0;
    bool storing = false;                    // stores of the last tile are behind the loads that are waited for
    uint32_t after;
    for (; tile < p.tiles; tile = after) {
        after = next(tile + gridDim.x);
        const TilePlace place(p, tile);
        const uint32_t m0 = place.m * TQ;
        const int n0 = (int)place.n * TP, i = lane & 15, g = lane >> 4;
        const int k0 = (int)((int64_t)place.part * p.k_part), k1 = p.k - k0 < p.k_part ? (int)p.k : k0 + (int)p.k_part;
        F4 acc[FP][FQ];
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
            for (int q = 0; q < FQ; ++q)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[f][q][r] = 0.0f;
        if (early) {
            const float* from = biases + n0 + wp + g * 8;
#pragma unroll
            for (int f = 0; f < FP; ++f) {
                const F4 b = *reinterpret_cast<const F4*>(from + f / 2 * 32 + f % 2 * 4);
#pragma unroll
                for (int q = 0; q < FQ; ++q) acc[f][q] = b;
            }
        }
        for (int k = k0; k < k1; k += K) {
            const char* here = lds + turn * STAGE;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                U4v fp[FP], fq[FQ];
#pragma unroll
                for (int f = 0; f < FP; ++f) {
                    if constexpr (INSIDE) fp[f] = inside_frag<true, BYTES>(here, wp, f, half);
                    else fp[f] = across_frag<E, TP>(here, wp + f * 16, half);
                }
#pragma unroll
                for (int f = 0; f < FQ; ++f) {
                    if constexpr (INSIDE) fq[f] = inside_frag<false, BYTES>(here + TP * BYTES, wq, f, half);
                    else fq[f] = across_frag<E, TQ>(here + TP * BYTES, wq + f * 16, half);
                }
#pragma unroll
                for (int f = 0; f < FP; ++f)
#pragma unroll
                    for (int q = 0; q < FQ; ++q) acc[f][q] = Frag<E>::times(fp[f], fq[q], acc[f][q]);
            }
            if (storing) wait_loads<STORES>();
            else wait_loads<0>();
            storing = false;
            barrier();
            load(turn);
            turn ^= 1;
        }
        const bool whole = n0 + TP <= p.n && m0 + TQ <= p.m;
        auto put = [&](auto kind) {
            constexpr Edge EDGE = decltype(kind)::value;
            constexpr bool WHOLE = EDGE == INNER;
            auto row = [&](int q) { return m0 + wq + q * 16 + i; };
            if (p.part) {
#pragma unroll
                for (int q = 0; q < FQ; ++q) {
                    const uint32_t m = row(q);
                    if (!WHOLE && m >= p.m) continue;
#pragma unroll
                    for (int f = 0; f < FP; ++f) {
                        const int n = n0 + wp + (INSIDE ? f / 2 * 32 + f % 2 * 4 + g * 8 : f * 16 + g * 4);
                        float v[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[f][q][r];
                        if (WHOLE || n < p.n) Finish<E, R>::template store<float, 4>(p.part + ((int64_t)place.part * p.m + m) * p.n + n, EDGE == VALUES ? p.n - n : 4, v);
                    }
                }
            } else if constexpr (INSIDE) {
                const int n = n0 + wp + g * 8;
                Pack<R, 8> residual[2][FP / 2];
                auto take = [&](int q) {
                    const uint32_t m = row(q);
#pragma unroll
                    for (int f = 0; f < FP / 2; ++f)
                        if (WHOLE || m < p.m) residual[q & 1][f] = p.finish.template take_residual<EDGE, 8>(m, n + f * 32);
                };
                take(0);
#pragma unroll
                for (int q = 0; q < FQ; ++q) {
                    if (q + 1 < FQ) take(q + 1);
                    const uint32_t m = row(q);
                    if (!WHOLE && m >= p.m) continue;
#pragma unroll
                    for (int f = 0; f < FP / 2; ++f) {
                        float v[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) v[r] = acc[2 * f + r / 4][q][r % 4];
                        if (late) {
                            const typename Finish<E, R>::template Bias<8> b = p.finish.template take_bias<EDGE, 8>(n + f * 32);
#pragma unroll
                            for (int r = 0; r < 8; ++r) v[r] += b.v[r];
                        }
                        p.finish.template put<EDGE, ACT>(m, n + f * 32, v, residual[q & 1][f]);
                    }
                }
            } else {
#pragma unroll
                for (int q = 0; q < FQ; ++q) {
                    const uint32_t m = row(q);
                    if (!WHOLE && m >= p.m) continue;
#pragma unroll
                    for (int f = 0; f < FP; ++f) {
                        float v[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[f][q][r];
                        p.finish.template put<EDGE, ACT>(m, n0 + wp + f * 16 + g * 4, v, Pack<R, 4>{});
                    }
                }
            }
        };
        if (whole) {
            put(std::integral_constant<Edge, INNER>{});
            storing = true;
        } else {
            if (p.n % 8 == 0) put(std::integral_constant<Edge, VECTORS>{});
            else put(std::integral_constant<Edge, VALUES>{});
            wait_loads<0>();
        }
    }
}

namespace host {

template <bool INSIDE, typename E, typename R> void launch_direct(const ProductParams<E, R>& p, int64_t tiles, bool large, hipStream_t st)
{
    // large tiles fill a compute unit one at a time: blocks go on to further ones
    const unsigned blocks = large && tiles > 256 ? 256 : blocks_in_turn(tiles);
    auto go = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (large) hipLaunchKernelGGL((k_product_direct<E, R, ACT, INSIDE, 4, 8, 4, 2>), dim3(blocks), dim3(512), 0, st, p);
        else hipLaunchKernelGGL((k_product_direct<E, R, ACT, INSIDE, 4, 4, 2, 2>), dim3(blocks), dim3(256), 0, st, p);
    };
    const int act = p.part ? CRAFTAX_ACT_NONE : p.finish.act;
    if constexpr (std::is_same_v<E, _Float16> && (!INSIDE || std::is_same_v<E, R>)) {
        if (act == ACT_SCALED) return go(std::integral_constant<int, ACT_SCALED>{});
    }
    if constexpr (INSIDE) {
        if (act == CRAFTAX_ACT_RELU) return go(std::integral_constant<int, CRAFTAX_ACT_RELU>{});
        if (act == CRAFTAX_ACT_SILU) return go(std::integral_constant<int, CRAFTAX_ACT_SILU>{});
        if (act == CRAFTAX_ACT_GELU_TANH) return go(std::integral_constant<int, CRAFTAX_ACT_GELU_TANH>{});
    }
    go(std::integral_constant<int, CRAFTAX_ACT_NONE>{});
}

template void launch_direct<true>(const ProductParams<__bf16, __bf16>&, int64_t, bool, hipStream_t);
template void launch_direct<true>(const ProductParams<__bf16, float>&, int64_t, bool, hipStream_t);
template void launch_direct<true>(const ProductParams<_Float16, _Float16>&, int64_t, bool, hipStream_t);
template void launch_direct<true>(const ProductParams<_Float16, float>&, int64_t, bool, hipStream_t);
template void launch_direct<false>(const ProductParams<__bf16, __bf16>&, int64_t, bool, hipStream_t);
template void launch_direct<false>(const ProductParams<__bf16, float>&, int64_t, bool, hipStream_t);
template void launch_direct<false>(const ProductParams<_Float16, _Float16>&, int64_t, bool, hipStream_t);
template void launch_direct<false>(const ProductParams<_Float16, float>&, int64_t, bool, hipStream_t);

}  // namespace host
}  // namespace mem
