// Matrix product with bias, activation and residual in its epilogue, and its backward pass.
//
//   out = residual + act(x weight^T + bias);   dp = dout act'(pre),  dx = dp weight,  dweight = dp^T x,  dbias = sum of dp
//
// Few rows (an actor's token) are bound by the latency of one pass over the operands, many by the matrix units or, at the
// widths of a policy, by memory.  Sums are in 32 bits; dp is rounded to the type of the activations, which the matrix instructions take.
//
// Products are cut in one of four ways, by a rule on their sizes (plan): fragments straight from memory, whose sums a block's wavefronts share along
// k (k_product_rows: 64 rows of 1,345 bfloat16 values onto 512, 6 us, a launch); tiles staged through registers, which take any
// stride, order and alignment (k_product); the same with float32 values in three bfloat16 parts (k_product_float); and, for 16-bit types, tiles that
// go straight to LDS (k_product_direct).  Sums too long for too few tiles are cut into parts, which a second kernel adds in order.
#include "memory_api.hpp"
#include "memory_common.hpp"
#include "memory_product.hpp"

#include <type_traits>

namespace mem {

// One operand's tile of TILE rows on its way from memory to LDS.
template <typename E, int TILE, int THREADS, bool INSIDE, int FP, bool IS_P> struct Stage {
    static constexpr int V = 16 / sizeof(E), CHUNKS = TILE * 8 / THREADS, ROW_CHUNKS = INSIDE ? 8 : TILE / V;
    const E* from[INSIDE ? CHUNKS : 1];      // rows
    U4v raw[CHUNKS];
    int side;                // values of a row before this thread's chunk
    int columns;             // across: of a row, from the tile's first on
    Operand<E> op;
    __device__ __forceinline__ static int row_of(int c) { return ((int)threadIdx.x + c * THREADS) / ROW_CHUNKS; }
    __device__ __forceinline__ static int chunk_of(int c) { return ((int)threadIdx.x + c * THREADS) % ROW_CHUNKS; }
    __device__ __forceinline__ Stage(const Operand<E>& o, uint32_t first, uint32_t rows) : op(o)
    {
        static_assert(THREADS % ROW_CHUNKS == 0, "a thread's chunks lie below one another");
        side = chunk_of(0) * V;
        columns = (int)(rows - first);
        if (INSIDE) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t r = first + row_of(c);
                from[c] = o.data + o.rows.at(r < rows ? r : rows - 1);
            }
        } else {
            from[0] = o.data + first;
        }
    }
    // values k .. k + tile of the sums; those at or behind `end` are 0
    __device__ __forceinline__ void load(int64_t k, int64_t end)
    {
        const bool whole = INSIDE ? k + tile_k<E>() <= end : columns >= TILE && k + tile_k<E>() <= end;
        auto row = [&](int c) {
            const int64_t r = k + row_of(c);
            return from[0] + op.rows.at((uint32_t)(r < end ? r : end - 1));
        };
        if (whole) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) raw[c] = load_chunk<false>(INSIDE ? from[c] + k + side : row(c) + side);
        } else {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (INSIDE) raw[c] = load_some<E>(from[c], k + side, end);
                else raw[c] = load_some<E>(row(c), side, k + row_of(c) < end ? columns : 0);
            }
        }
    }
    __device__ __forceinline__ void store(char* lds) const
    {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int r = row_of(c), key = INSIDE ? inside_key<FP, IS_P>(r) : across_key<E, TILE>(r);
            *reinterpret_cast<U4v*>(lds + (r * ROW_CHUNKS + (chunk_of(c) ^ key)) * 16) = raw[c];
        }
    }
    // float: each value in three parts of eight bits, hi + mid + lo, which are exactly the value (see k_product_float), one plane of 16-bit
    // values behind the other; whether one of the values is an infinity or NaN, or so large that hi is an infinity
    __device__ __forceinline__ bool store_parts(char* lds, int plane) const
    {
        bool odd = false;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            uint32_t part[3][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float a = __uint_as_float(raw[c][2 * j]), b = __uint_as_float(raw[c][2 * j + 1]);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    uint32_t q = __builtin_bit_cast(uint32_t, BF2{(__bf16)a, (__bf16)b});
                    pin(q);                    // or the compiler converts a again by itself
                    const float qa = __uint_as_float(q << 16), qb = __uint_as_float(q & 0xFFFF0000u);
                    if (k == 0) odd |= !__builtin_isfinite(qa) | !__builtin_isfinite(qb);
                    part[k][j] = q;
                    a -= qa;
                    b -= qb;
                }
            }
            const int r = row_of(c), v = chunk_of(c) * 4, key = INSIDE ? inside_key<FP, IS_P, 64>(r) : across_key<__bf16, TILE>(r);
            char* at = lds + (r * (INSIDE ? 4 : TILE / 8) + ((v / 8) ^ key)) * 16 + v % 8 * 2;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const Pack<uint32_t, 2> q{{part[k][0], part[k][1]}};
                *reinterpret_cast<Pack<uint32_t, 2>*>(at + k * plane) = q;
            }
        }
        return odd;
    }
    // the fragment of 16 rows whose first is `row`, 64 bytes along k from 64 * half on.  IS_P and k inside: place i of the fragment is row
    // i / 4 * 4 FP + i % 4 behind it.
    __device__ __forceinline__ static U4v frag(const char* lds, int row, int half)
    {
        const int lane = threadIdx.x & (WAVE - 1), i = lane & 15, g = lane >> 4;
        if constexpr (INSIDE) {
            const int r = row + (IS_P ? i / 4 * (4 * FP) + i % 4 : i);
            return *reinterpret_cast<const U4v*>(lds + (r * 8 + ((half * 4 + g) ^ inside_key<FP, IS_P>(r))) * 16);
        } else if constexpr (sizeof(E) == 2) {
            return across_frag<E, TILE>(lds, row, half);
        } else {
            U4v out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = half * 16 + g * 4 + j, col = row + i;
                out[j] = *reinterpret_cast<const uint32_t*>(lds + (k * ROW_CHUNKS + ((col / 4) ^ across_key<E, TILE>(k))) * 16 + col % 4 * 4);
            }
            return out;
        }
    }
};

// a wavefront's sums, 16 FP columns from n0 on of 16 FQ rows from m0 on
template <bool INSIDE, typename E, typename R, int FP, int FQ>
__device__ __forceinline__ void put_tile(const ProductParams<E, R>& p, uint32_t part, uint32_t m0, int n0, const F4 (&acc)[FP][FQ])
{
    const int lane = threadIdx.x & (WAVE - 1), i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
        const uint32_t m = m0 + q * 16 + i;
        if (m >= p.m) continue;
        auto put = [&](int n, auto& v) {
            constexpr int COUNT = sizeof(v) / sizeof(float);
            if (p.part) {
                if (n < p.n) Finish<E, R>::template store<float, COUNT>(p.part + ((int64_t)part * p.m + m) * p.n + n, p.n - n, v);
            } else {
                p.finish(m, n, v);
            }
        };
        if constexpr (INSIDE) {
            float v[4 * FP];
#pragma unroll
            for (int f = 0; f < FP; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[f * 4 + r] = acc[f][q][r];
            put(n0 + g * 4 * FP, v);
        } else {
#pragma unroll
            for (int f = 0; f < FP; ++f) {
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[f][q][r];
                put(n0 + f * 16 + g * 4, v);
            }
        }
    }
}

// A block of WP x WQ wavefronts computes 16 FP WP columns by 16 FQ WQ rows.
template <typename E, typename R, bool INSIDE, int FP, int FQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ) void k_product(const ProductParams<E, R> p)
{
    constexpr int THREADS = 64 * WP * WQ, TP = 16 * FP * WP, TQ = 16 * FQ * WQ, K = tile_k<E>();
    using StageP = Stage<E, TP, THREADS, INSIDE, FP, true>;
    using StageQ = Stage<E, TQ, THREADS, INSIDE, FP, false>;
    __shared__ __attribute__((aligned(16))) char lds[2][(TP + TQ) * TILE_BYTES];
    const TilePlace at(p, (uint32_t)spread_block(p.wide));
    if (!at.on) return;
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, wp = wave % WP * 16 * FP, wq = wave / WP * 16 * FQ;
    const uint32_t m0 = at.m * TQ;
    const int n0 = (int)at.n * TP;
    const int64_t k0 = (int64_t)at.part * p.k_part, k1 = p.k - k0 < p.k_part ? p.k : k0 + p.k_part;
    StageP sp(p.p, (uint32_t)n0, (uint32_t)p.n);
    StageQ sq(p.q, m0, p.m);
    F4 acc[FP][FQ] = {};
    sp.load(k0, k1);
    sq.load(k0, k1);
    sp.store(lds[0]);
    sq.store(lds[0] + TP * TILE_BYTES);
    __syncthreads();
    int turn = 0;
    for (int64_t k = k0; k < k1; k += K, turn ^= 1) {
        const bool more = k + K < k1;
        if (more) {
            sp.load(k + K, k1);
            sq.load(k + K, k1);
        }
        const char* tile = lds[turn];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            U4v fp[FP], fq[FQ];
#pragma unroll
            for (int f = 0; f < FP; ++f) fp[f] = StageP::frag(tile, wp + (INSIDE ? f * 4 : f * 16), half);
#pragma unroll
            for (int f = 0; f < FQ; ++f) fq[f] = StageQ::frag(tile + TP * TILE_BYTES, wq + f * 16, half);
#pragma unroll
            for (int f = 0; f < FP; ++f)
#pragma unroll
                for (int q = 0; q < FQ; ++q) acc[f][q] = Frag<E>::times(fp[f], fq[q], acc[f][q]);
        }
        if (more) {
            sp.store(lds[turn ^ 1]);
            sq.store(lds[turn ^ 1] + TP * TILE_BYTES);
        }
        __syncthreads();
    }
    put_tile<INSIDE>(p, at.part, m0 + wq, n0 + wp, acc);
}

// float32 on the matrix units of bfloat16, which are sixteen times as fast.  A float is exactly the sum of three bfloat16: hi = v rounded to eight
// bits, mid = v - hi rounded, lo = the rest, of seven bits at most.  Of the nine products of two such sums six are added, in 32 bits; the other three are
// below 2^-24 of the product in all, 2^-28 on average, of either sign: less than a float32 sum's own roundings.  (Of parts that are
// cut off they are up to 2^-21, 2^-24.5 on average, all of the product's sign.)  Six instructions of 16 cycles in place of eight of 32.  What is below
// 2^-133, bfloat16's smallest number, is lost: digits of values below 2^-110.  Infinities and NaN have no such parts (0 times infinity would come up), nor
// have values that round to infinity: a block that meets one computes its tile again as float32.
template <typename R, bool INSIDE, int FP, int FQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_product_float(const ProductParams<float, R> p)
{
    constexpr int THREADS = 64 * WP * WQ, TP = 16 * FP * WP, TQ = 16 * FQ * WQ, K = tile_k<float>(), PLANE = (TP + TQ) * 2 * K;
    using StageP = Stage<float, TP, THREADS, INSIDE, FP, true>;
    using StageQ = Stage<float, TQ, THREADS, INSIDE, FP, false>;
    __shared__ __attribute__((aligned(16))) char lds[3 * PLANE];
    __shared__ int again;
    const TilePlace at(p, (uint32_t)spread_block(p.wide));
    if (!at.on) return;
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, wp = wave % WP * 16 * FP, wq = wave / WP * 16 * FQ, i = lane & 15, g = lane >> 4;
    const uint32_t m0 = at.m * TQ;
    const int n0 = (int)at.n * TP;
    const int64_t k0 = (int64_t)at.part * p.k_part, k1 = p.k - k0 < p.k_part ? p.k : k0 + p.k_part;
    StageP sp(p.p, (uint32_t)n0, (uint32_t)p.n);
    StageQ sq(p.q, m0, p.m);
    F4 acc[FP][FQ] = {};
    if (threadIdx.x == 0) again = 0;
    bool odd = false;
    sp.load(k0, k1);
    sq.load(k0, k1);
    for (int64_t k = k0; k < k1; k += K) {
        odd |= sp.store_parts(lds, PLANE);
        odd |= sq.store_parts(lds + TP * 2 * K, PLANE);
        __syncthreads();
        if (k + K < k1) {
            sp.load(k + K, k1);
            sq.load(k + K, k1);
        }
        auto frag = [&](auto is_p, int part, int f) {
            constexpr bool IS_P = decltype(is_p)::value;
            const char* tile = lds + part * PLANE + (IS_P ? 0 : TP * 2 * K);
            if constexpr (INSIDE) {
                const int r = IS_P ? wp + f * 4 + i / 4 * (4 * FP) + i % 4 : wq + f * 16 + i;
                return *reinterpret_cast<const U4v*>(tile + r * 64 + (g ^ inside_key<FP, IS_P, 64>(r)) * 16);
            } else {
                return across_frag<__bf16, IS_P ? TP : TQ>(tile, (IS_P ? wp : wq) + f * 16, 0);
            }
        };
        U4v fq[3][FQ];
#pragma unroll
        for (int s = 0; s < 3; ++s)
#pragma unroll
            for (int f = 0; f < FQ; ++f) fq[s][f] = frag(std::false_type{}, s, f);
#pragma unroll
        for (int f = 0; f < FP; ++f) {
            U4v fp[3];
#pragma unroll
            for (int s = 0; s < 3; ++s) fp[s] = frag(std::true_type{}, s, f);
            // The matrix unit's own additions to a long sum cost digits: a step's products are summed from 0, small ones first, and added to the rest
            // by an addition that rounds.  Against 64 bits sums of 512 products are 0.9e-7 off (2-norm), of 4,000 1.4e-7.
            F4 sum[FQ] = {};
#pragma unroll
            for (int s = 2; s >= 0; --s)
#pragma unroll
                for (int u = s; u >= 0; --u)
#pragma unroll
                    for (int q = 0; q < FQ; ++q) sum[q] = Frag<__bf16>::times(fp[u], fq[s - u][q], sum[q]);
#pragma unroll
            for (int q = 0; q < FQ; ++q) acc[f][q] += sum[q];
        }
        __syncthreads();
    }
    if (odd) again = 1;
    __syncthreads();
    if (again) {
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
            for (int q = 0; q < FQ; ++q) acc[f][q] = F4{};
        for (int64_t k = k0; k < k1; k += K) {
            sp.load(k, k1);
            sq.load(k, k1);
            sp.store(lds);
            sq.store(lds + TP * TILE_BYTES);
            __syncthreads();
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int f = 0; f < FP; ++f) {
                    const U4v a = StageP::frag(lds, wp + (INSIDE ? f * 4 : f * 16), half);
#pragma unroll
                    for (int q = 0; q < FQ; ++q) acc[f][q] = Frag<float>::times(a, StageQ::frag(lds + TP * TILE_BYTES, wq + q * 16, half), acc[f][q]);
                }
            __syncthreads();
        }
    }
    put_tile<INSIDE>(p, at.part, m0 + wq, n0 + wp, acc);
}

// Few rows: a block is one fragment of 16 by 16, its wavefronts share the sums, and operands go from memory to registers.
template <typename E, typename R, bool ODD, int ROW_WAVES>
__global__ __launch_bounds__(64 * ROW_WAVES) void k_product_rows(const ProductParams<E, R> p)
{
    constexpr int V = 16 / sizeof(E), STEP = 4 * V, AHEAD = 4;
    __shared__ F4 sums[ROW_WAVES][WAVE];
    const uint32_t mt = blockIdx.x / p.n_tiles, nt = blockIdx.x % p.n_tiles;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), i = lane & 15, g = lane >> 4;
    const uint32_t m = mt * 16 + i;
    const int n = (int)nt * 16 + i;
    const E* q = p.q.data + p.q.rows.at(m < p.m ? m : p.m - 1);
    const E* w = p.p.data + p.p.rows.at((uint32_t)(n < p.n ? n : p.n - 1));
    F4 acc = {};
    const int64_t full = p.k / STEP;            // steps without an end of the sums in them
    for (int64_t s = wave; s < full; s += AHEAD * ROW_WAVES) {
        U4v a[AHEAD] = {}, b[AHEAD] = {};
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (s + j * ROW_WAVES < full) {
                a[j] = load_chunk<ODD>(w + (s + j * ROW_WAVES) * STEP + g * V);
                b[j] = load_chunk<ODD>(q + (s + j * ROW_WAVES) * STEP + g * V);
            }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) acc = Frag<E>::times(a[j], b[j], acc);
    }
    if (full * STEP < p.k && wave == ROW_WAVES - 1)
        acc = Frag<E>::times(load_some<E>(w, full * STEP + g * V, p.k), load_some<E>(q, full * STEP + g * V, p.k), acc);
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
    float v[4] = {};
#pragma unroll
    for (int s = 0; s < ROW_WAVES; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += sums[s][lane][r];
    if (m < p.m) p.finish(m, (int)nt * 16 + g * 4, v);
}

// Parts of sums added up, in a fixed order, and finished: four columns are LANES threads', which take the parts in turn.
template <typename E, typename R, int LANES>
__global__ __launch_bounds__(256) void k_product_sum(const float* part, int parts, uint32_t m, int n, uint32_t vectors, unsigned wide, const Finish<E, R> finish)
{
    constexpr int PLACES = 256 / LANES, GO = 4;
    __shared__ F4 sums[LANES > 1 ? LANES : 1][PLACES];
    const int place = threadIdx.x % PLACES, lane = threadIdx.x / PLACES;
    const int64_t at = spread_block(wide) * PLACES + place;
    const bool on = at < (int64_t)m * vectors;
    const uint32_t row = on ? (uint32_t)((uint64_t)at / vectors) : 0;
    const int c = on ? (int)((uint64_t)at % vectors) * 4 : 0;
    float v[4] = {};
    if (on) {
        const float* from = part + (int64_t)row * n + c;
        const int64_t step = (int64_t)m * n;
        int k = lane;
        for (; k + (GO - 1) * LANES < parts; k += GO * LANES) {
            float some[GO][4] = {};
#pragma unroll
            for (int g = 0; g < GO; ++g) Finish<E, R>::template add<float, 4>(from + (k + g * LANES) * step, n - c, some[g]);
#pragma unroll
            for (int g = 0; g < GO; ++g)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += some[g][j];
        }
        for (; k < parts; k += LANES) Finish<E, R>::template add<float, 4>(from + k * step, n - c, v);
    }
    if constexpr (LANES > 1) {
        sums[lane][place] = F4{v[0], v[1], v[2], v[3]};
        __syncthreads();
        if (lane != 0) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = 0.0f;
        for (int k = 0; k < LANES; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += sums[k][place][j];
    }
    if (on) finish(row, c, v);
}

// out[c][r] = in[r][c], in tiles of 32 by 32; rows of out are filled with 0 up to `out_row`, less than a tile
template <typename E>
__global__ __launch_bounds__(256) void k_turn(const E* in, int64_t in_row, E* out, int64_t out_row, int rows, int columns, unsigned x_tiles, unsigned wide)
{
    __shared__ E tile[32][32 + 4 / sizeof(E)];
    const uint32_t block = (uint32_t)spread_block(wide);
    const int x = threadIdx.x % 32, y = threadIdx.x / 32;
    const int64_t r0 = (int64_t)(block / x_tiles) * 32, c0 = (int64_t)(block % x_tiles) * 32;
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int64_t r = r0 + y + k, c = c0 + x;
        tile[y + k][x] = r < rows && c < columns ? in[r * in_row + c] : (E)0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        const int64_t c = c0 + y + k, r = r0 + x;
        if (r < out_row && c < columns) out[c * out_row + r] = tile[x][y + k];
    }
}

// Rows of `columns` values one behind the other, each filled with 0 up to a multiple of eight: what tiles that go straight to LDS ask for.
template <typename E>
__global__ __launch_bounds__(256) void k_fill_up(const Operand<E> in, E* out, uint32_t rows, int columns, uint32_t chunks, unsigned wide)
{
    constexpr int V = 8;
    const int64_t at = spread_block(wide) * 256 + threadIdx.x;
    if (at >= (int64_t)rows * chunks) return;
    const uint32_t row = (uint32_t)((uint64_t)at / chunks);
    const int c = (int)((uint64_t)at % chunks) * V;
    const E* from = in.data + in.rows.at(row);
    Pack<E, V> q;
    if (c + V <= columns) {
        q = *reinterpret_cast<const Pack<E, V>*>(from + c);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = c + j < columns ? from[c + j] : (E)0.0f;
    }
    *reinterpret_cast<Pack<E, V>*>(out + at * V) = q;
}

// dp = dout act'(pre), rounded to the activations' type (not stored where it is dout itself), and its sums over rows: a thread owns
// eight columns and goes on over the rows, 2^across threads lie side by side (64 of them, or as many as there are columns for: 164,595 rows of 44
// take 12 us in place of 110), blocks leave one partial row each.
constexpr int SLOPE_V = 8;
template <typename E, typename R> struct SlopeParams {
    const R* dout;
    const E* pre;
    E* dp;
    Rows dout_rows, pre_rows;
    int64_t dp_row;
    float* factor;           // what takes the power of two back that dp is stored with (see k_largest), or nullptr: stored as it is
    float* largest;          // of k_largest's blocks
    int blocks;
    float* part;
    uint32_t m;
    int n, across;
};
// a row's eight columns, or as many as there are, and the values of dp they are
template <Edge EDGE, typename P> __device__ __forceinline__ void slope_take(const P* from, int count, Pack<P, SLOPE_V>& to)
{
    if (EDGE == VECTORS || count >= SLOPE_V) {
        to = *reinterpret_cast<const Pack<P, SLOPE_V>*>(from);
    } else {
#pragma unroll
        for (int j = 0; j < SLOPE_V; ++j) to.v[j] = from[j < count ? j : 0];
    }
}

// The range of float16.  dp of a float32 gradient may be anything that float32 holds, and float16 ends at 65,504 and at 6e-8: dp is stored times a power of
// two that brings its largest value to 2^14 .. 2^15, which both products take back from their sums (ACT_SCALED).  Values keep their eleven bits down to
// 2^-29 of the largest, and an absolute 2^-40 of it below.  This pass finds the largest finite value of every block, k_slope that of all: it reads what
// k_slope reads once more (262,144 rows of 1,024, without and with an activation: 190 and 290 us).  At most LARGEST_X blocks lie side by side on the columns,
// since every block of k_slope goes over all of their values.
constexpr unsigned LARGEST_X = 2048;
__device__ __forceinline__ float block_largest(float most, float (&sums)[256])
{
    sums[threadIdx.x] = most;
    for (int half = 128; half > 0; half /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < half) sums[threadIdx.x] = __builtin_fmaxf(sums[threadIdx.x], sums[threadIdx.x + half]);
    }
    __syncthreads();
    return sums[0];
}
template <typename E, typename R, int ACT, Edge EDGE>
__global__ __launch_bounds__(256) void k_largest(const SlopeParams<E, R> p)
{
    __shared__ float sums[256];
    const int across = 1 << p.across, x = threadIdx.x & (across - 1), y = threadIdx.x >> p.across, pieces = (p.n - 1) / (across * SLOPE_V) + 1;
    const uint32_t rows = 256u >> p.across, step = gridDim.y * rows;
    float most = 0.0f;
    for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int c = (piece * across + x) * SLOPE_V, count = p.n - c;
        if (count <= 0) break;
        for (uint32_t m = blockIdx.y * rows + y; m < p.m; m += step) {
            Pack<R, SLOPE_V> d;
            Pack<E, SLOPE_V> v = {};
            slope_take<EDGE>(p.dout + p.dout_rows.at(m) + c, count, d);
            if (ACT != CRAFTAX_ACT_NONE) slope_take<EDGE>(p.pre + p.pre_rows.at(m) + c, count, v);
#pragma unroll
            for (int j = 0; j < SLOPE_V; ++j) {           // of a ragged end the first value comes up again
                float size = Elem<R>::up(d.v[j]);
                if (ACT != CRAFTAX_ACT_NONE) size *= slope_of<ACT>(Elem<E>::up(v.v[j]));
                size = __builtin_fabsf(size);
                most = size > most && size <= __FLT_MAX__ ? size : most;
            }
        }
    }
    most = block_largest(most, sums);
    if (threadIdx.x == 0) p.largest[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = most;
}
// The power of two of dp whose largest value is `most`, and what takes it back (`back`): both normal numbers.
__device__ __forceinline__ float power_for(float most, float& back)
{
    const int exponent = (int)(__float_as_uint(most) >> 23) - 127;          // -127: 0, or below the normal numbers
    const int by = most == 0.0f ? 0 : (14 - exponent < 126 ? 14 - exponent : 126);
    back = __uint_as_float((uint32_t)(127 - by) << 23);
    return __uint_as_float((uint32_t)(127 + by) << 23);
}
// EDGE: VECTORS where eight divide the columns, else VALUES.
template <typename E, typename R, int ACT, Edge EDGE>
__global__ __launch_bounds__(256) void k_slope(const SlopeParams<E, R> p)
{
    __shared__ float sums[SLOPE_V][256];
    const int across = 1 << p.across, x = threadIdx.x & (across - 1), y = threadIdx.x >> p.across, c = ((int)blockIdx.x * across + x) * SLOPE_V, count = p.n - c;
    float total[SLOPE_V] = {}, scale = 1.0f;
    constexpr bool SCALED = std::is_same_v<E, _Float16> && std::is_same_v<R, float>;
    if (SCALED && p.factor) {
        float most = 0.0f, back;
        for (int k = threadIdx.x; k < p.blocks; k += 256) most = __builtin_fmaxf(most, p.largest[k]);
        scale = power_for(block_largest(most, sums[0]), back);
        if (blockIdx.x + blockIdx.y + threadIdx.x == 0) *p.factor = back;
        __syncthreads();
    }
    if (count > 0) {
        const uint32_t rows = 256u >> p.across, step = gridDim.y * rows, last = p.m - 1;
        struct Raw { Pack<R, SLOPE_V> d; Pack<E, SLOPE_V> v; } raw;       // one row under way (two or four were no faster)
        auto load = [&](uint32_t row, Raw& q) {
            const uint32_t m = row < last ? row : last;
            slope_take<EDGE>(p.dout + p.dout_rows.at(m) + c, count, q.d);
            if (ACT != CRAFTAX_ACT_NONE) slope_take<EDGE>(p.pre + p.pre_rows.at(m) + c, count, q.v);
        };
        uint32_t m = blockIdx.y * rows + y;
        load(m, raw);
        for (; m < p.m; m += step) {
            float d[SLOPE_V];
#pragma unroll
            for (int j = 0; j < SLOPE_V; ++j) {
                d[j] = Elem<R>::up(raw.d.v[j]);
                if (ACT != CRAFTAX_ACT_NONE) d[j] *= slope_of<ACT>(Elem<E>::up(raw.v.v[j]));
                if (EDGE == VALUES && j >= count) d[j] = 0.0f;         // rows of dp are filled up to a multiple of eight
            }
            // the next row is under way in front of the stores: behind them the wait for it would be for those too
            load(m + step, raw);
#pragma unroll
            for (int j = 0; j < SLOPE_V; ++j) {
                total[j] += d[j];
                if (SCALED) d[j] *= scale;
            }
            if (p.dp) Finish<E, R>::template store<E, SLOPE_V>(p.dp + (int64_t)m * p.dp_row + c, SLOPE_V, d);
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int j = 0; j < SLOPE_V; ++j) sums[j][threadIdx.x] = total[j];
    for (int half = 128; half >= across; half /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < half) {
#pragma unroll
            for (int j = 0; j < SLOPE_V; ++j) total[j] += sums[j][threadIdx.x + half];
            if (half > across) {
#pragma unroll
                for (int j = 0; j < SLOPE_V; ++j) sums[j][threadIdx.x] = total[j];
            }
        }
    }
    if (y != 0 || count <= 0) return;
    Finish<E, R>::template store<float, SLOPE_V>(p.part + (int64_t)blockIdx.y * p.n + c, count, total);
}

struct PutBias {
    float* out;
    __device__ void operator()(int64_t column, float v) const { out[column] = v; }
};

namespace host {

// ---- how a product is cut ------------------------------------------------------------------------------
// ROWS: by fragments, straight from memory.  NARROW: results of up to 32 columns (heads), in tiles of 128 rows.  SMALL, LARGE: tiles of 64 x 64,
// 128 x 128 through registers.  DIRECT, DIRECT_LARGE: tiles of 128 x 128, 256 x 256 that go straight to LDS.
enum class Cut { ROWS, NARROW, SMALL, LARGE, DIRECT, DIRECT_LARGE };
struct Plan {
    Cut cut;
    uint32_t m_tiles, n_tiles;
    int parts;
    int64_t k_part;
    size_t part_bytes;
};
constexpr int64_t CHIP_UNITS = 256;
constexpr int64_t FRAGMENT_BYTES = 2 << 20;
constexpr int64_t MOST_VALUES = (int64_t)1 << 42;       // of a matrix: its tiles are counted in 32 bits

static int64_t tiles_of(int64_t m, int64_t n, int64_t side) { return ceil_div(m, side) * ceil_div(n, side); }
// The parts that a sum of k products may be cut into: eight tiles along k at least each, for the gradient of a weight, whose tiles are few, four.
// (A backward pass of 4,096 rows of 512 bfloat16 values onto 512 takes 42 us, with eight for both 54, with four for both 53; of 1,024 rows 30, 43
// and 32.)
static int64_t most_parts(int64_t k, size_t elem, bool inside)
{
    const int64_t parts = k * (int64_t)elem / ((inside ? 8 : 4) * TILE_BYTES);
    return parts > 1 ? parts : 1;
}
// Whether tiles of that size are enough for every compute unit, with long sums cut into parts, of sixteen tiles along k at least where k lies inside.
// (3,003 rows of 8,268 float32 values onto 256 are 48 of 128 x 128, in ten parts each: 104 us, in tiles of 64 x 64 160.  4,096 rows of 1,024
// bfloat16 values onto 512, 128 in two parts of eight, would take 25, in tiles of 64 x 64 16.  4,096 of 512 onto 1,024, 256 tiles: 11.7 and 14.5.)
static bool tiled(int64_t m, int64_t n, int64_t k, size_t elem, bool inside = true, int64_t side = 128)
{
    return m > side / 2 && n > side / 2 && tiles_of(m, n, side) * most_parts(inside ? k / 2 : k, elem, inside) >= CHIP_UNITS;
}

static Plan plan(int64_t m, int64_t n, int64_t k, size_t elem, bool inside, bool direct)
{
    Plan c{};
    const int64_t step = TILE_BYTES / (int64_t)elem;
    auto tiles = [&](int64_t side) { return tiles_of(m, n, side); };
    c.parts = 1;
    c.k_part = ceil_div(k, step) * step;
    // Fragments straight from memory leave no operand to read again, and each block goes along the whole of k: for few and short ones.  (512 rows of
    // bfloat16 onto 512, 1,024 fragments: 1,024 values a row 10.7 us, in tiles 12.0, 2,048 values 17.9 and 13.5, 8,192 59 and 23.  256 fragments:
    // 4,096 values 10.1 and 13.9, 8,192 17.4 and 13.2.)
    if (inside && tiles(16) <= 4 * CHIP_UNITS && tiles(16) * k * (int64_t)elem <= FRAGMENT_BYTES) {
        c.cut = Cut::ROWS;
        c.m_tiles = (uint32_t)ceil_div(m, 16);
        c.n_tiles = (uint32_t)ceil_div(n, 16);
        return c;
    }
    // A compute unit is taken to need 0.4 times as long for a tile of 128 x 128 as for one of 256 x 256.  With many tiles the large ones are 1.1 to 1.4
    // times as fast, short sums and heavy epilogues among them: bfloat16, tiles of 256 and of 128: 262,144 rows of 512 onto 1,024 337 and 459 us, with gelu
    // and its argument kept 455 and 593; 65,536 rows of 1,024 onto 512 67 and 77; 256 onto 1,024 47 and 63; 8,192 squared 1,070 and 1,197.  Two rounds of
    // large tiles for five of small ones are the rule's border and its worst case: 40,960 rows of 512 onto 512 37 and 33.
    const bool larger = 10 * ceil_div(tiles(256), CHIP_UNITS) <= 4 * ceil_div(tiles(128), CHIP_UNITS) || (!inside && tiled(m, n, k, elem, false, 256));
    if (direct) c.cut = larger ? Cut::DIRECT_LARGE : Cut::DIRECT;
    else c.cut = tiled(m, n, k, elem, inside) ? Cut::LARGE : Cut::SMALL;
    if (inside && n <= 32) c.cut = Cut::NARROW;
    const int64_t side = c.cut == Cut::DIRECT_LARGE ? 256 : c.cut == Cut::SMALL ? 64 : 128;
    c.m_tiles = (uint32_t)ceil_div(m, side);
    c.n_tiles = (uint32_t)ceil_div(n, c.cut == Cut::NARROW ? 32 : side);
    // long sums of few tiles are cut until every compute unit has what it holds at once
    const int64_t have = (int64_t)c.m_tiles * c.n_tiles, most = most_parts(k, elem, inside);
    const int64_t room = c.cut == Cut::DIRECT_LARGE ? CHIP_UNITS : c.cut == Cut::NARROW ? 4 * CHIP_UNITS : 2 * CHIP_UNITS;
    int64_t parts = have < room ? room / have : 1;
    if (parts > most) parts = most;
    if (parts > 1) {
        c.k_part = ceil_div(ceil_div(k, parts), step) * step;
        c.parts = (int)ceil_div(k, c.k_part);
        if (c.parts > 1) c.part_bytes = round256((size_t)c.parts * m * n * sizeof(float));
    }
    return c;
}

template <bool INSIDE, typename E, typename R>
static void launch_product(const Plan& c, ProductParams<E, R> p, float* part, hipStream_t st)
{
    p.m_tiles = c.m_tiles; p.n_tiles = c.n_tiles; p.k_part = c.k_part;
    p.part = c.parts > 1 ? part : nullptr;
    if constexpr (INSIDE) {
        if (c.cut == Cut::ROWS) {
            // rows that begin at odd places
            auto odd = [](const Operand<E>& o) { return !aligned(o.data, 4) || o.rows.step % 2 || o.rows.env % 2; };
            const uint32_t tiles = c.m_tiles * c.n_tiles;
            auto rows = [&](auto is_odd, auto waves) {
                hipLaunchKernelGGL((k_product_rows<E, R, decltype(is_odd)::value, decltype(waves)::value>), dim3(tiles), dim3(64 * decltype(waves)::value), 0, st, p);
            };
            auto waves = [&](auto is_odd) {
                if (tiles <= CHIP_UNITS && p.k * (int64_t)sizeof(E) >= 1024) rows(is_odd, std::integral_constant<int, 16>{});
                else rows(is_odd, std::integral_constant<int, 8>{});
            };
            if constexpr (sizeof(E) == 2) {
                if (odd(p.p) || odd(p.q)) return waves(std::true_type{});
            }
            return waves(std::false_type{});
        }
    }
    const int64_t tiles = ceil_div((int64_t)c.m_tiles * c.n_tiles * c.parts, DIES) * DIES;
    const Spread grid = spread(tiles, 256);
    p.tiles = (uint32_t)tiles;
    p.wide = grid.x;
    const dim3 blocks(grid.x, 1, grid.z);
    if (c.cut == Cut::DIRECT || c.cut == Cut::DIRECT_LARGE) {
        if constexpr (sizeof(E) == 2) launch_direct<INSIDE>(p, tiles, c.cut == Cut::DIRECT_LARGE, st);
    } else {
        auto staged = [&](auto fp, auto fq, auto wp, auto wq) {
            constexpr int FP = decltype(fp)::value, FQ = decltype(fq)::value, WP = decltype(wp)::value, WQ = decltype(wq)::value;
            if constexpr (sizeof(E) == 4) hipLaunchKernelGGL((k_product_float<R, INSIDE, FP, FQ, WP, WQ>), blocks, dim3(256), 0, st, p);
            else hipLaunchKernelGGL((k_product<E, R, INSIDE, FP, FQ, WP, WQ>), blocks, dim3(256), 0, st, p);
        };
        using std::integral_constant;
        constexpr integral_constant<int, 1> one;
        constexpr integral_constant<int, 2> two;
        constexpr integral_constant<int, 4> four;
        if (c.cut == Cut::LARGE) {
            staged(four, four, two, two);
        } else if (c.cut == Cut::SMALL) {
            staged(two, two, two, two);
        } else if constexpr (INSIDE) {
            staged(two, two, one, four);
        }
    }
    if (c.parts > 1) {
        const uint32_t vectors = (uint32_t)ceil_div(p.n, 4);
        auto sum = [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            const Spread wide = spread(ceil_div((int64_t)p.m * vectors, 256 / LANES), 256);
            hipLaunchKernelGGL((k_product_sum<E, R, LANES>), dim3(wide.x, 1, wide.z), dim3(256), 0, st, part, c.parts, p.m, p.n, vectors, wide.x, p.finish);
        };
        if (c.parts > 8) sum(std::integral_constant<int, 16>{});
        else sum(std::integral_constant<int, 1>{});
    }
}

// ---- arguments ---------------------------------------------------------------------------------------------
static bool flat(const craftax_projection_args* a, const craftax_view& v) { return a->steps == 1 || a->n == 1 || v.step == (int64_t)a->n * v.env; }
static Rows rows_of(const craftax_projection_args* a, const craftax_view& v)
{
    if (a->n == 1) return {v.step, 0, 1};
    if (flat(a, v)) return {v.env, 0, 1};
    return {v.step, v.env, (uint32_t)a->n};
}
static Rows dense_rows(int64_t stride) { return {stride, 0, 1}; }

// Batch first: environments count as steps, so that rows lie one behind the other.
static craftax_projection_args ordered(const craftax_projection_args* given)
{
    craftax_projection_args a = *given;
    if (a.x.step < a.x.env) {
        const int32_t steps = a.steps;
        a.steps = a.n;
        a.n = steps;
        for (craftax_view* v : {&a.x, &a.residual, &a.out, &a.pre, &a.dout, &a.dx}) *v = {v->data, v->env, v->step};
    }
    return a;
}

// the weight's rows lie with the inputs side by side
static bool by_rows(const craftax_projection_args* a) { return a->weight_column == 1 || a->inputs == 1; }

static bool countable(const craftax_projection_args* a)
{
    const int64_t rows = (int64_t)a->steps * a->n, wide = a->inputs > a->outputs ? a->inputs : a->outputs;
    return rows <= MOST_VALUES / wide && a->inputs <= MOST_VALUES / a->outputs;
}

static int projection_check(const craftax_projection_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->out_dtype != a->dtype && a->out_dtype != CRAFTAX_F32) return refuse(CRAFTAX_E_CONFIG, "out_dtype must be dtype or CRAFTAX_F32", why);
    if (a->act > CRAFTAX_ACT_GELU_TANH) return refuse(CRAFTAX_E_CONFIG, "unknown act", why);
    if (a->steps < 1 || a->n < 1 || a->inputs < 1 || a->outputs < 1) return refuse(CRAFTAX_E_COUNT, "steps, n, inputs and outputs must be positive", why);
    if ((int64_t)a->steps * a->n >= (int64_t)1 << 31) return refuse(CRAFTAX_E_COUNT, "steps * n must be below 2^31", why);
    if (a->inputs > MOST_COUNT || a->outputs > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "inputs and outputs must be below 2^31 - 4095", why);
    if (!countable(a)) return refuse(CRAFTAX_E_COUNT, "more values than memory holds", why);
    if (!by_rows(a) && a->weight_row != 1 && a->outputs != 1) return refuse(CRAFTAX_E_COUNT, "weight_row or weight_column must be 1", why);
    if (!a->weight || !a->x.data) return refuse(CRAFTAX_E_NULL, "weight or x is NULL", why);
    const size_t e = elem_bytes(a->dtype), r = elem_bytes(a->out_dtype);
    if (!aligned(a->weight, e) || !aligned(a->x.data, e) || !aligned(a->bias, 4) || !aligned(a->pre.data, e))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    if (!backward) {
        if (!a->out.data) return refuse(CRAFTAX_E_NULL, "out is NULL", why);
        if (!aligned(a->out.data, r) || !aligned(a->residual.data, r)) return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
        return CRAFTAX_OK;
    }
    if (!a->dout.data) return refuse(CRAFTAX_E_NULL, "dout is NULL", why);
    if (a->act != CRAFTAX_ACT_NONE && !a->pre.data) return refuse(CRAFTAX_E_NULL, "pre is NULL: the backward pass of an activation needs it", why);
    if (a->dweight_dtype != a->dtype && a->dweight_dtype != CRAFTAX_F32) return refuse(CRAFTAX_E_CONFIG, "dweight_dtype must be dtype or CRAFTAX_F32", why);
    if (!aligned(a->dout.data, r) || !aligned(a->dx.data, e) || !aligned(a->dweight, elem_bytes(a->dweight_dtype)) || !aligned(a->dbias, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    return CRAFTAX_OK;
}

// What a call does, and where in the workspace what lies.
struct Project {
    int64_t rows;
    Plan forward, dx, dweight;
    bool turn, fill_weight;  // the weight is turned, or its rows are filled up, first
    bool fill_x;             // the rows of x are
    int64_t weight_row, x_row, dp_row;   // of what lies in the workspace
    bool has_dp, scaled;     // dp lies in the workspace; times a power of two
    int slope_across;
    unsigned slope_x, slope_y, largest_x;
    size_t weight_at, x_at, dp_at, scale_at, sums_at, part_at, total;
};
// Where rows cannot go straight to LDS they are copied to where they can, if the product is worth it: reading and writing them takes as long as
// this many columns of the result gain by it, and a copy is a launch more.  (bfloat16: 16,384 rows of 333 values onto 1,024, 5.6e9 products, take 36 us,
// through registers 57; 262,144 rows of 1,345 onto 512 700 and 858; but 4,096 rows of 1,345 onto 512, 2.8e9 products, 33 and 23.)
constexpr int64_t WORTH_COLUMNS = 256;
constexpr double WORTH_PRODUCTS = 4e9;

static Project project(const craftax_projection_args* a, bool backward)
{
    Project c{};
    const size_t e = elem_bytes(a->dtype);
    c.rows = (int64_t)a->steps * a->n;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    auto filled = [](int64_t count) { return ceil_div(count, 8) * 8; };
    // whether rows can go straight to LDS, 16 bytes at a time: those of a tile lie within 2^32 bytes, one stride apart
    auto near = [&](int64_t row) { return e == 2 && row >= 0 && row < ((int64_t)1 << 23) - 512; };
    auto fits = [&](const void* data, int64_t row, int64_t count) { return near(row) && count % 8 == 0 && aligned(data, 16) && row % 8 == 0; };
    auto whole = [&](const craftax_view& v, int64_t count) { return flat(a, v) && fits(v.data, rows_of(a, v).step, count); };
    const bool large = (double)c.rows * a->inputs * a->outputs >= WORTH_PRODUCTS;
    c.x_row = filled(a->inputs);
    c.dp_row = filled(a->outputs);
    if (!backward) {
        c.weight_row = c.x_row;
        c.turn = !by_rows(a);
        bool direct = near(c.x_row) && tiled(c.rows, a->outputs, a->inputs, e);
        if (direct && !whole(a->x, a->inputs)) direct = c.fill_x = a->outputs >= WORTH_COLUMNS && large;
        if (direct && !c.turn) c.fill_weight = !fits(a->weight, a->weight_row, a->inputs);
        if (c.turn || c.fill_weight) c.weight_at = take((size_t)a->outputs * c.weight_row * e);
        if (c.fill_x) c.x_at = take((size_t)c.rows * c.x_row * e);
        c.forward = plan(c.rows, a->outputs, a->inputs, e, true, direct);
        c.part_at = take(c.forward.part_bytes);
    } else {
        c.weight_row = c.dp_row;
        c.turn = a->dx.data && by_rows(a) && a->weight_row != 1;
        c.has_dp = (a->act != CRAFTAX_ACT_NONE || a->out_dtype != a->dtype) && (a->dx.data || a->dweight);
        const bool wide = near(c.dp_row) && near(c.x_row) && c.rows < (int64_t)1 << 30, worth = wide && large;
        if (!c.has_dp && worth && !whole(a->dout, a->outputs)) c.has_dp = (a->dx.data || a->dweight) && a->inputs >= WORTH_COLUMNS;
        const bool dp_fits = wide && (c.has_dp || whole(a->dout, a->outputs));
        bool direct_dx = a->dx.data && dp_fits && tiled(c.rows, a->inputs, a->outputs, e), direct_dw = a->dweight && dp_fits;
        if (direct_dx && !c.turn) c.fill_weight = !fits(a->weight, a->weight_column, a->outputs);
        if (direct_dw && !whole(a->x, a->inputs)) direct_dw = c.fill_x = worth && a->outputs >= WORTH_COLUMNS;
        if (c.turn || c.fill_weight) c.weight_at = take((size_t)a->inputs * c.weight_row * e);
        if (c.fill_x) c.x_at = take((size_t)c.rows * c.x_row * e);
        if (c.has_dp) c.dp_at = take((size_t)c.rows * c.dp_row * e);
        while (c.slope_across < 6 && (SLOPE_V << c.slope_across) < a->outputs) ++c.slope_across;
        c.slope_x = (unsigned)ceil_div(a->outputs, SLOPE_V << c.slope_across);
        int64_t y = ceil_div(c.rows, 256 >> c.slope_across), most = ceil_div(2048, c.slope_x);
        c.slope_y = (unsigned)(y < most ? y : most);
        c.scaled = c.has_dp && a->dtype == CRAFTAX_F16 && a->out_dtype == CRAFTAX_F32;
        c.largest_x = c.slope_x < LARGEST_X ? c.slope_x : LARGEST_X;
        if (c.scaled) c.scale_at = take((1 + (size_t)c.largest_x * c.slope_y) * sizeof(float));
        if (a->dbias) c.sums_at = take((size_t)c.slope_y * a->outputs * sizeof(float));
        size_t part = 0;
        if (a->dx.data) {
            c.dx = plan(c.rows, a->inputs, a->outputs, e, true, direct_dx);
            part = c.dx.part_bytes;
        }
        if (a->dweight) {
            c.dweight = plan(a->outputs, a->inputs, c.rows, e, false, direct_dw);
            if (c.dweight.part_bytes > part) part = c.dweight.part_bytes;
        }
        c.part_at = take(part);
    }
    c.total = at;
    return c;
}

size_t projection_workspace_bytes(const craftax_projection_args* a, bool backward)
{
    if (!a || a->dtype > CRAFTAX_F16 || a->steps < 1 || a->n < 1 || a->inputs < 1 || a->outputs < 1 || a->inputs > MOST_COUNT || a->outputs > MOST_COUNT ||
        (int64_t)a->steps * a->n >= (int64_t)1 << 31 || !countable(a))
        return 0;
    const craftax_projection_args ours = ordered(a);
    return project(&ours, backward).total;
}

static int projection_room(const craftax_projection_args* a, size_t need, const char** why)
{
    if (need && !a->workspace) return refuse(CRAFTAX_E_NULL, "workspace is NULL", why);
    if (need && !aligned(a->workspace, 256)) return refuse(CRAFTAX_E_ALIGN, "workspace must be 256-byte aligned", why);
    if (a->workspace_bytes < need) return refuse(CRAFTAX_E_COUNT, "workspace smaller than craftax_projection_workspace_bytes", why);
    return CRAFTAX_OK;
}

template <typename E> static void turn(const E* in, int64_t in_row, E* out, int64_t out_row, int rows, int columns, hipStream_t st)
{
    const unsigned x = (unsigned)ceil_div(columns, 32);
    const Spread grid = spread(ceil_div(rows, 32) * x, 256);
    hipLaunchKernelGGL((k_turn<E>), dim3(grid.x, 1, grid.z), dim3(256), 0, st, in, in_row, out, out_row, rows, columns, x, grid.x);
}

template <typename E> static void fill_up(const Operand<E>& in, E* out, int64_t rows, int columns, hipStream_t st)
{
    const int64_t chunks = ceil_div(columns, 8);
    const Spread grid = spread(ceil_div(rows * chunks, 256), 256);
    hipLaunchKernelGGL((k_fill_up<E>), dim3(grid.x, 1, grid.z), dim3(256), 0, st, in, out, (uint32_t)rows, columns, (uint32_t)chunks, grid.x);
}
// x as the products read it
template <typename E> static Operand<E> x_of(const craftax_projection_args* a, const Project& c, char* work, hipStream_t st)
{
    const Operand<E> given{static_cast<const E*>(a->x.data), rows_of(a, a->x)};
    if (!c.fill_x) return given;
    E* ours = reinterpret_cast<E*>(work + c.x_at);
    fill_up<E>(given, ours, c.rows, a->inputs, st);
    return {ours, dense_rows(c.x_row)};
}

// calls f with values of the activations' and the outputs' type
template <typename F> static void with_types(uint32_t dtype, uint32_t out, F&& f)
{
    with_type(dtype, [&](auto e) {
        if (out == CRAFTAX_F32) f(e, float{});
        else f(e, e);
    });
}

int projection(const craftax_projection_args* given, void* stream, const char** why)
{
    if (int rc = projection_check(given, false, why)) return rc;
    const craftax_projection_args ours = ordered(given), *a = &ours;
    const Project c = project(a, false);
    if (int rc = projection_room(a, c.total, why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    char* work = static_cast<char*>(a->workspace);
    with_types(a->dtype, a->out_dtype, [&](auto e, auto r) {
        using E = decltype(e);
        using R = decltype(r);
        ProductParams<E, R> p{};
        const E* weight = static_cast<const E*>(a->weight);
        int64_t ld = a->weight_row;
        if (c.turn || c.fill_weight) {
            E* ours = reinterpret_cast<E*>(work + c.weight_at);
            if (c.turn) turn<E>(weight, a->weight_column, ours, c.weight_row, a->inputs, a->outputs, st);
            else fill_up<E>({weight, dense_rows(ld)}, ours, a->outputs, a->inputs, st);
            weight = ours;
            ld = c.weight_row;
        }
        p.p = {weight, dense_rows(ld)};
        p.q = x_of<E>(a, c, work, st);
        p.k = a->inputs; p.m = (uint32_t)c.rows; p.n = a->outputs;
        p.finish = {a->bias, static_cast<const R*>(a->residual.data), static_cast<R*>(a->out.data), static_cast<E*>(a->pre.data),
                    rows_of(a, a->residual), rows_of(a, a->out), rows_of(a, a->pre), (int)a->act, a->outputs, nullptr};
        launch_product<true>(c.forward, p, reinterpret_cast<float*>(work + c.part_at), st);
    });
    return launched(why);
}

int projection_backward(const craftax_projection_args* given, void* stream, const char** why)
{
    if (int rc = projection_check(given, true, why)) return rc;
    const craftax_projection_args ours = ordered(given), *a = &ours;
    const Project c = project(a, true);
    if (int rc = projection_room(a, c.total, why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    char* work = static_cast<char*>(a->workspace);
    with_types(a->dtype, a->out_dtype, [&](auto e, auto r) {
        using E = decltype(e);
        using R = decltype(r);
        E* own = c.has_dp ? reinterpret_cast<E*>(work + c.dp_at) : nullptr;
        float* factor = c.scaled ? reinterpret_cast<float*>(work + c.scale_at) : nullptr;
        if (own || a->dbias) {
            SlopeParams<E, R> s{};
            s.dout = static_cast<const R*>(a->dout.data); s.dout_rows = rows_of(a, a->dout);
            s.pre = a->act == CRAFTAX_ACT_NONE ? nullptr : static_cast<const E*>(a->pre.data); s.pre_rows = rows_of(a, a->pre);
            s.dp = own; s.dp_row = c.dp_row;
            s.factor = factor; s.largest = factor ? factor + 1 : nullptr; s.blocks = (int)(c.largest_x * c.slope_y);
            s.part = a->dbias ? reinterpret_cast<float*>(work + c.sums_at) : nullptr;
            s.m = (uint32_t)c.rows; s.n = a->outputs; s.across = c.slope_across;
            auto slope = [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                if constexpr (std::is_same_v<E, _Float16> && std::is_same_v<R, float>) {
                    if (factor) {
                        if (s.n % SLOPE_V == 0) hipLaunchKernelGGL((k_largest<E, R, ACT, VECTORS>), dim3(c.largest_x, c.slope_y), dim3(256), 0, st, s);
                        else hipLaunchKernelGGL((k_largest<E, R, ACT, VALUES>), dim3(c.largest_x, c.slope_y), dim3(256), 0, st, s);
                    }
                }
                if (s.n % SLOPE_V == 0) hipLaunchKernelGGL((k_slope<E, R, ACT, VECTORS>), dim3(c.slope_x, c.slope_y), dim3(256), 0, st, s);
                else hipLaunchKernelGGL((k_slope<E, R, ACT, VALUES>), dim3(c.slope_x, c.slope_y), dim3(256), 0, st, s);
            };
            if (a->act == CRAFTAX_ACT_NONE) slope(std::integral_constant<int, CRAFTAX_ACT_NONE>{});
            else if (a->act == CRAFTAX_ACT_RELU) slope(std::integral_constant<int, CRAFTAX_ACT_RELU>{});
            else if (a->act == CRAFTAX_ACT_SILU) slope(std::integral_constant<int, CRAFTAX_ACT_SILU>{});
            else slope(std::integral_constant<int, CRAFTAX_ACT_GELU_TANH>{});
            if (a->dbias) sum_rows(s.part, (int)c.slope_y, a->outputs, PutBias{a->dbias}, st);
        }
        const Operand<E> dp = own ? Operand<E>{own, dense_rows(c.dp_row)} : Operand<E>{static_cast<const E*>(a->dout.data), rows_of(a, a->dout)};
        float* part = reinterpret_cast<float*>(work + c.part_at);
        auto unscale = [&](auto& finish) {
            if (!factor) return;
            finish.act = ACT_SCALED;
            finish.factor = factor;
        };
        if (a->dx.data) {
            ProductParams<E, E> p{};
            unscale(p.finish);
            const E* weight = static_cast<const E*>(a->weight);
            int64_t ld = a->weight_column;
            if (c.turn || c.fill_weight) {
                E* ours = reinterpret_cast<E*>(work + c.weight_at);
                if (c.turn) turn<E>(weight, a->weight_row, ours, c.weight_row, a->outputs, a->inputs, st);
                else fill_up<E>({weight, dense_rows(ld)}, ours, a->inputs, a->outputs, st);
                weight = ours;
                ld = c.weight_row;
            }
            p.p = {weight, dense_rows(ld)};
            p.q = dp;
            p.k = a->outputs; p.m = (uint32_t)c.rows; p.n = a->inputs;
            p.finish.out = static_cast<E*>(a->dx.data); p.finish.out_rows = rows_of(a, a->dx); p.finish.columns = a->inputs;
            launch_product<true>(c.dx, p, part, st);
        }
        if (a->dweight) {
            auto weight = [&](auto w) {
                using W = decltype(w);
                ProductParams<E, W> p{};
                unscale(p.finish);
                p.p = x_of<E>(a, c, work, st);
                p.q = dp;
                p.k = c.rows; p.m = (uint32_t)a->outputs; p.n = a->inputs;
                p.finish.out = static_cast<W*>(a->dweight); p.finish.out_rows = dense_rows(a->inputs); p.finish.columns = a->inputs;
                launch_product<false>(c.dweight, p, part, st);
            };
            if (a->dweight_dtype == a->dtype) weight(E{});
            else weight(float{});
        }
    });
    return launched(why);
}

}  // namespace host
}  // namespace mem
