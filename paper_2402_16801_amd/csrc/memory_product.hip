// Matrix product with bias, activation and residual in its epilogue, and its backward pass.
//
//   out = residual + act(x weight^T + bias);   dp = dout act'(pre),  dx = dp weight,  dweight = dp^T x,  dbias = sum of dp
//
// Few rows (an actor's token) are bound by the latency of one pass over the operands, many by the matrix cores or, at the
// widths of a policy, by memory.  Sums are in 32 bits; dp is rounded to the type of the activations, which the matrix instructions take.
#include "memory_api.hpp"
#include "memory_common.hpp"
#include "memory_product.hpp"

#include <type_traits>

namespace mem {

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
    float* part;             // [parts][m][n], or nullptr: one part, finished here
    unsigned wide;
    Finish<E, R> finish;
};

// The place of a 16-byte chunk in a tile: exchanged within the row by a number of the row, so that the chunks that are read at once lie in
// different banks.
template <int FP, bool IS_P> __device__ __forceinline__ int inside_key(int row) { return IS_P ? (row & 3) | ((row / (4 * FP)) & 1) << 2 : row & 7; }
template <typename E, int TILE> __device__ __forceinline__ int across_key(int k)
{
    return (sizeof(E) == 2 ? ((k & 3) << 1) | ((k >> 3) & 1) << 3 : ((k >> 2) & 3) << 2) & (TILE * (int)sizeof(E) / 16 - 1);
}

// One operand's tile of TILE rows on its way from memory to LDS.
template <typename E, int TILE, int THREADS, bool INSIDE, int FP, bool IS_P> struct Stage {
    static constexpr int V = 16 / sizeof(E), CHUNKS = TILE * 8 / THREADS, ROW_CHUNKS = INSIDE ? 8 : TILE / V;
    const E* from[INSIDE ? CHUNKS : 1];
    U4v raw[CHUNKS];
    int side;                // chunks inside a row: values before this thread's
    int left;                // across: values of a row from its chunk on
    Operand<E> op;
    __device__ __forceinline__ static int row_of(int c) { return ((int)threadIdx.x + c * THREADS) / ROW_CHUNKS; }
    __device__ __forceinline__ static int chunk_of(int c) { return ((int)threadIdx.x + c * THREADS) % ROW_CHUNKS; }
    __device__ __forceinline__ Stage(const Operand<E>& o, uint32_t first, uint32_t rows) : op(o)
    {
        static_assert(THREADS % ROW_CHUNKS == 0, "a thread's chunks lie below one another");
        side = chunk_of(0) * V;
        left = (int)(rows - first) - side;
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
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (INSIDE) {
                const int64_t rest = end - (k + side);
                raw[c] = load_some<E>(from[c] + k + side, rest > V ? V : (int)rest);
            } else {
                const int64_t row = k + row_of(c);
                raw[c] = load_some<E>(from[0] + op.rows.at((uint32_t)(row < end ? row : end - 1)) + side, row < end ? left : 0);
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
    // the fragment of 16 rows whose first is `row`, 64 bytes along k from 64 * half on.  IS_P and k inside: place i of the fragment is row
    // i / 4 * 4 FP + i % 4 behind it.
    __device__ __forceinline__ static U4v frag(const char* lds, int row, int half)
    {
        const int lane = threadIdx.x & (WAVE - 1), i = lane & 15, g = lane >> 4;
        if constexpr (INSIDE) {
            const int r = row + (IS_P ? i / 4 * (4 * FP) + i % 4 : i);
            return *reinterpret_cast<const U4v*>(lds + (r * 8 + ((half * 4 + g) ^ inside_key<FP, IS_P>(r))) * 16);
        } else if constexpr (sizeof(E) == 2) {
            // a group of 16 lanes reads four rows of 16 values and gets them column by column
            U4v out;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = half * 32 + g * 8 + h * 4 + i / 4, col = row + i % 4 * 4;
                const char* at = lds + (k * ROW_CHUNKS + ((col / 8) ^ across_key<E, TILE>(k))) * 16 + col % 8 * 2;
                const S4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)(at));
                const uint64_t bits = __builtin_bit_cast(uint64_t, v);
                out[2 * h] = (uint32_t)bits;
                out[2 * h + 1] = (uint32_t)(bits >> 32);
            }
            return out;
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

// Which tile a block computes.  Consecutive blocks go to the eight dies in turn: the tiles of a row of tiles, which read the same rows of Q,
// follow one another on one die.
struct TilePlace {
    uint32_t m, n, part;
    bool on;
    template <typename P> __device__ __forceinline__ explicit TilePlace(const P& p)
    {
        constexpr uint32_t DIES = 8;
        const uint64_t block = (uint64_t)spread_block(p.wide);
        const uint32_t per_part = (p.m_tiles + DIES - 1) / DIES * DIES * p.n_tiles;
        part = (uint32_t)(block / per_part);
        const uint32_t at = (uint32_t)(block % per_part), turn = at / DIES;
        n = turn % p.n_tiles;
        m = turn / p.n_tiles * DIES + at % DIES;
        on = m < p.m_tiles && (int64_t)part * p.k_part < p.k;
    }
};

// A block of WP x WQ wavefronts computes 16 FP WP columns by 16 FQ WQ rows.
template <typename E, typename R, bool INSIDE, int FP, int FQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ) void k_product(const ProductParams<E, R> p)
{
    constexpr int THREADS = 64 * WP * WQ, TP = 16 * FP * WP, TQ = 16 * FQ * WQ, K = tile_k<E>();
    using StageP = Stage<E, TP, THREADS, INSIDE, FP, true>;
    using StageQ = Stage<E, TQ, THREADS, INSIDE, FP, false>;
    __shared__ __attribute__((aligned(16))) char lds[2][(TP + TQ) * TILE_BYTES];
    const TilePlace at(p);
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
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int q = 0; q < FQ; ++q) {
        const uint32_t m = m0 + wq + q * 16 + i;
        if (m >= p.m) continue;
        auto put = [&](int n, auto& v) {
            constexpr int COUNT = sizeof(v) / sizeof(float);
            if (p.part) {
                if (n < p.n) Finish<E, R>::template store<float, COUNT>(p.part + ((int64_t)at.part * p.m + m) * p.n + n, p.n - n, v);
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
            put(n0 + wp + g * 4 * FP, v);
        } else {
#pragma unroll
            for (int f = 0; f < FP; ++f) {
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[f][q][r];
                put(n0 + wp + f * 16 + g * 4, v);
            }
        }
    }
}

// Few rows: a block is one fragment of 16 by 16, its wavefronts share the sums, and operands go from memory to registers.
constexpr int ROW_WAVES = 8;
template <typename E, typename R>
__global__ __launch_bounds__(64 * ROW_WAVES) void k_product_rows(const ProductParams<E, R> p)
{
    constexpr int V = 16 / sizeof(E), STEP = 4 * V, AHEAD = 4;
    __shared__ F4 sums[ROW_WAVES][WAVE];
    const uint32_t mt = blockIdx.x / p.n_tiles, nt = blockIdx.x % p.n_tiles;
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), i = lane & 15, g = lane >> 4;
    const uint32_t m = mt * 16 + i;
    const int n = (int)nt * 16 + i;
    const E* q = p.q.data + p.q.rows.at(m < p.m ? m : p.m - 1) + g * V;
    const E* w = p.p.data + p.p.rows.at((uint32_t)(n < p.n ? n : p.n - 1)) + g * V;
    F4 acc = {};
    int64_t k = (int64_t)wave * STEP;
    for (; k + ((AHEAD - 1) * ROW_WAVES + 1) * STEP <= p.k; k += AHEAD * ROW_WAVES * STEP) {
        U4v a[AHEAD], b[AHEAD];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            a[s] = load_some<E>(w + k + s * ROW_WAVES * STEP, V);
            b[s] = load_some<E>(q + k + s * ROW_WAVES * STEP, V);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) acc = Frag<E>::times(a[s], b[s], acc);
    }
    for (; k < p.k; k += ROW_WAVES * STEP) {
        const int64_t rest = p.k - (k + g * V);
        const int count = rest > V ? V : (int)rest;
        acc = Frag<E>::times(load_some<E>(w + k, count), load_some<E>(q + k, count), acc);
    }
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

// Parts of sums added up, in order, and finished.
template <typename E, typename R>
__global__ __launch_bounds__(256) void k_product_sum(const float* part, int parts, uint32_t m, int n, uint32_t vectors, unsigned wide, const Finish<E, R> finish)
{
    const int64_t at = spread_block(wide) * 256 + threadIdx.x;
    if (at >= (int64_t)m * vectors) return;
    const uint32_t row = (uint32_t)((uint64_t)at / vectors);
    const int c = (int)((uint64_t)at % vectors) * 4;
    float v[4] = {};
    for (int k = 0; k < parts; ++k) Finish<E, R>::template add<float, 4>(part + ((int64_t)k * m + row) * n + c, n - c, v);
    finish(row, c, v);
}

// out[c][r] = in[r][c]
template <typename E>
__global__ __launch_bounds__(256) void k_turn(const E* in, int64_t in_row, E* out, int64_t out_row, int rows, int columns, unsigned x_tiles, unsigned wide)
{
    __shared__ E tile[64][64 + 4 / sizeof(E)];
    const uint32_t block = (uint32_t)spread_block(wide);
    const int x = threadIdx.x % 64, y = threadIdx.x / 64;
    const int64_t r0 = (int64_t)(block / x_tiles) * 64, c0 = (int64_t)(block % x_tiles) * 64;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t r = r0 + y + 4 * k, c = c0 + x;
        if (r < rows && c < columns) tile[y + 4 * k][x] = in[r * in_row + c];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t c = c0 + y + 4 * k, r = r0 + x;
        if (r < rows && c < columns) out[c * out_row + r] = tile[x][y + 4 * k];
    }
}

// dp = dout act'(pre), rounded to the activations' type (not stored where it is dout itself), and its sums over rows: a thread owns
// eight columns and goes on over the rows, blocks leave one partial row each.
constexpr int SLOPE_V = 8;
template <typename E, typename R> struct SlopeParams {
    const R* dout;
    const E* pre;
    E* dp;
    Rows dout_rows, pre_rows;
    int64_t dp_row;
    float* part;
    uint32_t m;
    int n, act;
};
template <typename P> __device__ __forceinline__ void load_row(const P* p, int count, float (&v)[SLOPE_V])
{
    if (count >= SLOPE_V) {
        const Pack<P, SLOPE_V> q = *reinterpret_cast<const Pack<P, SLOPE_V>*>(p);
#pragma unroll
        for (int j = 0; j < SLOPE_V; ++j) v[j] = Elem<P>::up(q.v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < SLOPE_V; ++j) v[j] = j < count ? Elem<P>::up(p[j]) : 0.0f;
    }
}
template <typename E, typename R>
__global__ __launch_bounds__(256) void k_slope(const SlopeParams<E, R> p)
{
    __shared__ float sums[SLOPE_V][256];
    const int x = threadIdx.x % 64, y = threadIdx.x / 64, c = ((int)blockIdx.x * 64 + x) * SLOPE_V, count = p.n - c;
    float total[SLOPE_V] = {};
    if (count > 0) {
        for (uint32_t m = blockIdx.y * 4 + y; m < p.m; m += gridDim.y * 4) {
            float d[SLOPE_V];
            load_row(p.dout + p.dout_rows.at(m) + c, count, d);
            if (p.pre) {
                float v[SLOPE_V];
                load_row(p.pre + p.pre_rows.at(m) + c, count, v);
#pragma unroll
                for (int j = 0; j < SLOPE_V; ++j) d[j] *= slope_of(v[j], p.act);
            }
            if (p.dp) Finish<E, R>::template store<E, SLOPE_V>(p.dp + (int64_t)m * p.dp_row + c, count, d);
#pragma unroll
            for (int j = 0; j < SLOPE_V; ++j) total[j] += d[j];
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int j = 0; j < SLOPE_V; ++j) sums[j][threadIdx.x] = total[j];
    __syncthreads();
    if (y != 0 || count <= 0) return;
#pragma unroll
    for (int j = 0; j < SLOPE_V; ++j) total[j] = (sums[j][x] + sums[j][x + 64]) + (sums[j][x + 128] + sums[j][x + 192]);
    Finish<E, R>::template store<float, SLOPE_V>(p.part + (int64_t)blockIdx.y * p.n + c, count, total);
}

struct PutBias {
    float* out;
    __device__ void operator()(int64_t column, float v) const { out[column] = v; }
};

namespace host {

// ---- how a product is cut ------------------------------------------------------------------------------
// ROWS: by fragments, straight from memory.  SMALL, LARGE: tiles of 64 x 64, 128 x 128.
enum class Cut { ROWS, SMALL, LARGE };
struct Plan {
    Cut cut;
    uint32_t m_tiles, n_tiles;
    int parts;
    int64_t k_part;
    size_t part_bytes;
};
constexpr int64_t CHIP_UNITS = 256;
constexpr int64_t MOST_VALUES = (int64_t)1 << 42;       // of a matrix: its tiles are counted in 32 bits

static Plan plan(int64_t m, int64_t n, int64_t k, size_t elem, bool inside)
{
    Plan c{};
    const int64_t step = TILE_BYTES / (int64_t)elem, small = ceil_div(m, 64) * ceil_div(n, 64), large = ceil_div(m, 128) * ceil_div(n, 128);
    c.parts = 1;
    c.k_part = ceil_div(k, step) * step;
    if (inside && ceil_div(m, 16) * ceil_div(n, 16) <= 4 * CHIP_UNITS) {
        c.cut = Cut::ROWS;
        c.m_tiles = (uint32_t)ceil_div(m, 16);
        c.n_tiles = (uint32_t)ceil_div(n, 16);
        return c;
    }
    c.cut = large >= CHIP_UNITS || (!inside && m >= 128 && n >= 128) ? Cut::LARGE : Cut::SMALL;
    const int64_t side = c.cut == Cut::LARGE ? 128 : 64, tiles = c.cut == Cut::LARGE ? large : small;
    c.m_tiles = (uint32_t)ceil_div(m, side);
    c.n_tiles = (uint32_t)ceil_div(n, side);
    // long sums of few tiles are cut, into parts of eight tiles along k at least
    int64_t parts = tiles < 2 * CHIP_UNITS ? 2 * CHIP_UNITS / tiles : 1;
    const int64_t most = k / (8 * step);
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
    if (c.cut == Cut::ROWS) {
        hipLaunchKernelGGL((k_product_rows<E, R>), dim3(c.m_tiles * c.n_tiles), dim3(64 * ROW_WAVES), 0, st, p);
        return;
    }
    const Spread grid = spread(ceil_div(c.m_tiles, 8) * 8 * (int64_t)c.n_tiles * c.parts, 256);
    p.wide = grid.x;
    const dim3 blocks(grid.x, 1, grid.z);
    if (c.cut == Cut::LARGE) hipLaunchKernelGGL((k_product<E, R, INSIDE, 4, 4, 2, 2>), blocks, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_product<E, R, INSIDE, 2, 2, 2, 2>), blocks, dim3(256), 0, st, p);
    if (c.parts > 1) {
        const uint32_t vectors = (uint32_t)ceil_div(p.n, 4);
        const Spread sum = spread(ceil_div((int64_t)p.m * vectors, 256), 256);
        hipLaunchKernelGGL((k_product_sum<E, R>), dim3(sum.x, 1, sum.z), dim3(256), 0, st, part, c.parts, p.m, p.n, vectors, sum.x, p.finish);
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

// the weight's rows lie with the inputs side by side
static bool by_rows(const craftax_projection_args* a) { return a->weight_column == 1 || a->inputs == 1; }

static int projection_check(const craftax_projection_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->out_dtype != a->dtype && a->out_dtype != CRAFTAX_F32) return refuse(CRAFTAX_E_CONFIG, "out_dtype must be dtype or CRAFTAX_F32", why);
    if (a->act > CRAFTAX_ACT_GELU_TANH) return refuse(CRAFTAX_E_CONFIG, "unknown act", why);
    if (a->steps < 1 || a->n < 1 || a->inputs < 1 || a->outputs < 1) return refuse(CRAFTAX_E_COUNT, "steps, n, inputs and outputs must be positive", why);
    if ((int64_t)a->steps * a->n >= (int64_t)1 << 31) return refuse(CRAFTAX_E_COUNT, "steps * n must be below 2^31", why);
    if (a->inputs > MOST_COUNT || a->outputs > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "inputs and outputs must be below 2^31 - 4095", why);
    const int64_t rows = (int64_t)a->steps * a->n, wide = a->inputs > a->outputs ? a->inputs : a->outputs;
    if (rows > MOST_VALUES / wide || a->inputs > MOST_VALUES / a->outputs) return refuse(CRAFTAX_E_COUNT, "more values than memory holds", why);
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
    bool turn;               // the weight is turned first
    int64_t turned_row, dp_row;
    bool has_dp;
    unsigned slope_x, slope_y;
    size_t turned_at, dp_at, sums_at, part_at, total;
};
static Project project(const craftax_projection_args* a, bool backward)
{
    Project c{};
    const size_t e = elem_bytes(a->dtype);
    c.rows = (int64_t)a->steps * a->n;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    if (!backward) {
        c.turn = !by_rows(a);
        c.turned_row = ceil_div(a->inputs, 8) * 8;
        if (c.turn) c.turned_at = take((size_t)a->outputs * c.turned_row * e);
        c.forward = plan(c.rows, a->outputs, a->inputs, e, true);
        c.part_at = take(c.forward.part_bytes);
    } else {
        c.turn = a->dx.data && by_rows(a) && a->weight_row != 1;
        c.turned_row = ceil_div(a->outputs, 8) * 8;
        if (c.turn) c.turned_at = take((size_t)a->inputs * c.turned_row * e);
        c.has_dp = (a->act != CRAFTAX_ACT_NONE || a->out_dtype != a->dtype) && (a->dx.data || a->dweight);
        c.dp_row = ceil_div(a->outputs, 8) * 8;
        if (c.has_dp) c.dp_at = take((size_t)c.rows * c.dp_row * e);
        c.slope_x = (unsigned)ceil_div(a->outputs, 64 * SLOPE_V);
        int64_t y = ceil_div(c.rows, 4), most = ceil_div(2048, c.slope_x);
        c.slope_y = (unsigned)(y < most ? y : most);
        if (a->dbias) c.sums_at = take((size_t)c.slope_y * a->outputs * sizeof(float));
        size_t part = 0;
        if (a->dx.data) {
            c.dx = plan(c.rows, a->inputs, a->outputs, e, true);
            part = c.dx.part_bytes;
        }
        if (a->dweight) {
            c.dweight = plan(a->outputs, a->inputs, c.rows, e, false);
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
        (int64_t)a->steps * a->n >= (int64_t)1 << 31)
        return 0;
    return project(a, backward).total;
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
    const unsigned x = (unsigned)ceil_div(columns, 64);
    const Spread grid = spread(ceil_div(rows, 64) * x, 256);
    hipLaunchKernelGGL((k_turn<E>), dim3(grid.x, 1, grid.z), dim3(256), 0, st, in, in_row, out, out_row, rows, columns, x, grid.x);
}

// calls f with values of the activations' and the outputs' type
template <typename F> static void with_types(uint32_t dtype, uint32_t out, F&& f)
{
    with_type(dtype, [&](auto e) {
        if (out == CRAFTAX_F32) f(e, float{});
        else f(e, e);
    });
}

int projection(const craftax_projection_args* a, void* stream, const char** why)
{
    if (int rc = projection_check(a, false, why)) return rc;
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
        if (c.turn) {
            E* turned = reinterpret_cast<E*>(work + c.turned_at);
            turn<E>(weight, a->weight_column, turned, c.turned_row, a->inputs, a->outputs, st);
            weight = turned;
            ld = c.turned_row;
        }
        p.p = {weight, dense_rows(ld)};
        p.q = {static_cast<const E*>(a->x.data), rows_of(a, a->x)};
        p.k = a->inputs; p.m = (uint32_t)c.rows; p.n = a->outputs;
        p.finish = {a->bias, static_cast<const R*>(a->residual.data), static_cast<R*>(a->out.data), static_cast<E*>(a->pre.data),
                    rows_of(a, a->residual), rows_of(a, a->out), rows_of(a, a->pre), (int)a->act, a->outputs};
        launch_product<true>(c.forward, p, reinterpret_cast<float*>(work + c.part_at), st);
    });
    return launched(why);
}

int projection_backward(const craftax_projection_args* a, void* stream, const char** why)
{
    if (int rc = projection_check(a, true, why)) return rc;
    const Project c = project(a, true);
    if (int rc = projection_room(a, c.total, why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    char* work = static_cast<char*>(a->workspace);
    with_types(a->dtype, a->out_dtype, [&](auto e, auto r) {
        using E = decltype(e);
        using R = decltype(r);
        E* own = c.has_dp ? reinterpret_cast<E*>(work + c.dp_at) : nullptr;
        if (own || a->dbias) {
            SlopeParams<E, R> s{};
            s.dout = static_cast<const R*>(a->dout.data); s.dout_rows = rows_of(a, a->dout);
            s.pre = a->act == CRAFTAX_ACT_NONE ? nullptr : static_cast<const E*>(a->pre.data); s.pre_rows = rows_of(a, a->pre);
            s.dp = own; s.dp_row = c.dp_row; s.act = (int)a->act;
            s.part = a->dbias ? reinterpret_cast<float*>(work + c.sums_at) : nullptr;
            s.m = (uint32_t)c.rows; s.n = a->outputs;
            hipLaunchKernelGGL((k_slope<E, R>), dim3(c.slope_x, c.slope_y), dim3(256), 0, st, s);
            if (a->dbias) sum_rows(s.part, (int)c.slope_y, a->outputs, PutBias{a->dbias}, st);
        }
        const Operand<E> dp = own ? Operand<E>{own, dense_rows(c.dp_row)} : Operand<E>{static_cast<const E*>(a->dout.data), rows_of(a, a->dout)};
        float* part = reinterpret_cast<float*>(work + c.part_at);
        if (a->dx.data) {
            ProductParams<E, E> p{};
            const E* weight = static_cast<const E*>(a->weight);
            int64_t ld = a->weight_column;
            if (c.turn) {
                E* turned = reinterpret_cast<E*>(work + c.turned_at);
                turn<E>(weight, a->weight_row, turned, c.turned_row, a->outputs, a->inputs, st);
                weight = turned;
                ld = c.turned_row;
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
                p.p = {static_cast<const E*>(a->x.data), rows_of(a, a->x)};
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
