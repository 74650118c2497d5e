// Between two blocks: norm after the block, gate, scale, residual, norm before the next block, in one
// pass over a row, and the backward pass.
//
//   out = residual + act(gate) scale post_weight y / rms(y),  u = pre_weight out / rms(out),  rms(v) = sqrt(mean(v v) + eps)
//
// and backward, with g = dL/dout + (pre_weight du)' through the second norm, where the gradient through a norm of v is
// (h - unit mean(h unit)) / rms(v) for h = weight times the gradient of its result and unit = v / rms(v).
//
// Bound by memory: a row is read once, kept in registers, and written once (forward 3 in, 2 out with a gate;
// backward 5 in, 3 out).  The backward pass computes the two roots again from the row, which is there
// anyway, so nothing is saved between the passes.  A row belongs to W wavefronts, as few as hold it with 16
// values per lane (backward 8); with one wavefront every sum stays inside it, with more the sums meet in LDS.
// Blocks go on to further rows with the weights, and in the backward pass their gradients, in registers.
// 262,144 rows of 512 values in bfloat16 with a gate: forward 250 us, 5.3 TB/s; backward 500 us, 4.3 TB/s, with vector issue
// at about half beside it (131,072 rows in float32: 258 us, 5.2 TB/s, and 418, 5.1).  Beyond 4,096 values the backward pass has no room for a
// row's eight arrays: 128 to 276 bytes of scratch a lane (16,384 rows of 8,192 bfloat16: 730 us, 2.9 TB/s).
#include "memory_api.hpp"
#include "memory_common.hpp"

#include <type_traits>

namespace mem {

template <typename E, typename R> struct NormParams {
    const float *post_weight, *scale, *pre_weight;
    Seq<const E> y, gate, du;
    Seq<const R> residual, dout;
    Seq<E> u, dy, dgate;
    Seq<R> out, dresidual;
    float* part;               // backward: [blocks][3][channels]
    uint32_t rows, n;
    int channels, gate_act;
    float eps;
};

// sum over the W wavefronts of a row, in every lane; slots: W floats of LDS for this row and this sum
template <int W>
__device__ __forceinline__ float row_sum(float v, float* slots)
{
    v = wave_sum(v);
    if constexpr (W > 1) {
        const int lane = threadIdx.x & (WAVE - 1), wave = (threadIdx.x / WAVE) % W;
        if (lane == 0) slots[wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) v += slots[k];
    }
    return v;
}

// 1 / sqrt(v), also of a subnormal number, as with a tiny eps: the instruction alone takes one for 0
__device__ __forceinline__ float inverse_root(float v)
{
    const bool tiny = v < 0x1p-126f;
    const float root = __builtin_amdgcn_rsqf(tiny ? v * 0x1p24f : v);
    return tiny ? root * 0x1p12f : root;
}

// act(gate) and its derivative; written as selections, so that no branch stands between the elements of a row
__device__ __forceinline__ float gate_value(float g, int act)
{
    const float s = sigmoid(g), both = g * s;
    const float v = act == CRAFTAX_GATE_SILU ? both : s;
    return act == CRAFTAX_GATE_LINEAR ? g : v;
}
// FULL: the registers are all taken.  The exponential is not kept beside the sigmoid through the sums of the row then, and what that leaves of 1 is a sigmoid,
// too (16,384 rows of 8,192 bfloat16 values 733 us, of 6,000 float16 values 641; with the exponential kept 829 and 819.  65,536 rows of 1,000: 234, and 233).
template <bool FULL> __device__ __forceinline__ float gate_slope(float g, int act)
{
    const float e = exp2_fast(-g * LOG2E), s = __builtin_amdgcn_rcpf(1.0f + e), t = FULL ? sigmoid(-g) : rest_of(s, e), of_sigmoid = s * t, of_silu = s * __builtin_fmaf(g, t, 1.0f);
    const float v = act == CRAFTAX_GATE_SILU ? of_silu : of_sigmoid;
    return act == CRAFTAX_GATE_LINEAR ? 1.0f : v;
}

// What is left of g without its part along the unit row, g - unit * mean(g * unit).  The mean of unit * unit is
// 1 - eps * root * root, so in a row of one value only eps * root * root * g is left, which the difference of the two
// terms would not show in 32 bits.
template <int W, typename P>
__device__ __forceinline__ float off_axis(const P& p, float g, float unit, float along, float root)
{
    if (W == 1 && p.channels == 1) return p.eps * root * root * g;
    return __builtin_fmaf(-unit, along, g);
}

template <int W> struct RowBlock {
    static constexpr int THREADS = W * WAVE > 256 ? W * WAVE : 256;
    static constexpr int ROWS = THREADS / (W * WAVE);      // rows a block works on at once
};

// How rows fit the lanes' chunks of V values.  WHOLE: exactly.  TAIL: a chunk that passes the end of the row is moved back to
// end with it: its first `old` values are another lane's too (those of a lane with nothing left: all V).  They are computed
// and stored like the other lane's, bit for bit, and only left out of the sums.  EVEN: the same where V divides the row, so that
// `old` is 0 or V and a chunk is left out by one selection instead of V (backward of 131,072 rows of 400 bfloat16 213 us, 220 as TAIL, of
// 1,000 487 and 504).  SHORT: rows of fewer than V values are read and written value by value, by one lane.
enum Fit { WHOLE, EVEN, TAIL, SHORT };
template <int CHUNKS, int V, Fit FIT> struct RowPlace {
    int at[CHUNKS], old[CHUNKS], channels;
    __device__ __forceinline__ RowPlace(int n, int side, int width) : channels(n)
    {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int first = (c * width + side) * V, last = FIT == SHORT ? 0 : n - V;
            at[c] = FIT == WHOLE || first <= last ? first : last;
            const int gone = first - at[c];
            old[c] = FIT == WHOLE ? 0 : (gone < V ? gone : V);
        }
    }
    __device__ __forceinline__ bool mine(int c, int j) const
    {
        if (FIT == WHOLE || FIT == EVEN) return FIT == WHOLE || old[c] == 0;
        return j >= old[c] && (FIT == TAIL || j < channels);
    }
    // s with value j's product added where it counts in this lane; values are added in order, and `before` is the sum in front of a chunk.
    // A selection, not a product with 0: the values that do not count may be infinite.  Of several chunks the first half is filled
    // in every row (see with_row) and needs none.
    __device__ __forceinline__ float add(int c, int j, float a, float b, float s, float& before) const
    {
        const float sum = __builtin_fmaf(a, b, s);
        if (FIT == WHOLE || c < CHUNKS / 2) return sum;
        if (FIT != EVEN) return mine(c, j) ? sum : s;
        if (j == 0) before = s;
        return j < V - 1 || old[c] == 0 ? sum : before;
    }
};

template <typename P, int CHUNKS, int V, Fit FIT>
__device__ __forceinline__ void fetch(const RowPlace<CHUNKS, V, FIT>& w, const P* p, Pack<P, V> (&q)[CHUNKS])
{
    if (FIT != SHORT) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) q[c] = *reinterpret_cast<const Pack<P, V>*>(p + w.at[c]);
    } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) q[c].v[j] = p[j < w.channels ? j : 0];
    }
}
template <typename P, int CHUNKS, int V>
__device__ __forceinline__ void expand(const Pack<P, V> (&q)[CHUNKS], float (&v)[CHUNKS][V])
{
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) v[c][j] = Elem<P>::up(q[c].v[j]);
}
template <typename P, int CHUNKS, int V, Fit FIT>
__device__ __forceinline__ void put(const RowPlace<CHUNKS, V, FIT>& w, P* p, const float (&v)[CHUNKS][V])
{
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        if (FIT != SHORT) {
            Pack<P, V> q;
#pragma unroll
            for (int j = 0; j < V; ++j) q.v[j] = Elem<P>::down(v[c][j]);
            if (FIT == WHOLE || w.old[c] < V) *reinterpret_cast<Pack<P, V>*>(p + w.at[c]) = q;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (w.mine(c, j)) p[j] = Elem<P>::down(v[c][j]);
        }
    }
}
// sums over rows: a value belongs to one lane
template <int CHUNKS, int V, Fit FIT>
__device__ __forceinline__ void put_mine(const RowPlace<CHUNKS, V, FIT>& w, float* p, const float (&v)[CHUNKS][V])
{
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (w.mine(c, j)) p[w.at[c] + j] = v[c][j];
}
template <int CHUNKS, int V, Fit FIT>
__device__ __forceinline__ void load_weight(const RowPlace<CHUNKS, V, FIT>& w, const float* p, float (&v)[CHUNKS][V])
{
    Pack<float, V> q[CHUNKS];
    if (p) {
        fetch(w, p, q);
        expand(q, v);
        return;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) v[c][j] = 1.0f;
}
// the values have arrived
template <typename P, int CHUNKS, int V> __device__ __forceinline__ void pin(Pack<P, V> (&q)[CHUNKS])
{
    uint32_t words[sizeof(q) / 4];
    __builtin_memcpy(words, q, sizeof(q));
    pin(words);
    __builtin_memcpy(q, words, sizeof(q));
}

// Wavefronts per SIMD at most: rows of 16 values per lane that do not fill the lanes are faster with two than with the three that
// their registers leave room for (131,072 rows of 1,000 bfloat16 264 us, 270 with three; 40,000 of 3,001 float16 285 and 290).
template <typename E, int CHUNKS, Fit FIT> constexpr int norm_waves() { return FIT != WHOLE && CHUNKS * 16 / sizeof(E) > 8 ? 2 : 8; }

template <typename E, typename R, int W, int CHUNKS, Fit FIT>
__global__ __launch_bounds__(RowBlock<W>::THREADS) __attribute__((amdgpu_waves_per_eu(2, norm_waves<E, CHUNKS, FIT>()))) void k_norm(const NormParams<E, R> p)
{
    constexpr int V = 16 / sizeof(E), ROWS = RowBlock<W>::ROWS;
    __shared__ float slots[2][ROWS][W];
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x / (W * WAVE));
    const RowPlace<CHUNKS, V, FIT> w(p.channels, threadIdx.x % (W * WAVE), W * WAVE);
    const bool gated = p.gate.data != nullptr;
    Pack<E, V> raw_y[CHUNKS], raw_g[CHUNKS];
    Pack<R, V> raw_r[CHUNKS];
    auto load = [&](uint32_t row) {
        const int t = (int)(row / p.n), i = (int)(row % p.n);
        fetch(w, p.y.at(t, i), raw_y);
        fetch(w, p.residual.at(t, i), raw_r);
        if (gated) fetch(w, p.gate.at(t, i), raw_g);
    };
    const uint32_t first = blockIdx.x * ROWS + which, stride = gridDim.x * ROWS, last = p.rows - 1;
    load(first < last ? first : last);
    float w1[CHUNKS][V], scale[CHUNKS][V], w2[CHUNKS][V];
    load_weight(w, p.post_weight, w1);
    load_weight(w, p.scale, scale);
    load_weight(w, p.pre_weight, w2);
    const float mean = 1.0f / (float)p.channels;
    for (uint32_t base = blockIdx.x * ROWS; base < p.rows; base += stride) {
        const uint32_t row = base + which;
        float y[CHUNKS][V], r[CHUNKS][V], g[CHUNKS][V] = {};
        expand(raw_y, y);
        expand(raw_r, r);
        if (gated) expand(raw_g, g);
        if (base + stride < p.rows) load(row + stride < last ? row + stride : last);
        float root = 1.0f;
        if (p.post_weight) {
            float s = 0.0f, before;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) s = w.add(c, j, y[c][j], y[c][j], s, before);
            root = inverse_root(__builtin_fmaf(row_sum<W>(s, slots[0][which]), mean, p.eps));
        }
        float s = 0.0f, before;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float act = gate_value(g[c][j], p.gate_act);
                r[c][j] = __builtin_fmaf(y[c][j] * root * w1[c][j] * scale[c][j], gated ? act : 1.0f, r[c][j]);
                s = w.add(c, j, r[c][j], r[c][j], s, before);
            }
        root = inverse_root(__builtin_fmaf(row_sum<W>(s, slots[1][which]), mean, p.eps));
        // the next row's values, waited for in front of the stores: behind them the wait would be for those too
        pin(raw_y);
        pin(raw_r);
        if (gated) pin(raw_g);
        if (row < p.rows) {
            const int t = (int)(row / p.n), i = (int)(row % p.n);
            put(w, p.out.at(t, i), r);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) r[c][j] = r[c][j] * root * w2[c][j];
            put(w, p.u.at(t, i), r);
        }
        if (W > 1) __syncthreads();
    }
}

template <typename E, typename R, int W, int CHUNKS, Fit FIT>
__global__ __launch_bounds__(RowBlock<W>::THREADS) void k_norm_backward(const NormParams<E, R> p)
{
    constexpr int V = 16 / sizeof(E), ROWS = RowBlock<W>::ROWS, THREADS = RowBlock<W>::THREADS;
    // Rows that are read ahead of the one that is computed, as many as the registers hold: two of 16-bit values (two
    // wavefronts per SIMD with one row each under way are 10 MB, what the memory's latency takes at its rate), one of floats,
    // none with 16 values per lane.
    constexpr int AHEAD = CHUNKS * V > 8 ? 0 : sizeof(E) == 2 ? 2 : 1, SLOTS = AHEAD ? AHEAD : 1;
    __shared__ float slots[4][ROWS][W];
    __shared__ float sums[ROWS > 1 ? THREADS * CHUNKS * V : 1];
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x / (W * WAVE)), side = threadIdx.x % (W * WAVE);
    const RowPlace<CHUNKS, V, FIT> w(p.channels, side, W * WAVE);
    const bool gated = p.gate.data != nullptr, through = p.dout.data != nullptr;
    struct Raw {
        Pack<E, V> y[CHUNKS], g[CHUNKS], du[CHUNKS];
        Pack<R, V> r[CHUNKS], dr[CHUNKS];
    } raw[SLOTS];
    const uint32_t stride = gridDim.x * ROWS, last = p.rows - 1;
    auto load = [&](Raw& q, uint32_t base) {
        const uint32_t row = base + which < last ? base + which : last;
        const int t = (int)(row / p.n), i = (int)(row % p.n);
        fetch(w, p.y.at(t, i), q.y);
        fetch(w, p.residual.at(t, i), q.r);
        if (gated) fetch(w, p.gate.at(t, i), q.g);
        fetch(w, p.du.at(t, i), q.du);
        if (through) fetch(w, p.dout.at(t, i), q.dr);
    };
    // the values have arrived: waited for in front of stores, since behind them the wait would be for those too
    auto arrive = [&](Raw& q) {
        pin(q.y);
        pin(q.r);
        if (gated) pin(q.g);
        pin(q.du);
        if (through) pin(q.dr);
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) load(raw[k], blockIdx.x * ROWS + k * stride < p.rows ? blockIdx.x * ROWS + k * stride : last);
    float w1[CHUNKS][V], scale[CHUNKS][V], w2[CHUNKS][V];
    load_weight(w, p.post_weight, w1);
    load_weight(w, p.scale, scale);
    load_weight(w, p.pre_weight, w2);
    float d1[CHUNKS][V] = {}, ds[CHUNKS][V] = {}, d2[CHUNKS][V] = {};
    const float mean = 1.0f / (float)p.channels;
    auto one = [&](uint32_t base, Raw& mine, Raw& next) {
        const uint32_t row = base + which;
        // Without a row of its own, one of two wavefronts of a row goes along with the last one, for the barriers: that adds nothing to
        // the weights' gradients, be it infinite.
        const bool on = W != 2 || row < p.rows;
        auto add = [&](float a, float b, float& sum) {
            const float with = __builtin_fmaf(a, b, sum);
            sum = on ? with : sum;
        };
        if (AHEAD == 0) load(mine, base);
        float y[CHUNKS][V], r[CHUNKS][V], g[CHUNKS][V] = {}, du[CHUNKS][V], dr[CHUNKS][V] = {};
        expand(mine.y, y);
        expand(mine.r, r);
        if (gated) expand(mine.g, g);
        expand(mine.du, du);
        if (through) expand(mine.dr, dr);
        if (AHEAD > 0 && base + AHEAD * stride < p.rows) load(mine, base + AHEAD * stride);
        float root_y = 1.0f;
        if (p.post_weight) {
            float s = 0.0f, before;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) s = w.add(c, j, y[c][j], y[c][j], s, before);
            root_y = inverse_root(__builtin_fmaf(row_sum<W>(s, slots[0][which]), mean, p.eps));
        }
        // out again, its root, and the sum over the row of (du w2) (out root)
        float s = 0.0f, m = 0.0f, before;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[c][j] *= root_y;                                   // from here on without its scale
                const float act = gate_value(g[c][j], p.gate_act);
                r[c][j] = __builtin_fmaf(y[c][j] * w1[c][j] * scale[c][j], gated ? act : 1.0f, r[c][j]);
                s = w.add(c, j, r[c][j], r[c][j], s, before);
            }
        const float root = inverse_root(__builtin_fmaf(row_sum<W>(s, slots[1][which]), mean, p.eps));
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                r[c][j] *= root;
                add(du[c][j], r[c][j], d2[c][j]);
                du[c][j] *= w2[c][j];
                m = w.add(c, j, du[c][j], r[c][j], m, before);
            }
        m = row_sum<W>(m, slots[2][which]) * mean;
        float q = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = __builtin_fmaf(root, off_axis<W>(p, du[c][j], r[c][j], m, root), dr[c][j]);
                dr[c][j] = d;
                const float value = gate_value(g[c][j], p.gate_act), act = gated ? value : 1.0f;
                const float v = y[c][j] * w1[c][j], dv = d * scale[c][j] * act;
                add(d * v, act, ds[c][j]);
                g[c][j] = d * v * scale[c][j] * gate_slope<(CHUNKS * V > 8)>(g[c][j], p.gate_act);
                add(dv, y[c][j], d1[c][j]);
                du[c][j] = dv * w1[c][j];
                q = w.add(c, j, du[c][j], y[c][j], q, before);
            }
        if (p.post_weight) {
            q = row_sum<W>(q, slots[3][which]) * mean;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) du[c][j] = root_y * off_axis<W>(p, du[c][j], y[c][j], q, root_y);
        }
        if (AHEAD > 0) arrive(next);
        if (row < p.rows) {
            const int t = (int)(row / p.n), i = (int)(row % p.n);
            put(w, p.dresidual.at(t, i), dr);
            if (gated) put(w, p.dgate.at(t, i), g);
            put(w, p.dy.at(t, i), du);
        }
        if (W > 1) __syncthreads();
    };
    for (uint32_t base = blockIdx.x * ROWS; base < p.rows; base += SLOTS * stride) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (base + k * stride + (W == 1 ? which : 0) < p.rows) one(base + k * stride, raw[k], raw[(k + 1) % SLOTS]);
    }
    if (p.part == nullptr) return;
    // one partial row per block and weight; the rows that a block works on at once are added up in LDS
    auto sum_up = [&](int weight, const float (&v)[CHUNKS][V]) {
        float* out = p.part + ((int64_t)blockIdx.x * 3 + weight) * p.channels;
        if constexpr (ROWS == 1) {
            put_mine(w, out, v);
        } else {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) sums[(c * V + j) * THREADS + threadIdx.x] = v[c][j];
            __syncthreads();
            if (which == 0) {
                float total[CHUNKS][V];
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        total[c][j] = 0.0f;
#pragma unroll
                        for (int k = 0; k < ROWS; ++k) total[c][j] += sums[(c * V + j) * THREADS + k * (W * WAVE) + side];
                    }
                put_mine(w, out, total);
            }
        }
    };
    sum_up(0, d1);
    sum_up(1, ds);
    sum_up(2, d2);
}

struct PutNorm {
    float* out[3];
    int channels;
    __device__ void operator()(int64_t column, float v) const
    {
        const int which = (int)(column / channels);
        float* p = which == 0 ? out[0] : which == 1 ? out[1] : out[2];
        if (p) p[column - (int64_t)which * channels] = v;
    }
};

namespace host {

constexpr int NORM_CHANNELS = 8192;
// Wavefronts per SIMD that are launched at most.  Backward all are there at once.  Forward a SIMD holds five to eight of the kernels with up to
// eight values per lane, and two or three of those with sixteen, so that these blocks follow one another.
constexpr int NORM_WAVES = 6, NORM_BACK_WAVES = 2;

static int norm_check(const craftax_norm_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->residual_dtype != a->dtype && a->residual_dtype != CRAFTAX_F32) return refuse(CRAFTAX_E_CONFIG, "residual_dtype must be dtype or CRAFTAX_F32", why);
    if (a->gate_act > CRAFTAX_GATE_LINEAR) return refuse(CRAFTAX_E_CONFIG, "unknown gate_act", why);
    if (!(a->eps > 0.0f)) return refuse(CRAFTAX_E_CONFIG, "eps must be positive", why);
    if (a->steps < 1 || a->n < 1) return refuse(CRAFTAX_E_COUNT, "steps and n must be positive", why);
    if ((int64_t)a->steps * a->n >= (int64_t)1 << 31) return refuse(CRAFTAX_E_COUNT, "steps * n must be below 2^31", why);
    if (a->channels < 1 || a->channels > NORM_CHANNELS) return refuse(CRAFTAX_E_COUNT, "channels must be 1..8192", why);
    if (!a->y.data || !a->residual.data) return refuse(CRAFTAX_E_NULL, "y or residual is NULL", why);
    const size_t e = elem_bytes(a->dtype), r = elem_bytes(a->residual_dtype);
    if (!aligned(a->y.data, e) || !aligned(a->gate.data, e) || !aligned(a->residual.data, r) || !aligned(a->post_weight, 4) ||
        !aligned(a->scale, 4) || !aligned(a->pre_weight, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    if (!backward) {
        if (!a->out.data || !a->u.data) return refuse(CRAFTAX_E_NULL, "out or u is NULL", why);
        if (!aligned(a->out.data, r) || !aligned(a->u.data, e)) return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
        return CRAFTAX_OK;
    }
    if (!a->du.data || !a->dy.data || !a->dresidual.data) return refuse(CRAFTAX_E_NULL, "du, dy or dresidual is NULL", why);
    if (a->gate.data && !a->dgate.data) return refuse(CRAFTAX_E_NULL, "dgate is NULL", why);
    if (!aligned(a->du.data, e) || !aligned(a->dy.data, e) || !aligned(a->dgate.data, e) || !aligned(a->dout.data, r) || !aligned(a->dresidual.data, r) ||
        !aligned(a->dpost_weight, 4) || !aligned(a->dscale, 4) || !aligned(a->dpre_weight, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    return CRAFTAX_OK;
}

template <typename E, typename R> static NormParams<E, R> norm_params(const craftax_norm_args* a)
{
    NormParams<E, R> p{};
    p.post_weight = a->post_weight; p.scale = a->scale; p.pre_weight = a->pre_weight;
    p.y = seq_in<E>(a->y); p.gate = seq_in<E>(a->gate); p.du = seq_in<E>(a->du);
    p.residual = seq_in<R>(a->residual); p.dout = seq_in<R>(a->dout);
    p.u = seq<E>(a->u); p.dy = seq<E>(a->dy); p.dgate = seq<E>(a->dgate);
    p.out = seq<R>(a->out); p.dresidual = seq<R>(a->dresidual);
    p.rows = (uint32_t)((int64_t)a->steps * a->n); p.n = (uint32_t)a->n; p.channels = a->channels; p.gate_act = (int)a->gate_act; p.eps = a->eps;
    return p;
}

// Wavefronts per row: as few (1, 2, 4, 8) as hold it with 16 values per lane, or with 8 in the backward pass, which holds five
// rows and three gradients (beyond 4,096 values 16 there too).
static int row_waves(int channels, bool backward)
{
    int w = 1;
    while (w < 8 && w * WAVE * (backward ? 8 : 16) < channels) w *= 2;
    return w;
}
static int row_threads(int w) { return w * WAVE > 256 ? w * WAVE : 256; }

// Blocks: all that the chip holds at once, then on to further rows.
static unsigned row_blocks(const craftax_norm_args* a, bool backward)
{
    const int waves_per_simd = backward ? NORM_BACK_WAVES : NORM_WAVES;
    const int w = row_waves(a->channels, backward), threads = row_threads(w);
    const int64_t need = ceil_div((int64_t)a->steps * a->n, threads / (w * WAVE));
    const int64_t most = (int64_t)CHIP_SIMDS * waves_per_simd * WAVE / threads;
    return (unsigned)(need < most ? need : most);
}

// calls f with the element types, the wavefronts per row, the chunks per lane and how they fit as constants
template <bool BACKWARD, typename F> static void with_row(const craftax_norm_args* a, F&& f)
{
    const int w = row_waves(a->channels, BACKWARD);
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        constexpr int V = 16 / sizeof(E);
        auto chunks = [&](auto r, auto wc) {
            constexpr int W = decltype(wc)::value;
            auto whole = [&](auto count) {
                constexpr int C = decltype(count)::value;
                if (a->channels == W * WAVE * V * C) f(e, r, wc, count, std::integral_constant<Fit, WHOLE>{});
                else if (a->channels % V == 0) f(e, r, wc, count, std::integral_constant<Fit, EVEN>{});
                else if (a->channels >= V) f(e, r, wc, count, std::integral_constant<Fit, TAIL>{});
                else if constexpr (W == 1 && C == 1) f(e, r, wc, count, std::integral_constant<Fit, SHORT>{});
            };
            // More than one chunk only where half as many would not hold the row: the first half is filled.
            constexpr int EIGHT = 8 / V;          // chunks of eight values
            // one wavefront takes a row of any length that fits it; more of them are taken for no fewer values per lane than half of
            // what they hold (see row_waves)
            if constexpr (W == 1) {
                if (V < 8 && a->channels <= WAVE * V) return whole(std::integral_constant<int, 1>{});
            }
            if constexpr (W == 1 || BACKWARD) {
                if (a->channels <= W * WAVE * 8) return whole(std::integral_constant<int, EIGHT>{});
            }
            if constexpr (!BACKWARD || W == 8) whole(std::integral_constant<int, 2 * EIGHT>{});
        };
        auto waves = [&](auto r) {
            if (w == 1) chunks(r, std::integral_constant<int, 1>{});
            else if (w == 2) chunks(r, std::integral_constant<int, 2>{});
            else if (w == 4) chunks(r, std::integral_constant<int, 4>{});
            else chunks(r, std::integral_constant<int, 8>{});
        };
        if (a->residual_dtype == CRAFTAX_F32) waves(float{});
        else waves(E{});
    });
}

int norm(const craftax_norm_args* a, void* stream, const char** why)
{
    if (int rc = norm_check(a, false, why)) return rc;
    with_row<false>(a, [&](auto e, auto r, auto w, auto chunks, auto fit) {
        using E = decltype(e);
        using R = decltype(r);
        constexpr int W = decltype(w)::value, C = decltype(chunks)::value;
        hipLaunchKernelGGL((k_norm<E, R, W, C, decltype(fit)::value>), dim3(row_blocks(a, false)), dim3(RowBlock<W>::THREADS), 0, (hipStream_t)stream,
                           (norm_params<E, R>(a)));
    });
    return launched(why);
}

size_t norm_workspace_bytes(const craftax_norm_args* a)
{
    if (!a || a->steps < 1 || a->n < 1 || a->channels < 1 || a->channels > NORM_CHANNELS) return 0;
    if (!a->dpost_weight && !a->dscale && !a->dpre_weight) return 0;
    return round256((size_t)row_blocks(a, true) * 3 * a->channels * sizeof(float));
}

int norm_backward(const craftax_norm_args* a, void* stream, const char** why)
{
    if (int rc = norm_check(a, true, why)) return rc;
    const size_t need = norm_workspace_bytes(a);
    if (need && !a->workspace) return refuse(CRAFTAX_E_NULL, "workspace is NULL", why);
    if (need && !aligned(a->workspace, 256)) return refuse(CRAFTAX_E_ALIGN, "workspace must be 256-byte aligned", why);
    if (a->workspace_bytes < need) return refuse(CRAFTAX_E_COUNT, "workspace smaller than craftax_residual_norm_workspace_bytes", why);
    const unsigned blocks = row_blocks(a, true);
    const hipStream_t st = (hipStream_t)stream;
    with_row<true>(a, [&](auto e, auto r, auto w, auto chunks, auto fit) {
        using E = decltype(e);
        using R = decltype(r);
        constexpr int W = decltype(w)::value, C = decltype(chunks)::value;
        NormParams<E, R> p = norm_params<E, R>(a);
        p.part = need ? static_cast<float*>(a->workspace) : nullptr;
        hipLaunchKernelGGL((k_norm_backward<E, R, W, C, decltype(fit)::value>), dim3(blocks), dim3(RowBlock<W>::THREADS), 0, st, p);
    });
    if (int rc = launched(why)) return rc;
    if (need)
        sum_rows(static_cast<const float*>(a->workspace), (int)blocks, (int64_t)3 * a->channels,
                 PutNorm{{a->post_weight ? a->dpost_weight : nullptr, a->dscale, a->dpre_weight}, a->channels}, st);
    return launched(why);
}

}  // namespace host
}  // namespace mem
