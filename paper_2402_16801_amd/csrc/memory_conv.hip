// Short causal convolution of every channel with an activation: whole sequences, single tokens
// (a sequence of one step) and the backward pass.
//
// Bound by memory: 2 (forward) or 3 (backward) activations move per step and channel against about 12
// and 30 instructions.  A thread owns V neighbouring channels of one environment (16 bytes forward)
// and walks along a stretch of steps with the last taps - 1 inputs in registers, so an input is read
// once but for the taps - 1 in front of a stretch.  Stretches exist only to fill the chip.
#include "memory_api.hpp"
#include "memory_common.hpp"

namespace mem {

constexpr int CONV_THREADS = 256;

template <typename E> struct ConvParams {
    const float *weight, *bias;
    Seq<const uint8_t> first;
    const int32_t* lengths;
    Seq<const E> x, dy;
    Seq<E> y, dx;
    const E *state_in, *dstate_out;
    E *state_out, *dstate_in;
    float* part;
    int steps, n, channels, stretch, vectors, silu;
    int lanes_log2;      // backward: threads of a block side by side on channels
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int steps, int i)
{
    if (lengths == nullptr) return steps;
    const int l = lengths[i];
    return l < 0 ? 0 : (l > steps ? steps : l);
}

// The last K - 1 inputs before step t as they count at step t - 1, for V channels from `c` on.
template <typename E, int K, int V>
__device__ __forceinline__ void window_before(const ConvParams<E>& p, int t, int i, int c, int count, float (&win)[K - 1][V])
{
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        const int s = t - (K - 1) + k;
        if (s >= 0) {
            if (p.first.data && *p.first.at(s, i)) {
#pragma unroll
                for (int m = 0; m < K - 1; ++m)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (m < k) win[m][j] = 0.0f;
            }
            load_row<E, V>(p.x.at(s, i) + c, count, win[k]);
        } else if (p.state_in) {
            load_row<E, V>(p.state_in + ((int64_t)i * (K - 1) + (s + K - 1)) * p.channels + c, count, win[k]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) win[k][j] = 0.0f;
        }
    }
}

template <int K, int V>
__device__ __forceinline__ void push(float (&win)[K - 1][V], const float (&x)[V])
{
#pragma unroll
    for (int k = 0; k + 1 < K - 1; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) win[k][j] = win[k + 1][j];
#pragma unroll
    for (int j = 0; j < V; ++j) win[K - 2][j] = x[j];
}

template <int K, int V>
__device__ __forceinline__ void clear(float (&win)[K - 1][V])
{
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) win[k][j] = 0.0f;
}

template <int K, int V> struct Taps {
    float w[K][V], bias[V];
    __device__ __forceinline__ void load(const float* weight, const float* b, int c, int count)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int d = c + (j < count ? j : 0);
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][j] = weight[(int64_t)d * K + k];
            bias[j] = b ? b[d] : 0.0f;
        }
    }
    __device__ __forceinline__ float sum(const float (&win)[K - 1][V], float x, int j) const
    {
        float s = bias[j];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) s = __builtin_fmaf(w[k][j], win[k][j], s);
        return __builtin_fmaf(w[K - 1][j], x, s);
    }
};

template <typename E, int K, int V>
__global__ __launch_bounds__(CONV_THREADS) void k_conv(const ConvParams<E> p)
{
    const uint32_t at = blockIdx.x * CONV_THREADS + threadIdx.x;
    const int i = (int)(at / (uint32_t)p.vectors);
    if (i >= p.n) return;
    const int c = (int)(at % (uint32_t)p.vectors) * V;
    const int count = p.channels - c < V ? p.channels - c : V;
    const int t0 = (int)blockIdx.y * p.stretch;
    const int t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
    const int length = length_of(p.lengths, p.steps, i);
    const int live = t1 < length ? t1 : length;       // steps of this stretch that count end here
    Taps<K, V> taps;
    taps.load(p.weight, p.bias, c, count);
    float win[K - 1][V];
    if (t0 < live || t0 == 0) window_before<E, K, V>(p, t0, i, c, count, win);
    constexpr int AHEAD = 4;
    int t = t0;
    for (; t < live; t += AHEAD) {
        float x[AHEAD][V];
        uint32_t starts = 0;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int s = t + a < live ? t + a : live - 1;
            load_row<E, V>(p.x.at(s, i) + c, count, x[a]);
            if (p.first.data) starts |= (uint32_t)(*p.first.at(s, i) != 0) << a;
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (t + a >= live) break;
            if (starts >> a & 1u) clear<K, V>(win);
            float out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = taps.sum(win, x[a][j], j);
                out[j] = p.silu ? v * sigmoid(v) : v;
            }
            push<K, V>(win, x[a]);
            store_row<E, V>(p.y.at(t + a, i) + c, count, out);
        }
    }
    float none[V];
#pragma unroll
    for (int j = 0; j < V; ++j) none[j] = 0.0f;
    for (t = t0 > live ? t0 : live; t < t1; ++t) store_row<E, V>(p.y.at(t, i) + c, count, none);
    // The thread of the first stretch, which alone reads the state, writes the new one too, so that it can
    // be the same memory.  With one stretch the window is what is wanted.
    if (p.state_out && blockIdx.y == 0) {
        if (live < length) window_before<E, K, V>(p, length, i, c, count, win);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store_row<E, V>(p.state_out + ((int64_t)i * (K - 1) + k) * p.channels + c, count, win[k]);
    }
}

// Backward.  With p the sum before the activation, dp = dy * act'(p):  an input s gets weight[K - 1 - j] * dp of
// step s + j for j = 0 .. K - 1 as far as no episode begins in (s, s + j], and the weight gets the products.  Walking
// forward, `due` holds the gradients of the last K - 1 inputs, of which the oldest is complete with every
// step; a stretch goes K - 1 steps beyond its end for the inputs at its end, without counting those steps
// for the weight.  A block sums its weight gradients in LDS and writes one partial row; rows are added in a
// fixed order by a second kernel.
template <typename E, int K, int V>
__global__ __launch_bounds__(CONV_THREADS) void k_conv_backward(const ConvParams<E> p)
{
    constexpr int COLS = V * (K + 1);
    __shared__ float sums[CONV_THREADS * COLS];
    const int lanes = 1 << p.lanes_log2, side = threadIdx.x >> p.lanes_log2, rows = CONV_THREADS >> p.lanes_log2;
    const int vec = (int)blockIdx.x * lanes + (threadIdx.x & (lanes - 1));
    const int c = vec * V;
    const int count = p.channels - c < V ? p.channels - c : V;
    const int stretches = (p.steps + p.stretch - 1) / p.stretch;
    float dw[K][V], db[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        db[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][j] = 0.0f;
    }
    if (count > 0) {
        Taps<K, V> taps;
        taps.load(p.weight, p.bias, c, count);
        const int64_t items = (int64_t)p.n * stretches;
        for (int64_t item = (int64_t)blockIdx.y * rows + side; item < items; item += (int64_t)gridDim.y * rows) {
            const int i = (int)(item % p.n), t0 = (int)(item / p.n) * p.stretch;
            const int t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
            const int length = length_of(p.lengths, p.steps, i);
            const int live = t1 < length ? t1 : length;
            const int end = length - t1 < K - 1 ? length : t1 + (K - 1);     // steps walked: up to here
            float none[V];
#pragma unroll
            for (int j = 0; j < V; ++j) none[j] = 0.0f;
            for (int t = t0 > live ? t0 : live; t < t1; ++t) store_row<E, V>(p.dx.at(t, i) + c, count, none);
            if (t0 >= live && t0 > 0) continue;
            float win[K - 1][V], due[K - 1][V];
            window_before<E, K, V>(p, t0, i, c, count, win);
            clear<K, V>(due);
            // steps since the last begin of an episode, as far as the window reaches back
            int age = K - 1;
            if (p.first.data)
                for (int s = t0 - (K - 1) > 0 ? t0 - (K - 1) : 0; s < t0; ++s)
                    age = *p.first.at(s, i) ? 0 : (age < K - 1 ? age + 1 : K - 1);
            constexpr int AHEAD = 2;
            for (int t = t0; t < end; t += AHEAD) {
                float x[AHEAD][V], dy[AHEAD][V];
                uint32_t starts = 0;
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    const int s = t + a < end ? t + a : end - 1;
                    load_row<E, V>(p.x.at(s, i) + c, count, x[a]);
                    load_row<E, V>(p.dy.at(s, i) + c, count, dy[a]);
                    if (p.first.data) starts |= (uint32_t)(*p.first.at(s, i) != 0) << a;
                }
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    if (t + a >= end) break;
                    if (starts >> a & 1u) { clear<K, V>(win); age = 0; }
                    else if (age < K - 1) ++age;
                    const bool counts = t + a < t1;
                    float now[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float dp = dy[a][j];
                        if (p.silu) {
                            const float v = taps.sum(win, x[a][j], j), g = sigmoid(v);
                            dp *= g * __builtin_fmaf(v, 1.0f - g, 1.0f);
                        }
                        now[j] = taps.w[K - 1][j] * dp;
#pragma unroll
                        for (int k = 0; k < K - 1; ++k)
                            if (age >= K - 1 - k) due[k][j] = __builtin_fmaf(taps.w[k][j], dp, due[k][j]);
                        if (counts) {
                            db[j] += dp;
#pragma unroll
                            for (int k = 0; k < K - 1; ++k) dw[k][j] = __builtin_fmaf(dp, win[k][j], dw[k][j]);
                            dw[K - 1][j] = __builtin_fmaf(dp, x[a][j], dw[K - 1][j]);
                        }
                    }
                    // the oldest input, t + a - (K - 1), is complete
                    const int s = t + a - (K - 1);
                    if (s >= t0) store_row<E, V>(p.dx.at(s, i) + c, count, due[0]);
                    else if (s < 0 && p.dstate_in)
                        store_row<E, V>(p.dstate_in + ((int64_t)i * (K - 1) + (s + K - 1)) * p.channels + c, count, due[0]);
                    push<K, V>(win, x[a]);
                    push<K, V>(due, now);
                }
            }
            // What the walk left: the inputs end - (K - 1) .. end - 1.  At the end of the sequence they are also the new
            // state.
            if (end == length) {
#pragma unroll
                for (int k = 0; k < K - 1; ++k) {
                    const int s = length - (K - 1) + k;
                    if (p.dstate_out && age >= K - 2 - k) {
                        float add[V];
                        load_row<E, V>(p.dstate_out + ((int64_t)i * (K - 1) + k) * p.channels + c, count, add);
#pragma unroll
                        for (int j = 0; j < V; ++j) due[k][j] += add[j];
                    }
                    if (s >= t0 && s < t1) store_row<E, V>(p.dx.at(s, i) + c, count, due[k]);
                    else if (s < 0 && p.dstate_in)
                        store_row<E, V>(p.dstate_in + ((int64_t)i * (K - 1) + (s + K - 1)) * p.channels + c, count, due[k]);
                }
            }
        }
    }
    if (p.part == nullptr) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int k = 0; k < K; ++k) sums[(j * (K + 1) + k) * CONV_THREADS + threadIdx.x] = dw[k][j];
        sums[(j * (K + 1) + K) * CONV_THREADS + threadIdx.x] = db[j];
    }
    __syncthreads();
    // partial row: [K + 1][channels]; slot q = (value, lane)
    float* row = p.part + (int64_t)blockIdx.y * (K + 1) * p.channels;
    for (int q = threadIdx.x; q < COLS * lanes; q += CONV_THREADS) {
        const int lane = q & (lanes - 1), value = q >> p.lanes_log2, j = value / (K + 1), k = value % (K + 1);
        const int d = ((int)blockIdx.x * lanes + lane) * V + j;
        if (d >= p.channels) continue;
        float s = 0.0f;
        for (int r = 0; r < rows; ++r) s += sums[value * CONV_THREADS + (r << p.lanes_log2) + lane];
        row[(int64_t)k * p.channels + d] = s;
    }
}

// dweight[d][k] and dbias[d] from columns [K + 1][channels]
struct PutConv {
    float *dweight, *dbias;
    int channels, taps;
    __device__ void operator()(int64_t column, float v) const
    {
        const int k = (int)(column / channels), d = (int)(column % channels);
        if (k == taps) { if (dbias) dbias[d] = v; }
        else if (dweight) dweight[(int64_t)d * taps + k] = v;
    }
};

namespace host {

static int conv_check(const craftax_conv_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->taps < 2 || a->taps > 4) return refuse(CRAFTAX_E_CONFIG, "taps must be 2..4", why);
    if (a->steps < 1 || a->n < 1 || a->channels < 1) return refuse(CRAFTAX_E_COUNT, "steps, n and channels must be positive", why);
    if ((int64_t)a->n * a->channels > ((int64_t)1 << 31) - 4096) return refuse(CRAFTAX_E_COUNT, "n * channels must be below 2^31", why);
    if (!a->weight || !a->x.data) return refuse(CRAFTAX_E_NULL, "weight or x is NULL", why);
    const size_t e = elem_bytes(a->dtype);
    if (!aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->lengths, 4) || !aligned(a->x.data, e) || !aligned(a->state_in, e))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    if (!backward) {
        if (!a->y.data) return refuse(CRAFTAX_E_NULL, "y is NULL", why);
        if (!aligned(a->y.data, e) || !aligned(a->state_out, e)) return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
        return CRAFTAX_OK;
    }
    if (!a->dy.data || !a->dx.data) return refuse(CRAFTAX_E_NULL, "dy or dx is NULL", why);
    if (!aligned(a->dy.data, e) || !aligned(a->dx.data, e) || !aligned(a->dstate_out, e) || !aligned(a->dstate_in, e) ||
        !aligned(a->dweight, 4) || !aligned(a->dbias, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    return CRAFTAX_OK;
}

template <typename E> static ConvParams<E> conv_params(const craftax_conv_args* a)
{
    ConvParams<E> p{};
    p.weight = a->weight; p.bias = a->bias; p.lengths = a->lengths;
    p.first = seq_in<uint8_t>(a->first);
    p.x = seq_in<E>(a->x); p.dy = seq_in<E>(a->dy); p.y = seq<E>(a->y); p.dx = seq<E>(a->dx);
    p.state_in = static_cast<const E*>(a->state_in); p.state_out = static_cast<E*>(a->state_out);
    p.dstate_out = static_cast<const E*>(a->dstate_out); p.dstate_in = static_cast<E*>(a->dstate_in);
    p.steps = a->steps; p.n = a->n; p.channels = a->channels; p.silu = a->silu != 0;
    return p;
}

// Steps per stretch: as many as leave `threads` threads, at least 8 (with 3 more read in front, a third
// of the reads of a stretch come a second time, from the L2).
static int stretch_of(int steps, int64_t threads_per_step, int64_t threads)
{
    const int64_t stretches = threads_per_step >= threads ? 1 : ceil_div(threads, threads_per_step);
    int64_t s = ceil_div(steps, stretches);
    if (s < 8) s = 8;
    if (ceil_div(steps, s) > 65535) s = ceil_div(steps, 65535);
    return (int)(s < steps ? s : steps);
}

constexpr int64_t CONV_FILL = (int64_t)CHIP_SIMDS * 4 * WAVE;     // four wavefronts per SIMD

int conv(const craftax_conv_args* a, void* stream, const char** why)
{
    if (int rc = conv_check(a, false, why)) return rc;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        constexpr int V = 16 / sizeof(E);
        ConvParams<E> p = conv_params<E>(a);
        p.vectors = (int)ceil_div(a->channels, V);
        const int64_t threads = (int64_t)a->n * p.vectors;
        p.stretch = stretch_of(a->steps, threads, CONV_FILL);
        const dim3 grid((unsigned)ceil_div(threads, CONV_THREADS), (unsigned)ceil_div(a->steps, p.stretch));
        const hipStream_t st = (hipStream_t)stream;
        if (a->taps == 2) hipLaunchKernelGGL((k_conv<E, 2, V>), grid, dim3(CONV_THREADS), 0, st, p);
        else if (a->taps == 3) hipLaunchKernelGGL((k_conv<E, 3, V>), grid, dim3(CONV_THREADS), 0, st, p);
        else hipLaunchKernelGGL((k_conv<E, 4, V>), grid, dim3(CONV_THREADS), 0, st, p);
    });
    return launched(why);
}

constexpr int CONV_BACK_V = 4;

// Blocks of the backward kernel: x over channels, y over environments and stretches.
struct ConvBack { int vectors, lanes_log2, stretch; unsigned x, y; };
static ConvBack conv_back(const craftax_conv_args* a)
{
    ConvBack b;
    b.vectors = (int)ceil_div(a->channels, CONV_BACK_V);
    b.lanes_log2 = 2;
    while (b.lanes_log2 < 6 && (1 << b.lanes_log2) < b.vectors) ++b.lanes_log2;
    const int lanes = 1 << b.lanes_log2, rows = CONV_THREADS / lanes;
    b.x = (unsigned)ceil_div(b.vectors, lanes);
    const int64_t wide = (int64_t)b.x * lanes;
    b.stretch = stretch_of(a->steps, wide * a->n, CONV_FILL);
    const int64_t items = (int64_t)a->n * ceil_div(a->steps, b.stretch);
    const int64_t most = ceil_div(CONV_FILL, wide * rows);       // no more partial rows than fill the chip
    const int64_t y = ceil_div(items, rows);
    b.y = (unsigned)(y < most ? y : most);
    return b;
}

size_t conv_workspace_bytes(const craftax_conv_args* a)
{
    if (!a || a->taps < 2 || a->taps > 4 || a->steps < 1 || a->n < 1 || a->channels < 1) return 0;
    if (!a->dweight && !a->dbias) return 0;
    return round256((size_t)conv_back(a).y * (a->taps + 1) * a->channels * sizeof(float));
}

int conv_backward(const craftax_conv_args* a, void* stream, const char** why)
{
    if (int rc = conv_check(a, true, why)) return rc;
    const size_t need = conv_workspace_bytes(a);
    if (need && !a->workspace) return refuse(CRAFTAX_E_NULL, "workspace is NULL", why);
    if (need && !aligned(a->workspace, 256)) return refuse(CRAFTAX_E_ALIGN, "workspace must be 256-byte aligned", why);
    if (a->workspace_bytes < need) return refuse(CRAFTAX_E_COUNT, "workspace smaller than craftax_causal_conv_workspace_bytes", why);
    const ConvBack b = conv_back(a);
    const hipStream_t st = (hipStream_t)stream;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        ConvParams<E> p = conv_params<E>(a);
        p.vectors = b.vectors; p.lanes_log2 = b.lanes_log2; p.stretch = b.stretch;
        p.part = need ? static_cast<float*>(a->workspace) : nullptr;
        const dim3 grid(b.x, b.y);
        if (a->taps == 2) hipLaunchKernelGGL((k_conv_backward<E, 2, CONV_BACK_V>), grid, dim3(CONV_THREADS), 0, st, p);
        else if (a->taps == 3) hipLaunchKernelGGL((k_conv_backward<E, 3, CONV_BACK_V>), grid, dim3(CONV_THREADS), 0, st, p);
        else hipLaunchKernelGGL((k_conv_backward<E, 4, CONV_BACK_V>), grid, dim3(CONV_THREADS), 0, st, p);
    });
    if (int rc = launched(why)) return rc;
    if (need)
        sum_rows(static_cast<const float*>(a->workspace), (int)b.y, (int64_t)a->channels * (a->taps + 1),
                 PutConv{a->dweight, a->dbias, a->channels, a->taps}, st);
    return launched(why);
}

}  // namespace host
}  // namespace mem
