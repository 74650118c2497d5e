// Short causal convolution of every channel with an activation: whole sequences, single tokens and the
// backward pass.
//
//   p_t = bias + sum over k of weight[k] x_(t - taps + 1 + k), of inputs since the last begin of an episode,  y = p sigmoid(p)
//
// Bound by memory: 2 (forward) or 3 (backward) activations move per step and channel against 18 and 34
// vector instructions.  A thread owns four neighbouring channels of one environment (eight of 16-bit types were no faster)
// and walks along a stretch of steps with the last taps - 1 inputs in registers, so an input is read
// once but for the taps - 1 in front of a stretch.  Stretches exist only to fill the chip.  Four steps are read ahead; eight
// were no faster.
//
// A row whose length is no multiple of V ends with a vector that overlaps the one before it: it is loaded whole,
// and only its own values are stored and counted.  Rows of fewer than V channels go value by value.
#include "memory_api.hpp"
#include "memory_common.hpp"
#include "memory_walk.hpp"

#include <type_traits>

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

// The last K - 1 inputs before step t as they count at step t - 1.  All loads are under way together.
template <typename E, int K, int V>
__device__ __forceinline__ void window_before(const ConvParams<E>& p, int t, int i, const Span& w, float (&win)[K - 1][V])
{
    Pack<E, V> raw[K - 1];
    bool begin[K - 1];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        const int s = t - (K - 1) + k;
        const E* from = s >= 0 || !p.state_in ? p.x.at(s < 0 ? 0 : s, i) : p.state_in + ((int64_t)i * (K - 1) + (s + K - 1)) * p.channels;
        fetch<E, V>(raw[k], from + w.c);
        begin[k] = p.first.data && s >= 0 && *p.first.at(s, i) != 0;
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        if (begin[k]) {
#pragma unroll
            for (int m = 0; m < K - 1; ++m)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (m < k) win[m][j] = 0.0f;
        }
        expand<E, V>(raw[k], win[k]);
        if (t - (K - 1) + k < 0 && !p.state_in) {
#pragma unroll
            for (int j = 0; j < V; ++j) win[k][j] = 0.0f;
        }
    }
}

template <int K, int V> struct Taps {
    float w[K][V], bias[V];
    __device__ __forceinline__ void load(const float* weight, const float* b, int c)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            Pack<float, K> q = *reinterpret_cast<const Pack<float, K>*>(weight + (int64_t)(c + j) * K);
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][j] = q.v[k];
        }
        const Pack<float, V> q = b ? *reinterpret_cast<const Pack<float, V>*>(b + c) : Pack<float, V>{};
#pragma unroll
        for (int j = 0; j < V; ++j) bias[j] = q.v[j];
    }
    __device__ __forceinline__ float sum(const float (&win)[K - 1][V], float x, int j) const
    {
        float s = bias[j];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) s = __builtin_fmaf(w[k][j], win[k][j], s);
        return __builtin_fmaf(w[K - 1][j], x, s);
    }
};

// CUTS: begins of episodes are given.  64 steps of 4,096 environments of 512 channels in bfloat16: 150 us, 3.6 TB/s; 2,048
// environments in float32 117 us, 4.6 TB/s.  Registers leave room for five wavefronts per SIMD (seven of 16-bit types without
// begins) where a rollout of that size launches eight.
template <typename E, int K, int V, bool CUTS>
__global__ __launch_bounds__(CONV_THREADS) void k_conv(const ConvParams<E> p)
{
    constexpr int AHEAD = 4;
    const uint32_t at = blockIdx.x * CONV_THREADS + threadIdx.x;
    const int i = (int)(at / (uint32_t)p.vectors);
    if (i >= p.n) return;
    const Span w = Span::of<V>((int)(at % (uint32_t)p.vectors), p.channels);
    const int t0 = (int)blockIdx.y * p.stretch;
    const int t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
    const int length = length_of(p.lengths, p.steps, i);
    const int live = t1 < length ? t1 : length;       // steps of this stretch that count end here
    float win[K - 1][V];
    if (t0 < live || t0 == 0) window_before<E, K, V>(p, t0, i, w, win);
    if (t0 < live) {
        Taps<K, V> taps;
        Stream<E, V, AHEAD> in;
        Begins<AHEAD> begins;
        in.start(p.x, t0, live, i, w.c);
        if (CUTS) begins.start(p.first, t0, live, i);
        taps.load(p.weight, p.bias, w.c);
        E* to = p.y.at(t0, i) + w.c;
        auto one = [&](int a) {
            float x[V], y[V];
            expand<E, V>(in.raw[a], x);
            in.refill(a);
            if (CUTS) {
                const bool begin = begins.flag[a] != 0;
                begins.refill(a);
#pragma unroll
                for (int k = 0; k < K - 1; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) win[k][j] = begin ? 0.0f : win[k][j];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = taps.sum(win, x[j], j), g = sigmoid(v);
                y[j] = v * (p.silu ? g : 1.0f);
            }
            push<K, V>(win, x);
            put<E, V>(to, w, shrink<E, V>(y));
            to += p.y.step;
            __builtin_amdgcn_sched_barrier(0);       // step by step: several at a time would take the registers of two more wavefronts
        };
        int t = t0;
        for (; t + AHEAD <= live; t += AHEAD) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) one(a);
        }
#pragma unroll
        for (int a = 0; a < AHEAD - 1; ++a)
            if (t + a < live) one(a);
    }
    for (int t = t0 > live ? t0 : live; t < t1; ++t) put<E, V>(p.y.at(t, i) + w.c, w, Pack<E, V>{});
    // The thread of the first stretch, which alone reads the state, writes the new one too, so that it can
    // be the same memory.  With one stretch the window is what is wanted.
    if (p.state_out && blockIdx.y == 0) {
        if (live < length) window_before<E, K, V>(p, length, i, w, win);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) put<E, V>(p.state_out + ((int64_t)i * (K - 1) + k) * p.channels + w.c, w, shrink<E, V>(win[k]));
    }
}

// One token: the state is read and written once, 2 K activations per channel.  A thread takes several environments one
// after the other, so that its weights (16 bytes per channel against 16 of activations) are read once.  4,096 environments of
// 1,024 channels in bfloat16: 15 us, 4.5 TB/s.
template <typename E, int K, int V>
__global__ __launch_bounds__(CONV_THREADS) void k_conv_token(const ConvParams<E> p)
{
    const uint32_t at = blockIdx.x * CONV_THREADS + threadIdx.x;
    int i = (int)(at / (uint32_t)p.vectors);
    if (i >= p.stretch) return;                 // here: environments that are taken side by side
    const Span w = Span::of<V>((int)(at % (uint32_t)p.vectors), p.channels);
    Taps<K, V> taps;
    taps.load(p.weight, p.bias, w.c);
    Pack<E, V> raw[K];
    uint32_t flag = 0;
    int length = 1;
    auto load = [&](int e) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
            fetch<E, V>(raw[k], (p.state_in ? p.state_in + ((int64_t)e * (K - 1) + k) * p.channels : p.x.at(0, e)) + w.c);
        fetch<E, V>(raw[K - 1], p.x.at(0, e) + w.c);
        if (p.first.data) flag = *p.first.at(0, e);
        if (p.lengths) length = p.lengths[e];
    };
    load(i);
    for (; i < p.n; i += p.stretch) {
        float win[K - 1][V], x[V], y[V];
        const bool live = length > 0, empty = !p.state_in || (flag && live);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) expand<E, V>(raw[k], win[k]);
        expand<E, V>(raw[K - 1], x);
        if (empty) clear<K, V>(win);
        Pack<E, V> keep[K - 1];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = !live ? win[k][j] : (k + 1 < K - 1 ? win[k + 1 < K - 1 ? k + 1 : 0][j] : x[j]);
            keep[k] = shrink<E, V>(v);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float v = taps.sum(win, x[j], j), g = sigmoid(v);
            y[j] = live ? v * (p.silu ? g : 1.0f) : 0.0f;
        }
        const int e = i;
        if (i + p.stretch < p.n) load(i + p.stretch);
        put<E, V>(p.y.at(0, e) + w.c, w, shrink<E, V>(y));
        if (p.state_out) {
#pragma unroll
            for (int k = 0; k < K - 1; ++k) put<E, V>(p.state_out + ((int64_t)e * (K - 1) + k) * p.channels + w.c, w, keep[k]);
        }
    }
}

// Backward.  With p the sum before the activation, dp = dy * act'(p):  an input s gets weight[K - 1 - j] * dp of
// step s + j for j = 0 .. K - 1 as far as no episode begins in (s, s + j], and the weight gets the products.  Walking
// forward, `due` holds the gradients of the last K - 1 inputs, of which the oldest is complete with every
// step; a stretch goes K - 1 steps beyond its end for the inputs at its end, without counting those steps
// for the weight.  A block sums its weight gradients in LDS and writes one partial row; rows are added in a
// fixed order by a second kernel.  Two wavefronts per SIMD is what the registers leave room for (weights, their gradients,
// both windows and what is read ahead); vector issue is at about two thirds of the time.  64 steps of 4,096 environments of 512 channels in
// bfloat16: 196 us, 4.1 TB/s, with begins 236 (their flags are loaded and tested by every thread for itself, step by step).
template <typename E, int K, int V, bool CUTS>
__global__ __launch_bounds__(CONV_THREADS) void k_conv_backward(const ConvParams<E> p)
{
    constexpr int COLS = V * (K + 1), AHEAD = 4;
    __shared__ float sums[CONV_THREADS * COLS];
    const int lanes = 1 << p.lanes_log2, side = threadIdx.x >> p.lanes_log2, rows = CONV_THREADS >> p.lanes_log2;
    const int vec = (int)blockIdx.x * lanes + (threadIdx.x & (lanes - 1));
    const int stretches = (p.steps - 1) / p.stretch + 1;
    float dw[K][V], db[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        db[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][j] = 0.0f;
    }
    if (vec < p.vectors) {
        const Span w = Span::of<V>(vec, p.channels);
        Taps<K, V> taps;
        taps.load(p.weight, p.bias, w.c);
        const int64_t items = (int64_t)p.n * stretches;
        for (int64_t item = (int64_t)blockIdx.y * rows + side; item < items; item += (int64_t)gridDim.y * rows) {
            const int i = (int)((uint64_t)item % (uint32_t)p.n), t0 = (int)((uint64_t)item / (uint32_t)p.n) * p.stretch;
            const int t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
            const int length = length_of(p.lengths, p.steps, i);
            const int live = t1 < length ? t1 : length;
            const int end = length - t1 < K - 1 ? length : t1 + (K - 1);     // steps walked: up to here
            for (int t = t0 > live ? t0 : live; t < t1; ++t) put<E, V>(p.dx.at(t, i) + w.c, w, Pack<E, V>{});
            if (t0 >= live && t0 > 0) continue;
            auto state_at = [&](int s) { return p.dstate_in + ((int64_t)i * (K - 1) + (s + K - 1)) * p.channels + w.c; };
            float win[K - 1][V], due[K - 1][V];
            window_before<E, K, V>(p, t0, i, w, win);
            clear<K, V>(due);
            // steps since the last begin of an episode, as far as the window reaches back
            int age = K - 1;
            if (CUTS)
                for (int s = t0 - (K - 1) > 0 ? t0 - (K - 1) : 0; s < t0; ++s)
                    age = *p.first.at(s, i) ? 0 : (age < K - 1 ? age + 1 : K - 1);
            if (t0 < live) {
                Stream<E, V, AHEAD> in_x, in_dy;
                Begins<AHEAD> begins;
                in_x.start(p.x, t0, live, i, w.c);
                in_dy.start(p.dy, t0, live, i, w.c);
                if (CUTS) begins.start(p.first, t0, live, i);
                E* to = p.dx.at(t0, i) + w.c;            // of the oldest input in the window, once that is in the stretch
                auto one = [&](int t, const Pack<E, V>& raw_x, const Pack<E, V>& raw_dy, bool begin, auto counts) {
                    float x[V], dy[V], now[V], grad[V];
                    expand<E, V>(raw_x, x);
                    expand<E, V>(raw_dy, dy);
                    // most steps of a wavefront are in nobody's first K - 1 of an episode and run like those without begins
                    const bool early = CUTS && __any(begin || age < K - 1);
                    if (early) {
                        age = begin ? 0 : age < K - 1 ? age + 1 : K - 1;
                        if (begin) clear<K, V>(win);
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = taps.sum(win, x[j], j), g = sigmoid(v), slope = g * __builtin_fmaf(v, 1.0f - g, 1.0f);
                        const float dp = dy[j] * (p.silu ? slope : 1.0f);
                        now[j] = taps.w[K - 1][j] * dp;
                        grad[j] = dp;
                        if (decltype(counts)::value) {
                            db[j] += dp;
#pragma unroll
                            for (int k = 0; k < K - 1; ++k) dw[k][j] = __builtin_fmaf(dp, win[k][j], dw[k][j]);
                            dw[K - 1][j] = __builtin_fmaf(dp, x[j], dw[K - 1][j]);
                        }
                    }
                    if (!early) {
#pragma unroll
                        for (int k = 0; k < K - 1; ++k)
#pragma unroll
                            for (int j = 0; j < V; ++j) due[k][j] = __builtin_fmaf(taps.w[k][j], grad[j], due[k][j]);
                    } else {
#pragma unroll
                        for (int k = 0; k < K - 1; ++k)
                            if (age >= K - 1 - k) {
#pragma unroll
                                for (int j = 0; j < V; ++j) due[k][j] = __builtin_fmaf(taps.w[k][j], grad[j], due[k][j]);
                            }
                    }
                    // the oldest input, t - (K - 1), is complete
                    const int s = t - (K - 1);
                    if (s >= t0) {
                        put<E, V>(to, w, shrink<E, V>(due[0]));
                        to += p.dx.step;
                    } else if (s < 0 && p.dstate_in) {
                        put<E, V>(state_at(s), w, shrink<E, V>(due[0]));
                    }
                    push<K, V>(win, x);
                    push<K, V>(due, now);
                    // all of a step is done in its turn: put off, the sums would keep several steps' factors in registers
                    pin(dw);
                    pin(db);
                    __builtin_amdgcn_sched_barrier(0);
                };
                auto streamed = [&](int t, int a, auto more) {
                    constexpr bool MORE = decltype(more)::value;
                    const Pack<E, V> raw_x = in_x.raw[a], raw_dy = in_dy.raw[a];
                    const bool begin = CUTS && begins.flag[a] != 0;
                    in_x.template refill<MORE>(a);
                    in_dy.template refill<MORE>(a);
                    if (CUTS) begins.template refill<MORE>(a);
                    one(t, raw_x, raw_dy, begin, std::true_type{});
                };
                int t = t0;
                // what is read ahead by these is in the stretch and not its last step
                for (; t + 2 * AHEAD < live; t += AHEAD) {
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a) streamed(t + a, a, std::true_type{});
                }
                for (; t + AHEAD <= live; t += AHEAD) {
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a) streamed(t + a, a, std::false_type{});
                }
#pragma unroll
                for (int a = 0; a < AHEAD - 1; ++a)
                    if (t + a < live) streamed(t + a, a, std::false_type{});
                // steps behind the stretch, for its last inputs
                for (t = live; t < end; ++t) {
                    Pack<E, V> raw_x, raw_dy;
                    fetch<E, V>(raw_x, p.x.at(t, i) + w.c);
                    fetch<E, V>(raw_dy, p.dy.at(t, i) + w.c);
                    one(t, raw_x, raw_dy, CUTS && *p.first.at(t, i) != 0, std::false_type{});
                }
            }
            // What the walk left: the inputs end - (K - 1) .. end - 1.  At the end of the sequence they are also the new
            // state.
            if (end == length) {
#pragma unroll
                for (int k = 0; k < K - 1; ++k) {
                    const int s = length - (K - 1) + k;
                    if (p.dstate_out && age >= K - 2 - k) {
                        Pack<E, V> raw;
                        float add[V];
                        fetch<E, V>(raw, p.dstate_out + ((int64_t)i * (K - 1) + k) * p.channels + w.c);
                        expand<E, V>(raw, add);
#pragma unroll
                        for (int j = 0; j < V; ++j) due[k][j] += add[j];
                    }
                    if (s >= t0 && s < t1) put<E, V>(p.dx.at(s, i) + w.c, w, shrink<E, V>(due[k]));
                    else if (s < 0 && p.dstate_in) put<E, V>(state_at(s), w, shrink<E, V>(due[k]));
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
        const int v = (int)blockIdx.x * lanes + lane;
        if (v >= p.vectors) continue;
        const Span w = Span::of<V>(v, p.channels);
        if (j < w.old) continue;
        float s = 0.0f;
        for (int r = 0; r < rows; ++r) s += sums[value * CONV_THREADS + (r << p.lanes_log2) + lane];
        row[(int64_t)k * p.channels + w.c + j] = s;
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
    if (a->steps > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "steps must be below 2^31 - 4095", why);
    if ((int64_t)a->n * a->channels > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "n * channels must be below 2^31 - 4095", why);
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

constexpr int64_t CONV_FILL = (int64_t)CHIP_SIMDS * 4 * WAVE;          // four wavefronts per SIMD
constexpr int64_t CONV_BACK_FILL = (int64_t)CHIP_SIMDS * 2 * WAVE;     // two of k_conv_backward, what the registers leave room for

// calls f with the taps and the channels per thread as constants
template <int WIDE, typename F> static void with_taps(const craftax_conv_args* a, F&& f)
{
    auto wide = [&](auto taps) {
        if (a->channels >= WIDE) f(taps, std::integral_constant<int, WIDE>{});
        else f(taps, std::integral_constant<int, 1>{});
    };
    if (a->taps == 2) wide(std::integral_constant<int, 2>{});
    else if (a->taps == 3) wide(std::integral_constant<int, 3>{});
    else wide(std::integral_constant<int, 4>{});
}

int conv(const craftax_conv_args* a, void* stream, const char** why)
{
    if (int rc = conv_check(a, false, why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        with_taps<4>(a, [&](auto taps, auto width) {
            constexpr int K = decltype(taps)::value, V = decltype(width)::value;
            ConvParams<E> p = conv_params<E>(a);
            p.vectors = (int)ceil_div(a->channels, V);
            const int64_t threads = (int64_t)a->n * p.vectors;
            if (a->steps == 1) {
                // environments side by side: two wavefronts per SIMD, each with several environments in turn, or all of them
                p.stretch = side_by_side(ceil_div(CONV_FILL / 2, p.vectors), a->n);
                const dim3 grid((unsigned)ceil_div((int64_t)p.stretch * p.vectors, CONV_THREADS));
                hipLaunchKernelGGL((k_conv_token<E, K, V>), grid, dim3(CONV_THREADS), 0, st, p);
                return;
            }
            p.stretch = stretch_of(a->steps, threads, 2 * CONV_FILL);
            const dim3 grid((unsigned)ceil_div(threads, CONV_THREADS), (unsigned)ceil_div(a->steps, p.stretch));
            if (p.first.data) hipLaunchKernelGGL((k_conv<E, K, V, true>), grid, dim3(CONV_THREADS), 0, st, p);
            else hipLaunchKernelGGL((k_conv<E, K, V, false>), grid, dim3(CONV_THREADS), 0, st, p);
        });
    });
    return launched(why);
}

constexpr int CONV_BACK_V = 4;

// Blocks of the backward kernel: x over channels, y over environments and stretches.
struct ConvBack { int vectors, lanes_log2, stretch; unsigned x, y; };
static ConvBack conv_back(const craftax_conv_args* a)
{
    ConvBack b;
    b.vectors = (int)ceil_div(a->channels, a->channels >= CONV_BACK_V ? CONV_BACK_V : 1);
    b.lanes_log2 = 2;
    while (b.lanes_log2 < 6 && (1 << b.lanes_log2) < b.vectors) ++b.lanes_log2;
    const int lanes = 1 << b.lanes_log2, rows = CONV_THREADS / lanes;
    b.x = (unsigned)ceil_div(b.vectors, lanes);
    const int64_t wide = (int64_t)b.x * lanes;
    b.stretch = stretch_of(a->steps, wide * a->n, CONV_BACK_FILL);
    const int64_t items = (int64_t)a->n * ceil_div(a->steps, b.stretch);
    const int64_t most = ceil_div(CONV_BACK_FILL, wide * rows);       // no more partial rows than fill the chip
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
        with_taps<CONV_BACK_V>(a, [&](auto taps, auto width) {
            constexpr int K = decltype(taps)::value, V = decltype(width)::value;
            if (p.first.data) hipLaunchKernelGGL((k_conv_backward<E, K, V, true>), grid, dim3(CONV_THREADS), 0, st, p);
            else hipLaunchKernelGGL((k_conv_backward<E, K, V, false>), grid, dim3(CONV_THREADS), 0, st, p);
        });
    });
    if (int rc = launched(why)) return rc;
    if (need)
        sum_rows(static_cast<const float*>(a->workspace), (int)b.y, (int64_t)a->channels * (a->taps + 1),
                 PutConv{a->dweight, a->dbias, a->channels, a->taps}, st);
    return launched(why);
}

}  // namespace host
}  // namespace mem
