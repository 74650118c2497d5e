// Selective state space scan: whole sequences, single tokens and the backward pass.
//
//   h = exp(D a) h + D x b,  y = (c . h + d x) z sigmoid(z)      per environment, channel and state
//
// Work: per step and channel 3 activations are read or written (4 with a gate), and per state there are
// an exponential and four multiplications and additions.  With 16 states that is 24 issue cycles times 16 against 6
// to 12 bytes: vector issue bounds sequences, memory bounds single tokens (the state is read and written
// for one step of work).
//
// Sequences: a lane is a channel and holds all of its states, so y is a sum inside the lane; a wavefront is
// 64 channels of one group of one environment, so b and c are the same in all lanes and come through
// scalar loads into scalar registers, which the multiplications take directly.  Where environments and
// channels do not fill the chip, the steps are split too ("parts"): a first kernel gives every part's
// effect on the state (its end from zero, and the sum of D, which is the exponent of the decay), a
// second carries the states through the parts, and the third runs the parts from their own starts.
#include "memory_api.hpp"
#include "memory_common.hpp"

#include <type_traits>

namespace mem {

constexpr int SCAN_THREADS = 256;                      // four wavefronts, each with a tile of its own
constexpr int SCAN_WAVES = SCAN_THREADS / WAVE;
constexpr int AHEAD = 8;                               // steps whose activations are loaded together

template <typename E> struct ScanParams {
    const float *a, *d, *delta_bias;
    Seq<const uint8_t> first;
    const int32_t* lengths;
    Seq<const E> x, delta, z, b, c, dy;
    Seq<E> y, dx, ddelta, dz;
    const float *state_in, *dstate_out;
    float *state_out, *dstate_in;
    float4* starts;        // states at the start of each part, tiled (see tiled_state)
    float2* decays;        // per part, environment, tile and lane: sum of D since the last begin of an episode, 1 if one began
    float4* saved;         // states before every SAVE_STEPS-th step, tiled
    float* shared_part;    // backward: [step][n][tiles][2 * N] sums over a tile for db and dc
    float* weight_part;    // backward: [rows][channels][N + 2] sums for da, dd and ddelta_bias
    int steps, n, channels, groups, group_channels, group_tiles, tiles, softplus;
    int part, parts;       // steps per part, number of parts
    int rows;              // backward: rows of weight_part
};

// What a wavefront works on: 64 channels of one group (`tile`) of one environment.
struct Tile {
    int tile, group, channel;      // channel of this lane; the group's last one where the lane has none
    bool owns;                     // the lane has a channel
};

template <typename E>
__device__ __forceinline__ Tile tile_of(const ScanParams<E>& p, int tile)
{
    Tile w;
    w.tile = tile;
    w.group = tile / p.group_tiles;
    const int in_group = (tile % p.group_tiles) * WAVE + (int)(threadIdx.x & (WAVE - 1));
    w.owns = in_group < p.group_channels;
    w.channel = w.group * p.group_channels + (w.owns ? in_group : p.group_channels - 1);
    return w;
}

template <typename E>
__device__ __forceinline__ int scan_length(const ScanParams<E>& p, int i)
{
    if (p.lengths == nullptr) return p.steps;
    const int l = __builtin_amdgcn_readfirstlane(p.lengths[i]);
    return l < 0 ? 0 : (l > p.steps ? p.steps : l);
}

// begins of episodes among the steps t .. t + 63 below `end`, one bit each
template <typename E>
__device__ __forceinline__ uint64_t begins(const ScanParams<E>& p, int t, int end, int i)
{
    if (p.first.data == nullptr) return 0;
    const int s = t + (int)(threadIdx.x & (WAVE - 1));
    const bool on = s < end && *p.first.at(s < end ? s : end - 1, i) != 0;
    return __ballot(on);
}

// N shared values of a step (b or c of the group), in scalar registers.
template <typename E, int N> struct Shared;
template <int N> struct Shared<float, N> {
    float v[N];
    __device__ __forceinline__ void load(const float* p)
    {
        const __attribute__((address_space(4))) float* q = (const __attribute__((address_space(4))) float*)(uintptr_t)p;
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = q[n];
    }
    __device__ __forceinline__ float operator[](int n) const { return v[n]; }
};
template <int N> struct Shared<__bf16, N> {
    uint32_t v[N / 2];
    __device__ __forceinline__ void load(const __bf16* p)
    {
        const __attribute__((address_space(4))) uint32_t* q = (const __attribute__((address_space(4))) uint32_t*)(uintptr_t)p;
#pragma unroll
        for (int n = 0; n < N / 2; ++n) v[n] = q[n];
    }
    __device__ __forceinline__ float operator[](int n) const { return __uint_as_float(n & 1 ? v[n / 2] & 0xffff0000u : v[n / 2] << 16); }
};
template <int N> struct Shared<_Float16, N> {
    uint32_t v[N / 2];
    __device__ __forceinline__ void load(const _Float16* p)
    {
        const __attribute__((address_space(4))) uint32_t* q = (const __attribute__((address_space(4))) uint32_t*)(uintptr_t)p;
#pragma unroll
        for (int n = 0; n < N / 2; ++n) v[n] = q[n];
    }
    __device__ __forceinline__ float operator[](int n) const
    {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(n & 1 ? v[n / 2] >> 16 : v[n / 2] & 0xffffu));
    }
};

// State in a workspace: [...][tile][N / 4][lane] float4, so that a wavefront moves whole kilobytes.
template <int N>
__device__ __forceinline__ float4* tiled_state(float4* base, int64_t index, const Tile& w, int tiles)
{
    return base + ((index * tiles + w.tile) * (N / 4)) * WAVE + (threadIdx.x & (WAVE - 1));
}
template <int N> __device__ __forceinline__ void load_tiled(const float4* q, float (&h)[N])
{
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const float4 v = q[k * WAVE];
        h[4 * k] = v.x; h[4 * k + 1] = v.y; h[4 * k + 2] = v.z; h[4 * k + 3] = v.w;
    }
}
template <int N> __device__ __forceinline__ void store_tiled(float4* q, const float (&h)[N])
{
#pragma unroll
    for (int k = 0; k < N / 4; ++k) q[k * WAVE] = make_float4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]);
}
// State as the caller has it: [n][channels][N].
template <int N> __device__ __forceinline__ void load_state(const float* state, int64_t index, float (&h)[N])
{
    const float4* q = reinterpret_cast<const float4*>(state + index * N);
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const float4 v = q[k];
        h[4 * k] = v.x; h[4 * k + 1] = v.y; h[4 * k + 2] = v.z; h[4 * k + 3] = v.w;
    }
}
template <int N> __device__ __forceinline__ void store_state(float* state, int64_t index, const float (&h)[N])
{
    float4* q = reinterpret_cast<float4*>(state + index * N);
#pragma unroll
    for (int k = 0; k < N / 4; ++k) q[k] = make_float4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]);
}
template <int N> __device__ __forceinline__ void zero(float (&h)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n) h[n] = 0.0f;
}

// The decay's exponent is taken to base 2: a is scaled once.
template <int N> __device__ __forceinline__ void load_rates(const float* a, int channel, float (&a2)[N])
{
    load_state<N>(a, channel, a2);
#pragma unroll
    for (int n = 0; n < N; ++n) a2[n] *= LOG2E;
}

// States are saved before every SAVE-th step for the backward pass, which holds SAVE * N of them per lane.
template <int N> struct Save { static constexpr int STEPS = 128 / N; };

// ---- forward ------------------------------------------------------------------------------------------
// One wavefront: the steps of one part of one tile of one environment.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan(const ScanParams<E> p)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + wave;
    if (item >= (int64_t)p.n * p.tiles) return;
    const int i = (int)(item / p.tiles);
    const Tile w = tile_of(p, (int)(item % p.tiles));
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    const int length = scan_length(p, i);
    const int end = t1 < length ? t1 : length;
    float a2[N], h[N];
    load_rates<N>(p.a, w.channel, a2);
    const float skip = p.d ? p.d[w.channel] : 0.0f;
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    if (part > 0) load_tiled<N>(tiled_state<N>(p.starts, (int64_t)part * p.n + i, w, p.tiles), h);
    else if (p.state_in) load_state<N>(p.state_in, (int64_t)i * p.channels + w.channel, h);
    else zero(h);
    uint64_t starts = 0;
    for (int t = t0; t < end; t += AHEAD) {
        if (((t - t0) & (WAVE - 1)) == 0) starts = begins(p, t, end, i);
        float x[AHEAD], delta[AHEAD], z[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = t + k < end ? t + k : end - 1;
            x[k] = Elem<E>::up(p.x.at(s, i)[w.channel]);
            delta[k] = Elem<E>::up(p.delta.at(s, i)[w.channel]);
            if (p.z.data) z[k] = Elem<E>::up(p.z.at(s, i)[w.channel]);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (t + k >= end) break;
            if (p.saved && (t + k) % Save<N>::STEPS == 0)
                store_tiled<N>(tiled_state<N>(p.saved, (int64_t)((t + k) / Save<N>::STEPS) * p.n + i, w, p.tiles), h);
            Shared<E, N> b, c;
            b.load(p.b.at(t + k, i) + w.group * N);
            c.load(p.c.at(t + k, i) + w.group * N);
            if (starts >> ((t + k - t0) & (WAVE - 1)) & 1u) zero(h);
            float size = delta[k] + bias;
            if (p.softplus) size = softplus(size);
            const float u = size * x[k];
            float y[4] = {skip * x[k], 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int n = 0; n < N; ++n) {
                h[n] = __builtin_fmaf(exp2_fast(size * a2[n]), h[n], u * b[n]);
                y[n & 3] = __builtin_fmaf(h[n], c[n], y[n & 3]);
            }
            float out = (y[0] + y[1]) + (y[2] + y[3]);
            if (p.z.data) out *= z[k] * sigmoid(z[k]);
            if (w.owns) p.y.at(t + k, i)[w.channel] = Elem<E>::down(out);
        }
    }
    if (w.owns) {
        for (int t = t0 > end ? t0 : end; t < t1; ++t) p.y.at(t, i)[w.channel] = Elem<E>::down(0.0f);
        if (p.state_out && p.parts == 1) store_state<N>(p.state_out, (int64_t)i * p.channels + w.channel, h);
    }
}

// What a part does to the state: its end from zero, and how the state before it decays.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_part(const ScanParams<E> p)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + wave;
    if (item >= (int64_t)p.n * p.tiles) return;
    const int i = (int)(item / p.tiles);
    const Tile w = tile_of(p, (int)(item % p.tiles));
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    const int length = scan_length(p, i);
    const int end = t1 < length ? t1 : length;
    float a2[N], h[N];
    load_rates<N>(p.a, w.channel, a2);
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    zero(h);
    float total = 0.0f, cut = 0.0f;
    uint64_t starts = 0;
    for (int t = t0; t < end; t += AHEAD) {
        if (((t - t0) & (WAVE - 1)) == 0) starts = begins(p, t, end, i);
        float x[AHEAD], delta[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = t + k < end ? t + k : end - 1;
            x[k] = Elem<E>::up(p.x.at(s, i)[w.channel]);
            delta[k] = Elem<E>::up(p.delta.at(s, i)[w.channel]);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (t + k >= end) break;
            Shared<E, N> b;
            b.load(p.b.at(t + k, i) + w.group * N);
            if (starts >> ((t + k - t0) & (WAVE - 1)) & 1u) { zero(h); total = 0.0f; cut = 1.0f; }
            float size = delta[k] + bias;
            if (p.softplus) size = softplus(size);
            const float u = size * x[k];
            total += size;
#pragma unroll
            for (int n = 0; n < N; ++n) h[n] = __builtin_fmaf(exp2_fast(size * a2[n]), h[n], u * b[n]);
        }
    }
    const int64_t index = (int64_t)part * p.n + i;
    store_tiled<N>(tiled_state<N>(p.starts, index, w, p.tiles), h);
    p.decays[(index * p.tiles + w.tile) * WAVE + (threadIdx.x & (WAVE - 1))] = make_float2(total, cut);
}

// Carries the state through the parts: starts[part] turns from the part's own end into the state at its
// start.  A thread takes four states of one channel.  Backward in time for the gradient of the state.
template <typename E, int N, bool BACK>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_carry(const ScanParams<E> p)
{
    constexpr int QUADS = N / 4;
    const int64_t item = ((int64_t)blockIdx.x * SCAN_THREADS + threadIdx.x) / WAVE;     // (environment, tile, four states)
    if (item >= (int64_t)p.n * p.tiles * QUADS) return;
    const int quad = (int)(item % QUADS);
    const int i = (int)(item / QUADS / p.tiles);
    const Tile w = tile_of(p, (int)(item / QUADS % p.tiles));
    const int lane = threadIdx.x & (WAVE - 1);
    const float4 a = *reinterpret_cast<const float4*>(p.a + (int64_t)w.channel * N + quad * 4);
    const float a2[4] = {a.x * LOG2E, a.y * LOG2E, a.z * LOG2E, a.w * LOG2E};
    const int64_t own = ((int64_t)i * p.channels + w.channel) * N + quad * 4;
    const float* in = BACK ? p.dstate_out : p.state_in;
    float* out = BACK ? p.dstate_in : p.state_out;
    float h[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (in) {
        const float4 v = *reinterpret_cast<const float4*>(in + own);
        h[0] = v.x; h[1] = v.y; h[2] = v.z; h[3] = v.w;
    }
    constexpr int GO = 8;
    for (int q0 = 0; q0 < p.parts; q0 += GO) {
        float4 end[GO];
        float2 decay[GO];
#pragma unroll
        for (int k = 0; k < GO; ++k) {
            const int q = q0 + k < p.parts ? q0 + k : p.parts - 1;
            const int64_t index = ((int64_t)(BACK ? p.parts - 1 - q : q) * p.n + i) * p.tiles + w.tile;
            end[k] = p.starts[(index * QUADS + quad) * WAVE + lane];
            decay[k] = p.decays[index * WAVE + lane];
        }
#pragma unroll
        for (int k = 0; k < GO; ++k) {
            const int q = q0 + k;
            if (q >= p.parts) break;
            const int64_t index = ((int64_t)(BACK ? p.parts - 1 - q : q) * p.n + i) * p.tiles + w.tile;
            p.starts[(index * QUADS + quad) * WAVE + lane] = make_float4(h[0], h[1], h[2], h[3]);
            const float e[4] = {end[k].x, end[k].y, end[k].z, end[k].w};
#pragma unroll
            for (int m = 0; m < 4; ++m) h[m] = decay[k].y != 0.0f ? e[m] : __builtin_fmaf(exp2_fast(decay[k].x * a2[m]), h[m], e[m]);
        }
    }
    if (out && w.owns) *reinterpret_cast<float4*>(out + own) = make_float4(h[0], h[1], h[2], h[3]);
}

// ---- one token -------------------------------------------------------------------------------------------
// Bound by the state, 2 * N * 4 bytes per channel: a thread takes four states of a channel (16 bytes, in the
// order of memory), N / 4 neighbouring threads add up their part of y.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_token(const ScanParams<E> p)
{
    constexpr int QUADS = N / 4;
    const int64_t at = (int64_t)blockIdx.x * SCAN_THREADS + threadIdx.x;
    const uint32_t per_env = (uint32_t)p.channels * QUADS;
    const int64_t total = (int64_t)p.n * per_env;
    const bool on = at < total;
    const int64_t mine = on ? at : total - 1;
    const int i = total <= 0xffffffffll ? (int)((uint32_t)mine / per_env) : (int)(mine / per_env);
    const uint32_t rest = (uint32_t)(mine - (int64_t)i * per_env);
    const int channel = (int)(rest / QUADS), quad = (int)(rest % QUADS);
    const int group = channel / p.group_channels;
    const bool alive = p.lengths == nullptr || p.lengths[i] > 0;
    const bool begin = p.first.data && *p.first.at(0, i) != 0;
    float h[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.state_in) {
        const float4 v = *reinterpret_cast<const float4*>(p.state_in + mine * 4);
        h[0] = v.x; h[1] = v.y; h[2] = v.z; h[3] = v.w;
    }
    float out = 0.0f;
    if (alive) {
        const float4 a = *reinterpret_cast<const float4*>(p.a + (int64_t)rest * 4);
        const float a4[4] = {a.x * LOG2E, a.y * LOG2E, a.z * LOG2E, a.w * LOG2E};
        float b[4], c[4];
        load_row<E, 4>(p.b.at(0, i) + group * N + quad * 4, 4, b);
        load_row<E, 4>(p.c.at(0, i) + group * N + quad * 4, 4, c);
        const float x = Elem<E>::up(p.x.at(0, i)[channel]);
        float size = Elem<E>::up(p.delta.at(0, i)[channel]) + (p.delta_bias ? p.delta_bias[channel] : 0.0f);
        if (p.softplus) size = softplus(size);
        const float u = size * x;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            h[m] = __builtin_fmaf(exp2_fast(size * a4[m]), begin ? 0.0f : h[m], u * b[m]);
            out = __builtin_fmaf(h[m], c[m], out);
        }
        // p.lengths is the same for the threads of a channel, so they add up together
        out += dpp<DPP_XOR1>(out);
        if constexpr (QUADS >= 4) out += dpp<DPP_XOR2>(out);
        if constexpr (QUADS >= 8) out += dpp<DPP_HALF_MIRROR>(out);
        if (p.d) out = __builtin_fmaf(p.d[channel], x, out);
        if (p.z.data) {
            const float z = Elem<E>::up(p.z.at(0, i)[channel]);
            out *= z * sigmoid(z);
        }
    }
    if (!on) return;
    if (p.state_out) *reinterpret_cast<float4*>(p.state_out + mine * 4) = make_float4(h[0], h[1], h[2], h[3]);
    if (quad == 0) p.y.at(0, i)[channel] = Elem<E>::down(out);
}

#include "memory_scan_backward.hpp"

// ---- host --------------------------------------------------------------------------------------------------
namespace host {

static int scan_check(const craftax_scan_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->states != 8 && a->states != 16 && a->states != 32) return refuse(CRAFTAX_E_CONFIG, "states must be 8, 16 or 32", why);
    if (a->steps < 1 || a->n < 1 || a->channels < 1) return refuse(CRAFTAX_E_COUNT, "steps, n and channels must be positive", why);
    if (a->groups < 1 || a->channels % a->groups != 0) return refuse(CRAFTAX_E_COUNT, "groups must divide channels", why);
    if ((int64_t)a->n * a->channels > ((int64_t)1 << 31) - 4096) return refuse(CRAFTAX_E_COUNT, "n * channels must be below 2^31", why);
    const craftax_view* need[] = {&a->x, &a->delta, &a->b, &a->c};
    for (const craftax_view* v : need)
        if (!v->data) return refuse(CRAFTAX_E_NULL, "x, delta, b or c is NULL", why);
    if (!a->a) return refuse(CRAFTAX_E_NULL, "a is NULL", why);
    const size_t e = elem_bytes(a->dtype);
    const craftax_view* all[] = {&a->x, &a->delta, &a->z, &a->b, &a->c};
    for (const craftax_view* v : all)
        if (!aligned(v->data, e)) return refuse(CRAFTAX_E_ALIGN, "an activation is not aligned to its elements", why);
    const craftax_view* rows[] = {&a->b, &a->c};
    for (const craftax_view* v : rows)
        if (!aligned(v->data, 4) || (a->steps > 1 && v->step * (int64_t)e % 4 != 0) || (a->n > 1 && v->env * (int64_t)e % 4 != 0))
            return refuse(CRAFTAX_E_ALIGN, "rows of b and c must be 4-byte aligned", why);
    if (!aligned(a->a, 16) || !aligned(a->state_in, 16) || !aligned(a->state_out, 16))
        return refuse(CRAFTAX_E_ALIGN, "a and the states must be 16-byte aligned", why);
    if (!aligned(a->d, 4) || !aligned(a->delta_bias, 4) || !aligned(a->lengths, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    if (!aligned(a->saved, 256)) return refuse(CRAFTAX_E_ALIGN, "saved must be 256-byte aligned", why);
    if (!backward) {
        if (!a->y.data) return refuse(CRAFTAX_E_NULL, "y is NULL", why);
        if (!aligned(a->y.data, e)) return refuse(CRAFTAX_E_ALIGN, "an activation is not aligned to its elements", why);
        return CRAFTAX_OK;
    }
    if (!a->saved) return refuse(CRAFTAX_E_NULL, "saved is NULL: run the forward pass with it", why);
    const craftax_view* grads[] = {&a->dy, &a->dx, &a->ddelta, &a->db, &a->dc};
    for (const craftax_view* v : grads) {
        if (!v->data) return refuse(CRAFTAX_E_NULL, "dy, dx, ddelta, db or dc is NULL", why);
        if (!aligned(v->data, e)) return refuse(CRAFTAX_E_ALIGN, "a gradient is not aligned to its elements", why);
    }
    if (a->z.data && !a->dz.data) return refuse(CRAFTAX_E_NULL, "dz is NULL", why);
    if (!a->da) return refuse(CRAFTAX_E_NULL, "da is NULL", why);
    if (!aligned(a->dz.data, e) || !aligned(a->dd, 4) || !aligned(a->ddelta_bias, 4))
        return refuse(CRAFTAX_E_ALIGN, "a gradient is not aligned to its elements", why);
    if (!aligned(a->da, 16) || !aligned(a->dstate_in, 16) || !aligned(a->dstate_out, 16))
        return refuse(CRAFTAX_E_ALIGN, "da and the gradients of states must be 16-byte aligned", why);
    return CRAFTAX_OK;
}

struct ScanTiles { int group_channels, group_tiles, tiles; };
static ScanTiles scan_tiles(const craftax_scan_args* a)
{
    ScanTiles t;
    t.group_channels = a->channels / a->groups;
    t.group_tiles = (int)ceil_div(t.group_channels, WAVE);
    t.tiles = t.group_tiles * a->groups;
    return t;
}

// Steps per part, a multiple of 64 (the begins of episodes are read 64 steps at a time).
struct ScanParts { int part, parts; };
static ScanParts scan_parts(const craftax_scan_args* a, int tiles, int64_t wavefronts)
{
    const int64_t waves = (int64_t)a->n * tiles;
    ScanParts s = {a->steps, 1};
    // Split steps cost the state's recurrence twice (about 1.7 times the work), so a chip half full is left as it is.
    if (2 * waves > wavefronts || a->steps <= WAVE) return s;
    const int64_t want = wavefronts / waves;
    int64_t part = (ceil_div(a->steps, want) + WAVE - 1) / WAVE * WAVE;
    if (ceil_div(a->steps, part) > 65535) part = (ceil_div(a->steps, 65535) + WAVE - 1) / WAVE * WAVE;
    s.part = (int)part;
    s.parts = (int)ceil_div(a->steps, part);
    if (s.parts == 1) s.part = a->steps;
    return s;
}

constexpr int64_t SCAN_FILL = (int64_t)CHIP_SIMDS * 2;           // wavefronts: two per SIMD
constexpr int64_t SCAN_BACK_FILL = (int64_t)CHIP_SIMDS * 2;

static bool scan_shape_ok(const craftax_scan_args* a)
{
    return a && (a->states == 8 || a->states == 16 || a->states == 32) && a->steps >= 1 && a->n >= 1 && a->channels >= 1 && a->groups >= 1 &&
           a->channels % a->groups == 0 && a->dtype <= CRAFTAX_F16;
}

static size_t state_bytes(const craftax_scan_args* a, int tiles) { return (size_t)a->n * tiles * WAVE * a->states * sizeof(float); }

size_t scan_saved_bytes(const craftax_scan_args* a)
{
    if (!scan_shape_ok(a)) return 0;
    return (size_t)ceil_div(a->steps, 128 / a->states) * state_bytes(a, scan_tiles(a).tiles);
}

// What lies where in a workspace.
struct ScanSpace { ScanParts parts; size_t starts, decays, shared, weights, bytes; int rows, turns; };
static ScanSpace scan_space(const craftax_scan_args* a, bool backward)
{
    const int tiles = scan_tiles(a).tiles;
    ScanSpace s{};
    s.parts = scan_parts(a, tiles, backward ? SCAN_BACK_FILL : SCAN_FILL);
    size_t at = 0;
    if (s.parts.parts > 1) {
        s.starts = at;
        at += round256((size_t)s.parts.parts * state_bytes(a, tiles));
        s.decays = at;
        at += round256((size_t)s.parts.parts * a->n * tiles * WAVE * sizeof(float2));
    }
    if (backward) {
        // a wavefront takes `turns` environments one after the other, so that no more rows of partial sums are written
        // than fill the chip
        const int64_t waves = (int64_t)a->n * tiles;
        int64_t turns = s.parts.parts > 1 ? 1 : waves / SCAN_BACK_FILL;
        if (turns < 1) turns = 1;
        s.turns = (int)turns;
        s.rows = (int)ceil_div(a->n, turns) * s.parts.parts;
        s.shared = at;
        at += round256((size_t)a->steps * a->n * tiles * 2 * a->states * sizeof(float));
        s.weights = at;
        at += round256((size_t)s.rows * a->channels * (a->states + 2) * sizeof(float));
    }
    s.bytes = at;
    return s;
}

size_t scan_workspace_bytes(const craftax_scan_args* a, bool backward)
{
    if (!scan_shape_ok(a)) return 0;
    if (!backward && a->steps == 1 && !a->saved) return 0;
    return scan_space(a, backward).bytes;
}

template <typename E> static ScanParams<E> scan_params(const craftax_scan_args* a)
{
    ScanParams<E> p{};
    const ScanTiles t = scan_tiles(a);
    p.a = a->a; p.d = a->d; p.delta_bias = a->delta_bias; p.lengths = a->lengths;
    p.first = seq_in<uint8_t>(a->first);
    p.x = seq_in<E>(a->x); p.delta = seq_in<E>(a->delta); p.z = seq_in<E>(a->z); p.b = seq_in<E>(a->b); p.c = seq_in<E>(a->c);
    p.dy = seq_in<E>(a->dy);
    p.y = seq<E>(a->y); p.dx = seq<E>(a->dx); p.ddelta = seq<E>(a->ddelta); p.dz = seq<E>(a->dz);
    p.state_in = a->state_in; p.dstate_out = a->dstate_out; p.state_out = a->state_out; p.dstate_in = a->dstate_in;
    p.saved = static_cast<float4*>(a->saved);
    p.steps = a->steps; p.n = a->n; p.channels = a->channels; p.groups = a->groups; p.softplus = a->softplus != 0;
    p.group_channels = t.group_channels; p.group_tiles = t.group_tiles; p.tiles = t.tiles;
    p.part = a->steps; p.parts = 1;
    return p;
}

// calls f with the number of states as a constant
template <typename F> static void with_states(int states, F&& f)
{
    if (states == 8) f(std::integral_constant<int, 8>{});
    else if (states == 16) f(std::integral_constant<int, 16>{});
    else f(std::integral_constant<int, 32>{});
}

static int check_workspace(const void* workspace, size_t given, size_t need, const char** why)
{
    if (need && !workspace) return refuse(CRAFTAX_E_NULL, "workspace is NULL", why);
    if (need && !aligned(workspace, 256)) return refuse(CRAFTAX_E_ALIGN, "workspace must be 256-byte aligned", why);
    if (given < need) return refuse(CRAFTAX_E_COUNT, "workspace smaller than craftax_selective_scan_workspace_bytes", why);
    return CRAFTAX_OK;
}

int scan(const craftax_scan_args* a, void* stream, const char** why)
{
    if (int rc = scan_check(a, false, why)) return rc;
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, scan_workspace_bytes(a, false), why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        ScanParams<E> p = scan_params<E>(a);
        with_states(a->states, [&](auto states) {
            constexpr int N = decltype(states)::value;
            if (a->steps == 1 && !a->saved) {
                const int64_t threads = (int64_t)a->n * a->channels * (N / 4);
                hipLaunchKernelGGL((k_scan_token<E, N>), dim3((unsigned)ceil_div(threads, SCAN_THREADS)), dim3(SCAN_THREADS), 0, st, p);
                return;
            }
            const ScanSpace s = scan_space(a, false);
            char* base = static_cast<char*>(a->workspace);
            p.part = s.parts.part; p.parts = s.parts.parts;
            const dim3 grid((unsigned)ceil_div((int64_t)a->n * p.tiles, SCAN_WAVES), (unsigned)p.parts);
            if (p.parts > 1) {
                p.starts = reinterpret_cast<float4*>(base + s.starts);
                p.decays = reinterpret_cast<float2*>(base + s.decays);
                const unsigned carry = (unsigned)ceil_div((int64_t)a->n * p.tiles * (N / 4), SCAN_WAVES);
                hipLaunchKernelGGL((k_scan_part<E, N>), grid, dim3(SCAN_THREADS), 0, st, p);
                hipLaunchKernelGGL((k_scan_carry<E, N, false>), dim3(carry), dim3(SCAN_THREADS), 0, st, p);
            }
            hipLaunchKernelGGL((k_scan<E, N>), grid, dim3(SCAN_THREADS), 0, st, p);
        });
    });
    return launched(why);
}

int scan_backward(const craftax_scan_args* a, void* stream, const char** why)
{
    if (int rc = scan_check(a, true, why)) return rc;
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, scan_workspace_bytes(a, true), why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    const ScanSpace s = scan_space(a, true);
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        ScanParams<E> p = scan_params<E>(a);
        char* base = static_cast<char*>(a->workspace);
        p.part = s.parts.part; p.parts = s.parts.parts; p.rows = s.rows;
        p.starts = reinterpret_cast<float4*>(base + s.starts);
        p.decays = reinterpret_cast<float2*>(base + s.decays);
        p.shared_part = reinterpret_cast<float*>(base + s.shared);
        p.weight_part = reinterpret_cast<float*>(base + s.weights);
        with_states(a->states, [&](auto states) {
            constexpr int N = decltype(states)::value;
            const dim3 parts_grid((unsigned)ceil_div((int64_t)a->n * p.tiles, SCAN_WAVES), (unsigned)p.parts);
            if (p.parts > 1) {
                const unsigned carry = (unsigned)ceil_div((int64_t)a->n * p.tiles * (N / 4), SCAN_WAVES);
                hipLaunchKernelGGL((k_scan_back_part<E, N>), parts_grid, dim3(SCAN_THREADS), 0, st, p);
                hipLaunchKernelGGL((k_scan_carry<E, N, true>), dim3(carry), dim3(SCAN_THREADS), 0, st, p);
            }
            const int env_rows = s.rows / p.parts;
            const dim3 grid((unsigned)ceil_div((int64_t)env_rows * p.tiles, SCAN_WAVES), (unsigned)p.parts);
            hipLaunchKernelGGL((k_scan_back<E, N>), grid, dim3(SCAN_THREADS), 0, st, p);
            const int64_t values = (int64_t)a->steps * a->n * a->groups * 2 * N;
            hipLaunchKernelGGL((k_scan_shared<E, N>), dim3((unsigned)ceil_div(values, SCAN_THREADS)), dim3(SCAN_THREADS), 0, st, p,
                               seq<E>(a->db), seq<E>(a->dc));
            sum_rows(p.weight_part, s.rows, (int64_t)a->channels * (N + 2), PutScan<N>{a->da, a->dd, a->ddelta_bias}, st);
        });
    });
    return launched(why);
}

}  // namespace host
}  // namespace mem
