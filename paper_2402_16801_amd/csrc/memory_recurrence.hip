// Gated linear recurrence of every channel, one state each: whole sequences, single tokens and the backward pass.
//
//   s = sigmoid(decay), L = rate s, a = exp(L), m = sqrt(1 - a a), h_t = a h_(t-1) + m sigmoid(intake) x,  y = h z sigmoid(z)
//
// Bound by memory: 4 activations move per step and channel (5 with a gate), 7 in the backward pass (9), and a float of state every REC_SPAN steps
// in each, beside some 40 and 115 vector instructions, 6 to 8 of them transcendental.  A thread owns V channels of one environment and walks
// along the steps, states in registers; nothing is exchanged between lanes.  64 steps of 4,096 environments of 512 bfloat16 channels: 318 us
// forward (1.50 GB, 4.7 TB/s), 650 backward (2.58 GB, 4.0 TB/s, 179 registers, which leave room for two wavefronts per SIMD); a token of 65,536 x 512 113 us (5.2 TB/s).
//
// Few environments are split into parts along time: a first kernel finds what each part does to the state (a factor and a term), and each block
// goes through the parts before its own.  That reads the inputs twice: 10,000 steps of one environment of 512 floats take 33 us in 625
// parts, one walk alone would take 10,000 steps' latency.
#include "memory_api.hpp"
#include "memory_common.hpp"
#include "memory_walk.hpp"

#include <type_traits>

namespace mem {

constexpr int REC_THREADS = 256;
constexpr int REC_SPAN = 4;             // steps between two saved states

template <typename E> struct RecParams {
    const float* rate;
    Seq<const uint8_t> first;
    const int32_t* lengths;
    Seq<const E> x, decay, intake, z, dy;
    Seq<E> y, dx, ddecay, dintake, dz;
    const float *state_in, *dstate_out;
    float *state_out, *dstate_in, *saved;
    float* sums;             // parts: [slot][2][n][channels], what a part does to the state (forward) or to its gradient (backward)
    float* part;             // backward: [rows of blocks][channels], gradients of the rates
    int steps, n, channels, vectors, lanes_log2;
    int parts, stretch;      // parts of a sequence, steps of one
    uint32_t items, xblocks; // sequences, and blocks side by side on channels
    uint32_t groups;         // of parts, of a sequence
    int group;               // parts in one
    int64_t stride;          // backward: a thread goes on to the sequence that many behind; with parts there is none
    unsigned wide;
};

// What a block works on: channels side by side on 2^lanes_log2 lanes, and rows: a sequence each, or, where sequences are split into parts, as many
// parts of one of them, one behind the other.
constexpr int REC_GROUP = 16;           // parts of a sequence that a block goes along, at most
template <bool SPLIT> struct RecPlace {
    int vec, side, group;
    uint32_t row_block;
    int64_t item;
    bool on;
    template <typename P> __device__ __forceinline__ explicit RecPlace(const P& p)
    {
        const uint32_t block = (uint32_t)spread_block(p.wide);
        const int lanes = 1 << p.lanes_log2, rows = SPLIT ? p.group : REC_THREADS >> p.lanes_log2;
        side = threadIdx.x >> p.lanes_log2;
        row_block = block / p.xblocks;
        vec = (int)(block % p.xblocks) * lanes + (threadIdx.x & (lanes - 1));
        group = SPLIT ? (int)(row_block % p.groups) : 0;
        item = SPLIT ? (int64_t)(row_block / p.groups) : (int64_t)row_block * rows + side;
        on = vec < p.vectors && item < (int64_t)p.items;
    }
};

// rates of minus infinity forget everything, as the smallest number does
template <int V> __device__ __forceinline__ void load_rates(const float* rate, int c, float (&v)[V])
{
    const Pack<float, V> q = *reinterpret_cast<const Pack<float, V>*>(rate + c);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = q.v[j] < -3.0e38f ? -3.0e38f : q.v[j];
}

// A sigmoid with all digits of what it leaves of 1, in one register: itself below 1/2, else its rest with a minus sign (-0 is a gate that is open).
struct Folded {
    float v;
    __device__ __forceinline__ static float of(float s, float e) { return s < 0.5f ? s : -(e * s); }
    __device__ __forceinline__ explicit Folded(float folded) : v(folded) {}
    __device__ __forceinline__ bool open() const { return (int)__float_as_uint(v) < 0; }
    __device__ __forceinline__ float other() const { return 1.0f - __builtin_fabsf(v); }
    __device__ __forceinline__ float sigmoid() const { return open() ? other() : v; }
    __device__ __forceinline__ float rest() const { return open() ? -v : other(); }
};

// The gate of one step: a = exp(rate s), and 1 - a a without the digits that the subtraction would lose where a is near 1:
// 1 - exp(-t) = t (1 - t / 2 + t^2 / 6 - ..) is below 2^-22 of its sum after eight terms for t < 1/2.
struct Gate {
    float e, s, a, rest;     // s = 1 / (1 + e), rest = 1 - a a, 0 where that is negative (rates above 0)
    __device__ __forceinline__ Gate(float decay, float rate)
    {
        e = exp2_fast(-decay * LOG2E);
        s = __builtin_amdgcn_rcpf(1.0f + e);
        const float l = rate * s, t = -2.0f * l;
        a = exp2_fast(l * LOG2E);
        float r = -1.0f / 40320.0f;
        r = __builtin_fmaf(r, t, 1.0f / 5040.0f);
        r = __builtin_fmaf(r, t, -1.0f / 720.0f);
        r = __builtin_fmaf(r, t, 1.0f / 120.0f);
        r = __builtin_fmaf(r, t, -1.0f / 24.0f);
        r = __builtin_fmaf(r, t, 1.0f / 6.0f);
        r = __builtin_fmaf(r, t, -0.5f);
        r = __builtin_fmaf(r, t, 1.0f) * t;
        rest = t < 0.5f ? r : __builtin_fmaf(-a, a, 1.0f);
        rest = rest < 0.0f ? 0.0f : rest;
    }
};

template <typename P> __device__ __forceinline__ float* sum_at(const P& p, int slot, int which, int i, int c)
{
    return p.sums + ((int64_t)(2 * slot + which) * p.n + i) * p.channels + c;
}

// What parts do to a state (or its gradient): factor * state + term; a factor below 0 stands for parts that forget what came before them,
// whatever that was.
template <int V> struct Effect {
    Pack<float, V> f, b;
    __device__ __forceinline__ static Effect none()
    {
        Effect e;
#pragma unroll
        for (int j = 0; j < V; ++j) { e.f.v[j] = 1.0f; e.b.v[j] = 0.0f; }
        return e;
    }
    __device__ __forceinline__ void then(const Effect& o)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const bool cut = o.f.v[j] < 0.0f;
            // A state of 0 stays one where the factor of many parts is infinite (rates above 0), and an infinite one where it is below all numbers.
            constexpr int ZERO_OR_INFINITE = 1 << 2 | 1 << 5 | 1 << 6 | 1 << 9;
            b.v[j] = cut ? o.b.v[j] : __builtin_fmaf(__builtin_amdgcn_classf(b.v[j], ZERO_OR_INFINITE) ? 1.0f : o.f.v[j], b.v[j], o.b.v[j]);
            f.v[j] = cut || f.v[j] < 0.0f ? -1.0f : f.v[j] * o.f.v[j];
        }
    }
};
// of `count` slots from `from` on, in steps of `by`
template <int V, typename P> __device__ __forceinline__ Effect<V> effect_of(const P& p, int from, int by, int count, int i, int c)
{
    constexpr int GO = 8;
    Effect<V> all = Effect<V>::none();
    for (int k = 0; k < count; k += GO) {
        Effect<V> e[GO];
#pragma unroll
        for (int g = 0; g < GO; ++g)
            if (k + g < count) {
                fetch<float, V>(e[g].f, sum_at(p, from + (k + g) * by, 0, i, c));
                fetch<float, V>(e[g].b, sum_at(p, from + (k + g) * by, 1, i, c));
            }
#pragma unroll
        for (int g = 0; g < GO; ++g)
            if (k + g < count) all.then(e[g]);
    }
    return all;
}
// The state behind `far` slots and then `near` rows of this block.  The rows share the slots; `own` is what this row's part does.
// FORWARD: the slots are those from 0 on and the rows those before this one, else the slots are those from `first` down and the rows those behind.
template <int V, bool FORWARD, typename P>
__device__ __forceinline__ void state_behind(const P& p, const RecPlace<true>& at, int first, int far, int own, int i, int c, bool rows_behind, Effect<V> (&maps)[2][REC_GROUP][WAVE],
                                             float (&h)[V])
{
    const int lane = threadIdx.x & ((1 << p.lanes_log2) - 1), each = (far + p.group - 1) / p.group, mine = at.side * each;
    const int count = far - mine < each ? far - mine : each;
    maps[0][at.side][lane] = at.on ? effect_of<V>(p, FORWARD ? mine : first - mine, FORWARD ? 1 : -1, count, i, c) : Effect<V>::none();
    maps[1][at.side][lane] = at.on && own >= 0 ? effect_of<V>(p, own, 1, 1, i, c) : Effect<V>::none();
    __syncthreads();
    Effect<V> all = Effect<V>::none();
    for (int s = 0; s < p.group; ++s) all.then(maps[0][s][lane]);
    if (FORWARD) {
        for (int s = 0; s < at.side; ++s) all.then(maps[1][s][lane]);
    } else if (rows_behind) {
        for (int s = p.group - 1; s > at.side; --s) all.then(maps[1][s][lane]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = all.f.v[j] < 0.0f ? all.b.v[j] : __builtin_fmaf(all.f.v[j], h[j], all.b.v[j]);
}

template <int V> __device__ __forceinline__ void put_sum(float* factor, float* term, const Span& w, const float (&f)[V], const float (&b)[V])
{
    put<float, V>(factor, w, shrink<float, V>(f));
    put<float, V>(term, w, shrink<float, V>(b));
}

// RUN: states and outputs.  SAVE: the states before every REC_SPAN steps as well.  PARTS: only what the parts do to the state; slot 0 is the
// state at the begin, slot 1 + q part q, and the last part is not asked for.
enum RecMode { RUN, SAVE, PARTS };

// SPLIT: sequences are split into parts, sixteen of one to a block.
template <typename E, int V, RecMode MODE, bool GATE, bool CUTS, bool SPLIT>
__global__ __launch_bounds__(SPLIT ? REC_GROUP * WAVE : REC_THREADS) void k_recurrence(const RecParams<E> p)
{
    // few wavefronts wait for memory more often than many
    constexpr int AHEAD = V == 1 ? 8 : 4;
    const RecPlace<SPLIT> at(p);
    if (!SPLIT && !at.on) return;
    const int i = at.on ? (int)at.item : 0, part = SPLIT ? at.group * p.group + at.side : 0;
    const bool on = at.on && part < p.parts - (MODE == PARTS ? 1 : 0);
    const Span w = Span::of<V>(at.on ? at.vec : 0, p.channels);
    const int t0 = on ? part * p.stretch : 0, t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
    const int length = length_of(p.lengths, p.steps, i);
    const int live = t1 < length ? t1 : length;
    const int64_t state_at = (int64_t)i * p.channels + w.c;
    float h[V] = {}, keep[V];
#pragma unroll
    for (int j = 0; j < V; ++j) keep[j] = 1.0f;
    if (on && part == 0 && (MODE == PARTS || !SPLIT)) {
        if (p.state_in) {
            const Pack<float, V> q = *reinterpret_cast<const Pack<float, V>*>(p.state_in + state_at);
            expand<float, V>(q, h);
        }
        if (MODE == PARTS) {
#pragma unroll
            for (int j = 0; j < V; ++j) keep[j] = -1.0f;
            put_sum<V>(sum_at(p, 0, 0, i, w.c), sum_at(p, 0, 1, i, w.c), w, keep, h);
        }
    }
    // With parts the state at the begin comes from slot 0: another thread may write the new state to its place.
    if constexpr (MODE != PARTS && SPLIT) {
        __shared__ Effect<V> maps[2][REC_GROUP][WAVE];
        state_behind<V, true>(p, at, 0, at.group * p.group + 1, part < p.parts - 1 ? part + 1 : -1, i, w.c, false, maps, h);
    }
    if (SPLIT && !on) return;
    if (t0 < live) {
        float rate[V];
        load_rates<V>(p.rate, w.c, rate);
        Stream<E, V, AHEAD> x, decay, intake, z;
        Begins<AHEAD> begins;
        x.start(p.x, t0, live, i, w.c);
        decay.start(p.decay, t0, live, i, w.c);
        intake.start(p.intake, t0, live, i, w.c);
        if (GATE && MODE != PARTS) z.start(p.z, t0, live, i, w.c);
        if (CUTS) begins.start(p.first, t0, live, i);
        E* to = MODE == PARTS ? nullptr : p.y.at(t0, i) + w.c;
        auto one = [&](int t, int a) {
            float vx[V], vd[V], vi[V], vz[V];
            expand<E, V>(x.raw[a], vx);
            expand<E, V>(decay.raw[a], vd);
            expand<E, V>(intake.raw[a], vi);
            if (GATE && MODE != PARTS) expand<E, V>(z.raw[a], vz);
            const bool begin = CUTS && begins.flag[a] != 0;
            x.refill(a);
            decay.refill(a);
            intake.refill(a);
            if (GATE && MODE != PARTS) z.refill(a);
            if (CUTS) begins.refill(a);
            if (MODE == SAVE && t % REC_SPAN == 0)
                put<float, V>(p.saved + ((int64_t)(t / REC_SPAN) * p.n + i) * p.channels + w.c, w, shrink<float, V>(h));
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const Gate g(vd[j], rate[j]);
                const float in = __builtin_amdgcn_sqrtf(g.rest) * sigmoid(vi[j]) * vx[j];
                h[j] = __builtin_fmaf(g.a, begin ? 0.0f : h[j], in);
                if (MODE == PARTS) keep[j] = begin || keep[j] < 0.0f ? -1.0f : keep[j] * g.a;
                else y[j] = GATE ? h[j] * vz[j] * sigmoid(vz[j]) : h[j];
            }
            if (MODE != PARTS) {
                put<E, V>(to, w, shrink<E, V>(y));
                to += p.y.step;
            }
            __builtin_amdgcn_sched_barrier(0);       // step by step: several at a time take the registers of further wavefronts
        };
        int t = t0;
        for (; t + AHEAD <= live; t += AHEAD) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) one(t + a, a);
        }
#pragma unroll
        for (int a = 0; a < AHEAD - 1; ++a)
            if (t + a < live) one(t + a, a);
    }
    if (MODE == PARTS) {
        put_sum<V>(sum_at(p, part + 1, 0, i, w.c), sum_at(p, part + 1, 1, i, w.c), w, keep, h);
        return;
    }
    for (int t = t0 > live ? t0 : live; t < t1; ++t) put<E, V>(p.y.at(t, i) + w.c, w, Pack<E, V>{});
    // the new state is that of the part which holds the last step that counts
    if (p.state_out && (t0 < length ? live == length : part == 0 && length == 0)) put<float, V>(p.state_out + state_at, w, shrink<float, V>(h));
}

// One token: a thread is V channels of one environment.
template <typename E, int V, bool GATE>
__global__ __launch_bounds__(REC_THREADS) void k_recurrence_token(const RecParams<E> p)
{
    const int64_t at = spread_block(p.wide) * REC_THREADS + threadIdx.x;
    if (at >= (int64_t)p.n * p.vectors) return;
    const int i = (int)((uint32_t)at / (uint32_t)p.vectors);
    const Span w = Span::of<V>((int)((uint32_t)at % (uint32_t)p.vectors), p.channels);
    const int64_t state_at = (int64_t)i * p.channels + w.c;
    Pack<E, V> rx, rd, ri, rz;
    Pack<float, V> rh = {};
    fetch<E, V>(rx, p.x.at(0, i) + w.c);
    fetch<E, V>(rd, p.decay.at(0, i) + w.c);
    fetch<E, V>(ri, p.intake.at(0, i) + w.c);
    if (GATE) fetch<E, V>(rz, p.z.at(0, i) + w.c);
    if (p.state_in) fetch<float, V>(rh, p.state_in + state_at);
    const bool begin = p.first.data && *p.first.at(0, i) != 0;
    float rate[V], x[V], d[V], q[V], z[V], h[V], y[V];
    load_rates<V>(p.rate, w.c, rate);
    expand<E, V>(rx, x);
    expand<E, V>(rd, d);
    expand<E, V>(ri, q);
    if (GATE) expand<E, V>(rz, z);
    expand<float, V>(rh, h);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const Gate g(d[j], rate[j]);
        h[j] = __builtin_fmaf(g.a, begin ? 0.0f : h[j], __builtin_amdgcn_sqrtf(g.rest) * sigmoid(q[j]) * x[j]);
        y[j] = GATE ? h[j] * z[j] * sigmoid(z[j]) : h[j];
    }
    put<E, V>(p.y.at(0, i) + w.c, w, shrink<E, V>(y));
    if (p.state_out) put<float, V>(p.state_out + state_at, w, shrink<float, V>(h));
}

// Backward.  With e = dy z sigmoid(z) the gradient of h_t is G_t = e_t + a_(t+1) G_(t+1), cut where an episode begins at t + 1, and
//   dx = G m q,  dintake = G m x q (1 - q),  dL = G (a h_(t-1) - q x a a / m),  ddecay = dL rate s (1 - s),  drate = sum of dL s
// (q = sigmoid(intake); the last term of dL is 0 where m is, at a decay of 1).  A thread walks its part of a sequence from the end in
// spans of REC_SPAN steps: forward through a span from its saved state, for the states, then back.  MODE PARTS: only what a part
// does to the gradient of the state; slot q is part q, from the second one on.
template <typename E, int V, bool GATE> struct RecRaw {
    Pack<E, V> x[REC_SPAN], decay[REC_SPAN], intake[REC_SPAN], z[GATE ? REC_SPAN : 1], dy[REC_SPAN];
    Pack<float, V> h;
    uint32_t first[REC_SPAN];
};

template <typename E, int V, RecMode MODE, bool GATE, bool CUTS, bool SPLIT>
__global__ __launch_bounds__(SPLIT ? REC_GROUP * WAVE : REC_THREADS) void k_recurrence_backward(const RecParams<E> p)
{
    __shared__ float sums[(SPLIT ? REC_GROUP * WAVE : REC_THREADS) * V];
    const RecPlace<SPLIT> at(p);
    float total[V] = {};
    for (int64_t item = SPLIT || at.on ? at.item : (int64_t)p.items; item < (int64_t)p.items; item += p.stride) {
        const int i = (int)item, part = SPLIT ? at.group * p.group + at.side : 0;
        const bool on = at.on && part < p.parts && (MODE != PARTS || part > 0);
        const Span w = Span::of<V>(at.on ? at.vec : 0, p.channels);
        const int t0 = on ? part * p.stretch : 0, t1 = p.steps - t0 < p.stretch ? p.steps : t0 + p.stretch;
        const int length = length_of(p.lengths, p.steps, i);
        const int live = t1 < length ? t1 : length;
        const int64_t state_at = (int64_t)i * p.channels + w.c;
        float g[V] = {}, keep[V];              // gradient of the state behind the step that is next
#pragma unroll
        for (int j = 0; j < V; ++j) keep[j] = 1.0f;
        const bool last = on && (t0 < length ? live == length : part == 0 && length == 0);
        if constexpr (MODE != PARTS && SPLIT) {
            // the parts behind this one, up to that of the last step that counts, which starts with the gradient of the state behind it
            __shared__ Effect<V> maps[2][REC_GROUP][WAVE];
            const int behind = length > 0 ? (length - 1) / p.stretch : 0, here = at.group * p.group + p.group - 1;
            state_behind<V, false>(p, at, behind, behind > here ? behind - here : 0, part > 0 && part <= behind ? part : -1, i, w.c, true, maps, g);
        }
        if (last && p.dstate_out) {
            Pack<float, V> q;
            fetch<float, V>(q, p.dstate_out + state_at);
            expand<float, V>(q, g);
        } else if (last) {
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = 0.0f;
        }
        if (last) {
#pragma unroll
            for (int j = 0; j < V; ++j) keep[j] = -1.0f;
        }
        if (!on) break;
        if (MODE != PARTS) {
            for (int t = t0 > live ? t0 : live; t < t1; ++t) {
                put<E, V>(p.dx.at(t, i) + w.c, w, Pack<E, V>{});
                put<E, V>(p.ddecay.at(t, i) + w.c, w, Pack<E, V>{});
                put<E, V>(p.dintake.at(t, i) + w.c, w, Pack<E, V>{});
                if (GATE) put<E, V>(p.dz.at(t, i) + w.c, w, Pack<E, V>{});
            }
        }
        if (t0 < live) {
            float rate[V];
            load_rates<V>(p.rate, w.c, rate);
            RecRaw<E, V, GATE> raw;
            auto load = [&](int t) {
#pragma unroll
                for (int k = 0; k < REC_SPAN; ++k) {
                    const int u = t + k < live ? t + k : live - 1;
                    if (MODE != PARTS) fetch<E, V>(raw.x[k], p.x.at(u, i) + w.c);
                    fetch<E, V>(raw.decay[k], p.decay.at(u, i) + w.c);
                    if (MODE != PARTS) fetch<E, V>(raw.intake[k], p.intake.at(u, i) + w.c);
                    if (GATE) fetch<E, V>(raw.z[k], p.z.at(u, i) + w.c);
                    fetch<E, V>(raw.dy[k], p.dy.at(u, i) + w.c);
                    raw.first[k] = CUTS ? *p.first.at(u, i) : 0;
                }
                if (MODE != PARTS) fetch<float, V>(raw.h, p.saved + ((int64_t)(t / REC_SPAN) * p.n + i) * p.channels + w.c);
            };
            int t = t0 + (live - 1 - t0) / REC_SPAN * REC_SPAN;
            load(t);
            for (; t >= t0; t -= REC_SPAN) {
                const int count = live - t < REC_SPAN ? live - t : REC_SPAN;
                float s[REC_SPAN][V], a[REC_SPAN][V], rest[REC_SPAN][V], q[REC_SPAN][V], before[REC_SPAN][V], e[REC_SPAN][V];
                Pack<E, V> x[REC_SPAN];
                uint32_t first[REC_SPAN];
                float h[V];
                if (MODE != PARTS) expand<float, V>(raw.h, h);
#pragma unroll
                for (int k = 0; k < REC_SPAN; ++k) {
                    float vx[V], vd[V], vi[V], vz[V], dz[V];
                    expand<E, V>(raw.decay[k], vd);
                    expand<E, V>(raw.dy[k], e[k]);
                    if (GATE) expand<E, V>(raw.z[k], vz);
                    first[k] = raw.first[k];
                    if (MODE != PARTS) {
                        x[k] = raw.x[k];
                        expand<E, V>(raw.x[k], vx);
                        expand<E, V>(raw.intake[k], vi);
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const Gate gate(vd[j], rate[j]);
                        s[k][j] = Folded::of(gate.s, gate.e);
                        a[k][j] = gate.a;
                        rest[k][j] = gate.rest;
                        if (MODE != PARTS) {
                            const float eq = exp2_fast(-vi[j] * LOG2E), vq = __builtin_amdgcn_rcpf(1.0f + eq);
                            q[k][j] = Folded::of(vq, eq);
                            before[k][j] = CUTS && first[k] ? 0.0f : h[j];
                            h[j] = __builtin_fmaf(gate.a, before[k][j], __builtin_amdgcn_sqrtf(gate.rest) * vq * vx[j]);
                        }
                        if (GATE) {
                            const float sg = sigmoid(vz[j]), open = vz[j] * sg;
                            if (MODE != PARTS) dz[j] = e[k][j] * h[j] * sg * __builtin_fmaf(vz[j], 1.0f - sg, 1.0f);
                            e[k][j] *= open;
                        }
                    }
                    if (MODE != PARTS) {               // folded here: kept as two numbers each they cost 15 registers more
                        pin(s[k]);
                        pin(q[k]);
                    }
                    if (MODE != PARTS && GATE && k < count) put<E, V>(p.dz.at(t + k, i) + w.c, w, shrink<E, V>(dz));
                }
                if (t > t0) load(t - REC_SPAN);
                float spans[V] = {};
#pragma unroll
                for (int k = REC_SPAN - 1; k >= 0; --k) {
                    if (k >= count) continue;
                    float dx[V], dd[V], di[V], vx[V];
                    if (MODE != PARTS) expand<E, V>(x[k], vx);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float G = g[j] + e[k][j];
                        if (MODE != PARTS) {
                            const float root = rest[k][j] < 0x1p-126f ? 0.0f : __builtin_amdgcn_rsqf(rest[k][j]);
                            const float m = rest[k][j] * root, gm = G * m;
                            const Folded fs(s[k][j]), fq(q[k][j]);
                            const float vq = fq.sigmoid();
                            dx[j] = gm * vq;
                            di[j] = dx[j] * vx[j] * fq.rest();
                            const float dl = G * a[k][j] * __builtin_fmaf(-vq * vx[j], a[k][j] * root, before[k][j]);
                            const float ds = dl * fs.sigmoid();
                            spans[j] += ds;
                            dd[j] = ds * rate[j] * fs.rest();
                        } else {
                            keep[j] = first[k] || keep[j] < 0.0f ? -1.0f : keep[j] * a[k][j];
                        }
                        g[j] = CUTS && first[k] ? 0.0f : a[k][j] * G;
                    }
                    if (MODE != PARTS) {
                        put<E, V>(p.dx.at(t + k, i) + w.c, w, shrink<E, V>(dx));
                        put<E, V>(p.ddecay.at(t + k, i) + w.c, w, shrink<E, V>(dd));
                        put<E, V>(p.dintake.at(t + k, i) + w.c, w, shrink<E, V>(di));
                    }
                }
#pragma unroll
                for (int j = 0; j < V; ++j) total[j] += spans[j];
            }
        }
        if (MODE == PARTS) put_sum<V>(sum_at(p, part, 0, i, w.c), sum_at(p, part, 1, i, w.c), w, keep, g);
        else if (part == 0 && p.dstate_in) put<float, V>(p.dstate_in + state_at, w, shrink<float, V>(g));
    }
    if (MODE == PARTS || p.part == nullptr) return;
    // one partial row per block
    constexpr int THREADS = SPLIT ? REC_GROUP * WAVE : REC_THREADS;
#pragma unroll
    for (int j = 0; j < V; ++j) sums[j * THREADS + threadIdx.x] = total[j];
    __syncthreads();
    if (at.side != 0 || at.vec >= p.vectors) return;
    const int rows = SPLIT ? p.group : REC_THREADS >> p.lanes_log2;
    const Span w = Span::of<V>(at.vec, p.channels);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float v = 0.0f;
        for (int r = 0; r < rows; ++r) v += sums[j * THREADS + (r << p.lanes_log2) + threadIdx.x];
        total[j] = v;
    }
    put<float, V>(p.part + (int64_t)at.row_block * p.channels + w.c, w, shrink<float, V>(total));
}

struct PutRate {
    float* out;
    __device__ void operator()(int64_t column, float v) const { out[column] = v; }
};

namespace host {

static int rec_check(const craftax_recurrence_args* a, bool backward, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->steps < 1 || a->n < 1 || a->channels < 1) return refuse(CRAFTAX_E_COUNT, "steps, n and channels must be positive", why);
    if (a->steps > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "steps must be below 2^31 - 4095", why);
    if ((int64_t)a->n * a->channels > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "n * channels must be below 2^31 - 4095", why);
    if (!a->rate || !a->x.data || !a->decay.data || !a->intake.data) return refuse(CRAFTAX_E_NULL, "rate, x, decay or intake is NULL", why);
    const size_t e = elem_bytes(a->dtype);
    if (!aligned(a->rate, 4) || !aligned(a->lengths, 4) || !aligned(a->x.data, e) || !aligned(a->decay.data, e) || !aligned(a->intake.data, e) ||
        !aligned(a->z.data, e) || !aligned(a->state_in, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    if (a->saved && !aligned(a->saved, 256)) return refuse(CRAFTAX_E_ALIGN, "saved must be 256-byte aligned", why);
    if (!backward) {
        if (!a->y.data) return refuse(CRAFTAX_E_NULL, "y is NULL", why);
        if (!aligned(a->y.data, e) || !aligned(a->state_out, 4)) return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
        return CRAFTAX_OK;
    }
    if (!a->saved) return refuse(CRAFTAX_E_NULL, "saved is NULL", why);
    if (!a->dy.data || !a->dx.data || !a->ddecay.data || !a->dintake.data) return refuse(CRAFTAX_E_NULL, "dy, dx, ddecay or dintake is NULL", why);
    if (a->z.data && !a->dz.data) return refuse(CRAFTAX_E_NULL, "dz is NULL", why);
    if (!aligned(a->dy.data, e) || !aligned(a->dx.data, e) || !aligned(a->ddecay.data, e) || !aligned(a->dintake.data, e) || !aligned(a->dz.data, e) ||
        !aligned(a->dstate_out, 4) || !aligned(a->dstate_in, 4) || !aligned(a->drate, 4))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    return CRAFTAX_OK;
}

// Wavefronts per SIMD from which on threads take several channels (of fewer, one), from which on sequences are walked whole, and that parts make;
// steps of the shortest part.  Measured with 512 channels of bfloat16, forward and backward (forward alone): REC_WIDE 1, 2, 4: 256 environments of 128
// steps 117, 105, 105 us, (512 of 64) 34, 28, 28, 1,024 of 64 184, 184, 188.  REC_ENOUGH 1, 2: (128 of 256) 45, 50, forward and backward 140, 134.
// REC_FILL 2, 4, 8: 40 ragged ones of 2,000 565, 417, 438, (one of 10,000) 42, 34, 49, 64 of 256 90, 83, 92.  REC_SHORTEST 8, 16, 32: (one of 10,000)
// 34, 34, 39; with 8 the workspace is twice as large for sequences of few channels.
constexpr int REC_WIDE = 2, REC_ENOUGH = 1, REC_FILL = 4, REC_SHORTEST = 16;
constexpr int REC_BLOCKS = 4096;

// How a call is cut: channels per thread, parts of a sequence, blocks.
struct RecCut {
    int width, vectors, lanes_log2, parts, stretch;
    uint32_t xblocks;
    // Blocks of few parts are placed more easily, those of many read fewer parts before their own (37 ragged sequences of 1,000 steps of 647 channels,
    // forward and backward, in groups of 4 and 16: 310 and 340 us; one of 10,000 steps of 512 channels, 512 parts, groups of 16: 32).
    int groups() const { return parts > 1 ? (int)ceil_div(parts, parts <= 128 ? 4 : REC_GROUP) : 1; }
    int group() const { return (int)ceil_div(parts, groups()); }
    // blocks over sequences, or groups of their parts; backward no more than fill the chip several times over, each with sequences in turn, for
    // their partial sums
    uint32_t row_blocks(int64_t n, bool backward) const
    {
        if (parts > 1) return (uint32_t)(n * groups());
        const int64_t need = ceil_div(n, REC_THREADS >> lanes_log2), most = ceil_div(REC_BLOCKS, xblocks);
        return (uint32_t)(backward && need > most ? most : need);
    }
};

static RecCut rec_cut(const craftax_recurrence_args* a, bool backward)
{
    RecCut c;
    c.width = backward ? 2 : 4;
    auto waves = [&] { return (int64_t)a->n * ceil_div(a->channels, c.width) / WAVE; };
    if (a->channels < c.width || waves() < REC_WIDE * CHIP_SIMDS) c.width = 1;
    c.vectors = (int)ceil_div(a->channels, c.width);
    c.lanes_log2 = 0;
    while (c.lanes_log2 < 6 && (1 << c.lanes_log2) < c.vectors) ++c.lanes_log2;
    c.xblocks = (uint32_t)ceil_div(c.vectors, 1 << c.lanes_log2);
    const int64_t have = waves() < 1 ? 1 : waves();
    // where lengths are given, about half of the parts have nothing to do
    int64_t parts = have >= REC_ENOUGH * CHIP_SIMDS ? 1 : (a->lengths ? REC_FILL * 3 / 2 : REC_FILL) * CHIP_SIMDS / have;
    if (parts > a->steps / REC_SHORTEST) parts = a->steps / REC_SHORTEST;
    if (parts < 1) parts = 1;
    c.stretch = (int)(ceil_div(ceil_div(a->steps, parts), REC_SPAN) * REC_SPAN);
    c.parts = (int)ceil_div(a->steps, c.stretch);
    return c;
}

// sizes that the calls take: of others no size is told, whose products might not fit one
static bool rec_shape_ok(const craftax_recurrence_args* a)
{
    return a && a->dtype <= CRAFTAX_F16 && a->steps >= 1 && a->n >= 1 && a->channels >= 1 && a->steps <= MOST_COUNT && (int64_t)a->n * a->channels <= MOST_COUNT;
}

size_t recurrence_saved_bytes(const craftax_recurrence_args* a)
{
    if (!rec_shape_ok(a)) return 0;
    return round256((size_t)ceil_div(a->steps, REC_SPAN) * a->n * a->channels * sizeof(float));
}

static size_t rec_sums_bytes(const craftax_recurrence_args* a, const RecCut& c)
{
    return c.parts > 1 ? round256((size_t)c.parts * 2 * a->n * a->channels * sizeof(float)) : 0;
}
size_t recurrence_workspace_bytes(const craftax_recurrence_args* a, bool backward)
{
    if (!rec_shape_ok(a)) return 0;
    const RecCut c = rec_cut(a, backward);
    size_t bytes = rec_sums_bytes(a, c);
    if (backward && a->drate) bytes += round256((size_t)c.row_blocks(a->n, true) * a->channels * sizeof(float));
    return bytes;
}

static int rec_room(const craftax_recurrence_args* a, size_t need, const char** why)
{
    if (need && !a->workspace) return refuse(CRAFTAX_E_NULL, "workspace is NULL", why);
    if (need && !aligned(a->workspace, 256)) return refuse(CRAFTAX_E_ALIGN, "workspace must be 256-byte aligned", why);
    if (a->workspace_bytes < need) return refuse(CRAFTAX_E_COUNT, "workspace smaller than craftax_gated_recurrence_workspace_bytes", why);
    return CRAFTAX_OK;
}

template <typename E> static RecParams<E> rec_params(const craftax_recurrence_args* a)
{
    RecParams<E> p{};
    p.rate = a->rate; p.lengths = a->lengths;
    p.first = seq_in<uint8_t>(a->first);
    p.x = seq_in<E>(a->x); p.decay = seq_in<E>(a->decay); p.intake = seq_in<E>(a->intake); p.z = seq_in<E>(a->z); p.dy = seq_in<E>(a->dy);
    p.y = seq<E>(a->y); p.dx = seq<E>(a->dx); p.ddecay = seq<E>(a->ddecay); p.dintake = seq<E>(a->dintake); p.dz = seq<E>(a->dz);
    p.state_in = a->state_in; p.state_out = a->state_out; p.dstate_out = a->dstate_out; p.dstate_in = a->dstate_in;
    p.saved = static_cast<float*>(a->saved);
    p.steps = a->steps; p.n = a->n; p.channels = a->channels;
    return p;
}
template <typename P> static void rec_place(P& p, const RecCut& c, const craftax_recurrence_args* a)
{
    p.vectors = c.vectors; p.lanes_log2 = c.lanes_log2; p.parts = c.parts; p.stretch = c.stretch; p.xblocks = c.xblocks;
    p.sums = static_cast<float*>(a->workspace);
}

// calls f with whether there is a gate and whether there are begins of episodes as constants
template <typename F> static void with_options(const craftax_recurrence_args* a, F&& f)
{
    auto cuts = [&](auto gate) {
        if (a->first.data) f(gate, std::true_type{});
        else f(gate, std::false_type{});
    };
    if (a->z.data) cuts(std::true_type{});
    else cuts(std::false_type{});
}

// launches over all sequences
template <typename P, typename K> static void rec_launch(K kernel, P& p, const RecCut& c, bool backward, hipStream_t st)
{
    const uint32_t blocks = c.row_blocks(p.n, backward);
    const int threads = c.parts > 1 ? c.group() << c.lanes_log2 : REC_THREADS;
    p.items = (uint32_t)p.n;
    p.groups = (uint32_t)c.groups();
    p.group = c.group();
    p.stride = c.parts > 1 ? (int64_t)1 << 40 : (int64_t)blocks * (REC_THREADS >> c.lanes_log2);
    const Spread grid = spread((int64_t)c.xblocks * blocks, threads);
    p.wide = grid.x;
    hipLaunchKernelGGL(kernel, dim3(grid.x, 1, grid.z), dim3(threads), 0, st, p);
}

template <typename E, int V> static void rec_token(const craftax_recurrence_args* a, hipStream_t st)
{
    RecParams<E> p = rec_params<E>(a);
    p.vectors = (int)ceil_div(a->channels, V);
    const Spread grid = spread(ceil_div((int64_t)a->n * p.vectors, REC_THREADS), REC_THREADS);
    p.wide = grid.x;
    if (a->z.data) hipLaunchKernelGGL((k_recurrence_token<E, V, true>), dim3(grid.x, 1, grid.z), dim3(REC_THREADS), 0, st, p);
    else hipLaunchKernelGGL((k_recurrence_token<E, V, false>), dim3(grid.x, 1, grid.z), dim3(REC_THREADS), 0, st, p);
}

int recurrence(const craftax_recurrence_args* a, void* stream, const char** why)
{
    if (int rc = rec_check(a, false, why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    if (a->steps == 1 && !a->saved && !a->lengths) {
        with_type(a->dtype, [&](auto e) {
            using E = decltype(e);
            constexpr int V = 16 / sizeof(E);
            if (a->channels >= V) rec_token<E, V>(a, st);
            else rec_token<E, 1>(a, st);
        });
        return launched(why);
    }
    if (int rc = rec_room(a, recurrence_workspace_bytes(a, false), why)) return rc;
    const RecCut c = rec_cut(a, false);
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        RecParams<E> p = rec_params<E>(a);
        rec_place(p, c, a);
        auto run = [&](auto width) {
            constexpr int V = decltype(width)::value;
            with_options(a, [&](auto gate, auto cuts) {
                constexpr bool GATE = decltype(gate)::value, CUTS = decltype(cuts)::value;
                if constexpr (V == 1) {
                    if (c.parts > 1) {
                        rec_launch(k_recurrence<E, V, PARTS, false, CUTS, true>, p, c, false, st);
                        if (a->saved) rec_launch(k_recurrence<E, V, SAVE, GATE, CUTS, true>, p, c, false, st);
                        else rec_launch(k_recurrence<E, V, RUN, GATE, CUTS, true>, p, c, false, st);
                        return;
                    }
                }
                if (a->saved) rec_launch(k_recurrence<E, V, SAVE, GATE, CUTS, false>, p, c, false, st);
                else rec_launch(k_recurrence<E, V, RUN, GATE, CUTS, false>, p, c, false, st);
            });
        };
        if (c.width == 4) run(std::integral_constant<int, 4>{});
        else run(std::integral_constant<int, 1>{});
    });
    return launched(why);
}

int recurrence_backward(const craftax_recurrence_args* a, void* stream, const char** why)
{
    if (int rc = rec_check(a, true, why)) return rc;
    if (int rc = rec_room(a, recurrence_workspace_bytes(a, true), why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    const RecCut c = rec_cut(a, true);
    float* part = a->drate ? reinterpret_cast<float*>(static_cast<char*>(a->workspace) + rec_sums_bytes(a, c)) : nullptr;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        RecParams<E> p = rec_params<E>(a);
        rec_place(p, c, a);
        p.part = part;
        auto run = [&](auto width) {
            constexpr int V = decltype(width)::value;
            with_options(a, [&](auto gate, auto cuts) {
                constexpr bool GATE = decltype(gate)::value, CUTS = decltype(cuts)::value;
                if constexpr (V == 1) {
                    if (c.parts > 1) {
                        rec_launch(k_recurrence_backward<E, V, PARTS, GATE, CUTS, true>, p, c, true, st);
                        rec_launch(k_recurrence_backward<E, V, RUN, GATE, CUTS, true>, p, c, true, st);
                        return;
                    }
                }
                rec_launch(k_recurrence_backward<E, V, RUN, GATE, CUTS, false>, p, c, true, st);
            });
        };
        if (c.width == 2) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 1>{});
    });
    if (int rc = launched(why)) return rc;
    if (part) sum_rows(part, (int)c.row_blocks(a->n, true), a->channels, PutRate{a->drate}, st);
    return launched(why);
}

}  // namespace host
}  // namespace mem
