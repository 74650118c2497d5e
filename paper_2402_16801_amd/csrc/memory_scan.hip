// Selective state space scan: whole sequences, single tokens and the backward pass.
//
//   h = exp(D a) h + D x b,  y = (c . h + d x) z sigmoid(z)      per environment, channel and state
//
// Work: per step and channel 3 activations are read or written (4 with a gate), and per state there are
// an exponential and four multiplications and additions: with 16 states about 320 issue cycles of a lane against 6 to 12
// bytes.  Vector issue bounds sequences, memory bounds single tokens (the state is read and written for one step of work).
//
// Sequences: a lane holds four states of a channel, so N / 4 neighbouring lanes are a channel and a wavefront
// is 64 / (N / 4) channels of one group of one environment.  It goes on by blocks of eight steps.  What a step
// needs of a channel (D and D x) is computed once, by the lane that owns the step, and handed to the
// channel's lanes through LDS, as are b and c, which all channels read; y of eight steps is summed over the
// channel's lanes by folding, which leaves each lane the steps it owns.  Everything in LDS belongs to one
// wavefront, so there are no barriers.  Where environments and channels do not fill the chip, the steps are
// split too ("parts"): a first kernel gives every part's effect on the state (its end from zero, and the
// sum of D, which is the exponent of the decay), and a second runs the parts from their own starts, which it finds from the
// effects of the parts before; of many parts a kernel in between does (see part_start).
#include "memory_api.hpp"
#include "memory_common.hpp"

#include <type_traits>

namespace mem {

constexpr int SCAN_THREADS = 512;                      // eight wavefronts, each with a tile of its own (see k_scan)
constexpr int SCAN_WAVES = SCAN_THREADS / WAVE;
constexpr int BLOCK = 8;                               // steps that are worked on together

typedef float Four __attribute__((ext_vector_type(4)));

// How N states lie on a wavefront.
template <int N> struct Lay {
    static constexpr int LANES = N / 4;                // lanes of a channel, four states each: 2, 4 or 8
    static constexpr int CHANNELS = WAVE / LANES;      // channels of a wavefront
    static constexpr int OWN = BLOCK / LANES;          // steps of a block that a lane owns: lane q the steps q * OWN ..
};

template <typename E> struct ScanParams {
    const float *a, *d, *delta_bias;
    Seq<const uint8_t> first;
    const int32_t* lengths;
    Seq<const E> x, delta, z, b, c, dy;
    Seq<E> y, dx, ddelta, dz;
    const float *state_in, *dstate_out;
    float *state_out, *dstate_in;
    float4* starts;        // states at the start of each part, [part][n][tile][lane]
    float2* decays;        // per part, environment, tile and channel: sum of D since the last begin of an episode, 1 if one began
    float4* saved;         // states before every block of steps, [block][n][tile][lane]
    float* shared_part;    // backward: [step][n][groups][group_blocks][2 * N] sums for db and dc
    float* weight_part;    // backward: [rows][channels][N + 2] sums for da, dd and ddelta_bias
    int steps, n, channels, groups, group_channels, group_tiles, tiles, softplus;
    int part, parts;       // steps per part (whole blocks), number of parts
    unsigned wide;         // blocks in x (see spread)
    int own_starts;        // wavefronts find the starts of their parts themselves (see part_start)
    int rows, group_blocks;          // backward: rows of weight_part, blocks per group
};

// What a wavefront works on: some channels of one group (`tile`) of one environment.
struct Tile {
    int tile, group, quad;         // quad: the lane's four states are 4 * quad ..
    uint32_t channel;              // channel of this lane; the group's last one where the lane has none
    bool owns;                     // the lane has a channel
};

template <int N, typename E>
__device__ __forceinline__ Tile tile_of(const ScanParams<E>& p, int tile)
{
    const int lane = (int)(threadIdx.x & (WAVE - 1));
    Tile w;
    w.tile = tile;
    w.group = tile / p.group_tiles;
    w.quad = lane % Lay<N>::LANES;
    const int in_group = (tile % p.group_tiles) * Lay<N>::CHANNELS + lane / Lay<N>::LANES;
    w.owns = in_group < p.group_channels;
    w.channel = (uint32_t)(w.group * p.group_channels + (w.owns ? in_group : p.group_channels - 1));
    return w;
}

template <typename E>
__device__ __forceinline__ int scan_length(const ScanParams<E>& p, int i)
{
    if (p.lengths == nullptr) return p.steps;
    const int l = __builtin_amdgcn_readfirstlane(p.lengths[i]);
    return l < 0 ? 0 : (l > p.steps ? p.steps : l);
}

// Begins of episodes in a block of steps: lane l brings the flag of step l % 8.
struct WalkFirst {
    const uint8_t* at;
    int64_t step;
    uint32_t flag;
    template <typename E> __device__ __forceinline__ void start(const ScanParams<E>& p, int t, int i)
    {
        step = p.first.step;
        at = p.first.data ? p.first.at(t, i) + (int)(threadIdx.x & (BLOCK - 1)) * step : nullptr;
        flag = 0;
    }
    __device__ __forceinline__ void move(int blocks) { at += blocks * BLOCK * step; }
    __device__ __forceinline__ void load(bool any, int count)
    {
        if (!any) return;
        const int row = (int)(threadIdx.x & (BLOCK - 1));
        const uint8_t* q = at;
        if (count < BLOCK && row >= count) q -= row * step;
        flag = *q;
    }
    __device__ __forceinline__ uint32_t cuts(int count) const
    {
        return (uint32_t)__ballot((int)(threadIdx.x & (WAVE - 1)) < count && flag != 0);
    }
};

// Four states of this lane in a workspace ([index][tile][lane]) and as the caller has them ([n][channels][N]).
__device__ __forceinline__ float4* tiled(float4* base, int64_t index, const Tile& w, int tiles)
{
    return base + (index * tiles + w.tile) * WAVE + (threadIdx.x & (WAVE - 1));
}
template <int N, typename P> __device__ __forceinline__ P* state_of(P* state, int channels, int i, const Tile& w)
{
    return state + ((int64_t)i * channels + w.channel) * N + w.quad * 4;
}
__device__ __forceinline__ void load4(const void* p, float (&h)[4])
{
    const float4 v = *static_cast<const float4*>(p);
    h[0] = v.x; h[1] = v.y; h[2] = v.z; h[3] = v.w;
}
__device__ __forceinline__ void store4(void* p, const float (&h)[4]) { *static_cast<float4*>(p) = make_float4(h[0], h[1], h[2], h[3]); }
__device__ __forceinline__ void zero(float (&h)[4]) { h[0] = h[1] = h[2] = h[3] = 0.0f; }

// The decay's exponent is taken to base 2: a is scaled once.  It stays finite, since steps that do not count have the size 0,
// and 0 times an infinity is no number; a step that counts decays to 0 by either.
template <int N> __device__ __forceinline__ void load_rates(const float* a, const Tile& w, float (&a2)[4])
{
    load4(a + (int64_t)w.channel * N + w.quad * 4, a2);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        a2[m] *= LOG2E;
        if (__builtin_fabsf(a2[m]) > __FLT_MAX__) a2[m] = __builtin_copysignf(__FLT_MAX__, a2[m]);
    }
}

// Where a lane reads or writes one sequence: its channel at its own first step of the current block of steps.
template <typename P, int N> __device__ __forceinline__ P* walk_from(const Seq<P>& q, int t, int i, const Tile& w)
{
    return q.data ? q.at(t + w.quad * Lay<N>::OWN, i) + w.channel : nullptr;
}
// The lane's own steps as they lie in memory, the block's first step behind the end.  Nothing is converted or tested
// here: the first use of a value waits for it, and that is to be a block of steps later.
template <typename E, int OWN>
__device__ __forceinline__ void load_own(const E* at, int64_t step, int own, int count, E (&v)[OWN])
{
    if (count >= BLOCK) {
#pragma unroll
        for (int k = 0; k < OWN; ++k) v[k] = at[k * step];
    } else {
#pragma unroll
        for (int k = 0; k < OWN; ++k) v[k] = at[(own + k < count ? k : -own) * step];
    }
}

// b and c of a block of steps, [step][2 N] (b first): every lane brings LANES values of one step.
template <typename E, int N> struct WalkShared {
    const E* at;
    int64_t step;
    uint32_t words[Lay<N>::LANES * sizeof(E) / 4];
    __device__ __forceinline__ void start(const ScanParams<E>& p, int t, int i, const Tile& w)
    {
        const int lane = (int)(threadIdx.x & (WAVE - 1)), piece = lane % 8;
        step = piece < 4 ? p.b.step : p.c.step;
        at = (piece < 4 ? p.b.at(t, i) : p.c.at(t, i)) + (int64_t)w.group * N + (piece & 3) * Lay<N>::LANES + lane / 8 * step;
    }
    __device__ __forceinline__ void move(int blocks) { at += blocks * BLOCK * step; }
    __device__ __forceinline__ void load(int count)
    {
        const int row = (int)(threadIdx.x & (WAVE - 1)) / 8;
        const E* q = at;
        if (count < BLOCK && row >= count) q -= row * step;
        const Pack<E, Lay<N>::LANES> v = *reinterpret_cast<const Pack<E, Lay<N>::LANES>*>(q);
        __builtin_memcpy(words, &v, sizeof(v));
    }
    // 0 behind the end
    __device__ __forceinline__ void stage(float4* lds, int count) const
    {
        const int row = (int)(threadIdx.x & (WAVE - 1)) / 8;
        Pack<E, Lay<N>::LANES> v;
        __builtin_memcpy(&v, words, sizeof(v));
        float* q = reinterpret_cast<float*>(lds) + (threadIdx.x & (WAVE - 1)) * Lay<N>::LANES;       // (step, piece) in a row
        if (count >= BLOCK) {
#pragma unroll
            for (int k = 0; k < Lay<N>::LANES; ++k) q[k] = Elem<E>::up(v.v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < Lay<N>::LANES; ++k) q[k] = row < count ? Elem<E>::up(v.v[k]) : 0.0f;
        }
    }
};

// LDS of one wavefront is written and then read by its lanes: in order for the hardware, and kept so for the compiler.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Sums of the values of eight steps over a channel's lanes; lane q is left with those of its steps q * OWN ..
template <int LANES>
__device__ __forceinline__ void fold_steps(float (&v)[BLOCK])
{
    const int lane = (int)(threadIdx.x & (WAVE - 1));
    int half = BLOCK / 2;
    if constexpr (LANES == 8) {
        const bool up = lane & 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = v[k] + dpp<DPP_HALF_MIRROR>(v[k]), b = v[k + 4] + dpp<DPP_HALF_MIRROR>(v[k + 4]);
            v[k] = up ? b : a;
        }
        half = 2;
    }
    if constexpr (LANES >= 4) {
        const bool up = lane & 2;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= half) break;
            const float a = v[k] + dpp<DPP_XOR2>(v[k]), b = v[k + half] + dpp<DPP_XOR2>(v[k + half]);
            v[k] = up ? b : a;
        }
        half /= 2;
    }
    const bool up = lane & 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k >= half) break;
        const float a = v[k] + dpp<DPP_XOR1>(v[k]), b = v[k + half] + dpp<DPP_XOR1>(v[k + half]);
        v[k] = up ? b : a;
    }
}

// The state behind a part, from the one before it and what the part does.
__device__ __forceinline__ void pass_part(const float (&a2)[4], float2 decay, const float (&end)[4], float (&h)[4])
{
#pragma unroll
    for (int m = 0; m < 4; ++m) h[m] = decay.y != 0.0f ? end[m] : __builtin_fmaf(exp2_fast(decay.x * a2[m]), h[m], end[m]);
}

// The state at the start of a part.  Of few parts (`own_starts`) every wavefront goes through the parts before its own, behind it
// backward in time, and is spared a kernel between the two; of many, that kernel, k_scan_carry, has left it in `starts`.
template <typename E, int N, bool BACK>
__device__ __forceinline__ void part_start(const ScanParams<E>& p, int part, int i, const Tile& w, const float (&a2)[4], float (&h)[4])
{
    constexpr int GO = 4;                       // parts whose effects are loaded together
    if (p.parts > 1 && !p.own_starts) {
        load4(tiled(p.starts, (int64_t)part * p.n + i, w, p.tiles), h);
        return;
    }
    const float* in = BACK ? p.dstate_out : p.state_in;
    if (in) load4(state_of<N>(in, p.channels, i, w), h);
    else zero(h);
    const int before = BACK ? p.parts - 1 - part : part;
    for (int q0 = 0; q0 < before; q0 += GO) {
        float end[GO][4];
        float2 decay[GO];
#pragma unroll
        for (int k = 0; k < GO; ++k) {
            const int q = q0 + k < before ? q0 + k : before - 1;
            const int64_t index = (int64_t)(BACK ? p.parts - 1 - q : q) * p.n + i;
            load4(tiled(p.starts, index, w, p.tiles), end[k]);
            decay[k] = p.decays[(index * p.tiles + w.tile) * Lay<N>::CHANNELS + (int)(threadIdx.x & (WAVE - 1)) / Lay<N>::LANES];
        }
#pragma unroll
        for (int k = 0; k < GO; ++k)
            if (q0 + k < before) pass_part(a2, decay[k], end[k], h);
    }
}

// ---- forward ------------------------------------------------------------------------------------------
// One wavefront: the steps of one part of one tile of one environment.  PART: only the part's effect on the
// state.  SAVE: the states before every block are kept for a backward pass (streamed: they are read long after).  The
// activations of the next block are under way while a block is computed.  Eight wavefronts to a block of threads put the
// rows of 128 channels side by side in time.  64 steps of 4,096 environments of 512 channels in 16 bits, with a gate:
// 750 us, with saved states 860 (998 with four wavefronts and cached stores); vector instructions issue 3/4 of the time.  That is 105 ns
// of its SIMD for a step of a wavefront.  A block is eight wavefronts, two to a SIMD, whatever the launch: two on a SIMD take 172 ns
// a step together, one alone 135 (measured in one block of one to four live wavefronts), so that few environments with long
// sequences run at 172 ns a step on the compute units that have a block, and the others idle.
enum ScanMode { RUN, SAVE, PART_ONLY };
template <typename E, int N, ScanMode MODE, bool GATE>
__global__ __launch_bounds__(SCAN_THREADS) __attribute__((amdgpu_waves_per_eu(5))) void k_scan(const ScanParams<E> p)
{
    constexpr int LANES = Lay<N>::LANES, CHANNELS = Lay<N>::CHANNELS, OWN = Lay<N>::OWN;
    constexpr bool PART = MODE == PART_ONLY;
    __shared__ float4 shared_lds[SCAN_WAVES][BLOCK * N / 2];
    __shared__ float2 step_lds[SCAN_WAVES][BLOCK * CHANNELS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = spread_block(p.wide) * SCAN_WAVES + wave;
    if (item >= (int64_t)p.n * p.tiles) return;
    const int i = (int)(item / p.tiles);
    const Tile w = tile_of<N>(p, (int)(item % p.tiles));
    const int mine = (int)(threadIdx.x & (WAVE - 1)) / LANES;
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    const int length = scan_length(p, i);
    const int end = t1 < length ? t1 : length;
    float a2[4], h[4];
    load_rates<N>(p.a, w, a2);
    const float skip = p.d ? p.d[w.channel] : 0.0f;
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    if (PART) zero(h);
    else part_start<E, N, false>(p, part, i, w, a2, h);
    float total = 0.0f, cut = 0.0f;
    const int own = w.quad * OWN;
    const E *at_x = walk_from<const E, N>(p.x, t0, i, w), *at_delta = walk_from<const E, N>(p.delta, t0, i, w);
    const E* at_z = walk_from<const E, N>(p.z, t0, i, w);
    E* at_y = walk_from<E, N>(p.y, t0, i, w);
    WalkShared<E, N> at_shared;
    WalkFirst at_first;
    at_shared.start(p, t0, i, w);
    at_first.start(p, t0, i);
    E x[OWN], delta[OWN], z[OWN];
    auto fetch = [&](int count) {
        at_first.load(p.first.data != nullptr, count);
        at_shared.load(count);
        load_own<E, OWN>(at_x, p.x.step, own, count, x);
        load_own<E, OWN>(at_delta, p.delta.step, own, count, delta);
        if (GATE) load_own<E, OWN>(at_z, p.z.step, own, count, z);
        at_first.move(1);
        at_shared.move(1);
        at_x += BLOCK * p.x.step;
        at_delta += BLOCK * p.delta.step;
        at_z += BLOCK * p.z.step;
    };
    if (t0 < end) fetch(end - t0);
    float4* at_saved = tiled(p.saved, (int64_t)(t0 / BLOCK) * p.n + i, w, p.tiles);
    for (int t = t0; t < end; t += BLOCK) {
        const int count = end - t < BLOCK ? end - t : BLOCK;
        const bool whole = count == BLOCK;
        const uint32_t cuts = at_first.cuts(count);
        float x_now[OWN], z_now[OWN];
        wave_fence();
        at_shared.stage(shared_lds[wave], count);
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            x_now[k] = Elem<E>::up(x[k]);
            z_now[k] = GATE ? Elem<E>::up(z[k]) : 0.0f;
            float size = Elem<E>::up(delta[k]) + bias;
            if (p.softplus) size = softplus(size);
            // steps behind the end leave the state as it is
            if (!whole && own + k >= count) size = x_now[k] = 0.0f;
            step_lds[wave][(own + k) * CHANNELS + mine] = make_float2(size, size * x_now[k]);
        }
        wave_fence();
        if (t + BLOCK < end) fetch(end - t - BLOCK);
        if (MODE == SAVE) {             // behind the loads: waiting for those must not be waiting for this
            __builtin_nontemporal_store(Four{h[0], h[1], h[2], h[3]}, reinterpret_cast<Four*>(at_saved));
            at_saved += (int64_t)p.n * p.tiles * WAVE;
        }
        float y[BLOCK];
        auto walk = [&](auto check) {
#pragma unroll
            for (int k = 0; k < BLOCK; ++k) {
                const float2 step = step_lds[wave][k * CHANNELS + mine];
                float b[4], c[4];
                load4(&shared_lds[wave][k * (N / 2) + w.quad], b);
                if (!PART) load4(&shared_lds[wave][k * (N / 2) + N / 4 + w.quad], c);
                if (decltype(check)::value && (cuts >> k & 1u)) {
                    zero(h);
                    if (PART) { total = 0.0f; cut = 1.0f; }
                }
                if (PART) total += step.x;
                float sum = 0.0f;
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    h[m] = __builtin_fmaf(exp2_fast(step.x * a2[m]), h[m], step.y * b[m]);
                    if (!PART) sum = m == 0 ? h[m] * c[m] : __builtin_fmaf(h[m], c[m], sum);
                }
                y[k] = sum;
                if (!PART) pin(y[k]);
                if (k % 2 == 1) __builtin_amdgcn_sched_barrier(0);     // the operands of two steps at a time, not of eight, are in registers
            }
        };
        // most blocks have no begin in them and run without a test per step
        if (cuts == 0) walk(std::false_type{});
        else walk(std::true_type{});
        if (PART) continue;
        fold_steps<LANES>(y);
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            float out = __builtin_fmaf(skip, x_now[k], y[k]);
            if (GATE) out *= z_now[k] * sigmoid(z_now[k]);
            y[k] = out;
        }
        // the next block's values, under way since before this one's steps, are waited for here: behind the stores, the wait
        // would be for those too
        pin(at_first.flag);
        pin(at_shared.words);
        pin(x);
        pin(delta);
        if (GATE) pin(z);
        if (w.owns) {
#pragma unroll
            for (int k = 0; k < OWN; ++k)
                if (whole || own + k < count) at_y[k * p.y.step] = Elem<E>::down(y[k]);
        }
        at_y += BLOCK * p.y.step;
    }
    if (PART) {
        const int64_t index = (int64_t)part * p.n + i;
        store4(tiled(p.starts, index, w, p.tiles), h);
        if (w.quad == 0) p.decays[(index * p.tiles + w.tile) * CHANNELS + mine] = make_float2(total, cut);
        return;
    }
    if (!w.owns) return;
    for (int t = (t0 > end ? t0 : end) + w.quad; t < t1; t += LANES) p.y.at(t, i)[w.channel] = Elem<E>::down(0.0f);
    if (p.state_out && part == p.parts - 1) store4(state_of<N>(p.state_out, p.channels, i, w), h);
}

// Carries the state through the parts: starts[part] turns from what the part does into the state at its start.  Backward in
// time for the gradient of the state.  A block is a tile of an environment; each of its wavefronts takes a run of
// parts, first adds up what they do together, and, once it knows what the runs before it do, goes through them again.
// One trip to memory for up to 192 parts (157 parts: 10.6 us; 22 where one wavefront makes one for every eight).
constexpr int CARRY_WAVES = 16;
template <typename E, int N, bool BACK>
__global__ __launch_bounds__(CARRY_WAVES* WAVE) void k_scan_carry(const ScanParams<E> p)
{
    constexpr int GO = 12;                      // parts whose effects are loaded together
    __shared__ float4 ends[CARRY_WAVES][WAVE];
    __shared__ float2 decays[CARRY_WAVES][WAVE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), waves = (int)blockDim.x / WAVE;
    const int lane = (int)(threadIdx.x & (WAVE - 1));
    const int i = (int)(blockIdx.x / (unsigned)p.tiles);
    const Tile w = tile_of<N>(p, (int)(blockIdx.x % (unsigned)p.tiles));
    const int mine = lane / Lay<N>::LANES;
    float a2[4], h[4], start[4];
    load_rates<N>(p.a, w, a2);
    const float* in = BACK ? p.dstate_out : p.state_in;
    if (in) load4(state_of<N>(in, p.channels, i, w), start);
    else zero(start);
    const int run = (p.parts + waves - 1) / waves, from = wave * run, to = from + run < p.parts ? from + run : p.parts;
    auto index_of = [&](int q) { return (int64_t)(BACK ? p.parts - 1 - q : q) * p.n + i; };
    float end[GO][4];
    float2 decay[GO];
    // what the last part does nobody asks for, and it is not there
    auto load = [&](int q0) {
#pragma unroll
        for (int k = 0; k < GO; ++k) {
            const int64_t index = index_of(q0 + k < p.parts - 1 ? q0 + k : p.parts - 2);
            load4(tiled(p.starts, index, w, p.tiles), end[k]);
            decay[k] = p.decays[(index * p.tiles + w.tile) * Lay<N>::CHANNELS + mine];
        }
    };
    // the run from zero, and its decay
    zero(h);
    float2 all = make_float2(0.0f, 0.0f);
    for (int q0 = from; q0 < to; q0 += GO) {
        load(q0);
#pragma unroll
        for (int k = 0; k < GO; ++k)
            if (q0 + k < to) {
                pass_part(a2, decay[k], end[k], h);
                all = decay[k].y != 0.0f ? decay[k] : make_float2(all.x + decay[k].x, all.y);
            }
    }
    store4(&ends[wave][lane], h);
    decays[wave][lane] = all;
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 4; ++m) h[m] = start[m];
    for (int v = 0; v < wave; ++v) {
        float before[4];
        load4(&ends[v][lane], before);
        pass_part(a2, decays[v][lane], before, h);
    }
    for (int q0 = from; q0 < to; q0 += GO) {
        if (run > GO) load(q0);
#pragma unroll
        for (int k = 0; k < GO; ++k)
            if (q0 + k < to) {
                store4(tiled(p.starts, index_of(q0 + k), w, p.tiles), h);
                pass_part(a2, decay[k], end[k], h);
            }
    }
}

// ---- one token -------------------------------------------------------------------------------------------
// Bound by the state, 2 * N * 4 bytes per channel: a thread takes four states of a channel (16 bytes, in the
// order of memory), N / 4 neighbouring threads add up their part of y.  It goes on to further environments with
// its rates in registers (another 16 bytes per thread otherwise), the next one's values under way.  65,536 environments of 512
// channels and 16 states: 935 us, 4.9 TB/s (1,153 with a thread for every four states and no second environment).
// STREAMED: the state passes the caches by (see TOKEN_STREAMED).
template <typename E, int N, bool STREAMED>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_token(const ScanParams<E> p)
{
    constexpr int QUADS = N / 4;
    const uint32_t per_env = (uint32_t)p.channels * QUADS;
    const uint32_t at = blockIdx.x * SCAN_THREADS + threadIdx.x;
    int i = (int)(at / per_env);
    const bool on = i < p.part;                // environments side by side; the other threads only follow their neighbours
    if (!on) i = p.part - 1;
    const uint32_t rest = at % per_env;
    const int channel = (int)(rest / QUADS), quad = (int)(rest % QUADS);
    const int64_t shared = (int64_t)(channel / p.group_channels) * N + quad * 4;
    float a4[4];
    load4(p.a + (int64_t)rest * 4, a4);
#pragma unroll
    for (int m = 0; m < 4; ++m) a4[m] *= LOG2E;
    const float skip = p.d ? p.d[channel] : 0.0f, bias = p.delta_bias ? p.delta_bias[channel] : 0.0f;
    const bool gate = p.z.data != nullptr;
    Four state = {0.0f, 0.0f, 0.0f, 0.0f};
    Pack<E, 4> b, c;
    E x, delta, z;
    uint32_t flag = 0;
    int length = 1;
    auto load = [&](int e) {
        if (p.state_in) {
            const Four* q = reinterpret_cast<const Four*>(p.state_in + ((int64_t)e * per_env + rest) * 4);
            state = STREAMED ? __builtin_nontemporal_load(q) : *q;
        }
        b = *reinterpret_cast<const Pack<E, 4>*>(p.b.at(0, e) + shared);
        c = *reinterpret_cast<const Pack<E, 4>*>(p.c.at(0, e) + shared);
        x = p.x.at(0, e)[channel];
        delta = p.delta.at(0, e)[channel];
        if (gate) z = p.z.at(0, e)[channel];
        if (p.first.data) flag = *p.first.at(0, e);
        if (p.lengths) length = p.lengths[e];
    };
    load(i);
    for (; i < p.n; i += p.part) {
        const bool alive = length > 0, begin = flag != 0;
        float size = Elem<E>::up(delta) + bias;
        if (p.softplus) size = softplus(size);
        const float input = Elem<E>::up(x), u = size * input, gated = gate ? Elem<E>::up(z) : 0.0f;
        const float old[4] = {state.x, state.y, state.z, state.w};
        float h[4], out = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const float next = __builtin_fmaf(exp2_fast(size * a4[m]), begin ? 0.0f : old[m], u * Elem<E>::up(b.v[m]));
            h[m] = alive ? next : old[m];
            out = __builtin_fmaf(next, Elem<E>::up(c.v[m]), out);
        }
        const int e = i;
        if (i + p.part < p.n) load(i + p.part);
        out += dpp<DPP_XOR1>(out);
        if constexpr (QUADS >= 4) out += dpp<DPP_XOR2>(out);
        if constexpr (QUADS >= 8) out += dpp<DPP_HALF_MIRROR>(out);
        out = __builtin_fmaf(skip, input, out);
        if (gate) out *= gated * sigmoid(gated);
        if (on) {
            if (p.state_out) {
                Four* q = reinterpret_cast<Four*>(p.state_out + ((int64_t)e * per_env + rest) * 4);
                const Four v = {h[0], h[1], h[2], h[3]};
                if (STREAMED) __builtin_nontemporal_store(v, q);
                else *q = v;
            }
            if (quad == 0) p.y.at(0, e)[channel] = Elem<E>::down(alive ? out : 0.0f);
        }
    }
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
    if (a->steps > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "steps must be below 2^31 - 4095", why);
    if ((int64_t)a->n * a->channels > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "n * channels must be below 2^31 - 4095", why);
    const craftax_view* need[] = {&a->x, &a->delta, &a->b, &a->c};
    for (const craftax_view* v : need)
        if (!v->data) return refuse(CRAFTAX_E_NULL, "x, delta, b or c is NULL", why);
    if (!a->a) return refuse(CRAFTAX_E_NULL, "a is NULL", why);
    const size_t e = elem_bytes(a->dtype);
    const craftax_view* all[] = {&a->x, &a->delta, &a->z, &a->b, &a->c};
    for (const craftax_view* v : all)
        if (!aligned(v->data, e)) return refuse(CRAFTAX_E_ALIGN, "an activation is not aligned to its elements", why);
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
    t.group_tiles = (int)ceil_div(t.group_channels, WAVE / (a->states / 4));
    t.tiles = t.group_tiles * a->groups;
    return t;
}

// Steps per part, whole blocks of steps, for about `want` parts.
struct ScanParts { int part, parts; };
static ScanParts scan_parts(const craftax_scan_args* a, int64_t want)
{
    if (want < 2 || a->steps < 4 * BLOCK) return {a->steps, 1};
    int64_t part = ceil_div(ceil_div(a->steps, want), BLOCK) * BLOCK;
    if (part < 2 * BLOCK) part = 2 * BLOCK;
    if (ceil_div(a->steps, part) > 65535) part = ceil_div(ceil_div(a->steps, 65535), BLOCK) * BLOCK;
    const int64_t parts = ceil_div(a->steps, part);
    return parts == 1 ? ScanParts{a->steps, 1} : ScanParts{(int)part, (int)parts};
}

// Parts that are few enough for every wavefront to go through them: 5 parts 28 us where the kernel between made it 37, 32 parts 41
// and 42, 53 parts 29 and 29.
constexpr int OWN_STARTS = 32;
static unsigned carry_threads(int parts) { return (unsigned)(parts < CARRY_WAVES ? parts : CARRY_WAVES) * WAVE; }

// States above this size (three quarters of the last-level cache) would push each other out of it between two tokens: 268 MB
// streamed 106 us, through the caches 117, 2.1 GB 924 and 998; below it a token finds the state of the one before
// (33 MB through the caches 12.6 us, streamed 14.8).
constexpr int64_t TOKEN_STREAMED = (int64_t)192 << 20;
// Wavefronts that a launch is to have for a full chip.  Registers leave room for five per SIMD of k_scan, but a block is eight or none, so
// that four are there at once and the last parts of a split sequence follow behind the others.
constexpr int64_t SCAN_FILL = (int64_t)CHIP_SIMDS * 5;
constexpr int64_t SCAN_BACK_FILL = (int64_t)CHIP_SIMDS * 2;      // k_scan_back: what is there at once,
constexpr int64_t TOKEN_FILL = (int64_t)CHIP_SIMDS * 8;          // k_scan_token: too

static bool scan_shape_ok(const craftax_scan_args* a)
{
    return a && (a->states == 8 || a->states == 16 || a->states == 32) && a->steps >= 1 && a->n >= 1 && a->channels >= 1 && a->groups >= 1 &&
           a->channels % a->groups == 0 && a->dtype <= CRAFTAX_F16;
}

// the states of all environments, tiled
static size_t tile_bytes(const craftax_scan_args* a, int tiles) { return (size_t)a->n * tiles * WAVE * sizeof(float4); }

size_t scan_saved_bytes(const craftax_scan_args* a)
{
    if (!scan_shape_ok(a)) return 0;
    return (size_t)ceil_div(a->steps, BLOCK) * tile_bytes(a, scan_tiles(a).tiles);
}

// What lies where in a workspace.
struct ScanSpace { ScanParts parts; size_t starts, decays, shared, weights, bytes; int rows, waves, group_blocks; };
static ScanSpace scan_space(const craftax_scan_args* a, bool backward)
{
    const ScanTiles t = scan_tiles(a);
    ScanSpace s{};
    if (backward) {
        // wavefronts of a block: as many as leave no more than a fifth of them without a tile, and fewer where more
        // parts of smaller blocks fit, which are shorter by a fifth at least (333 steps of 19 environments of 200 channels and 32
        // states: 73 us with blocks of two in four parts, 84 with blocks of four in three)
        s.waves = SCAN_BACK_WAVES;
        while (s.waves > 1 && ceil_div(t.group_tiles, s.waves) * s.waves * 4 > t.group_tiles * 5) s.waves /= 2;
        // Blocks are to be there all at once: a few more than that take twice the time.  Too few environments are split into parts
        // (the walk before costs a third); of too many, a block takes several one after the other, which also keeps the rows
        // of partial sums few.
        int64_t room, each;
        auto split = [&](int waves) {
            room = SCAN_BACK_FILL / waves;
            each = (int64_t)a->groups * ceil_div(t.group_tiles, waves);
            return scan_parts(a, room / (each * a->n));
        };
        s.parts = split(s.waves);
        while (s.waves > 1 && s.parts.parts > 1) {
            const ScanParts half = split(s.waves / 2);
            if (half.part * 5 > s.parts.part * 4) break;
            s.waves /= 2;
            s.parts = half;
        }
        s.parts = split(s.waves);           // room and each are those of the blocks taken
        s.group_blocks = (int)ceil_div(t.group_tiles, s.waves);
        const int64_t side = each < room ? room / each : 1, turns = ceil_div(a->n, side);
        s.rows = (int)ceil_div(a->n, turns) * s.parts.parts;
    } else {
        // Split steps cost the recurrence of the states twice, 1.7 times the work: sequences that fill a quarter of the chip are not split
        // (100 steps of 64 environments of 512 channels: 24 us, in two parts 46; 1,000 steps of them 162, in parts for two or four times
        // the wavefronts 198).  The line is between sizes, not at the best of each: 1,000 steps of 37 ragged environments of 648 channels
        // are not split, 173 us, and take 152 in such parts.
        const int64_t want = SCAN_FILL / ((int64_t)a->n * t.tiles);
        s.parts = scan_parts(a, want < 4 ? 1 : want);
    }
    size_t at = 0;
    if (s.parts.parts > 1) {
        s.starts = at;
        at += round256((size_t)s.parts.parts * tile_bytes(a, t.tiles));
        s.decays = at;
        at += round256((size_t)s.parts.parts * a->n * t.tiles * (WAVE / (a->states / 4)) * sizeof(float2));
    }
    if (backward) {
        s.shared = at;
        at += round256((size_t)a->steps * a->n * a->groups * s.group_blocks * 2 * a->states * sizeof(float));
        s.weights = at;
        at += round256((size_t)s.rows * a->channels * (a->states + 2) * sizeof(float));
    }
    s.bytes = at;
    return s;
}

size_t scan_workspace_bytes(const craftax_scan_args* a, bool backward)
{
    if (!scan_shape_ok(a)) return 0;
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

// whether the kernel for one token takes the call
static bool scan_token(const craftax_scan_args* a) { return a->steps == 1 && !a->saved && token_fits(a->channels, a->states); }

int scan(const craftax_scan_args* a, void* stream, const char** why)
{
    if (int rc = scan_check(a, false, why)) return rc;
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, scan_workspace_bytes(a, false), why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    int rc = CRAFTAX_OK;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        ScanParams<E> p = scan_params<E>(a);
        with_states(a->states, [&](auto states) {
            constexpr int N = decltype(states)::value;
            if (scan_token(a)) {
                // environments side by side: as many threads as the chip holds, each with several of them in turn, or all
                const int64_t per_env = (int64_t)a->channels * (N / 4);
                p.part = side_by_side(ceil_div(TOKEN_FILL * WAVE, per_env), a->n);
                const dim3 grid((unsigned)ceil_div(p.part * per_env, SCAN_THREADS));
                if (a->n * per_env * (int64_t)sizeof(float4) > TOKEN_STREAMED) hipLaunchKernelGGL((k_scan_token<E, N, true>), grid, dim3(SCAN_THREADS), 0, st, p);
                else hipLaunchKernelGGL((k_scan_token<E, N, false>), grid, dim3(SCAN_THREADS), 0, st, p);
                rc = launched(why);
                return;
            }
            const ScanSpace s = scan_space(a, false);
            char* base = static_cast<char*>(a->workspace);
            p.part = s.parts.part; p.parts = s.parts.parts;
            const Spread blocks = spread(ceil_div((int64_t)a->n * p.tiles, SCAN_WAVES), SCAN_THREADS);
            const dim3 grid(blocks.x, (unsigned)p.parts, blocks.z);
            p.wide = blocks.x;
            if (p.parts > 1) {
                p.starts = reinterpret_cast<float4*>(base + s.starts);
                p.decays = reinterpret_cast<float2*>(base + s.decays);
                hipLaunchKernelGGL((k_scan<E, N, PART_ONLY, false>), dim3(blocks.x, (unsigned)p.parts - 1, blocks.z), dim3(SCAN_THREADS), 0, st, p);
                if ((rc = launched(why))) return;
                // a state that is written in place is not there any more when the last parts ask for it
                p.own_starts = p.parts <= OWN_STARTS && !(p.state_in && p.state_in == p.state_out);
                if (!p.own_starts) hipLaunchKernelGGL((k_scan_carry<E, N, false>), dim3((unsigned)(a->n * p.tiles)), dim3(carry_threads(p.parts)), 0, st, p);
                if ((rc = launched(why))) return;
            }
            if (p.saved && p.z.data) hipLaunchKernelGGL((k_scan<E, N, SAVE, true>), grid, dim3(SCAN_THREADS), 0, st, p);
            else if (p.saved) hipLaunchKernelGGL((k_scan<E, N, SAVE, false>), grid, dim3(SCAN_THREADS), 0, st, p);
            else if (p.z.data) hipLaunchKernelGGL((k_scan<E, N, RUN, true>), grid, dim3(SCAN_THREADS), 0, st, p);
            else hipLaunchKernelGGL((k_scan<E, N, RUN, false>), grid, dim3(SCAN_THREADS), 0, st, p);
            rc = launched(why);
        });
    });
    return rc;
}

int scan_backward(const craftax_scan_args* a, void* stream, const char** why)
{
    if (int rc = scan_check(a, true, why)) return rc;
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, scan_workspace_bytes(a, true), why)) return rc;
    const hipStream_t st = (hipStream_t)stream;
    const ScanSpace s = scan_space(a, true);
    int rc = CRAFTAX_OK;
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        ScanParams<E> p = scan_params<E>(a);
        char* base = static_cast<char*>(a->workspace);
        p.part = s.parts.part; p.parts = s.parts.parts; p.rows = s.rows; p.group_blocks = s.group_blocks;
        p.starts = reinterpret_cast<float4*>(base + s.starts);
        p.decays = reinterpret_cast<float2*>(base + s.decays);
        p.shared_part = reinterpret_cast<float*>(base + s.shared);
        p.weight_part = reinterpret_cast<float*>(base + s.weights);
        with_states(a->states, [&](auto states) {
            constexpr int N = decltype(states)::value;
            if (p.parts > 1) {
                const Spread blocks = spread(ceil_div((int64_t)a->n * p.tiles, SCAN_WAVES), SCAN_THREADS);
                p.wide = blocks.x;
                hipLaunchKernelGGL((k_scan_back_part<E, N>), dim3(blocks.x, (unsigned)p.parts - 1, blocks.z), dim3(SCAN_THREADS), 0, st, p);
                if ((rc = launched(why))) return;
                p.own_starts = p.parts <= OWN_STARTS;
                if (!p.own_starts) hipLaunchKernelGGL((k_scan_carry<E, N, true>), dim3((unsigned)(a->n * p.tiles)), dim3(carry_threads(p.parts)), 0, st, p);
                if ((rc = launched(why))) return;
            }
            const Spread blocks = spread((int64_t)(s.rows / p.parts) * a->groups * s.group_blocks, s.waves * WAVE);
            const dim3 grid(blocks.x, (unsigned)p.parts, blocks.z);
            p.wide = blocks.x;
            if (p.z.data) hipLaunchKernelGGL((k_scan_back<E, N, true>), grid, dim3(s.waves * WAVE), s.waves * scan_back_lds<N>(), st, p);
            else hipLaunchKernelGGL((k_scan_back<E, N, false>), grid, dim3(s.waves * WAVE), s.waves * scan_back_lds<N>(), st, p);
            if ((rc = launched(why))) return;
            const Spread sums = spread(ceil_div((int64_t)a->steps * a->n * a->groups * 2 * N, SCAN_THREADS), SCAN_THREADS);
            p.wide = sums.x;
            hipLaunchKernelGGL((k_scan_shared<E, N>), dim3(sums.x, 1, sums.z), dim3(SCAN_THREADS), 0, st, p, seq<E>(a->db), seq<E>(a->dc));
            if ((rc = launched(why))) return;
            sum_rows(p.weight_part, s.rows, (int64_t)a->channels * (N + 2), PutScan<N>{a->da, a->dd, a->ddelta_bias}, st);
            rc = launched(why);
        });
    });
    return rc;
}

}  // namespace host
}  // namespace mem
