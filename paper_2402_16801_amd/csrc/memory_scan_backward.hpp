// Backward pass of the scan (part of memory_scan.hip).
//
// With g = dL/dh, walking back in time:
//   g   = c dy + (exp(D a) g of the step after it, 0 where an episode begins there)
//   dc  = sum over channels of dy h              db = sum over channels of g D x
//   dx  = D (g . b) + d dy                       dD = x (g . b) + sum over states of g a (exp(D a) h before)
//   da  = sum over steps of D g (exp(D a) h before)
// and dy here is dy z sigmoid(z) with a gate, dz = dy (c . h + d x) (z sigmoid(z))'.
//
// The layout is the forward pass's.  The states of a block of eight steps are computed again from the saved one
// and held in registers, as the decay exp(D a) and what decayed of the state before, from which h itself is
// one multiplication and addition away.  The sums over channels fold eight values (four states of db and dc)
// over the wavefront's channels, halving values and lanes at once; the wavefronts of a block, tiles of one group,
// meet in LDS once per block of steps, and what the blocks of a group leave is added up by a second kernel.
// The order is fixed, there are no atomics.

constexpr int SCAN_BACK_WAVES = 8;       // wavefronts of a block at most
constexpr int DPP_SHL4 = 0x104;

// Sums of v over the channels of the wavefront.  Value k ends in the lanes with fold_value(lane) == k that
// fold_writes<LANES>(lane) (the sums in the other lanes are not complete).
template <int LANES>
__device__ __forceinline__ float fold_channels(float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) { const Pair q = swap32(v[k], v[k + 4]); v[k] = q.a + q.b; }
#pragma unroll
    for (int k = 0; k < 2; ++k) { const Pair q = swap16(v[k], v[k + 2]); v[k] = q.a + q.b; }
    const float a = v[0] + dpp<DPP_ROR8>(v[0]), b = v[1] + dpp<DPP_ROR8>(v[1]);
    float r = threadIdx.x & 8 ? b : a;
    if constexpr (LANES <= 4) r += dpp<DPP_SHL4>(r);
    if constexpr (LANES <= 2) r += dpp<DPP_XOR2>(r);
    return r;
}
__device__ __forceinline__ int fold_value(int lane) { return (lane >> 5 & 1) * 4 + (lane >> 4 & 1) * 2 + (lane >> 3 & 1); }
template <int LANES> __device__ __forceinline__ bool fold_writes(int lane)
{
    return LANES == 8 || (LANES == 4 ? (lane & 4) == 0 : (lane & 6) == 0);
}

// LDS of a wavefront: b and c of a block of steps, what a step needs of each channel, and two turns of sums for db and dc.
template <int N> constexpr size_t scan_back_lds()
{
    return BLOCK * 2 * N * sizeof(float) + BLOCK * Lay<N>::CHANNELS * sizeof(float4) + 2 * BLOCK * 2 * N * sizeof(float);
}

template <typename E, int N>
__global__ __launch_bounds__(SCAN_BACK_WAVES* WAVE) __attribute__((amdgpu_waves_per_eu(2))) void k_scan_back(const ScanParams<E> p)
{
    constexpr int LANES = Lay<N>::LANES, CHANNELS = Lay<N>::CHANNELS, OWN = Lay<N>::OWN;
    extern __shared__ float4 lds[];
    const int lane = (int)(threadIdx.x & (WAVE - 1)), mine = lane / LANES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    float4* shared_lds = lds + wave * (BLOCK * N / 2);                                   // [step][2 N] floats
    float4* step_lds = lds + p.waves * (BLOCK * N / 2) + wave * (BLOCK * CHANNELS);      // [step][channel]: D, D x, dy, x
    float* sum_lds = reinterpret_cast<float*>(lds + p.waves * (BLOCK * N / 2 + BLOCK * CHANNELS));   // [turn][wave][step][2 N]
    const int group_block = (int)(blockIdx.x % (unsigned)(p.groups * p.group_blocks));
    const int env_row = (int)(blockIdx.x / (unsigned)(p.groups * p.group_blocks)), env_rows = p.rows / p.parts;
    const int group = group_block / p.group_blocks, in_group = (group_block % p.group_blocks) * p.waves + wave;
    const bool works = in_group < p.group_tiles;          // the other wavefronts only keep the barriers
    const Tile w = tile_of<N>(p, group * p.group_tiles + (works ? in_group : p.group_tiles - 1));
    const bool owns = works && w.owns;
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    float a2[4], g[4], da[4], dd = 0.0f, dbias = 0.0f;
    load_rates<N>(p.a, w, a2);
    zero(da);
    const float skip = p.d ? p.d[w.channel] : 0.0f;
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    const int slot = fold_value(lane) / 4 * N + w.quad * 4 + fold_value(lane) % 4;       // among the 2 N sums of a step
    const int own = w.quad * OWN;
    int turn = 0;
    for (int i = env_row; i < p.n; i += env_rows) {
        const int length = scan_length(p, i);
        const int end = t1 < length ? t1 : length;
        const int dead = t0 > end ? t0 : end;
        if (owns)
            for (int t = dead + w.quad; t < t1; t += LANES) {
                p.dx.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                p.ddelta.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                if (p.z.data) p.dz.at(t, i)[w.channel] = Elem<E>::down(0.0f);
            }
        for (int q = (int)threadIdx.x; q < (t1 - dead) * 2 * N; q += p.waves * WAVE)
            p.shared_part[(((int64_t)(dead + q / (2 * N)) * p.n + i) * (p.groups * p.group_blocks) + group_block) * (2 * N) + q % (2 * N)] = 0.0f;
        if (p.parts > 1) load4(tiled(p.starts, (int64_t)part * p.n + i, w, p.tiles), g);
        else if (p.dstate_out) load4(state_of<N>(p.dstate_out, p.channels, i, w), g);
        else zero(g);
        int t = t0 + (end - t0 - 1) / BLOCK * BLOCK;       // the last block of steps
        Walk<const E> at_x, at_delta, at_dy, at_z;
        Walk<E> at_dx, at_ddelta, at_dz;
        WalkShared<E, N> at_shared;
        at_x.template start<N>(p.x, t, i, w);
        at_delta.template start<N>(p.delta, t, i, w);
        at_dy.template start<N>(p.dy, t, i, w);
        at_z.template start<N>(p.z, t, i, w);
        at_dx.template start<N>(p.dx, t, i, w);
        at_ddelta.template start<N>(p.ddelta, t, i, w);
        at_dz.template start<N>(p.dz, t, i, w);
        at_shared.start(p, t, i, w);
        const float4* at_saved = tiled(p.saved, (int64_t)(t / BLOCK) * p.n + i, w, p.tiles);
        float next_x[OWN], next_delta[OWN], next_dy[OWN], next_z[OWN], shared[LANES], next_h[4];
        auto fetch = [&](int count) {
            at_shared.load(count, shared);
            at_x.load(own, count, next_x);
            at_delta.load(own, count, next_delta);
            at_dy.load(own, count, next_dy);
            if (p.z.data) at_z.load(own, count, next_z);
            load4(at_saved, next_h);
            at_shared.move(-BLOCK);
            at_x.move(-BLOCK);
            at_delta.move(-BLOCK);
            at_dy.move(-BLOCK);
            at_z.move(-BLOCK);
            at_saved -= (int64_t)p.n * p.tiles * WAVE;
        };
        if (t0 < end) fetch(end - t);
        for (; t0 < end && t >= t0; t -= BLOCK) {
            const int count = end - t < BLOCK ? end - t : BLOCK;
            const uint32_t starts = (uint32_t)begins(p, t, t + count, i);
            float slope[OWN], dz[OWN], h[4];
            wave_fence();
            stage_shared<N>(reinterpret_cast<float*>(shared_lds), shared);
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const float pre = next_delta[k] + bias;
                const float size = p.softplus ? softplus(pre) : pre;
                slope[k] = p.softplus ? sigmoid(pre) : 1.0f;
                float dout = next_dy[k];
                if (p.z.data) {
                    const float s = sigmoid(next_z[k]);
                    dz[k] = dout * (s * __builtin_fmaf(next_z[k], 1.0f - s, 1.0f));
                    dout *= next_z[k] * s;
                }
                // steps behind the end and channels that are none add nothing
                step_lds[(own + k) * CHANNELS + mine] = owns && own + k < count ? make_float4(size, size * next_x[k], dout, next_x[k])
                                                                               : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) h[m] = next_h[m];
            wave_fence();
            if (t > t0) fetch(BLOCK);
            // the states of these steps again: the decays, and what decayed of the state before
            float decay[BLOCK][4], kept[BLOCK][4], y[BLOCK];
#pragma unroll
            for (int k = 0; k < BLOCK; ++k) {
                const float4 step = step_lds[k * CHANNELS + mine];
                float b[4];
                load4(&shared_lds[k * (N / 2) + w.quad], b);
                if (starts >> k & 1u) zero(h);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    decay[k][m] = exp2_fast(step.x * a2[m]);
                    kept[k][m] = decay[k][m] * h[m];
                    h[m] = __builtin_fmaf(step.y, b[m], kept[k][m]);
                }
                if (p.z.data) {
                    float c[4];
                    load4(&shared_lds[k * (N / 2) + N / 4 + w.quad], c);
                    y[k] = h[0] * c[0];
#pragma unroll
                    for (int m = 1; m < 4; ++m) y[k] = __builtin_fmaf(h[m], c[m], y[k]);
                }
                if (p.z.data) pin(y[k]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (p.z.data) {
                fold_steps<LANES>(y);
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    const float x = step_lds[(own + k) * CHANNELS + mine].w;
                    if (owns && own + k < count) at_dz.at[k * at_dz.step] = Elem<E>::down(dz[k] * __builtin_fmaf(skip, x, y[k]));
                }
            }
            wave_fence();       // what is in LDS is read again rather than kept in registers: 64 more of them
            float gb[BLOCK], rate[BLOCK];
            float* sums = sum_lds + (turn * p.waves + wave) * (BLOCK * 2 * N);
#pragma unroll
            for (int k = BLOCK - 1; k >= 0; --k) {
                const float4 step = step_lds[k * CHANNELS + mine];
                float b[4], c[4], v[8];
                load4(&shared_lds[k * (N / 2) + w.quad], b);
                load4(&shared_lds[k * (N / 2) + N / 4 + w.quad], c);
                gb[k] = rate[k] = 0.0f;
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    v[4 + m] = step.z * __builtin_fmaf(step.y, b[m], kept[k][m]);
                    const float gm = __builtin_fmaf(c[m], step.z, g[m]);
                    v[m] = gm * step.y;
                    gb[k] = __builtin_fmaf(gm, b[m], gb[k]);
                    const float through = gm * kept[k][m];
                    rate[k] = __builtin_fmaf(through, a2[m], rate[k]);
                    da[m] = __builtin_fmaf(through, step.x, da[m]);
                    g[m] = decay[k][m] * gm;
                }
                if (starts >> k & 1u) zero(g);
                const float folded = fold_channels<LANES>(v);
                if (fold_writes<LANES>(lane)) sums[k * 2 * N + slot] = works ? folded : 0.0f;
                // all of a step is done in its turn: put off to the end, the sums would keep every step's factors in registers
                pin(gb[k]);
                pin(rate[k]);
#pragma unroll
                for (int m = 0; m < 4; ++m) pin(da[m]);
                __builtin_amdgcn_sched_barrier(0);
            }
            wave_fence();
            fold_steps<LANES>(gb);
            fold_steps<LANES>(rate);
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const float4 step = step_lds[(own + k) * CHANNELS + mine];
                const float dsize = slope[k] * __builtin_fmaf(gb[k], step.w, rate[k] * (1.0f / LOG2E));
                if (owns && own + k < count) {
                    dd = __builtin_fmaf(step.z, step.w, dd);
                    dbias += dsize;
                    at_dx.at[k * at_dx.step] = Elem<E>::down(__builtin_fmaf(gb[k], step.x, skip * step.z));
                    at_ddelta.at[k * at_ddelta.step] = Elem<E>::down(dsize);
                }
            }
            at_dx.move(-BLOCK);
            at_ddelta.move(-BLOCK);
            at_dz.move(-BLOCK);
            __syncthreads();
            // sums over the block's wavefronts; the next turn writes the other half, so one barrier is enough
            const float* from = sum_lds + turn * p.waves * (BLOCK * 2 * N);
            for (int q = (int)threadIdx.x; q < count * 2 * N; q += p.waves * WAVE) {
                float s = from[q];
                for (int v = 1; v < p.waves; ++v) s += from[v * (BLOCK * 2 * N) + q];
                p.shared_part[(((int64_t)(t + q / (2 * N)) * p.n + i) * (p.groups * p.group_blocks) + group_block) * (2 * N) + q % (2 * N)] = s;
            }
            turn ^= 1;
        }
        if (p.parts == 1 && p.dstate_in && owns) store4(state_of<N>(p.dstate_in, p.channels, i, w), g);
    }
    // a channel's lanes hold the sums of their own steps
    dd += dpp<DPP_XOR1>(dd);
    dbias += dpp<DPP_XOR1>(dbias);
    if constexpr (LANES >= 4) { dd += dpp<DPP_XOR2>(dd); dbias += dpp<DPP_XOR2>(dbias); }
    if constexpr (LANES >= 8) { dd += dpp<DPP_HALF_MIRROR>(dd); dbias += dpp<DPP_HALF_MIRROR>(dbias); }
    if (owns) {
        float* row = p.weight_part + ((int64_t)(part * env_rows + env_row) * p.channels + w.channel) * (N + 2);
#pragma unroll
        for (int m = 0; m < 4; ++m) row[w.quad * 4 + m] = da[m];
        if (w.quad == 0) { row[N] = dd; row[N + 1] = dbias; }
    }
}

// What a part does to the gradient of the state that comes from behind it: see k_scan with PART.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_back_part(const ScanParams<E> p)
{
    constexpr int LANES = Lay<N>::LANES, CHANNELS = Lay<N>::CHANNELS, OWN = Lay<N>::OWN;
    __shared__ float4 shared_lds[SCAN_WAVES][BLOCK * N / 2];
    __shared__ float2 step_lds[SCAN_WAVES][BLOCK * CHANNELS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + wave;
    if (item >= (int64_t)p.n * p.tiles) return;
    const int i = (int)(item / p.tiles);
    const Tile w = tile_of<N>(p, (int)(item % p.tiles));
    const int mine = (int)(threadIdx.x & (WAVE - 1)) / LANES;
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    const int length = scan_length(p, i);
    const int end = t1 < length ? t1 : length;
    float a2[4], g[4];
    load_rates<N>(p.a, w, a2);
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    zero(g);
    float total = 0.0f, cut = 0.0f;
    const int own = w.quad * OWN;
    int t = t0 + (end - t0 - 1) / BLOCK * BLOCK;
    Walk<const E> at_delta, at_dy, at_z;
    WalkShared<E, N> at_shared;
    at_delta.template start<N>(p.delta, t, i, w);
    at_dy.template start<N>(p.dy, t, i, w);
    at_z.template start<N>(p.z, t, i, w);
    at_shared.start(p, t, i, w);
    for (; t0 < end && t >= t0; t -= BLOCK) {
        const int count = end - t < BLOCK ? end - t : BLOCK;
        const uint32_t starts = (uint32_t)begins(p, t, t + count, i);
        float shared[LANES], delta[OWN], dy[OWN], z[OWN];
        at_shared.load(count, shared);
        at_delta.load(own, count, delta);
        at_dy.load(own, count, dy);
        if (p.z.data) at_z.load(own, count, z);
        at_shared.move(-BLOCK);
        at_delta.move(-BLOCK);
        at_dy.move(-BLOCK);
        at_z.move(-BLOCK);
        float2 step[OWN];
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            float size = delta[k] + bias;
            if (p.softplus) size = softplus(size);
            if (p.z.data) dy[k] *= z[k] * sigmoid(z[k]);
            step[k] = own + k < count ? make_float2(size, dy[k]) : make_float2(0.0f, 0.0f);
        }
        wave_fence();
        stage_shared<N>(reinterpret_cast<float*>(shared_lds[wave]), shared);
#pragma unroll
        for (int k = 0; k < OWN; ++k) step_lds[wave][(own + k) * CHANNELS + mine] = step[k];
        wave_fence();
#pragma unroll
        for (int k = BLOCK - 1; k >= 0; --k) {
            const float2 s = step_lds[wave][k * CHANNELS + mine];
            float c[4];
            load4(&shared_lds[wave][k * (N / 2) + N / 4 + w.quad], c);
            total += s.x;
#pragma unroll
            for (int m = 0; m < 4; ++m) g[m] = exp2_fast(s.x * a2[m]) * __builtin_fmaf(c[m], s.y, g[m]);
            if (starts >> k & 1u) { zero(g); total = 0.0f; cut = 1.0f; }
        }
    }
    const int64_t index = (int64_t)part * p.n + i;
    store4(tiled(p.starts, index, w, p.tiles), g);
    if (w.quad == 0) p.decays[(index * p.tiles + w.tile) * CHANNELS + mine] = make_float2(total, cut);
}

// db and dc: the blocks of a group added up
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_shared(const ScanParams<E> p, Seq<E> db, Seq<E> dc)
{
    const int64_t at = (int64_t)blockIdx.x * SCAN_THREADS + threadIdx.x;
    const int value = (int)(at % (2 * N));
    const int64_t row = at / (2 * N);                  // (step, environment, group)
    if (row >= (int64_t)p.steps * p.n * p.groups) return;
    const int group = (int)(row % p.groups);
    const int64_t token = row / p.groups;
    const float* q = p.shared_part + row * p.group_blocks * (2 * N) + value;
    float s = 0.0f;
    for (int k = 0; k < p.group_blocks; ++k) s += q[(int64_t)k * (2 * N)];
    const int t = (int)(token / p.n), i = (int)(token % p.n);
    if (value < N) db.at(t, i)[group * N + value] = Elem<E>::down(s);
    else dc.at(t, i)[group * N + value - N] = Elem<E>::down(s);
}

// da, dd and ddelta_bias from columns [channels][N + 2]
template <int N> struct PutScan {
    float *da, *dd, *ddelta_bias;
    __device__ void operator()(int64_t column, float v) const
    {
        const int channel = (int)(column / (N + 2)), value = (int)(column % (N + 2));
        if (value < N) da[(int64_t)channel * N + value] = v;
        else if (value == N) { if (dd) dd[channel] = v; }
        else if (ddelta_bias) ddelta_bias[channel] = v;
    }
};
