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
//
// Bound by vector issue: about 105 instructions per step of a wavefront (16 channels of 16 states), of which 20 are the states again
// and 20 the sums over channels, at two wavefronts per SIMD, what some 230 registers leave room for.  64 steps of 4,096 environments of
// 512 channels in bfloat16 with a gate: 2,050 us, and 50 for the second kernel.

constexpr int SCAN_BACK_WAVES = 8;       // wavefronts of a block at most
// The sums for da, dd and ddelta_bias over so many steps are added up apart before they join a wavefront's total: over
// 64 steps of 4,096 environments one running sum leaves da 1.1e-6 off, this 2.7e-7 (both relative), in the same time.
constexpr int SCAN_BACK_SPAN = 64;

// Two values each to the halves of a row of 16 lanes (bank masks name the quarters that an addition writes): lanes with bit 3
// clear get a's sum over bit 3, the others b's.  Then the same with bit 2.  Nothing else may stand between the
// instructions' registers and the moves across lanes that read them for two wait states, hence the s_nop.
__device__ __forceinline__ void fold_bit3(const float (&v)[8], float (&t)[4])
{
    asm("s_nop 1\n\t"
        "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %0, %8, %8 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %1, %9, %9 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %2, %6, %6 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %2, %10, %10 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %3, %7, %7 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %3, %11, %11 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "s_nop 1"
        : "=&v"(t[0]), "=&v"(t[1]), "=&v"(t[2]), "=&v"(t[3])
        : "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]));
}
__device__ __forceinline__ void fold_bit2(const float (&t)[4], float (&r)[2])
{
    asm("s_nop 1\n\t"
        "v_add_f32_dpp %0, %2, %2 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %0, %4, %4 row_shr:4 row_mask:0xf bank_mask:0xa\n\t"
        "v_add_f32_dpp %1, %3, %3 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %1, %5, %5 row_shr:4 row_mask:0xf bank_mask:0xa\n\t"
        "s_nop 1"
        : "=&v"(r[0]), "=&v"(r[1])
        : "v"(t[0]), "v"(t[1]), "v"(t[2]), "v"(t[3]));
}

// Sums of v over the channels of the wavefront.  Value k ends in the lanes with fold_value<LANES>(lane) == k that
// fold_writes<LANES>(lane).
template <int LANES>
__device__ __forceinline__ float fold_channels(const float (&v)[8])
{
    float t[4], r[2];
    fold_bit3(v, t);
    Pair q;
    if constexpr (LANES == 8) {
#pragma unroll
        for (int k = 0; k < 2; ++k) { q = swap16(t[k], t[k + 2]); r[k] = q.a + q.b; }
        q = swap32(r[0], r[1]);
        return q.a + q.b;
    } else {
        fold_bit2(t, r);
        q = swap16(r[0], r[1]);
        float s = q.a + q.b;
        q = swap32(s, s);
        s = q.a + q.b;
        if constexpr (LANES == 2) s += dpp<DPP_XOR2>(s);
        return s;
    }
}
template <int LANES> __device__ __forceinline__ int fold_value(int lane)
{
    return (lane >> 3 & 1) * 4 + (LANES == 8 ? (lane >> 4 & 1) * 2 + (lane >> 5 & 1) : (lane >> 2 & 1) * 2 + (lane >> 4 & 1));
}
template <int LANES> __device__ __forceinline__ bool fold_writes(int lane)
{
    return LANES == 8 || (LANES == 4 ? (lane & 32) == 0 : (lane & 34) == 0);
}

// LDS of a wavefront: b and c of a block of steps, what a step needs of each channel, and two turns of sums for db and dc.
template <int N> constexpr size_t scan_back_lds()
{
    return BLOCK * 2 * N * sizeof(float) + BLOCK * Lay<N>::CHANNELS * sizeof(float4) + 2 * BLOCK * 2 * N * sizeof(float);
}

// The arguments, read anew: strides and addresses that only the turn to another environment needs are not kept in scalar
// registers, of which they would take more than there are.
template <typename E> __device__ __forceinline__ const ScanParams<E>& arguments_again()
{
    uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const ScanParams<E>*)(const __attribute__((address_space(4))) void*)at;
}

template <typename E, int N, bool GATE>
__global__ __launch_bounds__(SCAN_BACK_WAVES* WAVE) __attribute__((amdgpu_waves_per_eu(2))) void k_scan_back(const ScanParams<E> given)
{
    constexpr int LANES = Lay<N>::LANES, CHANNELS = Lay<N>::CHANNELS, OWN = Lay<N>::OWN, SUMS = BLOCK * 2 * N;
    extern __shared__ float4 lds[];
    const int lane = (int)(threadIdx.x & (WAVE - 1)), mine = lane / LANES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), waves = (int)blockDim.x / WAVE;
    float4* shared_lds = lds + wave * (BLOCK * N / 2);                                   // [step][2 N] floats
    float4* step_lds = lds + waves * (BLOCK * N / 2) + wave * (BLOCK * CHANNELS);        // [step][channel]: D, D x, dy, x
    float* sum_lds = reinterpret_cast<float*>(lds + waves * (BLOCK * N / 2 + BLOCK * CHANNELS));   // [turn][wave][step][2 N]
    const int blocks = given.groups * given.group_blocks;
    const unsigned block = (unsigned)spread_block(given.wide);
    const int group_block = (int)(block % (unsigned)blocks);
    const int env_row = (int)(block / (unsigned)blocks), env_rows = given.rows / given.parts;
    if (env_row >= env_rows) return;
    const int group = group_block / given.group_blocks, in_group = (group_block % given.group_blocks) * waves + wave;
    const bool works = in_group < given.group_tiles;          // the other wavefronts only keep the barriers
    const Tile w = tile_of<N>(given, group * given.group_tiles + (works ? in_group : given.group_tiles - 1));
    const bool owns = works && w.owns;
    const int part = (int)blockIdx.y;
    float a2[4], g[4], da[4], dd = 0.0f, dbias = 0.0f, da_span[4], dd_span = 0.0f, dbias_span = 0.0f;
    load_rates<N>(given.a, w, a2);
    zero(da);
    zero(da_span);
    const float skip = given.d ? given.d[w.channel] : 0.0f;
    const float bias = given.delta_bias ? given.delta_bias[w.channel] : 0.0f;
    const int slot = fold_value<LANES>(lane) / 4 * N + w.quad * 4 + fold_value<LANES>(lane) % 4;       // among the 2 N sums of a step
    const int own = w.quad * OWN;
    // the sums of a step that this thread adds up over the block's wavefronts, and how many steps it goes on
    const int sum_row = (int)threadIdx.x / (2 * N), sum_value = (int)threadIdx.x % (2 * N), sum_rows = (int)blockDim.x / (2 * N);
    int turn = 0;
    for (int i = env_row; i < given.n; i += env_rows) {
        const ScanParams<E>& p = arguments_again<E>();
        const int t0 = part * p.part, t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
        const int length = scan_length(p, i);
        const int end = t1 < length ? t1 : length;
        const int dead = t0 > end ? t0 : end;
        if (owns)
            for (int t = dead + w.quad; t < t1; t += LANES) {
                p.dx.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                p.ddelta.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                if (GATE) p.dz.at(t, i)[w.channel] = Elem<E>::down(0.0f);
            }
        const int64_t sum_step = (int64_t)p.n * blocks * (2 * N);          // from one step's sums to the next one's
        float* at_sums = p.shared_part + ((int64_t)i * blocks + group_block) * (2 * N) + sum_value;
        for (int t = dead + sum_row; t < t1; t += sum_rows) at_sums[t * sum_step] = 0.0f;
        part_start<E, N, true>(p, part, i, w, a2, g);
        if (t0 < end) {
            int t = t0 + (end - t0 - 1) / BLOCK * BLOCK;       // the last block of steps
            const E *at_x = walk_from<const E, N>(p.x, t, i, w), *at_delta = walk_from<const E, N>(p.delta, t, i, w);
            const E *at_dy = walk_from<const E, N>(p.dy, t, i, w), *at_z = walk_from<const E, N>(p.z, t, i, w);
            E *at_dx = walk_from<E, N>(p.dx, t, i, w), *at_ddelta = walk_from<E, N>(p.ddelta, t, i, w), *at_dz = walk_from<E, N>(p.dz, t, i, w);
            WalkShared<E, N> at_shared;
            at_shared.start(p, t, i, w);
            const float4* at_saved = tiled(p.saved, (int64_t)(t / BLOCK) * p.n + i, w, p.tiles);
            const int64_t saved_step = (int64_t)p.n * p.tiles * WAVE;
            const int64_t step_x = p.x.step, step_delta = p.delta.step, step_dy = p.dy.step, step_z = p.z.step;
            const int64_t step_dx = p.dx.step, step_ddelta = p.ddelta.step, step_dz = p.dz.step;
            const bool soft = p.softplus != 0;
            WalkFirst at_first;
            at_first.start(p, t, i);
            at_sums += t * sum_step;
            E next_x[OWN], next_delta[OWN], next_dy[OWN], next_z[OWN];
            float next_h[4];
            auto fetch = [&](int count) {
                at_first.load(p.first.data != nullptr, count);
                at_shared.load(count);
                load_own<E, OWN>(at_x, step_x, own, count, next_x);
                load_own<E, OWN>(at_delta, step_delta, own, count, next_delta);
                load_own<E, OWN>(at_dy, step_dy, own, count, next_dy);
                if (GATE) load_own<E, OWN>(at_z, step_z, own, count, next_z);
                const Four v = __builtin_nontemporal_load(reinterpret_cast<const Four*>(at_saved));
                next_h[0] = v.x; next_h[1] = v.y; next_h[2] = v.z; next_h[3] = v.w;
                at_first.move(-1);
                at_shared.move(-1);
                at_x -= BLOCK * step_x;
                at_delta -= BLOCK * step_delta;
                at_dy -= BLOCK * step_dy;
                at_z -= BLOCK * step_z;
                at_saved -= saved_step;
            };
            fetch(end - t);
            for (; t >= t0; t -= BLOCK) {
                const int count = end - t < BLOCK ? end - t : BLOCK;
                const bool whole = count == BLOCK;
                const uint32_t cuts = at_first.cuts(count);
                float slope[OWN], dz[OWN], h[4];
                wave_fence();
                at_shared.stage(shared_lds, count);
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    const float pre = Elem<E>::up(next_delta[k]) + bias;
                    float size = soft ? softplus(pre) : pre;
                    slope[k] = soft ? sigmoid(pre) : 1.0f;
                    float dout = Elem<E>::up(next_dy[k]), x = Elem<E>::up(next_x[k]);
                    if (GATE) {
                        const float z = Elem<E>::up(next_z[k]), s = sigmoid(z);
                        dz[k] = dout * (s * __builtin_fmaf(z, 1.0f - s, 1.0f));
                        dout *= z * s;
                    }
                    // steps behind the end and channels that are none add nothing
                    if (!owns || (!whole && own + k >= count)) size = dout = x = 0.0f;
                    step_lds[(own + k) * CHANNELS + mine] = make_float4(size, size * x, dout, x);
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) h[m] = next_h[m];
                wave_fence();
                if (t > t0) fetch(BLOCK);
                // the states of these steps again: the decays, and what decayed of the state before
                float decay[BLOCK][4], kept[BLOCK][4], y[BLOCK];
                auto states = [&](auto check) {
                    float4 step = step_lds[mine];
                    float b[4], c[4];
                    load4(&shared_lds[w.quad], b);
                    if (GATE) load4(&shared_lds[N / 4 + w.quad], c);
#pragma unroll
                    for (int k = 0; k < BLOCK; ++k) {
                        float4 next_step = step;
                        float next_b[4] = {}, next_c[4] = {};
                        if (k + 1 < BLOCK) {
                            next_step = step_lds[(k + 1) * CHANNELS + mine];
                            load4(&shared_lds[(k + 1) * (N / 2) + w.quad], next_b);
                            if (GATE) load4(&shared_lds[(k + 1) * (N / 2) + N / 4 + w.quad], next_c);
                        }
                        if (decltype(check)::value && (cuts >> k & 1u)) zero(h);
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            decay[k][m] = exp2_fast(step.x * a2[m]);
                            kept[k][m] = decay[k][m] * h[m];
                            h[m] = __builtin_fmaf(step.y, b[m], kept[k][m]);
                        }
                        if (GATE) {
                            y[k] = h[0] * c[0];
#pragma unroll
                            for (int m = 1; m < 4; ++m) y[k] = __builtin_fmaf(h[m], c[m], y[k]);
                            pin(y[k]);
                        }
                        step = next_step;
#pragma unroll
                        for (int m = 0; m < 4; ++m) { b[m] = next_b[m]; c[m] = next_c[m]; }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (cuts == 0) states(std::false_type{});
                else states(std::true_type{});
                wave_fence();       // what is in LDS is read again rather than kept in registers: 64 more of them
                if (GATE) {
                    fold_steps<LANES>(y);
#pragma unroll
                    for (int k = 0; k < OWN; ++k) {
                        const float x = step_lds[(own + k) * CHANNELS + mine].w;
                        if (owns && (whole || own + k < count)) at_dz[k * step_dz] = Elem<E>::down(dz[k] * __builtin_fmaf(skip, x, y[k]));
                    }
                }
                float gb[BLOCK], rate[BLOCK];
                float* sums = sum_lds + (turn * waves + wave) * SUMS;
                auto back = [&](auto check) {
                    float4 step = step_lds[(BLOCK - 1) * CHANNELS + mine];
                    float b[4], c[4];
                    load4(&shared_lds[(BLOCK - 1) * (N / 2) + w.quad], b);
                    load4(&shared_lds[(BLOCK - 1) * (N / 2) + N / 4 + w.quad], c);
#pragma unroll
                    for (int k = BLOCK - 1; k >= 0; --k) {
                        float4 next_step = step;
                        float next_b[4] = {}, next_c[4] = {}, v[8];
                        if (k > 0) {
                            next_step = step_lds[(k - 1) * CHANNELS + mine];
                            load4(&shared_lds[(k - 1) * (N / 2) + w.quad], next_b);
                            load4(&shared_lds[(k - 1) * (N / 2) + N / 4 + w.quad], next_c);
                        }
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            v[4 + m] = step.z * __builtin_fmaf(step.y, b[m], kept[k][m]);
                            const float gm = __builtin_fmaf(c[m], step.z, g[m]);
                            v[m] = gm * step.y;
                            gb[k] = m == 0 ? gm * b[m] : __builtin_fmaf(gm, b[m], gb[k]);
                            const float through = gm * kept[k][m];
                            rate[k] = m == 0 ? through * a2[m] : __builtin_fmaf(through, a2[m], rate[k]);
                            da_span[m] = __builtin_fmaf(through, step.x, da_span[m]);
                            g[m] = decay[k][m] * gm;
                        }
                        if (decltype(check)::value && (cuts >> k & 1u)) zero(g);
                        const float folded = fold_channels<LANES>(v);
                        if (fold_writes<LANES>(lane)) sums[k * 2 * N + slot] = folded;
                        // all of a step is done in its turn: put off to the end, the sums would keep every step's factors in registers
                        pin(gb[k]);
                        pin(rate[k]);
#pragma unroll
                        for (int m = 0; m < 4; ++m) pin(da_span[m]);
                        step = next_step;
#pragma unroll
                        for (int m = 0; m < 4; ++m) { b[m] = next_b[m]; c[m] = next_c[m]; }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (cuts == 0) back(std::false_type{});
                else back(std::true_type{});
                wave_fence();
                fold_steps<LANES>(gb);
                fold_steps<LANES>(rate);
                float dx[OWN], dsize[OWN];
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    const float4 step = step_lds[(own + k) * CHANNELS + mine];
                    dsize[k] = slope[k] * __builtin_fmaf(gb[k], step.w, rate[k] * (1.0f / LOG2E));
                    dx[k] = __builtin_fmaf(gb[k], step.x, skip * step.z);
                    dd_span = __builtin_fmaf(step.z, step.w, dd_span);
                    if (whole || own + k < count) dbias_span += dsize[k];
                }
                if ((t - t0) % SCAN_BACK_SPAN == 0) {
#pragma unroll
                    for (int m = 0; m < 4; ++m) da[m] += da_span[m];
                    zero(da_span);
                    dd += dd_span;
                    dbias += dbias_span;
                    dd_span = dbias_span = 0.0f;
                }
                // the next block's values have been under way since before this one's steps; behind the stores, the wait would be for
                // those too
                pin(at_first.flag);
                pin(at_shared.words);
                pin(next_x);
                pin(next_delta);
                pin(next_dy);
                if (GATE) pin(next_z);
                pin(next_h);
                if (owns) {
#pragma unroll
                    for (int k = 0; k < OWN; ++k)
                        if (whole || own + k < count) {
                            at_dx[k * step_dx] = Elem<E>::down(dx[k]);
                            at_ddelta[k * step_ddelta] = Elem<E>::down(dsize[k]);
                        }
                }
                at_dx -= BLOCK * step_dx;
                at_ddelta -= BLOCK * step_ddelta;
                at_dz -= BLOCK * step_dz;
                __syncthreads();
                // sums over the block's wavefronts; the next turn writes the other half, so one barrier is enough
                const float* from = sum_lds + turn * waves * SUMS + sum_value;
                for (int k = sum_row; k < count; k += sum_rows) {
                    float s = from[k * 2 * N];
                    for (int v = 1; v < waves; ++v) s += from[v * SUMS + k * 2 * N];
                    at_sums[k * sum_step] = s;
                }
                at_sums -= BLOCK * sum_step;
                turn ^= 1;
            }
        }
        if (part == 0 && p.dstate_in && owns) store4(state_of<N>(p.dstate_in, p.channels, i, w), g);
    }
    // a channel's lanes hold the sums of their own steps
    dd += dpp<DPP_XOR1>(dd);
    dbias += dpp<DPP_XOR1>(dbias);
    if constexpr (LANES >= 4) { dd += dpp<DPP_XOR2>(dd); dbias += dpp<DPP_XOR2>(dbias); }
    if constexpr (LANES >= 8) { dd += dpp<DPP_HALF_MIRROR>(dd); dbias += dpp<DPP_HALF_MIRROR>(dbias); }
    if (owns) {
        float* row = given.weight_part + ((int64_t)(part * env_rows + env_row) * given.channels + w.channel) * (N + 2);
#pragma unroll
        for (int m = 0; m < 4; ++m) row[w.quad * 4 + m] = da[m];
        if (w.quad == 0) { row[N] = dd; row[N + 1] = dbias; }
    }
}

// What a part does to the gradient of the state that comes from behind it: see k_scan with PART.  No sums over channels and no
// parameters here, a third of the time of the walk behind it.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_back_part(const ScanParams<E> p)
{
    constexpr int LANES = Lay<N>::LANES, CHANNELS = Lay<N>::CHANNELS, OWN = Lay<N>::OWN;
    __shared__ float4 shared_lds[SCAN_WAVES][BLOCK * N / 2];
    __shared__ float2 step_lds[SCAN_WAVES][BLOCK * CHANNELS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = spread_block(p.wide) * SCAN_WAVES + wave;
    if (item >= (int64_t)p.n * p.tiles) return;
    const int i = (int)(item / p.tiles);
    const Tile w = tile_of<N>(p, (int)(item % p.tiles));
    const int mine = (int)(threadIdx.x & (WAVE - 1)) / LANES;
    const int part = (int)blockIdx.y + 1, t0 = part * p.part;          // what the first one does nobody asks for
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
    const E *at_delta = walk_from<const E, N>(p.delta, t, i, w), *at_dy = walk_from<const E, N>(p.dy, t, i, w), *at_z = walk_from<const E, N>(p.z, t, i, w);
    WalkShared<E, N> at_shared;
    WalkFirst at_first;
    at_shared.start(p, t, i, w);
    at_first.start(p, t, i);
    for (; t0 < end && t >= t0; t -= BLOCK) {
        const int count = end - t < BLOCK ? end - t : BLOCK;
        E delta[OWN], dy[OWN], z[OWN];
        at_first.load(p.first.data != nullptr, count);
        at_shared.load(count);
        load_own<E, OWN>(at_delta, p.delta.step, own, count, delta);
        load_own<E, OWN>(at_dy, p.dy.step, own, count, dy);
        if (p.z.data) load_own<E, OWN>(at_z, p.z.step, own, count, z);
        const uint32_t cuts = at_first.cuts(count);
        at_first.move(-1);
        at_shared.move(-1);
        at_delta -= BLOCK * p.delta.step;
        at_dy -= BLOCK * p.dy.step;
        at_z -= BLOCK * p.z.step;
        float2 step[OWN];
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            float size = Elem<E>::up(delta[k]) + bias, dout = Elem<E>::up(dy[k]);
            if (p.softplus) size = softplus(size);
            if (p.z.data) {
                const float v = Elem<E>::up(z[k]);
                dout *= v * sigmoid(v);
            }
            step[k] = own + k < count ? make_float2(size, dout) : make_float2(0.0f, 0.0f);
        }
        wave_fence();
        at_shared.stage(shared_lds[wave], count);
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
            if (cuts >> k & 1u) { zero(g); total = 0.0f; cut = 1.0f; }
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
    const int64_t at = spread_block(p.wide) * SCAN_THREADS + threadIdx.x;
    const int value = (int)(at % (2 * N));
    const int64_t row = at / (2 * N);                  // (step, environment, group)
    if (row >= (int64_t)p.steps * p.n * p.groups) return;
    const int64_t group = row % p.groups;
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
