// Backward pass of the scan (part of memory_scan.hip).
//
// With g = dL/dh, walking back in time:
//   g   = c dy + (exp(D a) g of the step after it, 0 where an episode begins there)
//   dc  = sum over channels of dy h              db = sum over channels of g D x
//   dx  = D (g . b) + d dy                       dD = x (g . b) + sum over states of g a (exp(D a) h before)
//   da  = sum over steps of D g (exp(D a) h before)
// and dy here is dy z sigmoid(z) with a gate, dz = dy (c . h + d x) (z sigmoid(z))'.
//
// The states of SAVE steps are computed again from a saved one and held in registers: what decayed of the
// state before (exp(D a) h), from which h itself is one multiplication and addition away.  Holding the decay
// as well would take twice the registers and leave one wavefront per SIMD; it is computed again.  The sums
// over channels fold 2 N values over the lanes, halving values and lanes at once, and leave one value
// per pair of lanes; tiles are added up by a second kernel in a fixed order, no atomics.

// Sums of the 2 N values v over the lanes of the wavefront: value i ends in the lanes l with fold_index<N>(l) == i.
template <int COUNT>
__device__ __forceinline__ float fold_lanes(float (&v)[COUNT])
{
    const int lane = threadIdx.x & (WAVE - 1);
    // halves of 32 lanes: value k + count / 2 goes to the upper ones
    if constexpr (COUNT >= 2) {
#pragma unroll
        for (int k = 0; k < COUNT / 2; ++k) { const Pair q = swap32(v[k], v[k + COUNT / 2]); v[k] = q.a + q.b; }
    }
    if constexpr (COUNT >= 4) {
#pragma unroll
        for (int k = 0; k < COUNT / 4; ++k) { const Pair q = swap16(v[k], v[k + COUNT / 4]); v[k] = q.a + q.b; }
    }
    if constexpr (COUNT >= 8) {
        const bool up = lane & 8;
#pragma unroll
        for (int k = 0; k < COUNT / 8; ++k) {
            const float a = v[k] + dpp<DPP_ROR8>(v[k]), b = v[k + COUNT / 8] + dpp<DPP_ROR8>(v[k + COUNT / 8]);
            v[k] = up ? b : a;
        }
    }
    if constexpr (COUNT >= 16) {
        const bool up = lane & 4;
#pragma unroll
        for (int k = 0; k < COUNT / 16; ++k) {
            const float a = v[k] + dpp<DPP_HALF_MIRROR>(v[k]), b = v[k + COUNT / 16] + dpp<DPP_HALF_MIRROR>(v[k + COUNT / 16]);
            v[k] = up ? b : a;
        }
    }
    if constexpr (COUNT >= 32) {
        const bool up = lane & 2;
#pragma unroll
        for (int k = 0; k < COUNT / 32; ++k) {
            const float a = v[k] + dpp<DPP_XOR2>(v[k]), b = v[k + COUNT / 32] + dpp<DPP_XOR2>(v[k + COUNT / 32]);
            v[k] = up ? b : a;
        }
    } else {
        v[0] += dpp<DPP_XOR2>(v[0]);
    }
    if constexpr (COUNT >= 64) {
        const bool up = lane & 1;
        const float a = v[0] + dpp<DPP_XOR1>(v[0]), b = v[1] + dpp<DPP_XOR1>(v[1]);
        v[0] = up ? b : a;
    } else {
        v[0] += dpp<DPP_XOR1>(v[0]);
    }
    return v[0];
}
// which of COUNT (16, 32 or 64) values a lane holds after fold_lanes
template <int COUNT> __device__ __forceinline__ int fold_index(int lane)
{
    int i = (lane >> 5 & 1) * (COUNT / 2) + (lane >> 4 & 1) * (COUNT / 4) + (lane >> 3 & 1) * (COUNT / 8) + (lane >> 2 & 1) * (COUNT / 16);
    if (COUNT >= 32) i += (lane >> 1 & 1) * (COUNT / 32);
    if (COUNT >= 64) i += lane & 1;
    return i;
}

template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_scan_back(const ScanParams<E> p)
{
    constexpr int SAVE = Save<N>::STEPS;
    const int lane = threadIdx.x & (WAVE - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int64_t item = (int64_t)blockIdx.x * SCAN_WAVES + wave;
    const int env_rows = p.rows / p.parts;
    if (item >= (int64_t)env_rows * p.tiles) return;
    const Tile w = tile_of(p, (int)(item % p.tiles));
    const int env_row = (int)(item / p.tiles);
    const int part = (int)blockIdx.y, t0 = part * p.part;
    const int t1 = p.steps - t0 < p.part ? p.steps : t0 + p.part;
    float a2[N], g[N], da[N], dd = 0.0f, dbias = 0.0f;
    load_rates<N>(p.a, w.channel, a2);
    zero(da);
    const float skip = p.d ? p.d[w.channel] : 0.0f;
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    const int slot = fold_index<2 * N>(lane);
    const bool writes = 2 * N == 64 || (lane & (64 / (2 * N) - 1)) == 0;
    for (int i = env_row; i < p.n; i += env_rows) {
        const int length = scan_length(p, i);
        const int end = t1 < length ? t1 : length;
        for (int t = t0 > end ? t0 : end; t < t1; ++t) {
            if (w.owns) {
                p.dx.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                p.ddelta.at(t, i)[w.channel] = Elem<E>::down(0.0f);
                if (p.z.data) p.dz.at(t, i)[w.channel] = Elem<E>::down(0.0f);
            }
            if (writes) p.shared_part[(((int64_t)t * p.n + i) * p.tiles + w.tile) * (2 * N) + slot] = 0.0f;
        }
        if (p.parts > 1) load_tiled<N>(tiled_state<N>(p.starts, (int64_t)part * p.n + i, w, p.tiles), g);
        else if (p.dstate_out) load_state<N>(p.dstate_out, (int64_t)i * p.channels + w.channel, g);
        else zero(g);
        for (int q = (end - t0 + SAVE - 1) / SAVE - 1; q >= 0; --q) {
            const int t = t0 + q * SAVE;
            const int count = end - t < SAVE ? end - t : SAVE;
            const uint64_t starts = begins(p, t, t + count, i);
            float x[SAVE], raw[SAVE], dy[SAVE], z[SAVE], core[SAVE];
#pragma unroll
            for (int k = 0; k < SAVE; ++k) {
                const int s = k < count ? t + k : t + count - 1;
                x[k] = Elem<E>::up(p.x.at(s, i)[w.channel]);
                raw[k] = Elem<E>::up(p.delta.at(s, i)[w.channel]);
                dy[k] = Elem<E>::up(p.dy.at(s, i)[w.channel]);
                if (p.z.data) z[k] = Elem<E>::up(p.z.at(s, i)[w.channel]);
            }
            // the states of these steps again: what decayed of the state before each
            float kept[SAVE][N], h[N];
            load_tiled<N>(tiled_state<N>(p.saved, (int64_t)(t / SAVE) * p.n + i, w, p.tiles), h);
#pragma unroll
            for (int k = 0; k < SAVE; ++k) {
                if (k >= count) break;
                if (starts >> k & 1u) zero(h);
                float size = raw[k] + bias;
                if (p.softplus) size = softplus(size);
                const float u = size * x[k];
                Shared<E, N> b;
                b.load(p.b.at(t + k, i) + w.group * N);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    kept[k][n] = exp2_fast(size * a2[n]) * h[n];
                    h[n] = __builtin_fmaf(u, b[n], kept[k][n]);
                }
                if (p.z.data) {
                    Shared<E, N> c;
                    c.load(p.c.at(t + k, i) + w.group * N);
                    float y[4] = {skip * x[k], 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int n = 0; n < N; ++n) y[n & 3] = __builtin_fmaf(h[n], c[n], y[n & 3]);
                    core[k] = (y[0] + y[1]) + (y[2] + y[3]);
                }
            }
#pragma unroll
            for (int k = SAVE - 1; k >= 0; --k) {
                if (k >= count) continue;
                Shared<E, N> b, c;
                b.load(p.b.at(t + k, i) + w.group * N);
                c.load(p.c.at(t + k, i) + w.group * N);
                const float pre = raw[k] + bias;
                const float size = p.softplus ? softplus(pre) : pre;
                const float u = size * x[k];
                float dout = dy[k];
                if (p.z.data) {
                    const float s = sigmoid(z[k]);
                    if (w.owns) p.dz.at(t + k, i)[w.channel] = Elem<E>::down(dout * core[k] * (s * __builtin_fmaf(z[k], 1.0f - s, 1.0f)));
                    dout *= z[k] * s;
                }
                if (!w.owns) dout = 0.0f;
                float gb[2] = {0.0f, 0.0f}, rate[2] = {0.0f, 0.0f}, sums[2 * N];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const float hn = __builtin_fmaf(u, b[n], kept[k][n]);
                    sums[N + n] = w.owns ? dout * hn : 0.0f;
                    const float gn = __builtin_fmaf(c[n], dout, g[n]);
                    sums[n] = w.owns ? gn * u : 0.0f;
                    gb[n & 1] = __builtin_fmaf(gn, b[n], gb[n & 1]);
                    const float through = gn * kept[k][n];
                    rate[n & 1] = __builtin_fmaf(through, a2[n], rate[n & 1]);
                    da[n] = __builtin_fmaf(through, size, da[n]);
                    g[n] = exp2_fast(size * a2[n]) * gn;
                }
                if (starts >> k & 1u) zero(g);
                const float folded = fold_lanes<2 * N>(sums);
                if (writes) p.shared_part[(((int64_t)(t + k) * p.n + i) * p.tiles + w.tile) * (2 * N) + slot] = folded;
                const float du = gb[0] + gb[1];
                float dsize = __builtin_fmaf(du, x[k], (rate[0] + rate[1]) * (1.0f / LOG2E));
                if (p.softplus) dsize *= sigmoid(pre);
                dd = __builtin_fmaf(dout, x[k], dd);
                dbias += dsize;
                if (w.owns) {
                    p.dx.at(t + k, i)[w.channel] = Elem<E>::down(__builtin_fmaf(du, size, skip * dout));
                    p.ddelta.at(t + k, i)[w.channel] = Elem<E>::down(dsize);
                }
            }
        }
        if (p.parts == 1 && p.dstate_in && w.owns) store_state<N>(p.dstate_in, (int64_t)i * p.channels + w.channel, g);
    }
    if (w.owns) {
        float* row = p.weight_part + ((int64_t)(part * env_rows + env_row) * p.channels + w.channel) * (N + 2);
#pragma unroll
        for (int n = 0; n < N; ++n) row[n] = da[n];
        row[N] = dd;
        row[N + 1] = dbias;
    }
}

// What a part does to the gradient of the state that comes from behind it: see k_scan_part.
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_back_part(const ScanParams<E> p)
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
    float a2[N], g[N];
    load_rates<N>(p.a, w.channel, a2);
    const float bias = p.delta_bias ? p.delta_bias[w.channel] : 0.0f;
    zero(g);
    float total = 0.0f, cut = 0.0f;
    for (int q = (end - t0 + AHEAD - 1) / AHEAD - 1; q >= 0; --q) {
        const int t = t0 + q * AHEAD;
        const int count = end - t < AHEAD ? end - t : AHEAD;
        const uint64_t starts = begins(p, t, t + count, i);
        float delta[AHEAD], dy[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = k < count ? t + k : t + count - 1;
            delta[k] = Elem<E>::up(p.delta.at(s, i)[w.channel]);
            dy[k] = Elem<E>::up(p.dy.at(s, i)[w.channel]);
            if (p.z.data) {
                const float z = Elem<E>::up(p.z.at(s, i)[w.channel]);
                dy[k] *= z * sigmoid(z);
            }
        }
#pragma unroll
        for (int k = AHEAD - 1; k >= 0; --k) {
            if (k >= count) continue;
            Shared<E, N> c;
            c.load(p.c.at(t + k, i) + w.group * N);
            float size = delta[k] + bias;
            if (p.softplus) size = softplus(size);
            total += size;
#pragma unroll
            for (int n = 0; n < N; ++n) g[n] = exp2_fast(size * a2[n]) * __builtin_fmaf(c[n], dy[k], g[n]);
            if (starts >> k & 1u) { zero(g); total = 0.0f; cut = 1.0f; }
        }
    }
    const int64_t index = (int64_t)part * p.n + i;
    store_tiled<N>(tiled_state<N>(p.starts, index, w, p.tiles), g);
    p.decays[(index * p.tiles + w.tile) * WAVE + (threadIdx.x & (WAVE - 1))] = make_float2(total, cut);
}

// db and dc: the tiles of a group added up
template <typename E, int N>
__global__ __launch_bounds__(SCAN_THREADS) void k_scan_shared(const ScanParams<E> p, Seq<E> db, Seq<E> dc)
{
    const int64_t at = (int64_t)blockIdx.x * SCAN_THREADS + threadIdx.x;
    const int value = (int)(at % (2 * N));
    const int64_t row = at / (2 * N);                  // (step, environment, group)
    if (row >= (int64_t)p.steps * p.n * p.groups) return;
    const int group = (int)(row % p.groups);
    const int64_t token = row / p.groups;
    const float* q = p.shared_part + (token * p.tiles + (int64_t)group * p.group_tiles) * (2 * N) + value;
    float s = 0.0f;
    for (int k = 0; k < p.group_tiles; ++k) s += q[(int64_t)k * (2 * N)];
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
