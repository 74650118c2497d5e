// Dropout onto a residual: out = residual + x / (1 - p) where the mask keeps x, residual alone where it does not.
//
// The mask is never stored.  Philox4x32-10 (Salmon et al., SC'11), keyed by a seed and counted by (eight channels, environment, step),
// gives eight numbers of 16 bits, one for each of a thread's eight channels; a value is dropped where its number is below
// round(p 2^16).  So an actor's token and a learner's rollout find the same mask, in any layout and number of threads, and the
// backward pass is the same call on the gradient.
//
// Bound by memory: 2 or 3 activations per value.  Ten rounds for eight values are some 60 vector instructions, 20 of them the wide
// multiplications at a quarter of the rate.  64 steps of 4,096 environments of 512 bfloat16 values, with and without a residual (forward
// and backward): 246 us, 5.4 TB/s of what has to move.
#include "common.hpp"
#include "memory_api.hpp"
#include "memory_common.hpp"

#include <type_traits>

namespace mem {

constexpr int DROP_THREADS = 256, DROP_V = 8;

template <typename E, typename O> struct DropParams {
    Seq<const E> x;
    Seq<const O> residual;
    Seq<O> out;
    uint32_t key0, key1, limit, env;
    uint64_t step;
    const int64_t* step_at;
    float scale;
    int64_t items;
    uint32_t vectors, n;
    int channels;
    unsigned wide;
};

template <typename P> __device__ __forceinline__ void drop_load(const P* p, int count, float (&v)[DROP_V])
{
    if (count >= DROP_V) {
        const Pack<P, DROP_V> q = *reinterpret_cast<const Pack<P, DROP_V>*>(p);
#pragma unroll
        for (int j = 0; j < DROP_V; ++j) v[j] = Elem<P>::up(q.v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < DROP_V; ++j) v[j] = j < count ? Elem<P>::up(p[j]) : 0.0f;
    }
}

template <typename E, typename O>
__global__ __launch_bounds__(DROP_THREADS) void k_dropout(const DropParams<E, O> p)
{
    const int64_t at = spread_block(p.wide) * DROP_THREADS + threadIdx.x;
    if (at >= p.items) return;
    const uint32_t row = (uint32_t)((uint64_t)at / p.vectors), vec = (uint32_t)((uint64_t)at % p.vectors);
    const int t = (int)(row / p.n), i = (int)(row % p.n);
    const int c = (int)vec * DROP_V, count = p.channels - c;
    float x[DROP_V], r[DROP_V] = {};
    drop_load(p.x.at(t, i) + c, count, x);
    if (p.residual.data) drop_load(p.residual.at(t, i) + c, count, r);
    const uint64_t step = p.step + (p.step_at ? (uint64_t)*p.step_at : 0) + (uint64_t)t;
    const cx::U4 u = cx::philox4x32_10(vec, p.env + (uint32_t)i, (uint32_t)step, (uint32_t)(step >> 32), p.key0, p.key1);
    O* out = p.out.at(t, i) + c;
    Pack<O, DROP_V> q;
#pragma unroll
    for (int j = 0; j < DROP_V; ++j) {
        const uint32_t number = j % 2 ? u.w[j / 2] >> 16 : u.w[j / 2] & 0xFFFFu;
        q.v[j] = Elem<O>::down(number < p.limit ? r[j] : __builtin_fmaf(x[j], p.scale, r[j]));
    }
    if (count >= DROP_V) {
        *reinterpret_cast<Pack<O, DROP_V>*>(out) = q;
    } else {
#pragma unroll
        for (int j = 0; j < DROP_V; ++j)
            if (j < count) out[j] = q.v[j];
    }
}

namespace host {

int dropout(const craftax_dropout_args* a, void* stream, const char** why)
{
    if (!a) return refuse(CRAFTAX_E_NULL, "args is NULL", why);
    if (a->dtype > CRAFTAX_F16) return refuse(CRAFTAX_E_CONFIG, "unknown dtype", why);
    if (a->out_dtype > CRAFTAX_F16 || (a->out_dtype != a->dtype && a->out_dtype != CRAFTAX_F32 && a->dtype != CRAFTAX_F32))
        return refuse(CRAFTAX_E_CONFIG, "out_dtype must be dtype, or one of the two CRAFTAX_F32", why);
    if (a->residual.data && a->out_dtype != a->dtype && a->out_dtype != CRAFTAX_F32)
        return refuse(CRAFTAX_E_CONFIG, "with a residual out_dtype must be dtype or CRAFTAX_F32", why);
    if (!(a->p >= 0.0 && a->p <= 1.0)) return refuse(CRAFTAX_E_CONFIG, "p must be 0..1", why);
    if (a->steps < 1 || a->n < 1 || a->channels < 1) return refuse(CRAFTAX_E_COUNT, "steps, n and channels must be positive", why);
    if ((int64_t)a->steps * a->n >= (int64_t)1 << 31) return refuse(CRAFTAX_E_COUNT, "steps * n must be below 2^31", why);
    if (a->channels > MOST_COUNT) return refuse(CRAFTAX_E_COUNT, "channels must be below 2^31 - 4095", why);
    if (a->env < 0 || a->env > ((int64_t)1 << 32) - a->n) return refuse(CRAFTAX_E_COUNT, "env + n must be within 0..2^32", why);
    if (a->step < 0 || a->step > INT64_MAX - a->steps) return refuse(CRAFTAX_E_COUNT, "step + steps must be within 0..2^63 - 1", why);
    if (!a->x.data || !a->out.data) return refuse(CRAFTAX_E_NULL, "x or out is NULL", why);
    if (!aligned(a->x.data, elem_bytes(a->dtype)) || !aligned(a->out.data, elem_bytes(a->out_dtype)) || !aligned(a->residual.data, elem_bytes(a->out_dtype)) ||
        !aligned(a->step_at, 8))
        return refuse(CRAFTAX_E_ALIGN, "a pointer is not aligned to its elements", why);
    const int64_t vectors = ceil_div(a->channels, DROP_V), rows = (int64_t)a->steps * a->n;
    const int64_t items = rows * vectors;
    if (ceil_div(items, DROP_THREADS) > ((int64_t)1 << 40)) return refuse(CRAFTAX_E_COUNT, "too many values for one call", why);
    const uint32_t limit = (uint32_t)(a->p * 65536.0 + 0.5);
    with_type(a->dtype, [&](auto e) {
        using E = decltype(e);
        auto launch = [&](auto o) {
            using O = decltype(o);
            DropParams<E, O> p{};
            p.x = seq_in<E>(a->x); p.residual = seq_in<O>(a->residual); p.out = seq<O>(a->out);
            p.key0 = (uint32_t)a->seed; p.key1 = (uint32_t)(a->seed >> 32);
            p.limit = limit; p.env = (uint32_t)a->env; p.step = (uint64_t)a->step; p.step_at = a->step_at;
            p.scale = limit < 65536 ? 65536.0f / (float)(65536 - limit) : 0.0f;
            p.items = items; p.vectors = (uint32_t)vectors; p.n = (uint32_t)a->n; p.channels = a->channels;
            const Spread grid = spread(ceil_div(items, DROP_THREADS), DROP_THREADS);
            p.wide = grid.x;
            hipLaunchKernelGGL((k_dropout<E, O>), dim3(grid.x, 1, grid.z), dim3(DROP_THREADS), 0, (hipStream_t)stream, p);
        };
        if (a->out_dtype == a->dtype) return launch(E{});
        if constexpr (std::is_same_v<E, float>) {
            if (a->out_dtype == CRAFTAX_BF16) launch(__bf16{});
            else launch(_Float16{});
        } else {
            launch(float{});
        }
    });
    return launched(why);
}

}  // namespace host
}  // namespace mem
