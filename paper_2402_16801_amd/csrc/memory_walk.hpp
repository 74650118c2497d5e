// What the policy memory operators that walk along the steps of a sequence share: the channels of a thread, and the steps read
// ahead of the one that is computed.
#pragma once

#include "memory_common.hpp"

namespace mem {

__device__ __forceinline__ int length_of(const int32_t* lengths, int steps, int i)
{
    if (lengths == nullptr) return steps;
    const int l = lengths[i];
    return l < 0 ? 0 : (l > steps ? steps : l);
}

// The channels of a thread: V from `c` on, of which the first `old` belong to the thread before it.  (A row whose length is no
// multiple of V ends with a vector that overlaps the one before it: it is loaded whole, and only its own values are stored and
// counted.)
struct Span {
    int c, old;
    template <int V> __device__ __forceinline__ static Span of(int vector, int channels)
    {
        const int c = vector * V, last = channels - V;
        return c <= last ? Span{c, 0} : Span{last, c - last};
    }
};

template <typename E, int V> __device__ __forceinline__ void fetch(Pack<E, V>& q, const E* p) { q = *reinterpret_cast<const Pack<E, V>*>(p); }
template <typename E, int V> __device__ __forceinline__ void expand(const Pack<E, V>& q, float (&v)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = Elem<E>::up(q.v[j]);
}
template <typename E, int V> __device__ __forceinline__ Pack<E, V> shrink(const float (&v)[V])
{
    Pack<E, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = Elem<E>::down(v[j]);
    return q;
}
template <typename E, int V> __device__ __forceinline__ void put(E* p, const Span& w, const Pack<E, V>& q)
{
    if (w.old == 0) {
        *reinterpret_cast<Pack<E, V>*>(p) = q;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= w.old) p[j] = q.v[j];
    }
}

// One sequence, read AHEAD steps in front of the step that is computed: raw[a] holds step t + a as it lies in memory and
// is refilled as soon as it is used.  Behind the last step that one is read again.
template <typename E, int V, int AHEAD> struct Stream {
    const E *next, *last;
    int64_t step;
    Pack<E, V> raw[AHEAD];
    template <bool MORE = false> __device__ __forceinline__ void refill(int a)       // MORE: there is a step behind this one
    {
        fetch<E, V>(raw[a], next);
        next = !MORE && next == last ? last : next + step;
    }
    __device__ __forceinline__ void start(const Seq<const E>& q, int t, int end, int i, int c)
    {
        step = q.step;
        next = q.at(t, i) + c;
        last = q.at(end - 1, i) + c;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) refill(a);
    }
};
// the same for the begins of episodes, where they are given
template <int AHEAD> struct Begins {
    const uint8_t *next, *last;
    int64_t step;
    uint32_t flag[AHEAD];
    template <bool MORE = false> __device__ __forceinline__ void refill(int a)
    {
        flag[a] = *next;
        next = !MORE && next == last ? last : next + step;
    }
    __device__ __forceinline__ void start(const Seq<const uint8_t>& q, int t, int end, int i)
    {
        step = q.step;
        next = q.at(t, i);
        last = q.at(end - 1, i);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) refill(a);
    }
};

}  // namespace mem
