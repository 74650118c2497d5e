// How launches of the policy memory operators are cut so that every size their header allows can be launched.  Plain C++ (no
// HIP types), so that the rules can be tested without a GPU.
#pragma once

#include <cstdint>

namespace mem {

// Kernels count steps in signed 32 bits and look some of them ahead, by less than 4,096.
constexpr int64_t MOST_COUNT = ((int64_t)1 << 31) - 4096;

// `blocks` blocks of `threads` threads: a dimension of a launch takes fewer than 2^32 threads, so that more blocks than that lie
// over x and z.  Some of the last ones in z may be too many.
struct Spread { unsigned x, z; };
inline Spread spread(int64_t blocks, int threads)
{
    const int64_t most = (((int64_t)1 << 32) - 1) / threads;
    const int64_t z = (blocks + most - 1) / most, x = (blocks + z - 1) / z;
    return {(unsigned)x, (unsigned)z};
}

// Blocks over `tiles` tiles, of a kernel whose blocks go on to the tile as many behind as there are blocks: one a tile, and of very many tiles as many
// as one dimension of a launch has threads for, so that the tiles' dies stay those of their blocks (the number is a multiple of eight, or all tiles).
inline unsigned blocks_in_turn(int64_t tiles)
{
    constexpr int64_t MOST = (int64_t)1 << 21;
    return (unsigned)(tiles < MOST ? tiles : MOST);
}

// Environments that are taken side by side by kernels whose threads go on by that many: `want` or all of them, and so few that what is
// behind the last one still has a number.
inline int side_by_side(int64_t want, int n)
{
    const int64_t room = ((int64_t)1 << 31) - n, side = want < n ? want : n;
    return (int)(side < room ? side : room);
}

// Whether the scan's kernel for one token can number its threads in 32 bits (states / 4 of them to a channel, and a chip full of them
// more); the kernel for sequences takes what it cannot.
inline bool token_fits(int64_t channels, int states) { return channels * (states / 4) <= (int64_t)1 << 31; }

}  // namespace mem
