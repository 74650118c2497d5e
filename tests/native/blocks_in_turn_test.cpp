// Host-only unit test of the number of blocks that go on from tile to tile (csrc/memory_grid.hpp).  Built with g++ and run by
// tests/test_policy_block_sizes.py.
#include <cstdio>
#include <initializer_list>

#include "../../paper_2402_16801_amd/csrc/memory_grid.hpp"

int main()
{
    int failures = 0;
    // 2^24 tiles: 2^31 - 1 rows of 65 to 128 columns; 2^33: more than the header's matrices have
    for (int64_t tiles : {(int64_t)8, (int64_t)264, (int64_t)1 << 16, ((int64_t)1 << 21) - 8, (int64_t)1 << 21, ((int64_t)1 << 21) + 8, (int64_t)1 << 24, (int64_t)1 << 33}) {
        const int64_t blocks = mem::blocks_in_turn(tiles);
        const bool ok = blocks >= 1 && blocks <= tiles && blocks % 8 == 0 && blocks * 512 < (int64_t)1 << 32 && (blocks == tiles || tiles > (int64_t)1 << 21);
        if (!ok) std::printf("FAILED: %lld tiles, %lld blocks\n", (long long)tiles, (long long)blocks), ++failures;
    }
    std::printf(failures ? "blocks_in_turn_test: %d failures\n" : "blocks_in_turn_test: ok\n", failures);
    return failures != 0;
}
