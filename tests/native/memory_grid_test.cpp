// Host-only unit test of how launches of the policy memory operators are cut (csrc/memory_grid.hpp).  Built with g++ and run
// by tests/test_native_checks.py.
#include <cstdio>
#include <initializer_list>

#include "../../paper_2402_16801_amd/csrc/memory_grid.hpp"

static int failures = 0;
static void expect(bool cond, const char* what, long long a, long long b)
{
    if (!cond) { std::printf("FAILED: %s (%lld, %lld)\n", what, a, b); ++failures; }
}

int main()
{
    using namespace mem;
    // every block there once, and every dimension within 2^32 threads and 65,535 blocks in z
    for (int threads : {64, 128, 256, 512})
        for (int64_t near : {(int64_t)1, (int64_t)1000, ((int64_t)1 << 32) / threads, 2 * (((int64_t)1 << 32) / threads), (int64_t)1 << 28, (int64_t)1 << 31, (int64_t)1 << 33})
            for (int64_t blocks = near > 3 ? near - 3 : 1; blocks <= near + 3; ++blocks) {
                const Spread s = spread(blocks, threads);
                expect((int64_t)s.x * threads < (int64_t)1 << 32, "threads in x", blocks, threads);
                expect(s.z >= 1 && s.z <= 65535, "blocks in z", blocks, threads);
                expect((int64_t)s.x * s.z >= blocks && (int64_t)s.x * (s.z - 1) < blocks, "all of the blocks", blocks, threads);
                if (blocks * threads < (int64_t)1 << 32) expect(s.z == 1 && s.x == blocks, "one dimension where it is enough", blocks, threads);
            }
    // what a kernel that numbers threads in 32 bits may be asked for: a call's channels plus a full chip and a block more
    for (int states : {8, 16, 32})
        for (int64_t channels : {(int64_t)1, (int64_t)512, ((int64_t)1 << 31) / (states / 4), ((int64_t)1 << 31) / (states / 4) + 1, ((int64_t)1 << 31) - 4096}) {
            const int64_t per_env = channels * (states / 4);
            if (token_fits(channels, states)) expect(per_env + 2 * 524288 + 512 < (int64_t)1 << 32, "threads of a token", channels, states);
            else expect(per_env > (int64_t)1 << 31, "a token that would fit", channels, states);
        }
    // environments side by side: at least one, no more than there are or are wanted, and the one behind the last is a number
    for (int64_t want : {(int64_t)1, (int64_t)512, (int64_t)131072, (int64_t)1 << 31, (int64_t)1 << 34})
        for (int n : {1, 2, 511, 4096, 131073, 2147483647 - 524288, (int)MOST_COUNT - 1, (int)MOST_COUNT}) {
            const int side = side_by_side(want, n);
            expect(side >= 1 && side <= n && side <= want && (int64_t)n - 1 + side <= 2147483647, "environments side by side", want, n);
            if (n <= 2147483647 - 524288 && want <= 524288) expect(side == (want < n ? want : n), "all that are wanted", want, n);
        }
    std::printf(failures ? "memory_grid_test: %d failures\n" : "memory_grid_test: ok\n", failures);
    return failures ? 1 : 0;
}
