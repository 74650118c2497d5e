"""Sizes that the policy block operators refuse, and launches of the largest that they take: without a GPU."""
import os
import subprocess

from paper_2402_16801_amd import binding

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


def test_a_refused_recurrence_saves_nothing():
    """As its workspace: 0 bytes of sizes that the calls refuse, whose product would not fit a size."""
    lib, most = binding.load(), 2 ** 31 - 4096
    for steps, n, channels in ((most + 1, 1, 1), (1, most + 1, 1), (1, 1, most + 1), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 16, 2 ** 15), (0, 1, 1), (1, -1, 1)):
        a = binding.RecurrenceArgs(dtype=1, steps=steps, n=n, channels=channels)
        assert lib.craftax_gated_recurrence_saved_bytes(a) == 0, (steps, n, channels)
        assert lib.craftax_gated_recurrence_workspace_bytes(a, 0) == 0 and lib.craftax_gated_recurrence_workspace_bytes(a, 1) == 0
    for steps, n, channels in ((1, 1, 1), (9, 3, 70), (most, 1, 1), (1, most, 1)):
        a = binding.RecurrenceArgs(dtype=1, steps=steps, n=n, channels=channels)
        need = -(-steps // 4) * n * channels * 4
        assert lib.craftax_gated_recurrence_saved_bytes(a) == -(-need // 256) * 256
    a.dtype = 7
    assert lib.craftax_gated_recurrence_saved_bytes(a) == 0


def test_blocks_that_go_on_from_tile_to_tile_can_be_launched(tmp_path):
    """A dimension of a launch takes fewer than 2^32 threads; 2^31 - 1 rows of 65 outputs, which fit a GPU, are 2^24 tiles (csrc/memory_grid.hpp)."""
    exe = str(tmp_path / "blocks_in_turn_test")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-o", exe,
                    os.path.join(NATIVE, "blocks_in_turn_test.cpp")], check=True)
    assert "blocks_in_turn_test: ok" in subprocess.run([exe], check=True, capture_output=True, text=True).stdout
