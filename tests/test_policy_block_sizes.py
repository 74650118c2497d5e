"""Sizes that the policy block operators refuse, and launches of the largest that they take: without a GPU."""
from paper_2402_16801_amd import binding


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
