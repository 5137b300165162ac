"""What the large-model operators settle on the host: which kernels a call launches (launches are noted instead of run: no
GPU needed)."""
import pytest

from launch_record import record


def test_no_launch_behind_the_last_tensor(tmp_path):
    """Empty tensors behind the last one of a full table of 64 need no table of their own: a launch with nothing in it would leave a
    norm of 0."""
    lists = [[4] * 64, [4] * 64 + [0], [0] + [4] * 64 + [0] * 70, [4] * 63 + [0, 0], [0, 0], [9000] * 64 + [0, 0], [0, 9000] * 64 + [0], [9000] * 128 + [0]]
    tables = [1, 1, 1, 1, 1, 1, 1, 2]
    for what in ("norm", "clip", "step"):
        for counts, n, (status, launches) in zip(lists, tables, record([[what, c] for c in lists], tmp_path)):
            assert status == 0
            small = sum(counts) <= 64 * 8
            assert len(launches) == (1 if small else n + 1 if what == "norm" else 2 * n), (what, counts, launches)
