"""The plan's sums over requests whose lengths add up beyond 2^30: they stop there, and the tokens in front have their slots all the same."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import CacheSpec

pytestmark = pytest.mark.gpu

MOST = 1 << 30
LONGEST = (1 << 31) - 1


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def planned(lengths, added, free, page, columns, tokens):
    """As the header has it, a request at a time; tables start as -7 everywhere, and only tokens with room are walked one by one."""
    table, slots, starts, missing, taken, first = [[-7] * columns for _ in lengths], [-7] * tokens, [0], 0, 0, 0
    for r, (n, a) in enumerate(zip(lengths, added)):
        n = max(0, n)
        a = max(0, min(a, n))
        have, need = -(-(n - a) // page), -(-n // page)
        fresh = max(0, min(need, columns) - have)
        missing += need - have - fresh
        for i in range(first, min(first + a, tokens)):
            t = n - a + i - first
            column = t // page
            if column >= columns:
                slots[i] = -1
                continue
            if t % page == 0:
                at = taken + column - have
                table[r][column] = free[at] if at < len(free) else -1
            id = table[r][column]
            slots[i] = id * page + t % page if id >= 0 else -1
        taken += fresh
        first += a
        starts.append(min(first, MOST))
    given = min(taken, len(free))
    return table, starts, slots, [given, min(min(taken, MOST) - given + min(missing, MOST), MOST)]


@pytest.mark.parametrize("lengths,added,page,columns", [
    ([MOST] * 2, [MOST] * 2, 16, 4), ([MOST] * 5, [MOST] * 5, 16, 4), ([5, MOST, 7, MOST, MOST, 3], [5, MOST, 7, MOST, MOST, 3], 16, 70),
    ([LONGEST] * 2, [LONGEST] * 2, 1, 1), ([LONGEST] * 4, [1] * 4, 1, 3), ([100, LONGEST] * 300, [100, LONGEST] * 300, 7, 20),
    ([MOST - 1, 2, 9], [MOST - 1, 2, 9], 128, 3), ([1 << 22] * 700, [1 << 22] * 700, 64, 6), ([40, 2100, MOST, 8], [40, 2100, MOST, 8], 16, 200)], ids=lambda v: None)
@pytest.mark.parametrize("tokens", [1, 90, 5000])
def test_sums_stop(lengths, added, page, columns, tokens):
    free = random.Random(len(lengths)).sample(range(1000), 300)
    spec = CacheSpec(len(lengths), 1, 1, 8, 1000, page, columns)
    table, starts, slots, state = ints([[-7] * columns] * len(lengths)), ints([-7] * (len(lengths) + 1)), ints([-7] * tokens), ints([-7, -7])
    B.dll_cache_plan(spec, ints(lengths), ints(added), ints(free), table, starts, slots, state)
    got = [table.tolist(), starts.tolist(), slots.tolist(), state.tolist()]
    for name, g, w in zip(("table", "starts", "slots", "state"), got, planned(lengths, added, free, page, columns, tokens)):
        assert g == w, name
