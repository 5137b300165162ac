"""What the attention operators settle on the host (launches are noted instead of run: no GPU needed)."""
import math
import random

import attention_sizes
from attention_launches import record


def sweep(seed, n):
    """Calls over the operators' ranges, sizes even over their logarithms."""
    rng = random.Random(seed)
    spread = lambda low, high: int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    calls = []
    while len(calls) < n:
        dtype, kv, dim = rng.choice(["bfloat16", "float32"]), spread(1, 64), rng.choice([rng.randint(1, 256), 32, 64, 96, 128, 256])
        heads = kv * rng.choice([1, 1, 2, 4, 8, 16])
        if rng.random() < 0.3:
            calls.append(["paged", spread(1, 2000), spread(1, 100000), heads, kv, dim, spread(1, 256), dtype])
            continue
        q = spread(1, 40000)
        k = q if rng.random() < 0.6 else spread(1, 40000)
        if max(q, k) * heads * dim < 1 << 31:
            calls.append([rng.choice(["forward", "backward"]), q, k, spread(1, max(1, min(q, 300))), heads, kv, dim, rng.random() < 0.7, dtype])
    return calls


def test_every_kernel_that_the_plans_choose_is_tested(tmp_path):
    """What a sweep of calls launches, the sizes of the GPU tests launch too."""
    covered = set()
    for status, names in record(attention_sizes.calls(), tmp_path):
        assert status == 0
        covered.update(names)
    calls = sweep(5, 12000)
    missing = {}
    for call, (status, names) in zip(calls, record(calls, tmp_path)):
        assert status == 0, call
        for name in set(names) - covered:
            missing.setdefault(name, call)
    assert not missing, missing


def test_what_a_sequence_of_one_length_launches(tmp_path):
    """One launch forward where there is enough work for the chip or none to share, and one that joins parts otherwise; two backward, and one for each
    gradient whose sums come in parts."""
    cases = {("forward", 4096, 4096, 1, 16, 16, 128, True, "bfloat16"): 1, ("forward", 37, 37, 1, 8, 8, 64, True, "float32"): 1,
             ("forward", 1, 100000, 1, 8, 8, 128, True, "bfloat16"): 2, ("backward", 4096, 4096, 1, 16, 16, 128, True, "bfloat16"): 2,
             ("backward", 2001, 2001, 3, 6, 3, 80, False, "float32"): 4, ("paged", 64, 8192, 32, 8, 128, 16, "bfloat16"): 2,
             ("paged", 64, 128, 32, 8, 128, 16, "bfloat16"): 1}
    for (call, n), (status, names) in zip(cases.items(), record([list(c) for c in cases], tmp_path)):
        assert status == 0 and len(names) == n, (call, names)
