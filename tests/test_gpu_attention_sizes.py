"""Every kernel that the attention operators' plans choose, against 64 bits (attention_sizes.py; a host test checks that none is left out)."""
import random

import pytest

torch = pytest.importorskip("torch")

from attention_sizes import BACKWARD, CACHES, FORWARD
from test_gpu_attention import Case
from test_gpu_paged_cache import Paged

pytestmark = pytest.mark.gpu

name = lambda v: v if isinstance(v, str) else "x".join(str(int(x)) for x in v)


def uneven(total, parts):
    """Lengths that add up, some of them short."""
    cuts = sorted(random.Random(total + parts).randint(0, total) for _ in range(parts - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def case(q, k, sequences, heads, kv_heads, dim, causal, dtype):
    nq = uneven(q, sequences)
    return Case(nq, nq if q == k else uneven(k, sequences), heads, kv_heads, dim, causal, dtype, seed=q + dim)


@pytest.mark.parametrize("dtype,size", [(t, s) for t, sizes in FORWARD.items() for s in sizes], ids=name)
def test_forward(size, dtype):
    c = case(*size, dtype)
    c.forward()
    c.check(backward=False)


@pytest.mark.parametrize("dtype,size", [(t, s) for t, sizes in BACKWARD.items() for s in sizes], ids=name)
def test_backward(size, dtype):
    c = case(*size, dtype)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype,size", [(t, s) for t, sizes in CACHES.items() for s in sizes], ids=name)
def test_paged(size, dtype):
    requests, longest, *rest = size
    rng = random.Random(longest)
    Paged([longest] + [rng.randint(0, longest) for _ in range(requests - 1)], *rest, dtype, columns=-(-longest // rest[-1])).run().check()
