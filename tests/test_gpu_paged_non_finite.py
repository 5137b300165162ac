"""One new token's attention over keys that are not finite: a key whose score is -infinity has no weight, whatever the head's size, and what is NaN stays with the
heads and requests that read it."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_paged_cache import Paged

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("element", [0, -1, -8], ids=["first", "last", "last run"])
@pytest.mark.parametrize("dim", [8, 13, 16, 24, 40, 64, 72, 80, 104, 128, 130, 136, 160, 200, 248, 256])
def test_scores_of_minus_infinity(dim, element, dtype):
    """Against the formula without these keys."""
    c = Paged([100, 333, 17], 6, 2, dim, 16, dtype, seed=11)
    c.q[..., element] = c.q[..., element].abs() + 0.25
    out = {0: [5, 99], 1: [0, 64, 200, 332], 2: [16]}
    for r, keys in out.items():
        for t in keys:
            c.k_cache[int(c.table[r, t // 16]), :, t % 16, element] = -INF
    c.run().check(out)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", [24, 80, 128, 200])
def test_nan_stays_where_it_is_read(dim, dtype):
    clean, bad = (Paged([100, 333, 17], 6, 2, dim, 16, dtype, seed=12) for _ in range(2))
    bad.k_cache[int(bad.table[1, 3]), 1, 2] = float("nan")
    clean.run()
    bad.run()
    for a, b in ((clean.o, bad.o), (clean.lse, bad.lse)):
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and torch.equal(a[1, :3], b[1, :3])   # heads 0 to 2 read the other key head
        assert torch.isnan(b[1, 3:]).all() or not torch.isfinite(b[1, 3:]).any()
