"""Values so large that the sums of their weighted numbers pass the largest one on the way to a mean that does not: the outputs are the formula's, and digit
for digit those of small values."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import Case
from test_gpu_paged_cache import TYPES, Paged

pytestmark = pytest.mark.gpu

FOLD = 2.0 ** 125   # of a normal number: below 1.9e38
# queries, keys, heads, key heads, elements: few queries with their keys between the wavefronts or in parts, 128 queries a workgroup, every size of a head
SIZES = [([1], [1], 1, 1, 8), ([40], [40], 2, 1, 64), ([70], [1500], 2, 1, 128), ([33, 1], [700, 20], 2, 2, 90), ([600], [600], 4, 2, 32), ([1, 0, 5], [3000, 2, 0], 2, 1, 64),
         ([105] * 20, [105] * 20, 32, 32, 64), ([300, 41], [300, 41], 2, 1, 200), ([777], [777], 16, 4, 64), ([65], [5000], 4, 4, 96)]
REQUESTS = [([1], 1, 1, 64, 16), ([1000], 16, 4, 128, 16), ([33, 600, 0, 31, 2], 8, 1, 96, 20), ([3000, 1], 24, 1, 64, 64), ([300, 20], 4, 2, 256, 16), ([9000, 400], 2, 2, 127, 7)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, causal, dtype):
    small, large = (Case(*size, causal, dtype, seed=50) for _ in range(2))
    large.v.mul_(FOLD)
    assert torch.isfinite(large.v).all()
    for c in (small, large):
        c.forward()
    assert torch.equal(large.lse, small.lse) and torch.equal(large.o, small.o * FOLD)
    small.check(backward=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("n", [130, 900])
def test_slowly_growing_scores(n, dim, dtype):
    """By a little less a tile than moves the running maximum, so that weights stand up to 2^8 above it."""
    c = Case([n], [n], 2, 1, dim, False, dtype, seed=51)
    c.k.copy_((torch.arange(n, device="cuda")[:, None, None] * (7.0 / 64) * 0.6931).expand(c.k.shape).to(c.k.dtype))
    c.q.fill_(1.0)
    c.scale = 1.0 / dim
    c.v.copy_((c.v.float().tanh() + 1.5).mul(1e38).to(c.v.dtype))
    c.forward()
    c.check(backward=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("requests", REQUESTS, ids=str)
def test_paged(requests, dtype):
    small, large = (Paged(*requests, dtype, seed=52) for _ in range(2))
    large.v_cache.mul_(FOLD)
    for c in (small, large):
        c.run()
    assert torch.equal(large.lse, small.lse) and torch.equal(large.o, small.o * FOLD)
    small.check()


def test_one_large_value_leaves_the_others_alone():
    """A workgroup that takes its tiles again leaves the digits of its other queries as they are."""
    for dtype in TYPES:
        clean, large = (Case([300], [300], 2, 1, 64, True, dtype, seed=53) for _ in range(2))
        large.v[200:202] = 2e38
        for c in (clean, large):
            c.forward()
        assert torch.equal(large.o[:200], clean.o[:200]) and torch.equal(large.lse, clean.lse) and torch.isfinite(large.o).all()
