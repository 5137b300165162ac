"""The ends of the scale's range: 0 and the smallest numbers against products near the largest ones, and the largest scale against small products."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import Case
from test_gpu_paged_cache import Paged

pytestmark = pytest.mark.gpu

# scale and the size of an element of q and k: products of 64 of them have a deviation of 8 times its square, at most 50 times
# (so none passes 2.3e38, and none of the largest scale's sums depends on numbers below 2^-126)
ENDS = [(0.0, 2e18), (-0.0, 2e18), (1e-40, 2e18), (-1e-39, 2e18), (2.0 ** -127, 2e18), (2.0 ** 127, 3e-19), (-(2.0 ** 126), 3e-19), (1e-45, 1.0)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("scale,size", ENDS, ids=str)
def test_packed(scale, size, causal, dtype):
    c = Case([100, 300], [100, 300], 2, 1, 64, causal, dtype, seed=60, scale=scale)
    for t in (c.q, c.k):
        t.mul_(size)
    c.forward()
    c.check(backward=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale,size", ENDS, ids=str)
def test_paged(scale, size, dtype):
    c = Paged([100, 900, 1], 4, 2, 64, 16, dtype, seed=61, scale=scale)
    for t in (c.q, c.k_cache, *c.k):
        t.mul_(size)
    c.run().check()
