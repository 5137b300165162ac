"""Attention under a causal mask with numbers that are not finite: they reach the results of those that see them, or are seen by them, and leave the
others' bits as they are."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu

SIZES = [([100], 2, 1, 64), ([300, 40], 4, 2, 128), ([700], 2, 2, 80), ([700, 33], 32, 32, 128), ([1500], 4, 1, 64), ([260], 2, 1, 200), ([2100], 32, 32, 64)]
AT = [0, 31, 70, 95]


def runs(size, dtype, spoil):
    """Forward and backward pass, clean and with what `spoil` does to the case."""
    n, heads, kv_heads, dim = size
    cases = [Case(n, n, heads, kv_heads, dim, True, dtype, seed=30) for _ in range(2)]
    spoil(cases[1])
    for c in cases:
        c.forward()
        c.backward()
    return cases


def same(a, b, rows, *names):
    for name in names:
        x, y = (getattr(c, name)[:, rows] if name == "lse" else getattr(c, name)[rows] for c in (a, b))
        assert torch.isfinite(x).all() and torch.equal(x, y), name


def lost(c, rows, *names):
    for name in names:
        assert not torch.isfinite(getattr(c, name)[rows]).any(), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("number", [float("nan"), float("inf"), -float("inf")], ids=str)
@pytest.mark.parametrize("at", AT)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_value(size, at, number, dtype):
    """One element of one value: the outputs of the queries from there on are NaN, lse is as it was."""
    n = size[0][0]

    def spoil(c):
        c.v[at, :, size[3] // 2] = number

    clean, bad = runs(size, dtype, spoil)
    same(clean, bad, slice(0, at), "o", "dq")
    same(clean, bad, slice(n, None), "o", "dq", "dk", "dv")
    same(clean, bad, slice(0, None), "lse")
    assert torch.isnan(bad.o[at:n, :, size[3] // 2]).all() or not torch.isfinite(bad.o[at:n, :, size[3] // 2]).any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("at", AT)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_key(size, at, dtype):
    n = size[0][0]

    def spoil(c):
        c.k[at] = float("nan")

    clean, bad = runs(size, dtype, spoil)
    same(clean, bad, slice(0, at), "o", "lse", "dq")
    same(clean, bad, slice(n, None), "o", "lse", "dq", "dk", "dv")
    lost(bad, slice(at, n), "o", "dq")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("number", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("at", AT)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_query_and_its_gradient(size, at, number, dtype):
    """Its own outputs and gradient, and the gradients of the keys that it sees."""
    n = size[0][0]

    def spoil_query(c):
        c.q[at] = float("nan")

    clean, bad = runs(size, dtype, spoil_query)
    same(clean, bad, slice(0, at), "o", "lse", "dq")
    same(clean, bad, slice(at + 1, None), "o", "lse", "dq", "dk", "dv")
    lost(bad, slice(at, at + 1), "o", "dq")
    lost(bad, slice(0, at + 1), "dk", "dv")

    def spoil_gradient(c):
        c.d_o[at, :, 0] = number

    clean, bad = runs(size, dtype, spoil_gradient)
    same(clean, bad, slice(0, None), "o", "lse")
    same(clean, bad, slice(0, at), "dq")
    same(clean, bad, slice(at + 1, None), "dq", "dk", "dv")
    lost(bad, slice(at, at + 1), "dq")
