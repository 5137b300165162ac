"""Thousands of short sequences, so that finding a tile's sequence takes three rounds of sixty-four probes, in all three kernels and with queries and keys that start at
different places: every output and gradient against 64 bits, all sequences of one pair of lengths at a time (each as heads of its own)."""
import pytest

torch = pytest.importorskip("torch")

import attention_ref
import large_ref as ref
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


def together(t, starts, n):
    """[n][sequences * heads][D] of the sequences that begin at `starts`."""
    rows = starts[:, None] + torch.arange(n, device=t.device)
    return t[rows].transpose(0, 1).reshape(n, len(starts) * t.shape[1], t.shape[2])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("same", [True, False], ids=["same", "apart"])
def test_against_64_bits(same, causal, dtype):
    count = 5000
    nq = [(7 * s) % 4 for s in range(count)]
    nk = nq if same else [(5 * s + s // 3) % 5 for s in range(count)]
    c = Case(nq, nk, 2, 1, 16, causal, dtype, seed=70)
    c.forward()
    c.backward()
    pairs = sorted(set(zip(nq, nk)))
    assert len(pairs) >= (4 if same else 18)
    for a, b in pairs:
        at = [s for s in range(count) if (nq[s], nk[s]) == (a, b)]
        qs, ks = (torch.tensor([x[s] for s in at], device="cuda") for x in (c.qs, c.ks))
        got = {name: together(getattr(c, name), s, n) for name, s, n in (("o", qs, a), ("dq", qs, a), ("dk", ks, b), ("dv", ks, b))}
        if a and not b:
            assert (got["o"] == 0).all() and (got["dq"] == 0).all()
            continue
        if a + b == 0:
            continue
        q, k, v, d_o = (together(t, s, n) for t, s, n in ((c.q, qs, a), (c.k, ks, b), (c.v, ks, b), (c.d_o, qs, a)))
        want = attention_ref.sequence(q, k, v, c.scale, causal, d_o)
        for name, t in got.items():
            ref.check(t, want[name], f"{name} of {a} queries and {b} keys")
        if a:
            lse = c.lse[:, qs[:, None] + torch.arange(a, device="cuda")].transpose(0, 1).reshape(2 * len(at), a)   # [sequences * heads][a]
            seen = torch.isfinite(want["lse"][0])
            assert torch.isneginf(lse[~seen]).all()
            ref.check(torch.where(seen, lse, 0.0), tuple(torch.where(seen, t, 0.0) for t in want["lse"]), f"lse of {a} queries and {b} keys")
            if a > 1 and b > 1:   # the bounds tell a sequence from its neighbour
                for name in ("o", "dq", "dk", "dv"):
                    with pytest.raises(AssertionError):
                        ref.check(got[name].roll(2, 1), want[name], name)
