"""Every kernel that the large-model operators' plans choose, against 64 bits (large_sizes.py; a host test checks that none is
left out)."""
import pytest

torch = pytest.importorskip("torch")

import large_ref as ref
from large_sizes import BLOCKS, LOSSES
from paper_1804_04512_amd.workloads import GatedSpec, VocabSpec
from test_gpu_large_edges import block, gated_inputs, head, vocab_inputs

pytestmark = pytest.mark.gpu

name = lambda v: v if isinstance(v, str) else "x".join(map(str, v))


@pytest.mark.parametrize("dtype,size", [(t, s) for t, sizes in BLOCKS.items() for s in sizes], ids=name)
def test_block(size, dtype):
    gate = ["silu", "gelu", "relu", "sigmoid"][sum(size) % 4]
    spec = GatedSpec(*size, gate, dtype)
    i, dy = gated_inputs(*size, dtype, seed=sum(size))
    got, want = block(spec, i, dy, 255), ref.gated(*i.values(), gate, dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype,size", [(t, s) for t, sizes in LOSSES.items() for s in sizes], ids=name)
def test_loss(size, dtype):
    spec = VocabSpec(*size, dtype)
    i = vocab_inputs(*size, dtype, seed=sum(size), ignored=0.05 if size[0] > 1 else 0.0)
    got, want = head(spec, i, 255), ref.vocab(*i.values())
    for k in got:
        ref.check(got[k], want[k.replace("fwd ", "")], k)
