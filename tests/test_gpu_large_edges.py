"""Edges of the large-model operators on the GPU: tables that are just full, workspaces that hold anything, rows that weigh nearly
everything."""
import math

import pytest

torch = pytest.importorskip("torch")

import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import GatedSpec, VocabSpec

pytestmark = pytest.mark.gpu

U32 = ref.U32
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


@pytest.mark.parametrize("counts", [[4] * 64 + [0], [4] * 63 + [0, 4, 0, 0], [0] + [9] * 64 + [0] * 65, [9000] * 64 + [0], [70] * 128 + [0, 0]],
                         ids=["64+1", "63+1+2", "1+64+65", "long", "two tables"])
def test_empty_tensors_behind_a_full_table(counts):
    """The norm of all three calls, and what clipping and the step leave."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(len(counts))
    g = [torch.randn(n, generator=gen, device="cuda") for n in counts]
    l = B.tensor_list(g)
    ws = B.workspace(B.dll_grad_norm_workspace_bytes(l)).fill_(255)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in g))
    norms = [torch.full((1,), float("nan"), device="cuda") for _ in range(3)]
    out, p, v = [torch.full_like(t, float("nan")) for t in g], [torch.ones_like(t) for t in g], [torch.zeros_like(t) for t in g]
    B.dll_grad_norm(l, g, norms[0], ws)
    B.dll_grad_clip(l, g, out, want / 2, norms[1], ws)
    B.dll_momentum_update_clipped(l, p, v, g, 1.0, 0.0, None, want / 2, norms[2], ws=ws)
    for n in norms:
        assert abs(float(n) - want) <= 2 * U32 * want   # the sum in 64 bits, the root's rounding to 32
    for a, b, c, d in zip(out, v, p, g):
        half = d.double() / 2
        bound = 3 * U32 * half.abs()   # max_norm, the factor and the product, rounded to 32 bits each
        ref.check(a, (half, bound), "clipped")
        ref.check(b, (-half, bound + U32 * half.abs()), "v")
        ref.check(c, (1 - half, bound + U32 * half.abs() + U32 * (1 - half).abs()), "theta")
