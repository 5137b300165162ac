"""One new token's outputs in bfloat16 are those of 32 bits but for their own rounding: what the weights lose on the way does not show."""
import pytest

torch = pytest.importorskip("torch")

import attention_ref
import large_ref as ref
from test_gpu_paged_cache import Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,heads,kv_heads,dim,page", [([2, 1000], 16, 4, 128, 16), ([33, 600, 0, 31], 8, 1, 96, 20), ([3000, 1], 24, 1, 64, 64), ([500], 5, 1, 256, 100),
                                                             ([300, 20], 4, 4, 32, 1), ([300, 77], 4, 2, 45, 16)], ids=str)
def test_outputs(lengths, heads, kv_heads, dim, page):
    c = Paged(lengths, heads, kv_heads, dim, page, "bfloat16", seed=13).run()
    for r in range(len(lengths)):
        q, k, v = (t.float() for t in (c.q[r:r + 1], c.k[r], c.v[r]))
        if not lengths[r]:
            continue
        value, bound = attention_ref.sequence(q, k, v, c.scale, False)["o"]
        size = attention_ref.sequence(q, k, v.abs(), c.scale, False)["o"][0]
        # bfloat16's half step of the output; a weight in two parts is off by 2^-8 of 2^-8 of it
        ref.check(c.o[r:r + 1], (value, bound + 2.0 ** -8 * (value.abs() + bound) + 2.0 ** -16 * size), f"o of request {r}")
