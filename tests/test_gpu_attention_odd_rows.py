"""Rows that do not come in whole 16-byte groups reach LDS by ordinary stores, the tile of zeros behind the last one among them: it has to lie there before
wavefronts that share a tile's keys leave their sums in its place.  Few queries, so that some wavefronts have nothing of the last tile and are early, and
an even number of tiles, so that those zeros go where the sums do."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import Case, both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True], ids=["whole", "causal"])
@pytest.mark.parametrize("dim", [13, 60, 90, 97, 127])
@pytest.mark.parametrize("queries,keys", [(1, 128), (20, 128), (32, 256), (5, 384), (32, 1024), (7, 2048), (33, 1024), (30, 3000)])   # 64 or 128 keys a tile
def test_forward(queries, keys, dim, causal):
    c = Case([queries], [keys], 2, 1, dim, causal, "bfloat16", seed=40)
    for _ in range(3):
        c.o.fill_(float("nan"))
        c.forward()
        c.check(backward=False)


@pytest.mark.parametrize("causal", [False, True], ids=["whole", "causal"])
@pytest.mark.parametrize("dim", [13, 60, 90, 97, 127, 201])
@pytest.mark.parametrize("queries,keys", [(64, 96), (20, 128), (1, 64), (32, 256), (60, 120), (9, 512)])
def test_backward(queries, keys, dim, causal):
    both([queries], [keys], 4, 2, dim, causal, "bfloat16", seed=41)
