"""Gated feed-forward block on the GPU against 64 bits, within bounds that follow from the sums' length and the types'
roundings (large_ref.py)."""
import pytest

torch = pytest.importorskip("torch")

import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import GatedSpec

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def inputs(T, D, H, dtype, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(s, generator=gen, device="cuda") * std).to(TYPES[dtype])
    return dict(x=n(T, D), w_gate=n(H, D, std=D ** -0.5), w_up=n(H, D, std=D ** -0.5), w_down=n(D, H, std=H ** -0.5)), n(T, D)


def nan(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def run(spec, i, dy, grads=("dx", "dw_gate", "dw_up", "dw_down"), stream=None):
    t = TYPES[spec.dtype]
    out = dict(y=nan(spec.tokens, spec.width, dtype=t), gate_pre=nan(spec.tokens, spec.hidden, dtype=t), up_pre=nan(spec.tokens, spec.hidden, dtype=t))
    ws = B.workspace(B.dll_gated_fwd_workspace_bytes(spec)).fill_(255)   # NaN in either type
    B.dll_gated_fwd(spec, **i, **out, ws=ws, stream=stream)
    g = {k: torch.full_like(i["x" if k == "dx" else k.replace("dw", "w")], float("nan")) for k in grads}
    ws = B.workspace(B.dll_gated_bwd_workspace_bytes(spec)).fill_(255)
    B.dll_gated_bwd(spec, **i, gate_pre=out["gate_pre"], up_pre=out["up_pre"], dy=dy, **g, ws=ws, stream=stream)
    return {**out, **g}


SIZES = [(1, 1, 1), (1, 8, 8), (3, 5, 7), (1, 64, 200), (2, 31, 9), (17, 33, 65), (16, 128, 72), (64, 100, 300), (129, 128, 64), (33, 260, 128), (257, 96, 130),
         (130, 259, 77)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_block(size, dtype):
    T, D, H = size
    gate = ["silu", "gelu", "relu", "sigmoid", "identity"][(T + D + H) % 5]
    spec = GatedSpec(T, D, H, gate, dtype)
    i, dy = inputs(T, D, H, dtype, seed=T + D + H)
    got, want = run(spec, i, dy), ref.gated(*i.values(), gate, dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("gate", ["identity", "sigmoid", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gates(gate, dtype):
    spec = GatedSpec(70, 48, 90, gate, dtype)
    i, dy = inputs(70, 48, 90, dtype, seed=5)
    i["x"] *= 8   # gate values far into both tails
    got, want = run(spec, i, dy), ref.gated(*i.values(), gate, dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_tiles(dtype):
    """Enough tiles of 256 x 256 in every product."""
    T, D, H = 1100, 1530, 8210
    spec = GatedSpec(T, D, H, "silu", dtype)
    i, dy = inputs(T, D, H, dtype, seed=9)
    got, want = run(spec, i, dy), ref.gated(*i.values(), "silu", dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("size", [(4095, 138, 4098), (138, 4098, 4096)], ids=lambda s: "x".join(map(str, s)))
def test_each_product_on_the_largest_tiles(size):
    """The forward products of the first size and the gradients of the second have 256 tiles of 256 x 256 and few slabs, the last
    slab with k ending inside 16 bytes."""
    spec = GatedSpec(*size, "silu", "bfloat16")
    i, dy = inputs(*size, "bfloat16", seed=10)
    got, want = run(spec, i, dy), ref.gated(*i.values(), "silu", dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("size", [(3, 40, 8250), (16, 33, 4100), (16, 32, 4098), (5, 40, 8251), (32, 24, 8250), (20, 1000, 2500), (32, 9, 4100)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_few_tokens(size, dtype):
    """On either side of where a few tokens' products change hands: rows of 16 KB, columns that fill half the compute units."""
    spec = GatedSpec(*size, "silu", dtype)
    i, dy = inputs(*size, dtype, seed=13)
    got, want = run(spec, i, dy), ref.gated(*i.values(), "silu", dy)
    for k in got:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("size", [(70, 33, 35), (70, 34, 38), (40, 1030, 1026), (300, 66, 37)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_lies_behind_a_row_is_not_multiplied(size, dtype):
    """Rows end inside 16 bytes, and the next row, which is another token's, holds NaN: it stays in that token's outputs."""
    T, D, H = size
    spec = GatedSpec(T, D, H, "silu", dtype)
    i, dy = inputs(T, D, H, dtype, seed=11)
    want = ref.gated(*i.values(), "silu", dy)
    odd = torch.arange(T, device="cuda") % 2 == 1
    i["x"][odd] = float("nan")
    dy[odd] = float("nan")
    got = run(spec, i, dy, ("dx",))
    for k in ("y", "gate_pre", "up_pre", "dx"):
        assert torch.isnan(got[k][odd]).all(), k
        ref.check(got[k][~odd], tuple(v[~odd] for v in want[k]), k)


@pytest.mark.parametrize("grads", [("dx",), ("dw_gate",), ("dw_up",), ("dw_down",), ("dw_gate", "dw_down"), ("dx", "dw_up")], ids="+".join)
def test_some_gradients(grads):
    spec = GatedSpec(40, 72, 56, "silu", "bfloat16")
    i, dy = inputs(40, 72, 56, "bfloat16")
    all_, some = run(spec, i, dy), run(spec, i, dy, grads)
    for k in grads:
        assert torch.equal(all_[k], some[k])


def test_inference_keeps_nothing_and_agrees():
    spec = GatedSpec(50, 72, 56, "gelu", "bfloat16")
    i, dy = inputs(50, 72, 56, "bfloat16")
    y = nan(50, 72, dtype=torch.bfloat16)
    B.dll_gated_fwd(spec, **i, y=y, ws=B.workspace(B.dll_gated_fwd_workspace_bytes(spec)))
    assert torch.equal(y, run(spec, i, dy)["y"])


def test_gradients_against_differences():
    """<gradient, direction> against the loss <y, dy> of 64-bit forward passes a step to either side; the gradients are the
    kernels' own.  Central differences with step e are off by the third derivative's e^2 / 6, far below 1e-6 here; the
    gradients' own error is bounded as elsewhere, by direction."""
    T, D, H = 9, 12, 20
    spec = GatedSpec(T, D, H, "gelu", "float32")
    i, dy = inputs(T, D, H, "float32", seed=3)
    got, want = run(spec, i, dy), ref.gated(*i.values(), "gelu", dy)
    names = {"x": "dx", "w_gate": "dw_gate", "w_up": "dw_up", "w_down": "dw_down"}
    wide = {k: v.double() for k, v in i.items()}
    loss = lambda v: float((ref.gated(*v.values(), "gelu")["y"][0] * dy.double()).sum())
    for k, g in names.items():
        gen = torch.Generator(device="cuda")
        gen.manual_seed(7)
        way = torch.randn(wide[k].shape, generator=gen, device="cuda", dtype=torch.float64)
        e = 1e-5
        slope = (loss({**wide, k: wide[k] + e * way}) - loss({**wide, k: wide[k] - e * way})) / (2 * e)
        mine = float((got[g].double() * way).sum())
        assert abs(mine - slope) <= float((want[g][1] * way.abs()).sum()) + 1e-6 * max(1.0, abs(slope))


def test_graph_and_streams():
    """Captured once, replayed several times on changed inputs with eager work in between; and the eager calls on a side stream."""
    spec = GatedSpec(33, 72, 130, "silu", "bfloat16")
    i, dy = inputs(33, 72, 130, "bfloat16")
    t = torch.bfloat16
    out = dict(y=nan(33, 72, dtype=t), gate_pre=nan(33, 130, dtype=t), up_pre=nan(33, 130, dtype=t))
    g = dict(dx=nan(33, 72, dtype=t), dw_gate=nan(130, 72, dtype=t), dw_up=nan(130, 72, dtype=t), dw_down=nan(72, 130, dtype=t))
    ws = B.workspace(max(B.dll_gated_fwd_workspace_bytes(spec), B.dll_gated_bwd_workspace_bytes(spec)))
    run(spec, i, dy)   # first use outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dll_gated_fwd(spec, **i, **out, ws=ws)
        B.dll_gated_bwd(spec, **i, gate_pre=out["gate_pre"], up_pre=out["up_pre"], dy=dy, **g, ws=ws)
    for seed in range(3):
        j, dy2 = inputs(33, 72, 130, t.__str__().split(".")[1], seed=50 + seed)
        for k in i:
            i[k].copy_(j[k])
        dy.copy_(dy2)
        graph.replay()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = run(spec, i, dy)
        side.synchronize()
        for k, v in {**out, **g}.items():
            assert torch.equal(v, eager[k]), k
