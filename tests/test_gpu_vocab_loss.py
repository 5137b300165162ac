"""Softmax cross entropy over a vocabulary on the GPU against 64 bits, within the bounds of large_ref.py."""
import pytest

torch = pytest.importorskip("torch")

import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import VocabSpec

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def inputs(T, D, V, dtype, bias=False, ignored=0.0, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(s, generator=gen, device="cuda") * std).to(TYPES[dtype])
    labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    out = torch.rand(T, generator=gen, device="cuda") < ignored
    return dict(x=n(T, D), w=n(V, D, std=2 * D ** -0.5), bias=n(V) if bias else None, labels=torch.where(out, torch.full_like(labels, -100), labels))


def nan(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def run_grad(spec, i, scale=1.0, grads=("dx", "dw", "dbias")):
    t = TYPES[spec.dtype]
    out = dict(row_loss=nan(spec.tokens), row_lse=nan(spec.tokens), loss=nan(1))
    g = dict(dx=nan(spec.tokens, spec.width, dtype=t), dw=nan(spec.classes, spec.width, dtype=t), dbias=nan(spec.classes, dtype=t))
    g = {k: v for k, v in g.items() if k in grads and (k != "dbias" or i["bias"] is not None)}
    ws = B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)).fill_(255)
    B.dll_vocab_loss_grad(spec, **i, scale=scale, **out, **g, ws=ws)
    return {**out, **g}


def run_fwd(spec, i):
    out = dict(row_loss=nan(spec.tokens), row_lse=nan(spec.tokens), loss=nan(1))
    B.dll_vocab_loss_fwd(spec, **i, **out, ws=B.workspace(B.dll_vocab_loss_fwd_workspace_bytes(spec)).fill_(255))
    return out


def compare(got, want):
    for k in got:
        ref.check(got[k], want[k], k)


SIZES = [(1, 1, 1), (1, 8, 16), (5, 3, 7), (1, 72, 1000), (16, 64, 500), (33, 40, 129), (64, 64, 64), (130, 50, 517), (200, 72, 1000), (257, 128, 300), (31, 260, 4099)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_loss_and_gradients(size, ignored, bias, dtype):
    spec = VocabSpec(*size, dtype)
    i = inputs(*size, dtype, bias, ignored, seed=sum(size))
    want = ref.vocab(*i.values(), scale=3.0)
    compare(run_grad(spec, i, 3.0), want)
    compare(run_fwd(spec, i), want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_tiles(dtype):
    spec = VocabSpec(1000, 1530, 12001, dtype)
    i = inputs(1000, 1530, 12001, dtype, True, 0.1, seed=2)
    compare(run_grad(spec, i), ref.vocab(*i.values()))


@pytest.mark.parametrize("size", [(4094, 134, 4096), (4300, 24, 70), (9001, 40, 33)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_tokens(size, dtype):
    """Logits on tiles of 256 x 256 (bfloat16); rows gathered by more than one launch, from 4097 tokens on."""
    spec = VocabSpec(*size, dtype)
    i = inputs(*size, dtype, True, 0.0 if size[0] < 4097 else 0.3, seed=6)
    want = ref.vocab(*i.values())
    compare(run_grad(spec, i), want)
    compare(run_fwd(spec, i), want)


@pytest.mark.parametrize("dtype,tokens", [("bfloat16", 700), ("float32", 300)])
def test_pieces(dtype, tokens):
    """More exponentials than are kept at a time: two pieces of tokens, the second not whole and partly not counted."""
    spec = VocabSpec(tokens, 8, 1 << 20, dtype)
    i = inputs(tokens, 8, 1 << 20, dtype, True, 0.05, seed=4)
    compare(run_grad(spec, i), ref.vocab(*i.values()))


def test_pieces_of_which_one_is_empty():
    spec = VocabSpec(300, 8, 1 << 20, "float32")
    i = inputs(300, 8, 1 << 20, "float32", True, 0.3, seed=4)   # about 210 of 256 rows of the first piece
    assert int((i["labels"] >= 0).sum()) <= 256
    compare(run_grad(spec, i), ref.vocab(*i.values()))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_row_counts(dtype):
    spec = VocabSpec(40, 24, 100, dtype)
    i = inputs(40, 24, 100, dtype, True)
    i["labels"].fill_(-1)
    for k, v in {**run_grad(spec, i), **run_fwd(spec, i)}.items():
        assert not v.float().any() and torch.isfinite(v.float()).all(), k


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_that_do_not_count_reach_nothing(dtype):
    """NaN, infinities and labels beyond the vocabulary in rows that do not count."""
    spec = VocabSpec(70, 40, 300, dtype)
    i = inputs(70, 40, 300, dtype, True, 0.5, seed=8)
    i["labels"][3], i["labels"][4] = 300, 2 ** 31 - 1
    out = (i["labels"] < 0) | (i["labels"] >= 300)
    clean = run_grad(spec, i)
    i["x"][out] = float("nan")
    i["x"][4] = float("inf")
    dirty = run_grad(spec, i)
    for k in clean:
        assert torch.equal(clean[k], dirty[k]), k
    assert not clean["dx"][out].any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_classes_taken_out(dtype):
    """A bias of -infinity, over whole groups of columns too: probability and gradient exactly 0, the rest as without these classes."""
    T, D, V = 50, 40, 400
    spec = VocabSpec(T, D, V, dtype)
    i = inputs(T, D, V, dtype, True, seed=1)
    off = torch.zeros(V, dtype=torch.bool, device="cuda")
    off[60:260] = True
    off[399] = True
    i["labels"] = torch.where(off[i["labels"].long()], torch.full_like(i["labels"], 7), i["labels"])
    i["bias"][off] = float("-inf")
    got = run_grad(spec, i)
    assert not got["dw"][off].any() and not got["dbias"][off].any()
    keep = (~off).nonzero()[:, 0]
    index = torch.zeros(V, dtype=torch.int32, device="cuda")
    index[keep] = torch.arange(len(keep), dtype=torch.int32, device="cuda")
    want = ref.vocab(i["x"], i["w"][keep], i["bias"][keep], index[i["labels"].long()])
    for k in ("row_loss", "row_lse", "loss", "dx"):
        ref.check(got[k], want[k], k)
    ref.check(got["dw"][keep], want["dw"], "dw")
    ref.check(got["dbias"][keep], want["dbias"], "dbias")


def test_lowest_bias_and_wide_logits():
    """Biases of the type's lowest value and logits of some hundreds: statistics stay finite."""
    T, D, V = 40, 32, 500
    spec = VocabSpec(T, D, V, "float32")
    i = inputs(T, D, V, "float32", True, seed=6)
    i["w"] *= 100
    i["bias"][100:300] = torch.finfo(torch.float32).min / 2
    got = run_grad(spec, i)
    want = ref.vocab(*i.values())
    on = (i["labels"] < 100) | (i["labels"] >= 300)   # a row whose label is out has a loss of 1e38
    for k in ("row_loss", "row_lse"):
        ref.check(got[k][on], tuple(v[on] for v in want[k]), k)
    for k in ("dx", "dw", "dbias"):
        ref.check(got[k], want[k], k)


def test_rows_without_a_finite_logit_and_nan_stay_in_their_rows():
    T, D, V = 20, 16, 130
    spec = VocabSpec(T, D, V, "float32")
    i = inputs(T, D, V, "float32", True, seed=3)
    want = ref.vocab(*i.values())
    i["x"][5, 3] = float("nan")
    bad = run_fwd(spec, i)
    rest = torch.arange(T, device="cuda") != 5
    # a tile with a sum that is not finite is multiplied again in single precision as it is, so the other rows' last digits may
    # differ from a run without the NaN; both are within the bounds of the same 64-bit result
    for k in ("row_loss", "row_lse"):
        ref.check(bad[k][rest], tuple(v[rest] for v in want[k]), k)
    assert torch.isnan(bad["row_loss"][5]) and torch.isnan(bad["loss"]).all()
    i["bias"].fill_(float("-inf"))
    assert torch.isnan(run_fwd(spec, i)["row_loss"]).all()


@pytest.mark.parametrize("grads", [("dx",), ("dw",), ("dbias",), ("dx", "dbias")], ids="+".join)
def test_some_gradients(grads):
    spec = VocabSpec(60, 48, 200, "bfloat16")
    i = inputs(60, 48, 200, "bfloat16", True, 0.2)
    all_, some = run_grad(spec, i), run_grad(spec, i, grads=grads)
    for k in some:
        assert torch.equal(all_[k], some[k]), k


@pytest.mark.parametrize("size", [(20, 64, 90), (20, 65, 90), (200, 72, 1000)], ids=lambda s: "x".join(map(str, s)))
def test_any_label(size):
    """The ends of the integers' range and of the classes."""
    spec = VocabSpec(*size, "bfloat16")
    i = inputs(*size, "bfloat16", True, seed=12)
    i["labels"][:6] = torch.tensor([-2 ** 31, 2 ** 31 - 1, size[2], -1, 0, size[2] - 1], dtype=torch.int32)
    want = ref.vocab(*i.values())
    compare(run_grad(spec, i), want)
    compare(run_fwd(spec, i), want)


def test_two_calls_at_once():
    """On two streams with a workspace each: the same bits as one after the other."""
    spec = VocabSpec(600, 256, 5003, "bfloat16")
    i = [inputs(600, 256, 5003, "bfloat16", True, 0.2, seed=k) for k in (1, 2)]
    alone = [run_grad(spec, j) for j in i]
    t = torch.bfloat16
    out = [dict(row_loss=nan(600), row_lse=nan(600), loss=nan(1), dx=nan(600, 256, dtype=t), dw=nan(5003, 256, dtype=t), dbias=nan(5003, dtype=t)) for _ in i]
    ws = [B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)) for _ in i]
    streams = [torch.cuda.Stream() for _ in i]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in (0, 1):
            B.dll_vocab_loss_grad(spec, **i[k], scale=1.0, **out[k], ws=ws[k], stream=streams[k])
    torch.cuda.synchronize()
    for k in (0, 1):
        for n in out[k]:
            assert torch.equal(out[k][n], alone[k][n]), n


def test_gradients_against_differences():
    T, D, V = 7, 12, 90
    spec = VocabSpec(T, D, V, "float32")
    i = inputs(T, D, V, "float32", True, 0.3, seed=11)
    got, want = run_grad(spec, i), ref.vocab(*i.values())
    wide = {k: v.double() if k != "labels" else v for k, v in i.items()}
    loss = lambda v: float(ref.vocab(*v.values())["loss"][0])
    for k in ("x", "w", "bias"):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(7)
        way = torch.randn(wide[k].shape, generator=gen, device="cuda", dtype=torch.float64)
        e = 1e-5   # central differences: e^2 / 6 of the third derivative
        slope = (loss({**wide, k: wide[k] + e * way}) - loss({**wide, k: wide[k] - e * way})) / (2 * e)
        assert abs(float((got["d" + k].double() * way).sum()) - slope) <= float((want["d" + k][1] * way.abs()).sum()) + 1e-6 * max(1.0, abs(slope))


def test_graph_replays():
    spec = VocabSpec(50, 40, 333, "bfloat16")
    i = inputs(50, 40, 333, "bfloat16", True, 0.2)
    run_grad(spec, i)
    t = torch.bfloat16
    out = dict(row_loss=nan(50), row_lse=nan(50), loss=nan(1), dx=nan(50, 40, dtype=t), dw=nan(333, 40, dtype=t), dbias=nan(333, dtype=t))
    ws = B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dll_vocab_loss_grad(spec, **i, scale=1.0, **out, ws=ws)
    for seed in range(3):
        j = inputs(50, 40, 333, "bfloat16", True, 0.3 * seed, seed=20 + seed)
        for k in i:
            i[k].copy_(j[k])
        graph.replay()
        torch.cuda.synchronize()
        eager = run_grad(spec, i)
        for k in out:
            assert torch.equal(out[k], eager[k]), k
