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


def gated_inputs(T, D, H, dtype, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(s, generator=gen, device="cuda") * std).to(TYPES[dtype])
    return dict(x=n(T, D), w_gate=n(H, D, std=D ** -0.5), w_up=n(H, D, std=D ** -0.5), w_down=n(D, H, std=H ** -0.5)), n(T, D)


def block(spec, i, dy, fill):
    """Forward and backward pass with workspaces that hold `fill` in every byte."""
    e = lambda *s: torch.empty(s, dtype=TYPES[spec.dtype], device="cuda")
    T, D, H = spec.tokens, spec.width, spec.hidden
    out = dict(y=e(T, D), gate_pre=e(T, H), up_pre=e(T, H))
    B.dll_gated_fwd(spec, **i, **out, ws=B.workspace(B.dll_gated_fwd_workspace_bytes(spec)).fill_(fill))
    g = dict(dx=e(T, D), dw_gate=e(H, D), dw_up=e(H, D), dw_down=e(D, H))
    B.dll_gated_bwd(spec, **i, gate_pre=out["gate_pre"], up_pre=out["up_pre"], dy=dy, **g,
                    ws=B.workspace(B.dll_gated_bwd_workspace_bytes(spec)).fill_(fill))
    return {**out, **g}


def vocab_inputs(T, D, V, dtype, seed=0, ignored=0.2):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(s, generator=gen, device="cuda") * std).to(TYPES[dtype])
    labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    out = torch.rand(T, generator=gen, device="cuda") < ignored
    return dict(x=n(T, D), w=n(V, D, std=2 * D ** -0.5), bias=n(V), labels=torch.where(out, torch.full_like(labels, -100), labels))


def head(spec, i, fill):
    """Loss, then loss with gradients, with workspaces that hold `fill` in every byte."""
    e = lambda *s, d=TYPES[spec.dtype]: torch.empty(s, dtype=d, device="cuda")
    T, D, V = spec.tokens, spec.width, spec.classes
    losses = lambda: dict(row_loss=e(T, d=torch.float32), row_lse=e(T, d=torch.float32), loss=e(1, d=torch.float32))
    fwd, out = losses(), dict(**losses(), dx=e(T, D), dw=e(V, D), dbias=e(V))
    B.dll_vocab_loss_fwd(spec, **i, **fwd, ws=B.workspace(B.dll_vocab_loss_fwd_workspace_bytes(spec)).fill_(fill))
    B.dll_vocab_loss_grad(spec, **i, scale=1.0, **out, ws=B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)).fill_(fill))
    return {**{"fwd " + k: v for k, v in fwd.items()}, **out}


# bytes of NaN, of the largest finite numbers' neighbourhood (beyond bfloat16's range in single precision: 3.39e38), of 1.7e38
FILLS = (0, 255, 0x7F, 0x7E)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(200, 72, 1000), (300, 260, 970), (1000, 500, 1337), (40, 1030, 1026), (130, 259, 77)], ids=lambda s: "x".join(map(str, s)))
def test_block_whatever_the_workspace_holds(size, dtype):
    """The same bits, and within the bounds, from every former content."""
    spec = GatedSpec(*size, "silu", dtype)
    i, dy = gated_inputs(*size, dtype, seed=sum(size))
    want = ref.gated(*i.values(), "silu", dy)
    first = block(spec, i, dy, FILLS[0])
    for k in first:
        ref.check(first[k], want[k], k)
    for fill in FILLS[1:]:
        got = block(spec, i, dy, fill)
        for k in first:
            assert torch.equal(got[k], first[k]), (k, fill)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(200, 72, 970), (128, 2048, 1000), (300, 40, 4099), (31, 260, 4099), (130, 50, 517)], ids=lambda s: "x".join(map(str, s)))
def test_loss_whatever_the_workspace_holds(size, dtype):
    spec = VocabSpec(*size, dtype)
    i = vocab_inputs(*size, dtype, seed=sum(size))
    want = ref.vocab(*i.values())
    first = head(spec, i, FILLS[0])
    for k in first:
        ref.check(first[k], want[k.replace("fwd ", "")], k)
    for fill in FILLS[1:]:
        got = head(spec, i, fill)
        for k in first:
            assert torch.equal(got[k], first[k]), (k, fill)


def test_single_precision_in_graphs_and_on_two_streams():
    """Captured once, replayed on changed inputs with eager work between; two calls at once with a workspace each."""
    gs, vs = GatedSpec(150, 72, 250, "gelu", "float32"), VocabSpec(150, 72, 970, "float32")
    i, dy = gated_inputs(150, 72, 250, "float32")
    j = vocab_inputs(150, 72, 970, "float32")
    e = lambda *s: torch.empty(s, device="cuda")
    kept = dict(gate_pre=e(150, 250), up_pre=e(150, 250))
    g = dict(dx=e(150, 72), dw_gate=e(250, 72), dw_up=e(250, 72), dw_down=e(72, 250))
    o = dict(row_loss=e(150), row_lse=e(150), loss=e(1), dx=e(150, 72), dw=e(970, 72), dbias=e(970))
    y = e(150, 72)
    ws = [B.workspace(max(B.dll_gated_fwd_workspace_bytes(gs), B.dll_gated_bwd_workspace_bytes(gs))), B.workspace(B.dll_vocab_loss_grad_workspace_bytes(vs))]

    def blocks(stream=None):
        B.dll_gated_fwd(gs, **i, y=y, **kept, ws=ws[0], stream=stream)
        B.dll_gated_bwd(gs, **i, **kept, dy=dy, **g, ws=ws[0], stream=stream)

    def loss(stream=None):
        B.dll_vocab_loss_grad(vs, **j, scale=1.0, **o, ws=ws[1], stream=stream)

    blocks(), loss()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blocks(), loss()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for seed in range(3):
        i2, dy2 = gated_inputs(150, 72, 250, "float32", seed=90 + seed)
        j2 = vocab_inputs(150, 72, 970, "float32", seed=90 + seed)
        for a, b in list(zip(i.values(), i2.values())) + list(zip(j.values(), j2.values())) + [(dy, dy2)]:
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in [y, *kept.values(), *g.values(), *o.values()]]
        eager = [*block(gs, i, dy, 255).values(), *(v for k, v in head(vs, j, 255).items() if "fwd" not in k)]
        assert all(torch.equal(a, b) for a, b in zip(replayed, eager))
        torch.cuda.synchronize()
        blocks(streams[0]), loss(streams[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([y, *kept.values(), *g.values(), *o.values()], eager))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(20, 64, 600), (31, 260, 4099), (32, 33, 9000), (5, 40, 300), (24, 72, 65), (32, 512, 33000)], ids=lambda s: "x".join(map(str, s)))
def test_few_rows_that_do_not_count_reach_nothing(size, dtype):
    """A forward pass of few rows, which are not gathered: NaN, infinities and the largest numbers in rows that do not count leave
    the others' bits as they are."""
    spec = VocabSpec(*size, dtype)
    i = vocab_inputs(*size, dtype, seed=sum(size), ignored=0.5)
    i["labels"][0], i["labels"][1] = 3, -1
    e = lambda *s: torch.full(s, float("nan"), device="cuda")
    T, out = size[0], i["labels"] < 0

    def fwd():
        o = dict(row_loss=e(T), row_lse=e(T), loss=e(1))
        B.dll_vocab_loss_fwd(spec, **i, **o, ws=B.workspace(B.dll_vocab_loss_fwd_workspace_bytes(spec)).fill_(255))
        return o

    clean, want = fwd(), ref.vocab(*i.values())
    for k in clean:
        ref.check(clean[k], want[k], k)
    for bad in (float("nan"), float("inf"), torch.finfo(torch.float32).max):
        i["x"][out] = bad
        dirty = fwd()
        for k in clean:
            assert torch.equal(clean[k], dirty[k]), (k, bad)


def sure_rows(T, V, D, dtype):
    """Logits that every way of multiplying gives exactly: row t of x is the t-th unit vector, so that z[t][v] = w[v][t], whole
    numbers of 8 bits.  The label's is 1024 (or in every third row 1008), the others' are at most 1008."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + V)
    x = torch.zeros(T, D, dtype=TYPES[dtype], device="cuda")
    x[torch.arange(T), torch.arange(T)] = 1
    w = (1008 - 16 * torch.randint(0, 8, (V, D), generator=gen, device="cuda")).to(TYPES[dtype])
    labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    w[labels.long(), torch.arange(T, device="cuda")] = 1024
    labels[2::3] = (labels[2::3] + 1) % V   # the label of another row is not there: rows are columns of w
    return x, w, labels


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(1, 900, 8), (20, 1000, 33), (20, 4000, 40), (100, 1000, 128), (300, 3001, 300)], ids=lambda s: "x".join(map(str, s)))
def test_loss_of_rows_that_are_nearly_sure(size, dtype):
    """The label has all but about 1e-5 of the probability at logits of 1024, whose last digit in 32 bits is 1.2e-4.
    Bound: the terms are at most 1.002 together, each with the error of its exponential (EXP, of the terms below the largest, which is
    exact); a row's sum has 8 terms a lane, 3 steps among lanes, ceil(groups / 64) <= 2 groups a thread, 2 and 16 steps: 31 roundings of
    2^-24 of the sum; logf two last digits; then the difference and its sum with the logarithm, 2^-24 of the loss each."""
    T, V, D = size
    x, w, labels = sure_rows(T, V, D, dtype)
    spec = VocabSpec(T, D, V, dtype)
    e = lambda *s, d=torch.float32: torch.full(s, float("nan"), dtype=d, device="cuda")
    z = w.double().t()[:T]
    top = z.amax(1)
    rest = torch.exp(z - top[:, None]).sum(1) - 1
    loss = torch.log1p(rest) + (top - z[torch.arange(T), labels.long()])
    bound = rest * ref.EXP + 31 * U32 * (1 + rest) + 4 * U32 * torch.log1p(rest) + 2 * U32 * loss
    assert float(loss.min()) < 2e-3 and float(bound[loss.argmin()]) < 8e-6   # below the last digit of 1024
    for call in ("fwd", "grad"):
        o = dict(row_loss=e(T), row_lse=e(T), loss=e(1))
        if call == "fwd":
            B.dll_vocab_loss_fwd(spec, x, w, None, labels, **o, ws=B.workspace(B.dll_vocab_loss_fwd_workspace_bytes(spec)).fill_(255))
        else:
            B.dll_vocab_loss_grad(spec, x, w, None, labels, 1.0, **o, dx=e(T, D, d=x.dtype), ws=B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)).fill_(255))
        ref.check(o["row_loss"], (loss, bound), call)
        ref.check(o["loss"], (loss.mean().reshape(1), bound.mean().reshape(1) + U32 * loss.mean()), call)
        ref.check(o["row_lse"], (top + torch.log1p(rest), bound + U32 * (top + 1)), call)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [(1, 900, 8), (20, 1000, 33), (100, 1000, 128), (300, 3001, 300)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_rows_that_are_nearly_sure(size, dtype):
    """dw[v][t] is dz[t][v] alone, as row t of x is the t-th unit vector.  Of a label with all but 1e-5 of the probability it is
    -1e-5 / count; p itself is off by the bound of the logarithm of the sum (31 roundings of a sum of about 1, and logf's
    last digits), by that of its exponential (EXP / 64: x is below 1e-3 there, so two last digits of 1) and, elsewhere, by EXP and
    the type's rounding of e; dz by the type's rounding and 4 of 32 bits."""
    T, V, D = size
    x, w, labels = sure_rows(T, V, D, dtype)
    spec = VocabSpec(T, D, V, dtype)
    e = lambda *s, d=torch.float32: torch.full(s, float("nan"), dtype=d, device="cuda")
    z = w.double().t()[:T]
    top = z.amax(1, keepdim=True)
    terms = torch.exp(z - top)
    at = torch.arange(T, device="cuda"), labels.long()
    best = z == top
    rest = torch.where(best, 0.0, terms).sum(1, keepdim=True) + (best.sum(1, keepdim=True) - 1)
    p = terms / (1 + rest)
    dz = p.clone()
    sure = torch.zeros_like(dz, dtype=torch.bool).index_put(at, torch.tensor(True, device="cuda")) & best
    dz[at] -= 1
    dz = torch.where(sure, (-rest / (1 + rest)).expand_as(dz), dz)
    u = ref.unit(x.dtype)
    log = 31 * U32 + 4 * U32 * torch.log1p(rest)
    edz = p * log + torch.where(best, p * 4 * U32, p * (ref.EXP + u)) + (u + 4 * U32) * dz.abs() + 2 * U32 + 2 * 2.0 ** -126
    o = dict(row_loss=e(T), row_lse=e(T), loss=e(1), dx=e(T, D, d=x.dtype), dw=e(V, D, d=x.dtype))
    B.dll_vocab_loss_grad(spec, x, w, None, labels, float(T), **o, ws=B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)).fill_(255))
    assert float(dz[sure].abs().min()) < 2.0 ** -14   # half a last digit of 1024 (scale / count = 1)
    want, bound = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    want[:, :T], bound[:, :T] = dz.t(), (edz + (ref.gamma(T) + u) * dz.abs()).t()
    ref.check(o["dw"], (want, bound), "dw")


@pytest.mark.parametrize("counts", [[8, 3], [40000, 9]], ids=["one workgroup", "many"])
def test_a_norm_beyond_32_bits_is_not_finite(counts):
    """Finite gradients whose norm 32 bits do not hold: the caller reads infinity, and then nothing was scaled and no step taken."""
    g = [torch.full((n,), 3e38, device="cuda") for n in counts]
    l, norm = B.tensor_list(g), torch.zeros(1, device="cuda")
    ws = B.workspace(B.dll_grad_norm_workspace_bytes(l)).fill_(255)
    B.dll_grad_norm(l, g, norm, ws)
    assert math.isinf(float(norm))
    out = [torch.zeros_like(t) for t in g]
    B.dll_grad_clip(l, g, out, 1.0, norm, ws)
    assert math.isinf(float(norm)) and all(torch.equal(a, b) for a, b in zip(out, g))
    p, v = [torch.ones_like(t) for t in g], [torch.full_like(t, 2) for t in g]
    B.dll_momentum_update_clipped(l, p, v, g, 0.1, 0.9, None, 1.0, norm, ws=ws)
    assert math.isinf(float(norm)) and all(bool((t == 1).all()) for t in p) and all(bool((t == 2).all()) for t in v)
    g = [t / 1e10 for t in g]   # and in reach again
    B.dll_grad_clip(l, g, out, 1.0, norm, ws)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in g))
    assert abs(float(norm) - want) <= 2 * U32 * want
    for a, b in zip(out, g):
        ref.check(a, (b.double() / want, 3 * U32 * b.double() / want), "clipped")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tokens", [1, 40])
def test_gelu_keeps_its_digits_in_the_tail(tokens, dtype):
    """a Phi(a) and its derivative one by one, relative to themselves: x is a unit vector, w_down a unit matrix, w_up ones, so that
    y[h] = gelu(a_h) and dw_gate[h][0] = tokens * gelu'(a_h).
    Single precision: the argument a / sqrt 2 is off by 1.5 * 2^-24 relative (its factor, the product), which erfc multiplies by
    x d/dx ln erfc <= a^2 + 2; 16 * 2^-24 for the library's function (a few last digits), 4 for the products; the density's exponent
    a^2 / 2 log2 e has three roundings and the hardware's 2^x a last digit.  Bfloat16: the handbook's formula with 64 bits shows what it
    leaves out; roundings on the way as in single precision, and the type's own (da and dw_gate, h and y: two each)."""
    a = torch.arange(-64 if dtype == "bfloat16" else -88, 65, device="cuda", dtype=torch.float64) / 8
    n = len(a)
    unit, low = ref.unit(TYPES[dtype]), TYPES[dtype]
    spec = GatedSpec(tokens, n, n, "gelu", dtype)
    x, wg, wu = (torch.zeros(s, device="cuda", dtype=torch.float64) for s in ((tokens, n), (n, n), (n, n)))
    x[:, 0], wg[:, 0], wu[:, 0] = 1, a, 1
    i = dict(x=x.to(low), w_gate=wg.to(low), w_up=wu.to(low), w_down=torch.eye(n, device="cuda", dtype=low))
    assert torch.equal(i["w_gate"][:, 0].double(), a)
    got = block(spec, i, torch.ones(tokens, n, device="cuda", dtype=low), 255)
    cdf, pdf = 0.5 * torch.special.erfc(-a * math.sqrt(0.5)), torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    ecdf = (1.5 * (a * a + 2) + 20) * U32 * cdf
    if dtype == "bfloat16":
        t = 1 / (1 + 0.3275911 * a.abs() * math.sqrt(0.5))
        half = 0.5 * t * (0.254829592 + t * (-0.284496736 + t * (1.421413741 + t * (-1.453152027 + t * 1.061405429)))) * torch.exp(-a * a / 2)
        form = torch.where(a < 0, half, 1 - half)
        ecdf = (form - cdf).abs() + (1.5 * (a * a + 2) + 40) * U32 * (half + (a > 0))   # the polynomial's terms are up to 6 times its value
    f, d = a * cdf, cdf + a * pdf
    ef = a.abs() * ecdf + U32 * f.abs()
    ed = ecdf + (2 * a * a + 20) * U32 * a.abs() * pdf + U32 * d.abs()
    roundings = 2 * unit if dtype == "bfloat16" else 2 * U32
    for row in got["y"]:
        ref.check(row, (f, ef + roundings * f.abs() * 1.01), "y")
    ref.check(got["dw_gate"][:, 0], (tokens * d, tokens * (ed + (roundings * 1.01 + ref.gamma(tokens)) * d.abs())), "dw_gate")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tokens,scale", [(7, 1.0), (3680, 1.0), (3682, 1.0), (3699, 1.0), (4800, 1.0), (3682, 65536.0), (3682, 2.0 ** -120)])
def test_the_factor_of_the_loss_is_rounded_with_the_results_alone(tokens, scale, dtype):
    """Every row's label is a class of nearly no probability, so that dz is -scale / count there: its sum over all rows is -scale, and
    a row's dx 40 scale / count.  Single precision is off by the factor's rounding, the sums' and the product's; what is rounded to
    bfloat16 is rounded from there once (dz with scale / count in it would be off by the same 0.3 % in every row at 3682)."""
    t, V, D = TYPES[dtype], 10, 8
    spec = VocabSpec(tokens, D, V, dtype)
    x, w = torch.zeros(tokens, D, dtype=t, device="cuda"), torch.zeros(V, D, dtype=t, device="cuda")
    x[:, 0], w[3, 0] = 1, -40
    e = lambda *s, d=t: torch.full(s, float("nan"), dtype=d, device="cuda")
    o = dict(row_loss=e(tokens, d=torch.float32), row_lse=e(tokens, d=torch.float32), loss=e(1, d=torch.float32), dx=e(tokens, D), dw=e(V, D), dbias=e(V))
    labels = torch.full((tokens,), 3, dtype=torch.int32, device="cuda")
    B.dll_vocab_loss_grad(spec, x, w, torch.zeros(V, dtype=t, device="cuda"), labels, scale, **o,
                          ws=B.workspace(B.dll_vocab_loss_grad_workspace_bytes(spec)).fill_(255))
    bound = ref.gamma(tokens) if dtype == "float32" else 0.0
    for got, want in ((o["dw"][3, 0], -scale), (o["dbias"][3], -scale), (o["dx"][0, 0], 40 * scale / tokens), (o["dx"][tokens - 1, 0], 40 * scale / tokens)):
        rounded = float(torch.tensor(want, dtype=torch.float64).float().to(t))
        assert abs(float(got) - rounded) <= bound * abs(want), (float(got), want)
