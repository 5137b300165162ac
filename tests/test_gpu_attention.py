"""Attention over packed sequences on the GPU against 64 bits, forward and backward, within bounds that follow from the sums' length
and the types' roundings (attention_ref.py)."""
import itertools

import pytest

torch = pytest.importorskip("torch")

import attention_ref
import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import AttentionSpec, GatedSpec, VocabSpec

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
NAN = float("nan")


def sums(counts, first=0):
    return list(itertools.accumulate(counts, initial=first))


class Case:
    """Packed sequences of nq and nk tokens, `gap` rows in front of the first and behind the last that belong to none.  Whatever belongs
    to nobody holds NaN, and so do all outputs before the calls."""

    def __init__(self, nq, nk, heads, kv_heads, dim, causal, dtype, seed=0, gap=0, fused=False, scale=None, off=0):
        self.nq, self.nk, self.causal, self.gap = nq, nk, causal, gap
        self.scale = dim ** -0.5 if scale is None else scale
        self.qs, self.ks = sums(nq, gap), sums(nk, gap)
        Tq, Tk, t = max(1, self.qs[-1] + gap), max(1, self.ks[-1] + gap), TYPES[dtype]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed + 7 * dim + heads)

        def normal(*shape):
            v = torch.full(shape, NAN, device="cuda")
            v[gap:shape[0] - gap if gap else None] = torch.randn((shape[0] - 2 * gap,) + shape[1:], generator=gen, device="cuda")
            return v.to(t)

        q, k, v, self.d_o = normal(Tq, heads, dim), normal(Tk, kv_heads, dim), normal(Tk, kv_heads, dim), normal(Tq, heads, dim)
        row = 0
        nan = lambda *s: torch.full(s, NAN, dtype=t, device="cuda")
        if fused:   # one buffer for all three, from an element that is no multiple of anything
            assert Tq == Tk
            row = (heads + 2 * kv_heads) * dim + off
            room = lambda: nan(Tq * row + off)[off:].unflatten(0, (Tq, row))[:, :row - off].unflatten(1, (heads + 2 * kv_heads, dim))
            self.buffer, self.dbuffer = room(), room()
            self.buffer.copy_(torch.cat((q, k, v), 1))
            q, k, v = self.buffer.split([heads, kv_heads, kv_heads], 1)
            self.dq, self.dk, self.dv = self.dbuffer.split([heads, kv_heads, kv_heads], 1)
        else:
            self.dq, self.dk, self.dv = nan(Tq, heads, dim), nan(Tk, kv_heads, dim), nan(Tk, kv_heads, dim)
        self.q, self.k, self.v = q, k, v
        self.spec = AttentionSpec(Tq, Tk, len(nq), heads, kv_heads, dim, causal, dtype, row, row)
        self.o, self.lse = nan(Tq, heads, dim), torch.full((heads, Tq), NAN, device="cuda")
        self.starts = [torch.tensor(s, dtype=torch.int32, device="cuda") for s in (self.qs, self.ks)]

    def inputs(self):
        return (self.q, self.k, self.v, *self.starts, self.scale)

    def forward(self, fill=255, stream=None):
        self.ws = B.workspace(B.dll_attention_fwd_workspace_bytes(self.spec)).fill_(fill)
        B.dll_attention_fwd(self.spec, *self.inputs(), self.o, self.lse, self.ws, stream)

    def backward(self, fill=255, stream=None, dq=True, dk=True, dv=True):
        self.ws_b = B.workspace(B.dll_attention_bwd_workspace_bytes(self.spec)).fill_(fill)
        B.dll_attention_bwd(self.spec, *self.inputs(), self.o, self.lse, self.d_o, self.dq if dq else None, self.dk if dk else None,
                            self.dv if dv else None, self.ws_b, stream)

    def outputs(self):
        return {k: getattr(self, k).clone() for k in ("o", "lse", "dq", "dk", "dv")}

    def check(self, backward=True):
        for s, (nq, nk) in enumerate(zip(self.nq, self.nk)):
            a, b = slice(self.qs[s], self.qs[s] + nq), slice(self.ks[s], self.ks[s] + nk)
            want = attention_ref.sequence(self.q[a], self.k[b], self.v[b], self.scale, self.causal, self.d_o[a] if backward else None)
            seen = torch.isfinite(want["lse"][0])
            assert torch.isneginf(self.lse[:, a][~seen]).all() and (self.o[a].transpose(0, 1)[~seen] == 0).all()
            ref.check(torch.where(seen, self.lse[:, a], 0.0), tuple(torch.where(seen, t, 0.0) for t in want["lse"]), f"lse of sequence {s}")
            for name, rows in (("o", a), ("dq", a), ("dk", b), ("dv", b)):
                if name == "o" or backward:
                    ref.check(getattr(self, name)[rows], want[name], f"{name} of sequence {s}")
        for t, ends in ((self.o, self.qs), (self.lse.t(), self.qs), (self.dq, self.qs), (self.dk, self.ks), (self.dv, self.ks)):   # nobody's rows
            assert torch.isnan(t[:ends[0]]).all() and torch.isnan(t[ends[-1]:]).all()


def both(*args, **kw):
    c = Case(*args, **kw)
    c.forward()
    c.backward()
    c.check()
    return c


EQUAL = [([1], 1, 1, 8), ([2], 1, 1, 64), ([31], 2, 1, 32), ([32, 33], 2, 2, 64), ([64, 1, 0, 63], 4, 2, 96), ([127, 128, 129], 3, 3, 128), ([300], 6, 2, 80),
         ([1] * 70, 2, 1, 64), ([517], 5, 1, 128), ([70, 5, 200], 4, 4, 256), ([260], 2, 2, 160), ([0, 0, 65, 0], 8, 1, 64)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("n,heads,kv_heads,dim", EQUAL, ids=str)
def test_sequences(n, heads, kv_heads, dim, causal, dtype):
    both(n, n, heads, kv_heads, dim, causal, dtype)


# more keys than queries (a prompt's later piece), fewer (queries in front see nothing), none at all
APART = [([1], [100]), ([5], [1000]), ([40], [130]), ([130], [40]), ([64, 0, 3], [0, 64, 3]), ([200], [1]), ([129, 1], [257, 300]), ([1], [0])]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("nq,nk", APART, ids=str)
def test_queries_and_keys_of_different_lengths(nq, nk, causal, dtype):
    both(nq, nk, 4, 2, 64, causal, dtype, seed=1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", [1, 3, 7, 16, 20, 33, 50, 66, 72, 100, 127, 129, 250, 255])
def test_head_sizes(dim, dtype):
    both([77, 20], [77, 20], 2, 1, dim, True, dtype, seed=2)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("off", [0, 1, 2, 3, 8])
@pytest.mark.parametrize("dim", [64, 40])
def test_one_buffer_for_all_three(dim, off, dtype):
    """q, k and v, and their gradients, side by side in rows of one projection, at any element."""
    c = both([50, 90], [50, 90], 4, 2, dim, True, dtype, seed=3, fused=True, off=off)
    assert torch.isfinite(c.dbuffer).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_of_nobody(dtype):
    """Rows in front of the first sequence and behind the last one hold NaN: nothing of them is used, nothing is written there."""
    both([30, 100], [30, 100], 2, 1, 64, True, dtype, seed=4, gap=37)
    both([30, 100], [64, 3], 2, 2, 72, False, dtype, seed=4, gap=5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale", [0.0, -0.125, 1.0, 3.0], ids=str)
def test_scales(scale, dtype):
    both([100], [100], 2, 2, 64, True, dtype, seed=5, scale=scale)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_growing_and_falling_scores(dtype):
    """Scores that grow along the keys, so that each tile raises the running maximum, and ones that fall, so that the rest vanishes."""
    for sign in (1.0, -1.0):
        c = Case([400], [400], 2, 2, 32, False, dtype, seed=6)
        c.k.copy_((c.k.float() * 0.1 + sign * torch.linspace(0, 20, 400, device="cuda")[:, None, None]).to(c.k.dtype))
        c.q.copy_((c.q.float() * 0.1 + 1.0).to(c.q.dtype))
        c.forward()
        c.backward()
        c.check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_other_sequences_hold(dtype):
    """A sequence full of NaN and one of infinities leave the others' bits as they are."""
    n = [50, 40, 129, 33]
    clean = both(n, n, 2, 1, 64, True, dtype, seed=7)
    dirty = Case(n, n, 2, 1, 64, True, dtype, seed=7)
    for t in (dirty.q, dirty.k, dirty.v, dirty.d_o):
        t[50:90] = NAN
        t[219:] = float("inf")
    dirty.forward()
    dirty.backward()
    for name in ("o", "dq", "dk", "dv"):
        for rows in (slice(0, 50), slice(90, 219)):
            assert torch.equal(getattr(dirty, name)[rows], getattr(clean, name)[rows]), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradients_that_are_not_asked_for(dtype):
    c = both([150, 20], [150, 20], 4, 2, 64, True, dtype, seed=8)
    want = c.outputs()
    for dq, dk, dv in itertools.product([True, False], repeat=3):
        if not (dq or dk or dv):
            continue
        for name in ("dq", "dk", "dv"):
            getattr(c, name).fill_(NAN)
        c.backward(0, None, dq, dk, dv)
        for name, asked in (("dq", dq), ("dk", dk), ("dv", dv)):
            assert torch.equal(getattr(c, name), want[name]) if asked else torch.isnan(getattr(c, name)).all()


def test_without_lse():
    c = Case([100], [100], 2, 2, 64, True, "bfloat16")
    c.forward()
    want = c.o.clone()
    B.dll_attention_fwd(c.spec, *c.inputs(), c.o.fill_(NAN), None, c.ws)
    assert torch.equal(c.o, want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradients_are_differences_quotients(dtype):
    """Directional derivatives of the 64-bit forward pass, by central differences, against the kernels' gradients."""
    c = both([40, 9], [40, 9], 4, 2, 16, True, dtype, seed=9)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    h = 1e-4
    for name in ("q", "k", "v"):
        t = getattr(c, name)
        step = torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends, slack = [], 0.0
        for sign in (1, -1):
            total = 0.0
            for s, n in enumerate(c.nq):
                r = slice(c.qs[s], c.qs[s] + n)
                moved = {k: getattr(c, k)[r].double() for k in ("q", "k", "v")}
                moved[name] = moved[name] + sign * h * step[r]
                total += float((attention_ref.sequence(**moved, scale=c.scale, causal=True)["o"][0] * c.d_o[r].double()).sum())
            ends.append(total)
        got = float((getattr(c, "d" + name).double() * step).sum())
        for s, n in enumerate(c.nq):   # what the gradients' bounds leave, and the differences' third derivatives at this step
            r = slice(c.qs[s], c.qs[s] + n)
            slack += float((attention_ref.sequence(c.q[r], c.k[r], c.v[r], c.scale, True, c.d_o[r])["d" + name][1] * step[r].abs()).sum())
        assert abs((ends[0] - ends[1]) / (2 * h) - got) <= slack + 1e-4, name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_whatever_the_workspace_holds(dtype):
    c = both([300, 41], [300, 41], 4, 2, 128, True, dtype, seed=10)
    want = c.outputs()
    for fill in (0, 0x7F, 0x7E):
        c.forward(fill)
        c.backward(fill)
        for k, v in c.outputs().items():
            assert torch.equal(v, want[k]), k


def test_captured_and_replayed():
    """Replays with other inputs in the same places, the program's own work between them, against eager calls."""
    c = Case([200, 57], [200, 57], 4, 2, 64, True, "bfloat16", seed=11)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dll_attention_fwd(c.spec, *c.inputs(), c.o, c.lse, c.ws)
        B.dll_attention_bwd(c.spec, *c.inputs(), c.o, c.lse, c.d_o, c.dq, c.dk, c.dv, c.ws_b)
    for turn in range(3):
        other = Case([200, 57], [200, 57], 4, 2, 64, True, "bfloat16", seed=20 + turn)
        for t in ("q", "k", "v", "d_o"):
            getattr(c, t).copy_(getattr(other, t))
        if turn == 2:   # lengths are read on the device
            other = Case([57, 200], [57, 200], 4, 2, 64, True, "bfloat16", seed=20 + turn)
            for s, t in zip(c.starts, other.starts):
                s.copy_(t)
        for t in (c.o, c.lse, c.dq, c.dk, c.dv):
            t.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        other.forward()
        other.backward()
        torch.cuda.synchronize()
        for k, v in c.outputs().items():
            assert torch.equal(v, getattr(other, k)), (turn, k)


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    cases = [Case([500, 100], [500, 100], 8, 2, 128, True, "bfloat16", seed=12 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            c.forward(stream=s)
            c.backward(stream=s)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


@pytest.mark.parametrize("dtype,n,heads,kv_heads,dim", [("bfloat16", 2500, 2, 1, 128), ("bfloat16", 1500, 1, 1, 64), ("float32", 1100, 2, 2, 128)])
def test_long_sequences(dtype, n, heads, kv_heads, dim):
    both([n, 3], [n, 3], heads, kv_heads, dim, True, dtype, seed=14)


def test_many_sequences():
    """More than sixty-four times sixty-four: the search for a tile's sequence takes three rounds."""
    n = [(7 * s) % 4 for s in range(5000)]
    c = Case(n, n, 1, 1, 16, True, "float32", seed=15)
    c.forward()
    c.backward()
    # one token: itself; two or three: the formula, all at once for sequences of one length
    for length in (1, 2, 3):
        at = torch.tensor([a for a, k in zip(c.qs, n) if k == length], device="cuda")
        rows = at[:, None] + torch.arange(length, device="cuda")
        q, k, v = (t[rows, 0].double() for t in (c.q, c.k, c.v))
        z = torch.where(torch.ones(length, length, device="cuda").tril() > 0, q @ k.transpose(1, 2) * c.scale, -torch.inf)
        want = torch.softmax(z, 2) @ v
        # sums of at most 16 and 3 terms of numbers below 6, exponents below 40
        assert (c.o[rows, 0] - want).abs().max() <= 6 * (ref.EXP * 2 + 64 * ref.gamma(16))
    assert torch.isfinite(c.dq).all() and torch.isfinite(c.dk).all() and torch.isfinite(c.dv).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_training_step(dtype):
    """Attention, a gated block and the loss over a vocabulary, then their gradients back to one buffer of q, k and v, cut to a norm.  Every operator is checked on
    what it was given; the step is captured and replayed with other inputs."""
    lengths, H, KV, D, hidden, classes = [70, 1, 129], 4, 2, 32, 96, 300
    T, width, t = sum(lengths), H * D, TYPES[dtype]
    c = Case(lengths, lengths, H, KV, D, True, dtype, seed=31, fused=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(32)
    wg, wu, wd, wv = (torch.randn(s, generator=gen, device="cuda").mul(0.1).to(t) for s in ((hidden, width), (hidden, width), (width, hidden), (classes, width)))
    labels = torch.randint(-30, classes, (T,), generator=gen, device="cuda", dtype=torch.int32)
    block, head = GatedSpec(T, width, hidden, "silu", dtype), VocabSpec(T, width, classes, dtype)
    nan = lambda *s, t=t: torch.full(s, NAN, dtype=t, device="cuda")
    y, dy, a, b = nan(T, width), nan(T, width), nan(T, hidden), nan(T, hidden)
    dwg, dwu, dwd, dwv = nan(hidden, width), nan(hidden, width), nan(width, hidden), nan(classes, width)
    row_loss, row_lse, loss, norm = nan(T, t=torch.float32), nan(T, t=torch.float32), nan(1, t=torch.float32), nan(1, t=torch.float32)
    grads = [c.dbuffer, dwg, dwu, dwd, dwv]
    cut, several = [torch.full_like(g, NAN) for g in grads], B.tensor_list(grads)
    ws = {f: B.workspace(getattr(B, f + "_workspace_bytes")(s)) for f, s in (
        ("dll_attention_fwd", c.spec), ("dll_attention_bwd", c.spec), ("dll_gated_fwd", block), ("dll_gated_bwd", block), ("dll_vocab_loss_grad", head),
        ("dll_grad_norm", several))}

    def step():
        B.dll_attention_fwd(c.spec, *c.inputs(), c.o, c.lse, ws["dll_attention_fwd"])
        rows = c.o.view(T, width)
        B.dll_gated_fwd(block, rows, wg, wu, wd, y, a, b, ws["dll_gated_fwd"])
        B.dll_vocab_loss_grad(head, y, wv, None, labels, 8.0, row_loss, row_lse, loss, dy, dwv, None, ws["dll_vocab_loss_grad"])
        B.dll_gated_bwd(block, rows, wg, wu, wd, a, b, dy, c.d_o.view(T, width), dwg, dwu, dwd, ws["dll_gated_bwd"])
        B.dll_attention_bwd(c.spec, *c.inputs(), c.o, c.lse, c.d_o, c.dq, c.dk, c.dv, ws["dll_attention_bwd"])
        B.dll_grad_clip(several, grads, cut, 0.25, norm, ws["dll_grad_norm"])

    results = lambda: [r.clone() for r in (c.o, c.lse, c.d_o, y, dy, loss, row_loss, row_lse, norm, *grads, *cut)]
    step()
    c.check()
    rows = c.o.view(T, width)
    want = ref.gated(rows, wg, wu, wd, "silu", dy)
    for k, v in {"y": y, "gate_pre": a, "up_pre": b, "dx": c.d_o.view(T, width), "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}.items():
        ref.check(v, want[k], k)
    want = ref.vocab(y, wv, None, labels, scale=8.0)
    for k, v in {"loss": loss, "row_loss": row_loss, "row_lse": row_lse, "dx": dy, "dw": dwv}.items():
        ref.check(v, want[k], k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        c.buffer.copy_(Case(lengths, lengths, H, KV, D, True, dtype, seed=33 + turn, fused=True).buffer)
        step()
        eager = results()
        for r in (c.o, c.lse, c.d_o, y, a, b, dy, loss, row_loss, row_lse, norm, *grads, *cut):
            r.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, z) in enumerate(zip(results(), eager)):
            assert torch.isfinite(z).all() and torch.equal(x, z), (turn, i)
