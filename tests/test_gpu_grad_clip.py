"""Global gradient norm, clipping and the clipped momentum step on the GPU against 64 bits; and the large-model operators
together, as a training loop uses them."""
import math

import pytest

torch = pytest.importorskip("torch")

import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd import workloads as wl
from paper_1804_04512_amd.workloads import GatedSpec, VocabSpec

pytestmark = pytest.mark.gpu

U32 = ref.U32
LISTS = {"one": [1], "few": [200, 8, 1600, 8, 19200, 150, 1500, 10], "empty": [0, 5, 0], "nothing": [0], "odd": [8191, 8192, 8193, 1, 7, 100003], "many": [3 + 5 * k for k in range(150)],
         "long": [3000001]}


def tensors(counts, dtypes, std=1.0, seed=0, shift=0):
    """Views into one buffer each, `shift` elements behind a 16-byte boundary."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return [(torch.randn(n + shift, generator=gen, device="cuda") * std).to(d)[shift:] for n, d in zip(counts, dtypes)]


def types(name, n):
    return [{"float32": torch.float32, "bfloat16": torch.bfloat16, "mixed": [torch.float32, torch.bfloat16][k % 2]}[name] for k in range(n)]


def exact_norm(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def ws_of(l):
    return B.workspace(B.dll_grad_norm_workspace_bytes(l)).fill_(255)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "mixed"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("name", LISTS)
def test_norm_and_clip(name, shift, dtype):
    counts = LISTS[name]
    g = tensors(counts, types(dtype, len(counts)), seed=len(counts), shift=shift)
    l, norm = B.tensor_list(g), torch.full((1,), float("nan"), device="cuda")
    B.dll_grad_norm(l, g, norm, ws_of(l))
    want = exact_norm(g)
    assert abs(float(norm) - want) <= 2 * U32 * want
    for max_norm, c in ((want / 3, 1 / 3), (2 * want + 1, 1.0), (math.inf, 1.0)):
        if max_norm == 0:
            continue
        c32 = min(1.0, max_norm / want) if want else 1.0
        out, norm2 = [torch.full_like(t, float("nan")) for t in g], torch.zeros(1, device="cuda")
        B.dll_grad_clip(l, g, out, max_norm, norm2, ws_of(l))
        assert torch.equal(norm, norm2)
        for a, b in zip(out, g):
            v = b.double() * c32   # the factor rounded to 32 bits, the product rounded to 32 bits, then to its type
            ref.check(a, (v, (3 * U32 + ref.unit(a.dtype)) * v.abs() + 2.0 ** -149), name)
        again = [t.clone() for t in g]
        B.dll_grad_clip(l, again, again, max_norm, norm2, ws_of(l))
        assert all(torch.equal(a, b) for a, b in zip(again, out))


def test_extremes():
    """Squares that 32 bits do not hold, either way; zeros; norms that are not finite."""
    norm = torch.zeros(1, device="cuda")
    for scale in (1e30, 1e-30):
        g = [torch.full((1000,), scale, device="cuda"), torch.full((24,), scale, device="cuda")]
        l = B.tensor_list(g)
        out = [torch.empty_like(t) for t in g]
        B.dll_grad_clip(l, g, out, 16 * scale, norm, ws_of(l))
        assert abs(float(norm) / (32 * scale) - 1) < 1e-6   # sqrt(1024); the inputs themselves are rounded to 2^-24
        assert abs(float(out[0][5]) / (scale / 2) - 1) < 1e-6
    z = [torch.zeros(100, device="cuda")]
    l = B.tensor_list(z)
    B.dll_grad_clip(l, z, z, 1.0, norm, ws_of(l))
    assert float(norm) == 0 and not z[0].any()
    for bad in (float("inf"), float("nan")):
        g = [torch.ones(100, device="cuda"), torch.tensor([bad, 2.0], device="cuda")]
        l, out = B.tensor_list(g), [torch.empty(100, device="cuda"), torch.empty(2, device="cuda")]
        B.dll_grad_clip(l, g, out, 1.0, norm, ws_of(l))
        assert not math.isfinite(float(norm)) and torch.equal(out[0], g[0]) and float(out[1][1]) == 2
        p, v = [torch.ones(100, device="cuda"), torch.ones(2, device="cuda")], [torch.ones(100, device="cuda"), torch.ones(2, device="cuda")]
        B.dll_momentum_update_clipped(l, p, v, g, 0.1, 0.9, None, 1.0, norm, ws=ws_of(l))
        assert not math.isfinite(float(norm)) and all(bool((t == 1).all()) for t in p + v)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "mixed"])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("name", ["one", "few", "empty", "odd", "many"])
def test_momentum_step(name, shift, dtype):
    counts = LISTS[name]
    n = len(counts)
    g = tensors(counts, types(dtype, n), seed=1, shift=shift)
    p, v = (tensors(counts, [torch.float32] * n, s, seed=k, shift=shift) for k, s in ((2, 1.0), (3, 0.1)))
    copies = [torch.full_like(t, float("nan"), dtype=torch.bfloat16) if k % 3 != 1 else None for k, t in enumerate(p)]
    decay = [0.01 * (k % 2) for k in range(n)]
    l, norm = B.tensor_list(g), torch.zeros(1, device="cuda")
    lr, mu, max_norm = 0.1, 0.9, exact_norm(g) / 2
    c = 0.5
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))
    want = []
    for k in range(n):
        gk, pk, vk = g[k].double(), p[k].double(), v[k].double()
        nv = f32(mu) * vk - f32(lr) * (c * gk + f32(decay[k]) * pk)
        # six roundings on the way to v, one more to theta
        ev = 8 * U32 * (f32(mu) * vk.abs() + f32(lr) * (c * gk.abs() + f32(decay[k]) * pk.abs()))
        want.append(((pk + nv, ev + U32 * (pk + nv).abs()), (nv, ev)))
    B.dll_momentum_update_clipped(l, p, v, g, lr, mu, decay, max_norm, norm, copies, ws=ws_of(l))
    for k in range(n):
        ref.check(p[k], want[k][0], "theta")
        ref.check(v[k], want[k][1], "v")
        if copies[k] is not None:
            assert torch.equal(copies[k], p[k].to(torch.bfloat16))


def test_same_as_the_network_step():
    """Gradients of the MNIST network from its step, then the update on its own: what the network's momentum step does."""
    w = wl.config2(batch=20)
    net = B.net_desc(w.conv, w.dense, w.classes)
    ws = B.workspace(B.dll_cnn_workspace_bytes(net))
    x, labels, loss = torch.from_numpy(w.x).cuda(), torch.from_numpy(w.labels).cuda(), torch.zeros(1, device="cuda")
    theta = [torch.from_numpy(t).cuda() for t in w.params]
    vel = [0.01 * torch.randn_like(t) for t in theta]
    mine, vmine = [t.clone() for t in theta], [t.clone() for t in vel]
    grads = [torch.empty_like(t) for t in theta]
    B.dll_cnn_train_step(net, mine, grads, x, labels, 0.0, loss, None, None, ws)
    l, norm = B.tensor_list(grads), torch.zeros(1, device="cuda")
    decay = [1e-3 * (k % 2 == 0) for k in range(len(grads))]
    B.dll_momentum_update_clipped(l, mine, vmine, grads, 0.1, 0.9, decay, math.inf, norm, ws=ws_of(l))
    B.dll_cnn_train_step_momentum(net, theta, vel, None, x, labels, 0.1, 0.9, 1e-3, loss, None, None, ws)
    for a, b, va, vb in zip(mine, theta, vmine, vel):
        # the same rule on the same gradients; contraction of its products and sums may differ by a rounding each
        assert float((a - b).abs().max()) <= 4 * U32 * float(b.abs().max() + vb.abs().max())
        assert float((va - vb).abs().max()) <= 8 * U32 * float(vb.abs().max() + 0.1 * b.abs().max())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_together(dtype):
    """Three steps of a block with a vocabulary behind it: forward, loss with gradients, backward, clipped step.  Each step's
    outputs are checked against 64 bits from the operands that the step itself saw."""
    T, D, H, V = 48, 64, 96, 301
    t = {"float32": torch.float32, "bfloat16": torch.bfloat16}[dtype]
    torch.manual_seed(0)
    master = [torch.randn(s, device="cuda") * s[-1] ** -0.5 for s in ((H, D), (H, D), (D, H), (V, D))]
    work = [m.to(t) if t != torch.float32 else m for m in master]
    vel = [torch.zeros_like(m) for m in master]
    gs, vs = GatedSpec(T, D, H, "silu", dtype), VocabSpec(T, D, V, dtype)
    x, labels = torch.randn(T, D, device="cuda").to(t), torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32)
    e = lambda *s, d=t: torch.empty(s, dtype=d, device="cuda")
    y, a, b, dy = e(T, D), e(T, H), e(T, H), e(T, D)
    grads = [torch.empty_like(w) for w in work]
    losses, loss, norm = [], e(1, d=torch.float32), e(1, d=torch.float32)
    l = B.tensor_list(grads)
    ws = B.workspace(max(B.dll_gated_fwd_workspace_bytes(gs), B.dll_gated_bwd_workspace_bytes(gs), B.dll_vocab_loss_grad_workspace_bytes(vs),
                         B.dll_grad_norm_workspace_bytes(l)))
    for step in range(3):
        before = [w.clone() for w in work]
        B.dll_gated_fwd(gs, x, *work[:3], y, a, b, ws=ws)
        B.dll_vocab_loss_grad(vs, y, work[3], None, labels, 1.0, None, None, loss, dy, grads[3], ws=ws)
        B.dll_gated_bwd(gs, x, *work[:3], a, b, dy, None, *grads[:3], ws=ws)
        B.dll_momentum_update_clipped(l, master, vel, grads, 0.5, 0.9, None, 0.5, norm, None if t == torch.float32 else work, ws=ws)
        block = ref.gated(x, *before[:3], "silu", dy)
        head = ref.vocab(y, before[3], None, labels)
        ref.check(y, block["y"], "y")
        ref.check(loss, head["loss"], "loss")
        ref.check(dy, head["dx"], "dy")
        ref.check(grads[3], head["dw"], "dw")
        for k, n in enumerate(("dw_gate", "dw_up", "dw_down")):
            ref.check(grads[k], block[n], n)
        assert abs(float(norm) / exact_norm(grads) - 1) <= 2 * U32
        if t != torch.float32:
            assert all(torch.equal(w, m.to(t)) for w, m in zip(work, master))


def test_graph_replays():
    counts = LISTS["few"] + [70000] * 70
    g = tensors(counts, types("mixed", len(counts)))
    p, v = tensors(counts, [torch.float32] * len(counts), seed=1), tensors(counts, [torch.float32] * len(counts), seed=2)
    l, norm, norm2 = B.tensor_list(g), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    out = [torch.zeros_like(t) for t in g]
    ws = ws_of(l)
    B.dll_grad_clip(l, g, out, 1.0, norm, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dll_grad_clip(l, g, out, 1.0, norm, ws)
        B.dll_momentum_update_clipped(l, p, v, out, 0.1, 0.9, None, 0.5, norm2, ws=ws)
    pe, ve = [t.clone() for t in p], [t.clone() for t in v]
    for k in range(3):
        for t in g:
            t.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        oe, ne = [torch.zeros_like(t) for t in g], torch.zeros(1, device="cuda")
        B.dll_grad_clip(l, g, oe, 1.0, ne, ws_of(l))
        assert torch.equal(ne, norm) and all(torch.equal(a, b) for a, b in zip(oe, out))
        B.dll_momentum_update_clipped(l, pe, ve, oe, 0.1, 0.9, None, 0.5, ne, ws=ws_of(l))
        assert torch.equal(ne, norm2) and all(torch.equal(a, b) for a, b in zip(pe + ve, p + v))
