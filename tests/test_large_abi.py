"""Refusals and workspace queries of the large-model operators: on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import GatedSpec, VocabSpec

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
P = [C.c_void_p(0x10000 * k) for k in range(1, 16)]   # never dereferenced: every call below is refused
BIG = 1 << 40


def gated(**over):
    d = B.gated_desc(GatedSpec(16, 24, 40, "silu", "bfloat16"))
    for k, v in over.items():
        setattr(d, k, v)
    return C.byref(d)


def vocab(**over):
    d = B.vocab_desc(VocabSpec(16, 24, 40, "float32"))
    for k, v in over.items():
        setattr(d, k, v)
    return C.byref(d)


BAD_SIZES = [(dict(tokens=0), SHAPE), (dict(tokens=-1), SHAPE), (dict(width=0), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
             (dict(tokens=(1 << 24) + 1), UNSUPPORTED), (dict(width=(1 << 20) + 1), UNSUPPORTED), (dict(tokens=1 << 24, width=128), UNSUPPORTED)]


@pytest.mark.parametrize("over,status", BAD_SIZES + [(dict(hidden=0), SHAPE), (dict(gate=5), UNSUPPORTED), (dict(gate=-1), UNSUPPORTED),
                                                     (dict(hidden=1 << 20, width=1 << 11), UNSUPPORTED), (dict(tokens=1 << 20, hidden=1 << 11), UNSUPPORTED)])
def test_gated_descriptors(over, status):
    L = B.lib()
    d = gated(**over)
    assert L.dll_gated_fwd_workspace_bytes(d) == 0 and L.dll_gated_bwd_workspace_bytes(d) == 0
    assert L.dll_gated_fwd(d, *P[:7], P[7], BIG, None) == status
    assert L.dll_gated_bwd(d, *P[:11], P[11], BIG, None) == status


@pytest.mark.parametrize("over,status", BAD_SIZES + [(dict(classes=0), SHAPE), (dict(classes=(1 << 20) + 1), UNSUPPORTED)])
def test_vocab_descriptors(over, status):
    L = B.lib()
    d = vocab(**over)
    assert L.dll_vocab_loss_fwd_workspace_bytes(d) == 0 and L.dll_vocab_loss_grad_workspace_bytes(d) == 0
    assert L.dll_vocab_loss_fwd(d, *P[:7], P[7], BIG, None) == status
    assert L.dll_vocab_loss_grad(d, *P[:4], 1.0, *P[4:10], P[10], BIG, None) == status


def test_gated_pointers():
    L = B.lib()
    d, need = gated(), B.dll_gated_fwd_workspace_bytes(GatedSpec(16, 24, 40, "silu", "bfloat16"))
    assert need > 0 and need % 256 == 0
    for k in range(5):   # x, w_gate, w_up, w_down, y
        a = list(P[:7])
        a[k] = None
        assert L.dll_gated_fwd(d, *a, P[7], BIG, None) == NULL
    assert L.dll_gated_fwd(d, *P[:5], P[5], None, P[7], BIG, None) == NULL            # one of the kept pair alone
    assert L.dll_gated_fwd(d, *P[:4], P[0], None, None, P[7], BIG, None) == SHAPE     # y is x
    assert L.dll_gated_fwd(d, *P[:5], P[5], P[5], P[7], BIG, None) == SHAPE           # one buffer for both kept
    assert L.dll_gated_fwd(d, *P[:5], None, None, P[4], BIG, None) == SHAPE           # y is the workspace
    assert L.dll_gated_fwd(d, C.c_void_p(0x10008), *P[1:5], None, None, P[7], BIG, None) == SHAPE   # 8 bytes off
    assert L.dll_gated_fwd(d, *P[:5], None, None, None, BIG, None) == WORKSPACE
    assert L.dll_gated_fwd(d, *P[:5], None, None, P[7], need - 1, None) == WORKSPACE
    assert L.dll_gated_fwd(d, *P[:5], None, None, C.c_void_p(0x80010), BIG, None) == WORKSPACE
    for k in range(7):   # inputs of the backward pass
        a = list(P[:11])
        a[k] = None
        assert L.dll_gated_bwd(d, *a, P[11], BIG, None) == NULL
    assert L.dll_gated_bwd(d, *P[:7], None, None, None, None, P[11], BIG, None) == NULL      # nothing asked for
    assert L.dll_gated_bwd(d, *P[:7], P[6], None, None, None, P[11], BIG, None) == SHAPE     # dx is dy
    assert L.dll_gated_bwd(d, *P[:7], None, P[8], P[8], None, P[11], BIG, None) == SHAPE     # one buffer for two gradients
    assert L.dll_gated_bwd(d, *P[:11], P[11], 256, None) == WORKSPACE
    assert L.dll_gated_fwd(None, *P[:7], P[7], BIG, None) == NULL and L.dll_gated_bwd(None, *P[:11], P[11], BIG, None) == NULL


def test_vocab_pointers():
    L = B.lib()
    d = vocab()
    x, w, bias, labels, row, lse, loss, dx, dw, db, ws = P[:11]
    for a in ((None, w, bias, labels, row, lse, loss), (x, None, bias, labels, row, lse, loss), (x, w, bias, None, row, lse, loss), (x, w, bias, labels, row, lse, None)):
        assert L.dll_vocab_loss_fwd(d, *a, ws, BIG, None) == NULL
        assert L.dll_vocab_loss_grad(d, *a[:4], 1.0, *a[4:], dx, dw, db, ws, BIG, None) == NULL
    assert L.dll_vocab_loss_grad(d, x, w, bias, labels, 1.0, row, lse, loss, None, None, None, ws, BIG, None) == NULL
    assert L.dll_vocab_loss_grad(d, x, w, None, labels, 1.0, row, lse, loss, dx, dw, db, ws, BIG, None) == NULL      # dbias without bias
    assert L.dll_vocab_loss_grad(d, x, w, bias, labels, 1.0, row, lse, loss, x, dw, db, ws, BIG, None) == SHAPE      # dx is x
    assert L.dll_vocab_loss_grad(d, x, w, bias, labels, 1.0, row, lse, loss, dx, dx, db, ws, BIG, None) == SHAPE
    assert L.dll_vocab_loss_fwd(d, x, w, bias, labels, row, row, loss, ws, BIG, None) == SHAPE
    assert L.dll_vocab_loss_fwd(d, x, C.c_void_p(0x20004), bias, labels, row, lse, loss, ws, BIG, None) == SHAPE
    assert L.dll_vocab_loss_fwd(d, x, w, bias, labels, row, lse, loss, ws, 255, None) == WORKSPACE
    assert L.dll_vocab_loss_grad(d, x, w, bias, labels, 1.0, row, lse, loss, dx, dw, db, None, BIG, None) == WORKSPACE
    assert L.dll_vocab_loss_fwd(None, x, w, bias, labels, row, lse, loss, ws, BIG, None) == NULL


def test_workspaces_do_not_grow_with_tokens_times_classes():
    """The exponentials of a piece of tokens: 1 GiB however many tokens there are."""
    one = B.dll_vocab_loss_grad_workspace_bytes(VocabSpec(1 << 13, 64, 1 << 17, "bfloat16"))
    many = B.dll_vocab_loss_grad_workspace_bytes(VocabSpec(1 << 20, 64, 1 << 17, "bfloat16"))
    assert one < many < 2 * one and many < 3 << 30
    assert B.dll_vocab_loss_fwd_workspace_bytes(VocabSpec(1 << 20, 64, 1 << 17, "bfloat16")) < 1 << 30


def pointers(*p):
    return (C.c_void_p * len(p))(*p)


def test_tensor_lists():
    L = B.lib()

    def listed(counts, dtypes, n=None):
        k = len(counts)
        return C.byref(B.dll_tensor_list(k if n is None else n, (C.c_size_t * k)(*counts), (C.c_int * k)(*dtypes)))

    l = listed([3, 0, 5], [0, 1, 1])
    need = L.dll_grad_norm_workspace_bytes(l)
    assert need > 0 and need % 256 == 0
    g, norm, ws = pointers(0x1000, None, 0x2002), P[0], P[1]
    assert L.dll_grad_norm_workspace_bytes(None) == 0 and L.dll_grad_norm(None, g, norm, ws, BIG, None) == NULL
    assert L.dll_grad_norm_workspace_bytes(listed([1], [0], 0)) == 0 and L.dll_grad_norm(listed([1], [0], 0), g, norm, ws, BIG, None) == SHAPE
    assert L.dll_grad_norm(listed([1], [2]), g, norm, ws, BIG, None) == UNSUPPORTED
    assert L.dll_grad_norm(listed([1 << 40], [0]), g, norm, ws, BIG, None) == UNSUPPORTED
    assert L.dll_grad_norm(l, None, norm, ws, BIG, None) == NULL and L.dll_grad_norm(l, g, None, ws, BIG, None) == NULL
    assert L.dll_grad_norm(l, pointers(0x1000, None, None), norm, ws, BIG, None) == NULL      # 5 elements at NULL
    assert L.dll_grad_norm(l, pointers(0x1002, None, 0x2002), norm, ws, BIG, None) == SHAPE   # fp32 at an odd place
    assert L.dll_grad_norm(l, g, norm, None, BIG, None) == WORKSPACE and L.dll_grad_norm(l, g, norm, ws, need - 1, None) == WORKSPACE
    for bad in (0.0, -1.0, float("nan")):
        assert L.dll_grad_clip(l, g, g, bad, norm, ws, BIG, None) == SHAPE
        assert L.dll_momentum_update_clipped(l, g, g, g, 0.1, 0.9, None, bad, norm, None, ws, BIG, None) == SHAPE
    assert L.dll_grad_clip(l, g, None, 1.0, norm, ws, BIG, None) == NULL
    assert L.dll_grad_clip(l, g, pointers(0x1000, None, None), 1.0, norm, ws, BIG, None) == NULL
    assert L.dll_grad_clip(l, g, pointers(0x1000, None, 0x2001), 1.0, norm, ws, BIG, None) == SHAPE
    assert L.dll_grad_clip(l, g, g, 1.0, norm, ws, 0, None) == WORKSPACE
    p, v = pointers(0x3000, None, 0x4000), pointers(0x5000, None, 0x6000)
    assert L.dll_momentum_update_clipped(l, None, v, g, 0.1, 0.9, None, 1.0, norm, None, ws, BIG, None) == NULL
    assert L.dll_momentum_update_clipped(l, p, pointers(0x5000, None, None), g, 0.1, 0.9, None, 1.0, norm, None, ws, BIG, None) == NULL
    assert L.dll_momentum_update_clipped(l, p, p, g, 0.1, 0.9, None, 1.0, norm, None, ws, BIG, None) == SHAPE     # velocity is theta
    assert L.dll_momentum_update_clipped(l, p, v, p, 0.1, 0.9, None, 1.0, norm, None, ws, BIG, None) == SHAPE     # gradient is theta
    assert L.dll_momentum_update_clipped(l, p, v, g, 0.1, 0.9, None, 1.0, norm, p, ws, BIG, None) == SHAPE        # copy is theta
    assert L.dll_momentum_update_clipped(l, pointers(0x3002, None, 0x4000), v, g, 0.1, 0.9, None, 1.0, norm, None, ws, BIG, None) == SHAPE
    assert L.dll_momentum_update_clipped(l, p, v, g, 0.1, 0.9, None, 1.0, norm, None, None, BIG, None) == WORKSPACE


def test_no_tensor_is_written_twice():
    """Every list is refused for an output that is another output, another tensor's gradient or the norm."""
    L, ws = B.lib(), P[1]
    for n in (2, 3, 150):   # addresses on the stack, and more than fit there
        l = C.byref(B.dll_tensor_list(n, (C.c_size_t * n)(*[4] * n), (C.c_int * n)(*[0] * n)))
        at = lambda base, **over: pointers(*[over.get(f"k{k}", base + 64 * k) for k in range(n)])
        g, p, v, c = 0x100000, 0x200000, 0x300000, 0x400000
        last = f"k{n - 1}"
        clip = lambda out, norm=P[0]: L.dll_grad_clip(l, at(g), out, 1.0, norm, ws, 0, None)
        assert clip(at(g)) == clip(at(p)) == WORKSPACE   # nothing else to refuse
        assert clip(at(p, **{last: p})) == SHAPE         # two outputs
        assert clip(at(p, **{last: g})) == SHAPE         # another tensor's gradient
        assert clip(at(g, **{last: g})) == SHAPE
        assert clip(at(p), C.c_void_p(p)) == clip(at(p), C.c_void_p(g)) == SHAPE
        twice = at(g, **{last: g})
        assert L.dll_grad_clip(l, twice, twice, 1.0, P[0], ws, 0, None) == SHAPE      # the same tensor twice, in place
        assert L.dll_grad_clip(l, twice, at(p), 1.0, P[0], ws, 0, None) == WORKSPACE  # read twice, written apart
        step = lambda params, vel, copies=None, grads=None, norm=P[0]: L.dll_momentum_update_clipped(
            l, params, vel, grads or at(g), 0.1, 0.9, None, 1.0, norm, copies, ws, 0, None)
        assert step(at(p), at(v)) == step(at(p), at(v), at(c)) == step(at(p), at(v), pointers(*[None] * n)) == WORKSPACE
        assert step(at(p, **{last: p}), at(v)) == step(at(p), at(v, **{last: v})) == step(at(p), at(v), at(c, **{last: c})) == SHAPE
        assert step(at(p), at(v, **{last: p})) == step(at(p), at(v), at(c, k0=p)) == step(at(p, **{last: g}), at(v)) == SHAPE
        assert step(at(p), at(v), at(c, **{last: g})) == step(at(p), at(v), norm=C.c_void_p(v)) == SHAPE


def test_binding_checks_what_an_address_cannot_say():
    cpu = torch.device("cpu")
    t = torch.zeros(4, 6)
    assert B._tensor(t, (4, 6), torch.float32, "x", cpu) == t.data_ptr()
    assert B._tensor(None, (4, 6), torch.float32, "x", cpu, True) is None
    for bad in (None, t.to(torch.bfloat16), torch.zeros(6, 4), torch.zeros(6, 4).t(), torch.zeros(4, 6, device="meta")):
        with pytest.raises(ValueError):
            B._tensor(bad, (4, 6), torch.float32, "x", cpu)
    g = [torch.zeros(3), torch.zeros(2, 5, dtype=torch.bfloat16), torch.zeros(0)]
    l = B.tensor_list(g)
    assert list(l.counts) == [3, 10, 0] and list(l.dtypes) == [0, 1, 0]
    assert len(B._list_ptrs(g, l, l.torch_types, "grads", cpu)) == 3
    for bad in (g[:2], [g[0], g[1].float(), g[2]], [g[0], None, g[2]], [torch.zeros(4), g[1], g[2]], [torch.zeros(6)[::2], g[1], g[2]]):
        with pytest.raises(ValueError):
            B._list_ptrs(bad, l, l.torch_types, "grads", cpu)
    with pytest.raises(ValueError):
        B.tensor_list([torch.zeros(3, dtype=torch.float16)])
    with pytest.raises(ValueError):
        B._ws(torch.zeros(8, device="meta"), cpu)
    with pytest.raises(KeyError):
        B.gated_desc(GatedSpec(1, 1, 1, "tanh", "float32"))
    with pytest.raises(KeyError):
        B.vocab_desc(VocabSpec(1, 1, 1, "float16"))
