"""Refusals and workspace queries of attention and the paged cache: on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import AttentionSpec, CacheSpec

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
P = [C.c_void_p(0x10000 * k) for k in range(1, 20)]   # never dereferenced: every call below is refused
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")


def attention(**over):
    d = B.attention_desc(AttentionSpec(16, 24, 2, 4, 2, 64, True, "bfloat16"))
    for k, v in over.items():
        setattr(d, k, v)
    return C.byref(d)


def forward(L, d, p=P, scale=1.0, ws=P[14], room=BIG, lse=P[6]):
    return L.dll_attention_fwd(d, *p[:5], scale, p[5], lse, ws, room, None)


def backward(L, d, p=P, scale=1.0, ws=P[14], room=BIG):
    return L.dll_attention_bwd(d, *p[:5], scale, *p[5:11], ws, room, None)


@pytest.mark.parametrize("over,status", [
    (dict(q_tokens=0), SHAPE), (dict(kv_tokens=-1), SHAPE), (dict(sequences=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(heads=5), SHAPE), (dict(heads=1), SHAPE), (dict(q_row=255), SHAPE), (dict(kv_row=127), SHAPE),
    (dict(q_row=-1), SHAPE), (dict(kv_row=-256), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(causal=2), UNSUPPORTED), (dict(causal=-1), UNSUPPORTED),
    (dict(head_dim=257), UNSUPPORTED), (dict(heads=4098), UNSUPPORTED), (dict(q_tokens=(1 << 24) + 1), UNSUPPORTED),
    (dict(q_tokens=1 << 23), UNSUPPORTED), (dict(kv_tokens=1 << 24), UNSUPPORTED), (dict(kv_tokens=1 << 12, kv_row=1 << 19), UNSUPPORTED),
    (dict(q_row=(1 << 20) + 1), UNSUPPORTED), (dict(sequences=(1 << 20) + 1), UNSUPPORTED), (dict(sequences=1 << 20, heads=4094), UNSUPPORTED)], ids=str)
def test_attention_descriptors(over, status):
    L = B.lib()
    d = attention(**over)
    assert L.dll_attention_fwd_workspace_bytes(d) == 0 and L.dll_attention_bwd_workspace_bytes(d) == 0
    assert forward(L, d) == status and backward(L, d) == status


def test_attention_pointers():
    L = B.lib()
    d = attention()
    need, need_b = L.dll_attention_fwd_workspace_bytes(d), L.dll_attention_bwd_workspace_bytes(d)
    assert need > 0 and need % 256 == 0 and need_b > 0 and need_b % 256 == 0
    swap = lambda k, v: [*P[:k], v, *P[k + 1:]]
    at = lambda k, off: C.c_void_p(P[k].value + off)
    for k in range(6):
        assert forward(L, d, swap(k, None)) == NULL
    for k in range(8):   # q, k, v, starts, o, lse, d_o
        assert backward(L, d, swap(k, None)) == NULL
    assert backward(L, d, [*P[:8], None, None, None]) == NULL
    for k in (0, 1, 2):   # q, k and v at any element, but no part of one
        assert forward(L, d, swap(k, at(k, 2)), room=0) == WORKSPACE and forward(L, d, swap(k, at(k, 1))) == SHAPE
        assert backward(L, d, swap(k, at(k, 2)), room=0) == WORKSPACE and backward(L, d, swap(k, at(k, 1))) == SHAPE
    assert forward(L, d, swap(5, at(5, 8))) == SHAPE and backward(L, d, swap(5, at(5, 8))) == SHAPE and backward(L, d, swap(7, at(7, 8))) == SHAPE
    for k in (3, 4):
        assert forward(L, d, swap(k, at(k, 2))) == SHAPE and backward(L, d, swap(k, at(k, 2))) == SHAPE
    assert forward(L, d, lse=at(6, 2)) == SHAPE and backward(L, d, swap(6, at(6, 2))) == SHAPE
    for k in (8, 9, 10):
        assert backward(L, d, swap(k, at(k, 2)), room=0) == WORKSPACE and backward(L, d, swap(k, at(k, 1))) == SHAPE
    assert forward(L, d, swap(4, P[3]), room=0) == WORKSPACE   # one array for both starts
    assert forward(L, d, swap(5, P[0])) == SHAPE               # o is q
    assert forward(L, d, lse=P[5]) == SHAPE and forward(L, d, ws=P[1]) == SHAPE
    assert backward(L, d, swap(8, P[7])) == SHAPE              # dq is d_o
    assert backward(L, d, swap(9, P[8])) == SHAPE              # one buffer for two gradients
    for bad in (INF, -INF, NAN):
        assert forward(L, d, scale=bad) == SHAPE and backward(L, d, scale=bad) == SHAPE
    assert forward(L, d, room=need - 1) == WORKSPACE and forward(L, d, ws=None) == WORKSPACE and forward(L, d, ws=at(14, 16)) == WORKSPACE
    assert backward(L, d, room=need_b - 1) == WORKSPACE and backward(L, d, ws=None) == WORKSPACE
    assert forward(L, None) == NULL and backward(L, None) == NULL
    assert L.dll_attention_fwd_workspace_bytes(None) == 0


def test_binding_checks_rows():
    cpu = torch.device("cpu")
    buffer = torch.zeros(5, 8, 16)
    q, k, _ = buffer.split([4, 2, 2], 1)
    assert B._head_rows(q, (5, 4, 16), 128, torch.float32, "q", cpu) == buffer.data_ptr()
    assert B._head_rows(k, (5, 2, 16), 128, torch.float32, "k", cpu) == buffer.data_ptr() + 4 * 64
    assert B._head_rows(k[:1], (1, 2, 16), 0, torch.float32, "k", cpu) == k.data_ptr()   # one token: no next row
    assert B._head_rows(None, (5, 2, 16), 0, torch.float32, "dk", cpu, True) is None
    for bad, row in ((k, 0), (k, 64), (q.transpose(1, 2), 128), (q.to(torch.bfloat16), 128), (q[:, :3], 128), (None, 128)):
        with pytest.raises(ValueError):
            B._head_rows(bad, (5, 2 if bad is k else 4, 16), row, torch.float32, "k", cpu)
    with pytest.raises(KeyError):
        B.attention_desc(AttentionSpec(1, 1, 1, 1, 1, 1, True, "float16"))


def cache(**over):
    d = B.cache_desc(CacheSpec(4, 8, 2, 64, 100, 16, 10, "float32"))
    for k, v in over.items():
        setattr(d, k, v)
    return C.byref(d)


def plan(L, d, p=P, n_free=5, free_at=P[17], tokens=9):
    return L.dll_cache_plan(d, p[0], p[1], p[2], n_free, free_at, *p[3:6], tokens, p[6], None)


def store(L, d, p=P, tokens=9, row=0):
    return L.dll_cache_write(d, tokens, row, *p[:5], None)


def paged(L, d, p=P, scale=1.0, lse=P[12], ws=P[14], room=BIG):
    return L.dll_paged_attention(d, *p[:5], scale, p[5], lse, ws, room, None)


@pytest.mark.parametrize("over,status", [
    (dict(requests=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=7), SHAPE), (dict(kv_heads=-2), SHAPE), (dict(head_dim=0), SHAPE), (dict(pages=0), SHAPE),
    (dict(page_tokens=0), SHAPE), (dict(table_pages=-1), SHAPE), (dict(dtype=5), UNSUPPORTED), (dict(head_dim=257), UNSUPPORTED),
    (dict(requests=(1 << 16) + 1), UNSUPPORTED), (dict(requests=1 << 14, heads=1 << 11), UNSUPPORTED), (dict(pages=1 << 28), UNSUPPORTED),
    (dict(table_pages=(1 << 26) + 1), UNSUPPORTED), (dict(requests=1 << 12, table_pages=1 << 19), UNSUPPORTED)], ids=str)
def test_cache_descriptors(over, status):
    L = B.lib()
    d = cache(**over)
    assert L.dll_paged_attention_workspace_bytes(d) == 0
    assert plan(L, d) == store(L, d) == paged(L, d) == status


def test_cache_pointers():
    L = B.lib()
    d = cache()
    swap = lambda k, v: [*P[:k], v, *P[k + 1:]]
    at = lambda k, off: C.c_void_p(P[k].value + off)
    for k in range(7):
        assert plan(L, d, swap(k, None)) == NULL and plan(L, d, swap(k, at(k, 2))) == SHAPE
    assert plan(L, None) == store(L, None) == paged(L, None) == NULL
    assert plan(L, d, n_free=-1) == SHAPE and plan(L, d, tokens=0) == SHAPE and plan(L, d, tokens=(1 << 24) + 1) == UNSUPPORTED
    assert plan(L, d, free_at=P[6]) == SHAPE and plan(L, d, free_at=at(17, 2)) == SHAPE   # other workgroups still read it
    assert plan(L, d, swap(3, P[2])) == SHAPE and plan(L, d, swap(4, P[0])) == SHAPE and plan(L, d, swap(5, P[4])) == SHAPE
    for k in range(5):
        assert store(L, d, swap(k, None)) == NULL
    for k, off in ((0, 2), (1, 1), (2, 2), (3, 8), (4, 4)):
        assert store(L, d, swap(k, at(k, off))) == SHAPE
    assert store(L, d, tokens=0) == SHAPE and store(L, d, row=127) == SHAPE and store(L, d, row=-1) == SHAPE
    assert store(L, d, tokens=(1 << 24) + 1) == store(L, d, row=(1 << 20) + 1) == store(L, d, tokens=1 << 20, row=1 << 11) == UNSUPPORTED
    assert store(L, d, swap(3, P[0])) == SHAPE and store(L, d, swap(4, P[3])) == SHAPE
    need = L.dll_paged_attention_workspace_bytes(d)
    assert need > 0 and need % 256 == 0
    for k in range(6):
        assert paged(L, d, swap(k, None)) == NULL
    for k, off in ((0, 8), (1, 8), (2, 8), (3, 2), (4, 2), (5, 8)):
        assert paged(L, d, swap(k, at(k, off))) == SHAPE
    assert paged(L, d, lse=at(12, 2)) == SHAPE and paged(L, d, lse=P[5]) == SHAPE and paged(L, d, swap(5, P[0])) == SHAPE
    for bad in (INF, NAN):
        assert paged(L, d, scale=bad) == SHAPE
    assert paged(L, d, room=need - 1) == paged(L, d, ws=None) == paged(L, d, ws=at(14, 16)) == WORKSPACE
    assert paged(L, d, lse=None, room=0) == WORKSPACE
