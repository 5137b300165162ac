"""Strides and counts beyond the library's 32-bit arguments are refused where the binding makes arguments of them (no GPU needed: tensors without memory)."""
import pytest
import torch

from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import AttentionSpec, CacheSpec

META = torch.device("meta")


class Refuses:
    """In the library's place."""

    def __getattr__(self, name):
        return lambda *args: pytest.fail("the call went on")


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    monkeypatch.setattr(B, "_call_stream", lambda stream: B._CurrentStream(META, 0))
    monkeypatch.setattr(B, "lib", Refuses)


def rows(tokens, heads, dim, row):
    return torch.empty_strided((tokens, heads, dim), (row, dim, 1), dtype=torch.bfloat16, device=META)


def test_rows_too_far_apart():
    far = (1 << 32) + 16   # the lower half is a row's length
    spec = AttentionSpec(2, 2, 1, 1, 1, 16, q_row=far, kv_row=far)
    q, starts, o = rows(2, 1, 16, far), torch.empty(2, dtype=torch.int32, device=META), rows(2, 1, 16, 16)
    with pytest.raises(ValueError, match="apart"):
        B.dll_attention_fwd(spec, q, q, q, starts, starts, 1.0, o)
    with pytest.raises(ValueError, match="apart"):
        B.dll_attention_bwd(spec, q, q, q, starts, starts, 1.0, o, None, o, q)
    cache = torch.empty(4, 1, 4, 16, dtype=torch.bfloat16, device=META)
    with pytest.raises(ValueError, match="apart"):
        B.dll_cache_write(CacheSpec(1, 1, 1, 16, 4, 4, 4), q, q, starts, cache, cache)


def test_too_many_entries():
    spec, many = CacheSpec(1, 1, 1, 16, 4, 4, 4), torch.empty((1 << 32) + 5, dtype=torch.int32, device=META)
    one, table, two = (torch.empty(s, dtype=torch.int32, device=META) for s in (1, (1, 4), 2))
    with pytest.raises(ValueError, match="entries"):
        B.dll_cache_plan(spec, one, one, many, table, two, one, two)
    with pytest.raises(ValueError, match="entries"):
        B.dll_cache_plan(spec, one, one, one, table, two, many, two)
