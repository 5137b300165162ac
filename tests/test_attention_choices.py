"""Which kernels of the backward pass stand on both sides of a size, found out without a GPU: the choice goes by how the call fills the chip, and neighbours of
a size take the same way."""
import pytest

from attention_launches import record


def ways(calls, folder):
    """(groups of 32 queries a workgroup of dq, whether values lie in LDS) for each."""
    out = []
    for status, names in record([["backward", *c, "bfloat16"] for c in calls], folder):
        assert status == 0
        dq = next(n for n in names if "attention_dq_kernel" in n)
        dkv = next(n for n in names if "attention_dkv_kernel" in n)
        out.append((2 if "ELi2ELNS" in dq else 4, "4FormE1" in dkv))
    return out


@pytest.mark.parametrize("heads,kv_heads,around", [(16, 16, 4096), (8, 8, 8192), (32, 32, 2048), (32, 8, 8192), (16, 4, 16384)])
def test_neighbours_take_the_same_way(heads, kv_heads, around, tmp_path):
    """Keys and values: 6 % more tokens, and one more, change nothing; a call of one more changes neither."""
    calls = [(t, t, 1, heads, kv_heads, 128, True) for t in (around - 1, around, around + 1, around + around // 16)]
    assert len({less for _, less in ways(calls, tmp_path)}) == 1


def test_fewer_tokens_with_as_many_heads(tmp_path):
    """16 heads of 128: parts would cost more than they win below 4096 tokens, too, and dq's workgroups are small until the chip is full."""
    calls = [(t, t, 1, 16, 16, 128, True) for t in (2304, 2560, 3328, 3712, 3968, 4096, 4224, 4992, 5632, 8192)]
    assert ways(calls, tmp_path) == [(2, False)] * 6 + [(4, False)] * 2 + [(4, True)] * 2


def test_short_sequences(tmp_path):
    """Two workgroups a unit where nothing is cut; the tokens' count alone does not decide."""
    assert ways([(3000, 3000, 30, 16, 16, 128, True), (4096, 4096, 8, 16, 16, 128, True), (2000, 2000, 20, 8, 8, 128, True)], tmp_path) == [(4, True), (4, True), (4, False)]
