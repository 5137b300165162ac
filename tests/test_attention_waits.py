"""Barriers of the attention kernels: no wavefront goes past one with LDS accesses of its own on their way, as the others may write or read the same
places next.  Read from the compiled kernels, for every way through them."""
import pytest

import device_code
from paper_1804_04512_amd import binding as B

pytestmark = pytest.mark.skipif(not device_code.available(), reason="no disassembler")


def step(op, operands, pending):
    if op.startswith("ds_") and not op.startswith(("ds_bpermute", "ds_permute", "ds_swizzle", "ds_nop")):
        return True
    if op == "s_waitcnt" and "lgkmcnt(0)" in operands:
        return False
    return pending


@pytest.mark.parametrize("kernel", ["attention_fwd_kernel", "attention_dq_kernel", "attention_dkv_kernel", "paged_attention_kernel"])
def test_nothing_in_flight_at_a_barrier(kernel, tmp_path):
    B.lib()
    found = device_code.kernels(B.LIB_PATH, tmp_path, kernel)
    assert len(found) >= 10
    bad = {}
    for name, code in found.items():
        ops = {op for _, op, _, _ in code}
        assert {"s_barrier", "s_endpgm"} <= ops and "s_swappc_b64" not in ops, name
        before = device_code.reaching(code, step)
        at = [hex(code[i][0]) for i, pending in before.items() if pending and code[i][1] == "s_barrier"]
        if at:
            bad[name] = at
    assert not bad, bad


def test_the_walk_itself():
    code = [(0, "ds_write_b128", "", None), (8, "s_cbranch_scc1", "", 20), (12, "s_waitcnt", "vmcnt(0) lgkmcnt(0)", None), (16, "s_barrier", "", None),
            (20, "s_waitcnt", "vmcnt(0)", None), (24, "s_barrier", "", None), (28, "s_endpgm", "", None)]
    before = device_code.reaching(code, step)
    assert not before[3] and before[5]


def test_registers_that_are_spilled(tmp_path):
    """Sums and rows of heads up to 96 elements stay in registers: no gradient kernel writes any of them to memory and reads them again."""
    for kernel in ("attention_dq_kernel", "attention_dkv_kernel"):
        for name, code in device_code.kernels(B.LIB_PATH, tmp_path, kernel).items():
            if any(f"Li{dim}EL" in name for dim in (32, 64, 96)) and not any(f"Li{dim}EL" in name for dim in (128, 256)):
                assert not any(op.startswith("scratch_") for _, op, _, _ in code), name
