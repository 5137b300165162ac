"""What the large-model operators settle on the host: which kernels a call launches (launches are noted instead of run: no
GPU needed)."""
import ctypes as C
import math
import random

from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import VocabSpec

import large_sizes
from launch_record import record

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4


def test_no_launch_behind_the_last_tensor(tmp_path):
    """Empty tensors behind the last one of a full table of 64 need no table of their own: a launch with nothing in it would leave a
    norm of 0."""
    lists = [[4] * 64, [4] * 64 + [0], [0] + [4] * 64 + [0] * 70, [4] * 63 + [0, 0], [0, 0], [9000] * 64 + [0, 0], [0, 9000] * 64 + [0], [9000] * 128 + [0]]
    tables = [1, 1, 1, 1, 1, 1, 1, 2]
    for what in ("norm", "clip", "step"):
        for counts, n, (status, launches) in zip(lists, tables, record([[what, c] for c in lists], tmp_path)):
            assert status == 0
            small = sum(counts) <= 64 * 8
            assert len(launches) == (1 if small else n + 1 if what == "norm" else 2 * n), (what, counts, launches)


def test_norm_and_workspace_are_no_tensor_of_the_list():
    """The norm of a list is refused where it lies on one of its gradients, as clipping and the step refuse it, and so is a workspace
    there or on the norm.  A gradient that is listed twice may be read twice."""
    L = B.lib()
    for n in (2, 150):   # addresses on the stack, and more than fit there
        l = C.byref(B.dll_tensor_list(n, (C.c_size_t * n)(*[4] * n), (C.c_int * n)(*[0] * n)))
        at = lambda base, step=256: (C.c_void_p * n)(*[base + step * k for k in range(n)])
        g, p, v = at(0x100000), at(0x200000), at(0x300000)
        norm, ws, first, last = (C.c_void_p(a) for a in (0x10000, 0x20000, 0x100000, 0x100000 + 256 * (n - 1)))
        calls = (lambda norm, ws, g=g: L.dll_grad_norm(l, g, norm, ws, 0, None), lambda norm, ws, g=g: L.dll_grad_clip(l, g, p, 1.0, norm, ws, 0, None),
                 lambda norm, ws, g=g: L.dll_momentum_update_clipped(l, p, v, g, 0.1, 0.9, None, 1.0, norm, None, ws, 0, None))
        for call in calls:
            assert call(norm, ws) == call(norm, ws, at(0x100000, 0)) == WORKSPACE   # nothing else to refuse
            assert call(first, ws) == call(last, ws) == call(norm, last) == call(norm, norm) == SHAPE
        assert L.dll_grad_clip(l, g, g, 1.0, norm, ws, 0, None) == WORKSPACE and L.dll_grad_clip(l, g, p, 1.0, norm, C.c_void_p(0x200000), 0, None) == SHAPE


def test_labels_losses_and_norms_lie_at_their_elements():
    """At any multiple of four bytes; refused elsewhere, before any launch."""
    L = B.lib()
    d = C.byref(B.vocab_desc(VocabSpec(16, 24, 40, "float32")))
    at = lambda k, off=0: C.c_void_p(0x10000 * (k + 1) + off)
    ws, out = at(9), [at(10), at(11), at(12)]
    for k in range(4):   # labels, row_loss, row_lse, loss
        for off, status in ((0, WORKSPACE), (4, WORKSPACE), (1, SHAPE), (2, SHAPE)):
            labels, *losses = [at(4 + i, off if i == k else 0) for i in range(4)]
            assert L.dll_vocab_loss_fwd(d, at(0), at(1), at(2), labels, *losses, ws, 0, None) == status
            assert L.dll_vocab_loss_grad(d, at(0), at(1), at(2), labels, 1.0, *losses, *out, ws, 0, None) == status
    l, one = C.byref(B.dll_tensor_list(1, (C.c_size_t * 1)(4), (C.c_int * 1)(0))), lambda k: (C.c_void_p * 1)(at(k).value)
    for off, status in ((0, WORKSPACE), (4, WORKSPACE), (2, SHAPE)):
        norm = at(5, off)
        assert L.dll_grad_norm(l, one(0), norm, ws, 0, None) == L.dll_grad_clip(l, one(0), one(1), 1.0, norm, ws, 0, None) == status
        assert L.dll_momentum_update_clipped(l, one(1), one(2), one(0), 0.1, 0.9, None, 1.0, norm, None, ws, 0, None) == status


# tokens, width, hidden units, type, whether the weights go straight from memory: either side of the line, where the other way was
# measured slower
FEW = [(1, 2048, 8192, "bfloat16", True), (1, 2048, 11008, "bfloat16", True), (1, 512, 14336, "bfloat16", False), (16, 2048, 4096, "bfloat16", True),
       (16, 2048, 8192, "bfloat16", False), (16, 63, 22015, "bfloat16", False), (1, 4095, 22015, "bfloat16", True), (4, 255, 8191, "bfloat16", False),
       (24, 1000, 2730, "bfloat16", True), (24, 2047, 8191, "bfloat16", False), (32, 2048, 2730, "bfloat16", True), (33, 1000, 2730, "bfloat16", False),
       (1, 2048, 8192, "float32", True), (1, 2048, 11008, "float32", True), (1, 512, 8192, "float32", False), (16, 4096, 8192, "float32", True), (16, 2048, 8192, "float32", False),
       (4, 4096, 14336, "float32", True), (16, 64, 4096, "float32", False), (24, 784, 500, "float32", True), (1, 7, 100, "float32", False)]


def test_blocks_of_few_tokens_take_the_faster_way(tmp_path):
    calls = [["gated_fwd", T, D, H, "silu", dtype] for T, D, H, dtype, _ in FEW]
    for call, case, (status, launches) in zip(calls, FEW, record(calls, tmp_path)):
        assert status == 0 and ("skinny_kernel" in launches[0][0]) == case[-1], (call, launches)


# tokens, width, classes, type, whether the weights go straight from memory
SCORED = [(1, 1024, 5000, "bfloat16", True), (16, 1024, 32000, "bfloat16", True), (17, 1024, 32000, "bfloat16", False), (1, 1024, 100000, "float32", True),
          (16, 4098, 32000, "bfloat16", True), (16, 4098, 32000, "float32", False), (1, 8192, 100000, "bfloat16", True), (16, 8194, 500, "bfloat16", False),
          (4, 8191, 5000, "float32", False), (16, 1001, 32000, "bfloat16", True), (32, 513, 8000, "bfloat16", True), (16, 16001, 500, "bfloat16", False),
          (32, 4095, 32000, "bfloat16", False), (1, 4095, 500, "bfloat16", False), (1, 4095, 32000, "bfloat16", True), (3, 7, 50, "bfloat16", False)]


def test_losses_of_few_tokens_take_the_faster_way(tmp_path):
    calls = [["loss_fwd", T, D, V, dtype] for T, D, V, dtype, _ in SCORED]
    for call, case, (status, launches) in zip(calls, SCORED, record(calls, tmp_path)):
        assert status == 0 and ("skinny_kernel" in launches[0][0]) == case[-1], (call, launches)


def products(launches):
    """The product kernels among a call's launches; gradients also by whether their k is split."""
    names = [l[0] for l in launches]
    split = any("sum_splits" in n for n in names)
    return {(n, "gradient_kernel" in n and split) for n in names if n.startswith("_ZN4dllk4tile") and "sum_splits" not in n}


def sweep(seed, n):
    """Calls over the operators' ranges, sizes even over their logarithms, and losses of more exponentials than are kept at a time."""
    rng = random.Random(seed)
    spread = lambda low, high: int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    calls = []
    for _ in range(n):
        what, dtype = rng.choice(["gated_fwd", "gated_bwd", "loss_fwd", "loss_grad"]), rng.choice(["bfloat16", "float32"])
        calls.append([what, spread(1, 8192), spread(1, 8192), spread(1, 16384), "silu", dtype] if what.startswith("gated") else
                     [what, spread(1, 8192), spread(1, 8192), spread(1, 110000), dtype])
    for _ in range(n // 20):
        pieces = ((1 << 20) + spread(1, 400000), spread(3, 40), spread(3, 40)) if rng.random() < 0.5 else (spread(257, 1500), spread(8, 40), (1 << 20) - rng.randint(0, 9))
        calls.append(["loss_grad", *pieces, rng.choice(["bfloat16", "float32"])])
    return calls


def test_every_kernel_that_the_plans_choose_is_tested(tmp_path):
    """What a sweep of calls launches, the sizes of the GPU tests launch too: a change of the plans' constants that leaves a kernel without
    a test shows here."""
    covered = set().union(*[products(launches) for _, launches in record(large_sizes.calls(), tmp_path)])
    calls = sweep(3, 16000)
    for call, (status, launches) in zip(calls, record(calls, tmp_path)):
        assert status == 0
        assert products(launches) <= covered, (call, products(launches) - covered)
    largest = {(what, split) for name, split in covered if "Li256ELi256E" in name
               for what in ("7GateEpi", "11GateBackEpi", "8StoreEpiIDF16b", "10PartialEpi", "Lb0EEE", "Lb1EEE", "gradient_kernel") if what in name}
    assert {("7GateEpi", False), ("11GateBackEpi", False), ("8StoreEpiIDF16b", False), ("10PartialEpi", False), ("gradient_kernel", False), ("gradient_kernel", True)} <= largest
    assert sum("LogitEpi" in name and "Li256ELi256E" in name for name, _ in covered) == 2   # with and without the exponentials
