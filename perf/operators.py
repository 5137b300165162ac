"""The large-model operators whose speed is watched: a gated feed-forward block, softmax cross entropy over a
large vocabulary, and clipping by the global gradient norm with the momentum step behind it.

A case is a dict of plain values.  `listed()` names a dozen of them, `draw(rng)` gives more of the same ranges,
`prepare` builds what a program holds before the call, `run` is one pass (through the library where `own` is set,
in elementary torch operations otherwise), `exact` the same result in 64 bits.

Kinds of case:
  gated_fwd     forward pass of the block, as a server or an evaluation runs it
  gated_train   forward pass that keeps what the backward pass needs, and the backward pass
  loss_fwd      losses of given tokens, as a scoring run asks for them
  loss_grad     loss and its gradients by input, weights and bias, as a training step asks for them
  clip          gradients of many tensors scaled so that their common norm is at most `max_norm`
  update        momentum step with weight decay on such clipped gradients, 32-bit parameters and their bfloat16 copies
"""
import itertools
import math

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


# ---------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------
def listed():
    return [
        # one token through a block between the large-image network's dense widths: a server's decoding step
        dict(name="gated_fwd_one_token_bf16", kind="gated_fwd", tokens=1, width=2048, hidden=8192, gate="silu", dtype="bfloat16"),
        # a small batch in single precision on the MNIST network's widths: latency
        dict(name="gated_fwd_b24_mnist_fp32", kind="gated_fwd", tokens=24, width=784, hidden=500, gate="gelu", dtype="float32"),
        # a prompt of a length that fills no tile
        dict(name="gated_fwd_prompt_777_bf16", kind="gated_fwd", tokens=777, width=1000, hidden=2730, gate="gelu", dtype="bfloat16"),
        # a training step's worth of tokens: the block's largest case
        dict(name="gated_train_4096_bf16", kind="gated_train", tokens=4096, width=2048, hidden=8192, gate="silu", dtype="bfloat16"),
        # training in single precision on odd sizes
        dict(name="gated_train_odd_fp32", kind="gated_train", tokens=1000, width=500, hidden=1337, gate="relu", dtype="float32"),
        # scoring a few candidate tokens of a request
        dict(name="loss_fwd_16_bf16", kind="loss_fwd", tokens=16, width=1024, classes=32000, ignored=0.0, bias=False, dtype="bfloat16"),
        # a training batch over a large vocabulary of odd size, a tenth of it padding: the largest case
        dict(name="loss_grad_4096_bf16", kind="loss_grad", tokens=4096, width=2048, classes=50257, ignored=0.1, bias=False, dtype="bfloat16"),
        # the large-image network's own last layer and loss
        dict(name="loss_grad_imagenet_fp32", kind="loss_grad", tokens=128, width=2048, classes=1000, ignored=0.0, bias=True, dtype="float32"),
        # a ragged batch in single precision
        dict(name="loss_grad_odd_fp32", kind="loss_grad", tokens=1023, width=784, classes=10007, ignored=0.25, bias=True, dtype="float32"),
        # the gradients of the MNIST network: eight small tensors
        dict(name="clip_mnist_fp32", kind="clip", sizes="mnist", layers=0, width=0, hidden=0, classes=0, dtype="float32"),
        # the gradients of the large-image network: 75 MB, nearly all in two tensors of twelve
        dict(name="clip_imagenet_fp32", kind="clip", sizes="imagenet", layers=0, width=0, hidden=0, classes=0, dtype="float32"),
        # the step of a model of 24 blocks and its vocabulary: 194 tensors from 1024 to 33 million elements
        dict(name="update_blocks_bf16", kind="update", sizes="blocks", layers=24, width=1024, hidden=2816, classes=32000, dtype="bfloat16"),
    ]


_MAX_FLOP = 1.2e12     # of a drawn case: under the largest listed one in time and size
_MAX_LOGITS = 1 << 27


def _spread(rng, low, high):
    """A whole number, even over its logarithm; every other one is a multiple of 8 where there is room for that."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if n >= 16 and rng.random() < 0.5:
        n -= n % 8
    return max(low, min(high, n))


def draw(rng):
    kind = rng.choice(["gated_fwd", "gated_train", "loss_fwd", "loss_grad", "clip", "update"])
    dtype = rng.choice(["bfloat16", "float32"])
    # the plain form's rate does not depend on the type: one limit for both
    while True:
        tokens, width = _spread(rng, 1, 4096), _spread(rng, 64, 4096)
        hidden, classes = _spread(rng, 64, 8192), _spread(rng, 500, 65536)
        if kind.startswith("gated"):
            if 18.0 * tokens * width * hidden <= _MAX_FLOP:
                return dict(kind=kind, tokens=tokens, width=width, hidden=hidden, gate=rng.choice(["silu", "gelu", "relu", "sigmoid"]), dtype=dtype)
        elif kind.startswith("loss"):
            if 6.0 * tokens * width * classes <= _MAX_FLOP and tokens * classes <= _MAX_LOGITS:
                return dict(kind=kind, tokens=tokens, width=width, classes=classes, ignored=rng.choice([0.0, 0.1, 0.5]), bias=rng.random() < 0.5, dtype=dtype)
        else:
            layers = _spread(rng, 1, 24)
            width, hidden, classes = _spread(rng, 16, 1024), _spread(rng, 16, 2816), _spread(rng, 100, 32000)
            return dict(kind=kind, sizes="blocks", layers=layers, width=width, hidden=hidden, classes=classes, dtype=dtype)


def _shapes(case):
    """Element counts of the tensors of a clip or update case."""
    if case["sizes"] == "mnist":
        return [8 * 25, 8, 8 * 8 * 25, 8, 150 * 128, 150, 10 * 150, 10]
    if case["sizes"] == "imagenet":
        return [16 * 27, 16, 16 * 144, 16, 32 * 144, 32, 32 * 288, 32, 2048 * 8192, 2048, 1000 * 2048, 1000]
    D, H, V = case["width"], case["hidden"], case["classes"]
    return [V * D] + [D * D, D * D, D * D, D * D, H * D, H * D, D * H, D] * case["layers"] + [D]


def _places(counts):
    """Where each tensor starts in one buffer that holds them all, each at a multiple of 64 elements, and the buffer's length."""
    ends = list(itertools.accumulate(-(-n // 64) * 64 for n in counts))
    return [0] + ends[:-1], ends[-1]


def _views(flat, counts):
    """The tensors of one buffer that holds them all."""
    return [flat[i:i + n] for i, n in zip(_places(counts)[0], counts)]


def _flat(tensors):
    """One buffer with the given tensors, zeros between them."""
    counts = [t.numel() for t in tensors]
    flat = torch.zeros(_places(counts)[1], dtype=tensors[0].dtype, device=tensors[0].device)
    torch._foreach_copy_(_views(flat, counts), tensors)
    return flat


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _inputs(case, seed):
    """The inputs in their own types, on the GPU."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 18040451)
    kind, dtype = case["kind"], _TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dtype):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)

    if kind.startswith("gated"):
        T, D, H = case["tokens"], case["width"], case["hidden"]
        s = dict(x=normal(T, D), w_gate=normal(H, D, std=D ** -0.5), w_up=normal(H, D, std=D ** -0.5), w_down=normal(D, H, std=H ** -0.5))
        if kind == "gated_train":
            s["dy"] = normal(T, D)
        return s
    if kind.startswith("loss"):
        T, D, V = case["tokens"], case["width"], case["classes"]
        s = dict(x=normal(T, D), w=normal(V, D, std=2.0 * D ** -0.5), bias=normal(V, std=0.5) if case["bias"] else None)
        labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
        out = torch.rand(T, generator=gen, device="cuda") < case["ignored"]
        out[T // 2] = False   # one row counts at least
        s["labels"] = torch.where(out, torch.full_like(labels, -1), labels)
        return s
    counts = _shapes(case)
    s = dict(grads=_views(_flat([normal(n, std=0.01) for n in counts]), counts))
    s["max_norm"] = 0.005 * math.sqrt(sum(counts))   # half of the norm: clipping takes place, as it does early in training
    if kind == "update":
        s["flat_params"] = _flat([normal(n, std=0.05, dtype=torch.float32) for n in counts])
        s["flat_velocity"] = _flat([normal(n, std=1e-4, dtype=torch.float32) for n in counts])
        s["params"], s["velocity"] = _views(s["flat_params"], counts), _views(s["flat_velocity"], counts)
        s["decay"] = [0.01 if n > case["width"] else 0.0 for n in counts]   # matrices only
        s["lr"], s["momentum"] = 1e-3, 0.9
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = s["kind"] = case["kind"]
    s["case"] = case
    dtype = _TYPES[case["dtype"]]

    def empty(*shape, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind.startswith("gated"):
        T, D, H = case["tokens"], case["width"], case["hidden"]
        s["y"] = empty(T, D)
        if kind == "gated_train":
            s.update(gate_pre=empty(T, H), up_pre=empty(T, H), dx=empty(T, D), dw_gate=empty(H, D), dw_up=empty(H, D), dw_down=empty(D, H))
    elif kind.startswith("loss"):
        T, D, V = case["tokens"], case["width"], case["classes"]
        s.update({k: empty(T, dtype=torch.float32) for k in ("row_loss", "row_lse")}, loss=empty(1, dtype=torch.float32))
        if kind == "loss_grad":
            s.update(dx=empty(T, D), dw=empty(V, D), dbias=empty(V) if case["bias"] else None)
    else:
        s["norm"] = empty(1, dtype=torch.float32)
        if kind == "clip":
            s["flat_out"] = _flat([torch.zeros_like(g) for g in s["grads"]])
            s["out"] = _views(s["flat_out"], _shapes(case))
        else:
            s["flat_copies"] = torch.zeros_like(s["flat_params"], dtype=torch.bfloat16)
            s["copies"] = _views(s["flat_copies"], _shapes(case))
    if own:
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    """The handle and the workspace that a program of the library keeps."""
    from paper_1804_04512_amd import binding as B
    from paper_1804_04512_amd.workloads import GatedSpec, VocabSpec
    kind = case["kind"]
    if kind.startswith("gated"):
        s["spec"] = GatedSpec(case["tokens"], case["width"], case["hidden"], case["gate"], case["dtype"])
        n = B.dll_gated_fwd_workspace_bytes(s["spec"])
        if kind == "gated_train":
            n = max(n, B.dll_gated_bwd_workspace_bytes(s["spec"]))
    elif kind.startswith("loss"):
        s["spec"] = VocabSpec(case["tokens"], case["width"], case["classes"], case["dtype"])
        n = B.dll_vocab_loss_fwd_workspace_bytes(s["spec"]) if kind == "loss_fwd" else B.dll_vocab_loss_grad_workspace_bytes(s["spec"])
    else:
        s["spec"] = B.tensor_list(s["grads"])
        n = B.dll_grad_norm_workspace_bytes(s["spec"])
    s["ws"] = B.workspace(n)


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _run_own(s):
    from paper_1804_04512_amd import binding as B
    kind, spec, ws = s["kind"], s["spec"], s["ws"]
    if kind == "gated_fwd":
        B.dll_gated_fwd(spec, s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"], ws=ws)
        return {"y": s["y"]}
    if kind == "gated_train":
        B.dll_gated_fwd(spec, s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"], s["gate_pre"], s["up_pre"], ws=ws)
        B.dll_gated_bwd(spec, s["x"], s["w_gate"], s["w_up"], s["w_down"], s["gate_pre"], s["up_pre"], s["dy"], s["dx"],
                        s["dw_gate"], s["dw_up"], s["dw_down"], ws=ws)
        return {k: s[k] for k in ("y", "dx", "dw_gate", "dw_up", "dw_down")}
    if kind == "loss_fwd":
        B.dll_vocab_loss_fwd(spec, s["x"], s["w"], s["bias"], s["labels"], s["row_loss"], s["row_lse"], s["loss"], ws=ws)
        return {k: s[k] for k in ("row_loss", "row_lse", "loss")}
    if kind == "loss_grad":
        B.dll_vocab_loss_grad(spec, s["x"], s["w"], s["bias"], s["labels"], 1.0, s["row_loss"], s["row_lse"], s["loss"],
                              s["dx"], s["dw"], s["dbias"], ws=ws)
        return {k: s[k] for k in ("row_loss", "row_lse", "loss", "dx", "dw", "dbias") if s[k] is not None}
    if kind == "clip":
        B.dll_grad_clip(spec, s["grads"], s["out"], s["max_norm"], s["norm"], ws=ws)
        return {"norm": s["norm"], "grads": s["flat_out"]}
    B.dll_momentum_update_clipped(spec, s["params"], s["velocity"], s["grads"], s["lr"], s["momentum"], s["decay"], s["max_norm"],
                                  s["norm"], s["copies"], ws=ws)
    return {"norm": s["norm"], "params": s["flat_params"], "velocity": s["flat_velocity"], "copies": s["flat_copies"]}


def _act(name, a):
    """The gate's activation and its derivative."""
    if name == "relu":
        return a.clamp(min=0), (a > 0).to(a.dtype)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-a))
    if name == "sigmoid":
        return sig, sig * (1 - sig)
    return a * sig, sig * (1 + a * (1 - sig))


def _plain_gated_fwd(s):
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    h = _act(s["case"]["gate"], x @ wg.t())[0] * (x @ wu.t())
    return {"y": (h @ wd.t()).to(s["x"].dtype)}


def _plain_gated_train(s):
    dtype = s["x"].dtype
    x, wg, wu, wd, dy = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down", "dy"))
    a, b = x @ wg.t(), x @ wu.t()
    f, d = _act(s["case"]["gate"], a)
    h, dh = f * b, dy @ wd
    da, db = dh * b * d, dh * f
    out = {"y": h @ wd.t(), "dx": da @ wg + db @ wu, "dw_gate": da.t() @ x, "dw_up": db.t() @ x, "dw_down": dy.t() @ h}
    return {k: v.to(dtype) for k, v in out.items()}


def _plain_loss_fwd(s):
    return _plain_loss(s, False)


def _plain_loss_grad(s):
    return _plain_loss(s, True)


def _plain_loss(s, grad):
    dtype = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    counted = s["labels"] >= 0
    label = s["labels"].clamp(min=0).long()[:, None]
    n = counted.sum()
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"].float()
    top = z.amax(1, keepdim=True)
    hit = z.gather(1, label)
    z -= top
    z.exp_()
    lse = top + z.sum(1, keepdim=True).log()
    zero = torch.zeros((), device=x.device)
    row_loss = torch.where(counted, (lse - hit)[:, 0], zero)
    out = {"row_loss": row_loss, "row_lse": torch.where(counted, lse[:, 0], zero), "loss": (row_loss.sum(dtype=torch.float64) / n).float().reshape(1)}
    if grad:
        share = (counted.float() / n)[:, None]
        z *= torch.exp(top - lse) * share
        z.scatter_add_(1, label, -share)
        out.update(dx=(z @ w).to(dtype), dw=(z.t() @ x).to(dtype))
        if s["bias"] is not None:
            out["dbias"] = z.sum(0).to(dtype)
    return out


def _norm(grads):
    """In 64 bits: a sum of up to hundreds of millions of squares."""
    return torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt()


def _plain_clip(s):
    norm = _norm(s["grads"])
    c = (s["max_norm"] / norm).clamp(max=1.0).float()
    _ = [o.copy_(g.float() * c) for o, g in zip(s["out"], s["grads"])]
    return {"norm": norm.float().reshape(1), "grads": s["flat_out"]}


def _plain_update(s):
    norm = _norm(s["grads"])
    c = (s["max_norm"] / norm).clamp(max=1.0).float()
    lr, mu = s["lr"], s["momentum"]
    _ = [_plain_step(*t, c, lr, mu) for t in zip(s["params"], s["velocity"], s["copies"], s["grads"], s["decay"])]
    return {"norm": norm.float().reshape(1), "params": s["flat_params"], "velocity": s["flat_velocity"], "copies": s["flat_copies"]}


def _plain_step(p, v, copy, g, wd, c, lr, mu):
    v.mul_(mu).sub_((g.float() * c + p * wd) * lr)
    p.add_(v)
    copy.copy_(p)


_PLAIN = {"gated_fwd": _plain_gated_fwd, "gated_train": _plain_gated_train, "loss_fwd": _plain_loss_fwd, "loss_grad": _plain_loss_grad,
          "clip": _plain_clip, "update": _plain_update}


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bfloat16" else 4
    kind = case["kind"]
    if kind.startswith("gated"):
        T, D, H = case["tokens"], case["width"], case["hidden"]
        if kind == "gated_fwd":
            return {"bytes": e * (2 * T * D + 3 * D * H), "flops": 6.0 * T * D * H}
        return {"bytes": e * (4 * T * D + 6 * D * H), "flops": 18.0 * T * D * H}
    if kind.startswith("loss"):
        T, D, V = case["tokens"], case["width"], case["classes"]
        b = V * (1 if case["bias"] else 0)
        if kind == "loss_fwd":
            return {"bytes": e * (T * D + V * D + b) + 12 * T, "flops": 2.0 * T * D * V}
        return {"bytes": 2 * e * (T * D + V * D + b) + 12 * T, "flops": 6.0 * T * D * V}
    n = sum(_shapes(case))
    if kind == "clip":
        return {"bytes": 2 * e * n, "flops": 3.0 * n}
    return {"bytes": (e + 4 * 4 + 2) * n, "flops": 8.0 * n}


# ---------------------------------------------------------------------------------------
# the result in 64 bits
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("gated"):
        x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
        a = torch.matmul(x, wg.t()).requires_grad_()
        gate = {"relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu, "sigmoid": torch.sigmoid}[case["gate"]](a)
        b = torch.matmul(x, wu.t())
        h = gate.detach() * b
        out = {"y": torch.matmul(h, wd.t())}
        if kind == "gated_train":
            dy = s["dy"].double()
            dh = torch.matmul(dy, wd)
            da = torch.autograd.grad(gate, a, dh * b)[0]
            db = dh * gate.detach()
            out.update(dx=torch.matmul(torch.cat((da, db), 1), torch.cat((wg, wu), 0)), dw_gate=torch.matmul(x.t(), da).t().contiguous(),
                       dw_up=torch.matmul(x.t(), db).t().contiguous(), dw_down=torch.matmul(h.t(), dy).t().contiguous())
        return out
    if kind.startswith("loss"):
        x, w, labels = s["x"].double(), s["w"].double(), s["labels"]
        rows = (labels >= 0).nonzero()[:, 0]
        lab = labels[rows].long()
        logits = torch.matmul(x[rows], w.t())
        if s["bias"] is not None:
            logits = logits + s["bias"].double()
        logp = torch.log_softmax(logits, 1)
        each = -logp[torch.arange(len(rows), device=x.device), lab]
        full = lambda v: torch.zeros((len(labels),) + v.shape[1:], dtype=v.dtype, device=v.device).index_copy(0, rows, v)  # noqa: E731
        out = {"row_loss": full(each), "row_lse": full((logits - logp).select(1, 0)), "loss": each.mean().reshape(1)}
        if kind == "loss_grad":
            d = logp.exp()
            d[torch.arange(len(rows), device=x.device), lab] -= 1.0
            d /= len(rows)
            out.update(dx=full(torch.matmul(d, w)), dw=torch.matmul(d.t(), x[rows]))
            if s["bias"] is not None:
                out["dbias"] = d.sum(0)
        return out
    counts = _shapes(case)
    g = _flat([t.double() for t in s["grads"]])
    norm = torch.linalg.vector_norm(g)
    c = torch.clamp(s["max_norm"] / norm, max=1.0)
    if kind == "clip":
        return {"norm": norm.reshape(1), "grads": g * c}
    d = torch.zeros_like(g)
    for view, wd in zip(_views(d, counts), s["decay"]):
        view.fill_(wd)
    p = s["flat_params"].double()
    v = s["momentum"] * s["flat_velocity"].double() - s["lr"] * (c * g + d * p)
    return {"norm": norm.reshape(1), "params": p + v, "velocity": v, "copies": p + v}
