"""The attention operators whose speed is watched: attention over packed prompts with its gradients, and the paged cache
of keys and values: its tables and slots, the store of new tokens, and the attention of one new token a request.

A case is a dict of plain values.  `listed()` names a dozen of them, `draw(rng)` gives more of the same ranges,
`prepare` builds what a program holds before the call, `run` is one pass (through the library where `own` is set,
in elementary torch operations otherwise), `exact` the same result in 64 bits.

Kinds of case:
  prompt   attention of packed sequences, forward pass, as a server runs it on prompts
  train    forward and backward pass, q, k and v side by side in one projection's output and their gradients in another's
  decode   attention of one new token a request over a paged cache
  plan     pages for new tokens from a list of free ones, block tables and slots, from the requests' lengths
  store    keys and values of new tokens written into the cache by slot
"""
import itertools
import math
import random

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


# ---------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------
def listed():
    return [
        # one short prompt in single precision: latency
        dict(name="prompt_37_fp32", kind="prompt", tokens=37, sequences=1, heads=8, kv_heads=8, dim=64, causal=True, dtype="float32"),
        # one prompt of a length that fills no tile, four heads to a key
        dict(name="prompt_777_bf16", kind="prompt", tokens=777, sequences=1, heads=16, kv_heads=4, dim=64, causal=True, dtype="bfloat16"),
        # a server's batch of prompts of all lengths, packed: the largest forward pass
        dict(name="prompt_packed_16384_bf16", kind="prompt", tokens=16384, sequences=5, heads=16, kv_heads=4, dim=128, causal=True, dtype="bfloat16"),
        # a training step's sequence at the large-image network's dense width
        dict(name="train_4096_bf16", kind="train", tokens=4096, sequences=1, heads=16, kv_heads=16, dim=128, causal=True, dtype="bfloat16"),
        # ragged sequences that see both ways, in single precision with heads of a size between the usual ones
        dict(name="train_ragged_fp32", kind="train", tokens=2001, sequences=3, heads=6, kv_heads=3, dim=80, causal=False, dtype="float32"),
        # one request with a short history: the step of a single conversation
        dict(name="decode_one_bf16", kind="decode", requests=1, longest=1000, heads=16, kv_heads=4, dim=128, page=16, dtype="bfloat16"),
        # a server's batch, every length up to 8192
        dict(name="decode_64_bf16", kind="decode", requests=64, longest=8192, heads=32, kv_heads=8, dim=128, page=16, dtype="bfloat16"),
        # few requests with a long history, single precision, pages that fill no tile
        dict(name="decode_long_fp32", kind="decode", requests=3, longest=60000, heads=8, kv_heads=8, dim=96, page=20, dtype="float32"),
        # tables and slots of a decoding step
        dict(name="plan_step_64", kind="plan", requests=64, longest=8192, added=1, page=16),
        # tables and slots of many prompts at once
        dict(name="plan_prompts_2000", kind="plan", requests=2000, longest=1500, added=300, page=16),
        # the store of a decoding step
        dict(name="store_64_bf16", kind="store", requests=64, longest=2048, added=1, kv_heads=8, dim=128, page=16, dtype="bfloat16"),
        # the store of a batch of prompts
        dict(name="store_prompts_fp32", kind="store", requests=33, longest=3000, added=1000, kv_heads=8, dim=128, page=20, dtype="float32"),
    ]


_MAX_PAIRS = 1 << 28     # pairs of a token and one it may look at, by head size and heads / 2048: of the listed cases' order at most
_MAX_CACHE = 1 << 28     # elements of the keys of a drawn cache


def _spread(rng, low, high):
    """A whole number, even over its logarithm; every other one is a multiple of 8 where there is room for that."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if n >= 16 and rng.random() < 0.5:
        n -= n % 8
    return max(low, min(high, n))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "decode", "decode", "plan", "store"])
    dtype = rng.choice(["bfloat16", "float32"])
    while True:
        kv_heads, group = rng.choice([1, 2, 3, 4, 8, 12, 16]), rng.choice([1, 1, 2, 4, 5, 8])
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        heads, page = kv_heads * group, rng.choice([8, 16, 16, 20, 32, 64, 100])
        if heads > 48:
            continue
        if kind in ("prompt", "train"):
            tokens, sequences = _spread(rng, 16, 16384), _spread(rng, 1, 64)
            if sequences > tokens:
                continue
            case = dict(kind=kind, tokens=tokens, sequences=sequences, heads=heads, kv_heads=kv_heads, dim=dim, causal=rng.random() < 0.75, dtype=dtype)
            cost = _pairs(case) * heads * dim / 2048.0 * (3.5 if kind == "train" else 1.0)
            if cost <= 0.4 * _MAX_PAIRS:
                return case
        elif kind == "decode":
            requests, longest = _spread(rng, 1, 256), _spread(rng, 16, 65536)
            if requests * longest * kv_heads * dim <= _MAX_CACHE and requests * longest * heads <= _MAX_CACHE // 8:
                return dict(kind=kind, requests=requests, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)
        else:
            requests, longest, added = _spread(rng, 1, 2048), _spread(rng, 16, 8192), rng.choice([1, 1, _spread(rng, 2, 2048)])
            if added > longest or requests * added > 600000:
                continue
            if kind == "plan":
                return dict(kind=kind, requests=requests, longest=longest, added=added, page=page)
            if requests * longest * kv_heads * dim <= _MAX_CACHE and requests * added * kv_heads * dim <= 34000000:
                return dict(kind=kind, requests=requests, longest=longest, added=added, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)


def _fixed(case):
    """Lengths belong to the case: a generator that depends on its sizes alone."""
    return random.Random(",".join(f"{k}={case[k]}" for k in sorted(case) if k != "name"))


def _sequence_lengths(case):
    """Lengths of the packed sequences, uneven, none empty, that add up to the case's tokens."""
    n, left = case["sequences"], case["tokens"]
    rng = _fixed(case)
    weights = [rng.uniform(0.2, 2.0) for _ in range(n)]
    total = sum(weights)
    lengths = [1 + int(w / total * (left - n)) for w in weights]
    lengths[-1] += left - sum(lengths)
    return lengths



def _request_lengths(case):
    """Tokens that each request has in the cache, and how many of these are new."""
    rng, n, longest = _fixed(case), case["requests"], case["longest"]
    lengths = [longest] + [rng.randint(1, longest) for _ in range(n - 1)]
    rng.shuffle(lengths)
    most = case.get("added", 1)
    added = [min(k, most if most == 1 else rng.randint(1, most)) for k in lengths]
    return lengths, added


def _pairs(case):
    """Pairs of a token and one that it may look at."""
    return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _sequence_lengths(case))


def _sums(counts):
    return [0] + list(itertools.accumulate(counts))


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _inputs(case, seed):
    """The inputs in their own types, on the GPU, and what the program knows of them on the host."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 18040452)
    kind = case["kind"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(_TYPES[case["dtype"]])

    def ints(v):
        return torch.tensor(v, dtype=torch.int32).cuda()

    s = dict(case=case, kind=kind)
    if kind in ("prompt", "train"):
        T, H, KV, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        s["scale"] = D ** -0.5
        s["bounds"] = _sums(_sequence_lengths(case))
        s["starts"] = ints(s["bounds"])
        if kind == "train":
            s["qkv"], s["do"] = normal(T, H + 2 * KV, D), normal(T, H, D)
            s["q"], s["k"], s["v"] = s["qkv"].split([H, KV, KV], 1)
        else:
            s["q"], s["k"], s["v"] = normal(T, H, D), normal(T, KV, D), normal(T, KV, D)
        return s
    lengths, added = _request_lengths(case)
    page, R = case["page"], case["requests"]
    need = [-(-n // page) for n in lengths]
    have = [-(-(n - a) // page) for n, a in zip(lengths, added)]
    columns, pages = -(-case["longest"] // page), sum(need) + 8
    s.update(lengths=ints(lengths), added=ints(added), columns=columns, pages=pages, tokens=sum(added))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    # the table as the requests' histories left it; a decoding case's has the new token's page too
    held = need if kind == "decode" else have
    host, at = torch.full((R, columns), -1, dtype=torch.int64), 0
    for r, n in enumerate(held):
        host[r, :n] = torch.arange(at, at + n)
        at += n
    host = host.cuda()
    s["table"] = torch.where(host >= 0, order[host.clamp(min=0)], torch.full_like(order[:1], -1))
    s["free"] = order[at:].contiguous()
    if kind == "decode":
        H, KV, D = case["heads"], case["kv_heads"], case["dim"]
        s["scale"] = D ** -0.5
        s["q"], s["k_cache"], s["v_cache"] = normal(R, H, D), normal(pages, KV, page, D), normal(pages, KV, page, D)
    elif kind == "store":
        KV, D = case["kv_heads"], case["dim"]
        s["k"], s["v"] = normal(s["tokens"], KV, D), normal(s["tokens"], KV, D)
        s["k_cache"], s["v_cache"] = (torch.zeros(pages, KV, page, D, dtype=_TYPES[case["dtype"]], device="cuda") for _ in range(2))
        slots = _slots(s)[2]
        s["slots"] = slots.to(torch.int32)
    return s


def _slots(s):
    """Table, starts and slots in whole numbers of 64 bits; also the state: the first free entry left, and how many pages were missing."""
    page, lengths, added, table, free = s["case"]["page"], s["lengths"].long(), s["added"].long(), s["table"].long(), s["free"].long()
    have, need = (lengths - added + page - 1) // page, (lengths + page - 1) // page
    fresh = need - have
    first = fresh.cumsum(0) - fresh
    column = torch.arange(table.shape[1], device=table.device)[None]
    new = (column >= have[:, None]) & (column < need[:, None])
    place = first[:, None] + column - have[:, None]
    table = torch.where(new, free[place.clamp(0, len(free) - 1)], table)
    zero = torch.zeros(1, dtype=torch.int64, device=table.device)
    starts = torch.cat((zero, added.cumsum(0)))
    row = torch.repeat_interleave(torch.arange(len(added), device=table.device), added, output_size=s["tokens"])
    at = (lengths - added)[row] + torch.arange(s["tokens"], device=table.device) - starts[row]
    slots = table[row, at // page] * page + at % page
    return table, starts, slots, torch.cat((fresh.sum().reshape(1), zero))


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]

    def empty(*shape, dtype=None):
        return torch.empty(shape, dtype=dtype or _TYPES[case["dtype"]], device="cuda")

    if kind in ("prompt", "train"):
        T, H, KV, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        s["o"], s["lse"] = empty(T, H, D), empty(H, T, dtype=torch.float32)
        if kind == "train":
            s["dqkv"] = empty(T, H + 2 * KV, D)
            s["dq"], s["dk"], s["dv"] = s["dqkv"].split([H, KV, KV], 1)
    elif kind == "decode":
        s["o"] = empty(case["requests"], case["heads"], case["dim"])
    elif kind == "plan":
        i = torch.int32
        s["slots"], s["starts"], s["state"] = empty(s["tokens"], dtype=i), empty(case["requests"] + 1, dtype=i), empty(2, dtype=i)
    if own:
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    """The handle and the workspace that a program of the library keeps."""
    from paper_1804_04512_amd import binding as B
    from paper_1804_04512_amd.workloads import AttentionSpec, CacheSpec
    kind = case["kind"]
    if kind in ("prompt", "train"):
        T, H, KV, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        row = (H + 2 * KV) * D if kind == "train" else 0
        s["spec"] = AttentionSpec(T, T, case["sequences"], H, KV, D, case["causal"], case["dtype"], row, row)
        n = B.dll_attention_fwd_workspace_bytes(s["spec"])
        if kind == "train":
            n = max(n, B.dll_attention_bwd_workspace_bytes(s["spec"]))
        s["ws"] = B.workspace(n)
    else:
        s["spec"] = CacheSpec(case["requests"], case.get("heads", case.get("kv_heads", 1)), case.get("kv_heads", 1), case.get("dim", 64),
                              s["pages"], case["page"], s["columns"], case.get("dtype", "bfloat16"))
        if kind == "decode":
            s["ws"] = B.workspace(B.dll_paged_attention_workspace_bytes(s["spec"]))


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _run_own(s):
    from paper_1804_04512_amd import binding as B
    kind, spec = s["kind"], s["spec"]
    if kind in ("prompt", "train"):
        B.dll_attention_fwd(spec, s["q"], s["k"], s["v"], s["starts"], s["starts"], s["scale"], s["o"], s["lse"], ws=s["ws"])
        if kind == "prompt":
            return {"o": s["o"], "lse": s["lse"]}
        B.dll_attention_bwd(spec, s["q"], s["k"], s["v"], s["starts"], s["starts"], s["scale"], s["o"], s["lse"], s["do"],
                            s["dq"], s["dk"], s["dv"], ws=s["ws"])
        return {"o": s["o"], "lse": s["lse"], "dqkv": s["dqkv"]}
    if kind == "decode":
        B.dll_paged_attention(spec, s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["scale"], s["o"], ws=s["ws"])
        return {"o": s["o"]}
    if kind == "plan":
        B.dll_cache_plan(spec, s["lengths"], s["added"], s["free"], s["table"], s["starts"], s["slots"], s["state"])
        return {k: s[k] for k in ("table", "starts", "slots", "state")}
    B.dll_cache_write(spec, s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _heads_first(t, group=1):
    """[tokens][heads][dim] in its type -> [heads * group][tokens][dim] in 32 bits."""
    t = t.float().transpose(0, 1)
    return (t.repeat_interleave(group, 0) if group > 1 else t).contiguous()


def _scores(s, a, b, group):
    """Softmax over one sequence: q and k with the heads first, probabilities and the logarithms of their sums."""
    q, k = _heads_first(s["q"][a:b]), _heads_first(s["k"][a:b], group)
    z = torch.matmul(q, k.transpose(1, 2).contiguous())
    z *= s["scale"]
    if s["case"]["causal"]:
        at = torch.arange(b - a, device=z.device)
        z.masked_fill_(at[None, :] > at[:, None], -math.inf)
    top = z.amax(2, keepdim=True)
    z -= top
    z.exp_()
    total = z.sum(2, keepdim=True)
    z /= total
    return q, k, z, (top + total.log())[..., 0]


def _plain_prompt(s):
    case = s["case"]
    group = case["heads"] // case["kv_heads"]
    for a, b in zip(s["bounds"][:-1], s["bounds"][1:]):
        p, lse = _scores(s, a, b, group)[2:]
        s["o"][a:b] = torch.matmul(p, _heads_first(s["v"][a:b], group)).transpose(0, 1)
        s["lse"][:, a:b] = lse
    return {"o": s["o"], "lse": s["lse"]}


def _plain_train(s):
    case = s["case"]
    KV, group = case["kv_heads"], case["heads"] // case["kv_heads"]
    for a, b in zip(s["bounds"][:-1], s["bounds"][1:]):
        q, k, p, lse = _scores(s, a, b, group)
        v, do = _heads_first(s["v"][a:b], group), _heads_first(s["do"][a:b])
        o = torch.matmul(p, v)
        dv = torch.matmul(p.transpose(1, 2).contiguous(), do)
        ds = torch.matmul(do, v.transpose(1, 2).contiguous())
        ds -= (do * o).sum(2, keepdim=True)
        ds *= p
        ds *= s["scale"]
        dk = torch.matmul(ds.transpose(1, 2).contiguous(), q)
        s["o"][a:b], s["lse"][:, a:b] = o.transpose(0, 1), lse
        s["dq"][a:b] = torch.matmul(ds, k).transpose(0, 1)
        for out, d in (("dk", dk), ("dv", dv)):
            s[out][a:b] = d.reshape(KV, group, b - a, -1).sum(1).transpose(0, 1)
    return {"o": s["o"], "lse": s["lse"], "dqkv": s["dqkv"]}


def _plain_decode(s):
    case = s["case"]
    R, H, KV, D, L = case["requests"], case["heads"], case["kv_heads"], case["dim"], s["columns"] * case["page"]
    pages = s["table"].clamp(min=0).long()
    out = torch.arange(L, device=pages.device)[None, :] >= s["lengths"][:, None]
    q = s["q"].float().reshape(R, KV, H // KV, D)
    k = s["k_cache"][pages].float().transpose(1, 2).reshape(R, KV, L, D)
    z = torch.matmul(q, k.transpose(2, 3))
    del k
    z *= s["scale"]
    z.masked_fill_(out[:, None, None], -math.inf)
    z -= z.amax(3, keepdim=True)
    z.exp_()
    z /= z.sum(3, keepdim=True)
    v = s["v_cache"][pages].float().transpose(1, 2).reshape(R, KV, L, D)
    s["o"].copy_(torch.matmul(z, v).reshape(R, H, D))
    return {"o": s["o"]}


def _plain_plan(s):
    out = _slots(s)
    for name, v in zip(("table", "starts", "slots", "state"), out):
        s[name].copy_(v)
    return {k: s[k] for k in ("table", "starts", "slots", "state")}


def _plain_store(s):
    page, slots = s["case"]["page"], s["slots"].long()
    s["k_cache"][slots // page, :, slots % page] = s["k"]
    s["v_cache"][slots // page, :, slots % page] = s["v"]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


_PLAIN = {"prompt": _plain_prompt, "train": _plain_train, "decode": _plain_decode, "plan": _plain_plan, "store": _plain_store}


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    e = 2 if case.get("dtype") == "bfloat16" else 4
    kind = case["kind"]
    if kind in ("prompt", "train"):
        T, H, KV, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        rows, pairs = e * T * D, _pairs(case)
        if kind == "prompt":
            return {"bytes": rows * 2 * (H + KV) + 4 * T * H, "flops": 4.0 * D * H * pairs}
        return {"bytes": rows * (4 * H + 4 * KV) + 4 * T * H, "flops": 14.0 * D * H * pairs}
    lengths, added = _request_lengths(case)
    page, R = case["page"], case["requests"]
    if kind == "decode":
        tokens = sum(lengths)
        return {"bytes": e * case["dim"] * (2 * case["kv_heads"] * tokens + 2 * case["heads"] * R) + 4 * (sum(-(-n // page) for n in lengths) + R),
                "flops": 4.0 * case["dim"] * case["heads"] * tokens}
    if kind == "plan":
        # lengths and new tokens, starts and state; a free page in and a table entry out for each new page, a slot for each token
        fresh = sum(-(-n // page) + (-(n - a) // page) for n, a in zip(lengths, added))
        return {"bytes": 4 * (3 * R + 3 + 2 * fresh + sum(added)), "flops": 8.0 * sum(added)}
    return {"bytes": 4 * e * sum(added) * case["kv_heads"] * case["dim"] + 4 * sum(added), "flops": 0.0}


# ---------------------------------------------------------------------------------------
# the result in 64 bits
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("prompt", "train"):
        T, H, KV, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        o = torch.zeros(T, H, D, dtype=torch.float64, device="cuda")
        lse, dqkv = torch.zeros(H, T, dtype=torch.float64, device="cuda"), torch.zeros(T, H + 2 * KV, D, dtype=torch.float64, device="cuda")
        for (a, b), h in itertools.product(zip(s["bounds"][:-1], s["bounds"][1:]), range(H)):
            j = h * KV // H
            q, k, v = s["q"][a:b, h].double(), s["k"][a:b, j].double(), s["v"][a:b, j].double()
            z = torch.mm(q, k.t()) * s["scale"]
            if case["causal"]:
                z = z + torch.triu(torch.full_like(z, -math.inf), 1)
            logs = torch.logsumexp(z, 1)
            p = torch.exp(z - logs[:, None])
            lse[h, a:b] = logs
            o[a:b, h] = torch.mm(p, v)
            if kind == "train":
                g = s["do"][a:b, h].double()
                dp = torch.mm(g, v.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                dqkv[a:b, h] = torch.mm(ds, k)
                dqkv[a:b, H + j] += torch.mm(ds.t(), q)
                dqkv[a:b, H + KV + j] += torch.mm(p.t(), g)
        return {"o": o, "lse": lse, "dqkv": dqkv} if kind == "train" else {"o": o, "lse": lse}
    page, lengths, added = case["page"], s["lengths"].tolist(), s["added"].tolist()
    if kind == "decode":
        H, KV, D = case["heads"], case["kv_heads"], case["dim"]
        o = torch.empty(case["requests"], H, D, dtype=torch.float64, device="cuda")
        for r, n in enumerate(lengths):
            row = s["table"][r, :-(-n // page)].long()
            for j in range(KV):
                k, v = (s[c][row, j].reshape(-1, D)[:n].double() for c in ("k_cache", "v_cache"))
                at = slice(j * (H // KV), (j + 1) * (H // KV))
                o[r, at] = torch.mm(torch.softmax(torch.mm(s["q"][r, at].double(), k.t()) * s["scale"], 1), v)
        return {"o": o}
    if kind == "plan":
        table, free, at = s["table"].tolist(), s["free"].tolist(), 0
        starts, slots = _sums(added), []
        for r, (n, a) in enumerate(zip(lengths, added)):
            for t in range(n - a, n):
                if t % page == 0:
                    table[r][t // page] = free[at]
                    at += 1
                slots.append(table[r][t // page] * page + t % page)
        out = dict(table=table, starts=starts, slots=slots, state=[at, 0])
        return {k: torch.tensor(v, dtype=torch.int32).cuda() for k, v in out.items()}
    out = {}
    for name in ("k", "v"):
        cache = torch.zeros(s["pages"] * page, case["kv_heads"], case["dim"], dtype=torch.float64, device="cuda")
        cache[s["slots"].long()] = s[name].double()
        out[name + "_cache"] = cache.reshape(s["pages"], page, case["kv_heads"], case["dim"]).transpose(1, 2).contiguous()
    return out
