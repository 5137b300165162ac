"""The paged cache of keys and values on the GPU: tables and slots against a plain loop, the store, the attention of new tokens against 64 bits
(attention_ref.py), and all of them together as a server uses them."""
import random

import pytest

torch = pytest.importorskip("torch")

import attention_ref
import large_ref as ref
from paper_1804_04512_amd import binding as B
from paper_1804_04512_amd.workloads import AttentionSpec, CacheSpec, GatedSpec

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
NAN = float("nan")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ plan
def planned(lengths, added, free, at, table, pages, page, tokens, slots):
    """The plain loop: new table, starts, slots and state."""
    table, slots, starts, missing, next_free = [list(r) for r in table], list(slots), [0], 0, at
    for r, (n, a) in enumerate(zip(lengths, added)):
        n = max(0, n)
        a = max(0, min(a, n))
        for t in range(n - a, n):
            i, column = starts[-1] + t - (n - a), t // page
            new = t % page == 0
            if column >= len(table[r]):
                missing += new
                slot = -1
            else:
                if new:
                    id = free[next_free] if next_free < len(free) else -1
                    missing += next_free >= len(free)
                    next_free += next_free < len(free)
                    if i < tokens:
                        table[r][column] = id
                id = table[r][column]
                slot = id * page + t % page if 0 <= id < pages else -1
            if i < tokens:
                slots[i] = slot
        starts.append(starts[-1] + a)
    return table, starts, slots, [next_free, missing]


def check_plan(lengths, added, page, columns, n_free, at=None, room=None, seed=0, pages=None):
    rng = random.Random(seed)
    R = len(lengths)
    total = sum(max(0, min(a, n)) for n, a in zip(lengths, added))
    tokens = max(1, total) + 5 if room is None else room
    pages = pages or max(1, n_free + sum(-(-max(n, 0) // page) for n in lengths))
    free = rng.sample(range(pages), min(n_free, pages))
    table = [[rng.randrange(pages) if rng.random() < 0.95 else rng.choice([-1, pages, -(1 << 31)]) for _ in range(columns)] for _ in range(R)]
    spec = CacheSpec(R, 1, 1, 8, pages, page, columns)
    t, starts, slots, state = ints(table), ints([-7] * (R + 1)), ints([-7] * tokens), ints([-7, -7])
    args = (spec, ints(lengths), ints(added), ints(free), t, starts, slots, state, None if at is None else ints([at]))
    B.dll_cache_plan(*args)
    first = max(0, min(at or 0, len(free)))
    want = planned(lengths, added, free, first, table, pages, page, tokens, [-7] * tokens)
    got = [t.tolist(), starts.tolist(), slots.tolist(), state.tolist()]
    for name, g, w in zip(("table", "starts", "slots", "state"), got, want):
        assert g == w, name
    B.dll_cache_plan(*args)   # repeated: the same
    assert [t.tolist(), starts.tolist(), slots.tolist(), state.tolist()] == got
    return got



@pytest.mark.parametrize("page", [1, 3, 16, 20, 128])
@pytest.mark.parametrize("R,longest,most", [(1, 1, 1), (1, 5000, 5000), (3, 40, 1), (64, 300, 1), (70, 100, 50), (1500, 60, 8), (2500, 30, 1)])
def test_plan(R, longest, most, page):
    rng = random.Random(R + page)
    lengths = [rng.randint(0, longest) if R > 1 else longest for _ in range(R)]
    added = [min(n, rng.randint(0, most) if most > 1 else 1) for n in lengths]
    check_plan(lengths, added, page, -(-longest // page) + rng.randint(0, 2), sum(lengths) // page + R + 3, seed=R)


def test_plan_edges():
    check_plan([0, 0, 0], [0, 0, 0], 16, 2, 4)                                       # nothing to do
    check_plan([-5, 7, 3], [2, 9, -1], 4, 3, 10)                                     # below zero, more new than there are
    check_plan([100, 50], [100, 50], 8, 30, 5)                                       # the list is too short
    check_plan([100, 50], [10, 10], 8, 30, 0)                                        # and empty
    check_plan([100, 50, 9], [60, 50, 9], 8, 6, 40)                                  # the table is too narrow
    check_plan([100, 50, 9], [60, 50, 9], 8, 6, 40, room=70)                         # no room for all slots
    for at in (0, 3, 17, 1000, -4):
        check_plan([30, 40], [30, 1], 8, 10, 20, at=at)                              # from a later entry
    check_plan([3000, 0, 0, 2100, 1], [3000, 0, 0, 1100, 1], 16, 200, 400)           # several workgroups' tokens
    check_plan([1] * 1023 + [2, 1, 1], [1] * 1026, 16, 1, 1100)                      # a request on the border of two workgroups
    check_plan([64] * 8, [64] * 8, 16, 4, 32, pages=33)


# ------------------------------------------------------------------------------------------------ store
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tokens,heads,dim,page,off", [(1, 1, 1, 1, 0), (7, 2, 64, 16, 0), (50, 3, 33, 5, 1), (130, 8, 128, 16, 3), (1000, 4, 80, 20, 0), (5, 1, 256, 7, 2)])
def test_store(tokens, heads, dim, page, off, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens)
    pages = tokens // page + 3
    row = 2 * heads * dim + off
    both = torch.randn(tokens * row + off, generator=gen, device="cuda").to(TYPES[dtype])[off:].unflatten(0, (tokens, row))[:, :row - off].unflatten(1, (2 * heads, dim))
    k, v = both.split([heads, heads], 1)
    spec = CacheSpec(1, heads, heads, dim, pages, page, 1, dtype)
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:tokens].to(torch.int32)
    if tokens > 4:
        slots[1], slots[3], slots[4] = -1, pages * page, -(1 << 31)   # left out
    caches = [torch.full((pages, heads, page, dim), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    want = [c.transpose(1, 2).reshape(pages * page, heads, dim).clone() for c in caches]
    ok = (slots >= 0) & (slots < pages * page)
    for w, t in zip(want, (k, v)):
        w[slots[ok].long()] = t[ok]
    B.dll_cache_write(spec, k, v, slots, *caches)
    for c, w in zip(caches, want):
        assert torch.equal(c.transpose(1, 2).reshape(w.shape), w)


# ------------------------------------------------------------------------------------------------ attention
class Paged:
    """Requests of the given lengths with their pages strewn over a cache that holds NaN everywhere else."""

    def __init__(self, lengths, heads, kv_heads, dim, page, dtype, seed=0, spare=3, scale=None, columns=None):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed + dim)
        t, R = TYPES[dtype], len(lengths)
        self.lengths, self.scale = lengths, dim ** -0.5 if scale is None else scale
        need = [-(-n // page) for n in lengths]
        pages = sum(need) + spare
        columns = columns or max(1, *need) + 1
        self.spec = CacheSpec(R, heads, kv_heads, dim, pages, page, columns, dtype)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        self.table, at = torch.full((R, columns), -1, dtype=torch.int32, device="cuda"), 0
        self.q = torch.randn(R, heads, dim, generator=gen, device="cuda").to(t)
        self.k_cache, self.v_cache = (torch.full((pages, kv_heads, page, dim), NAN, dtype=t, device="cuda") for _ in range(2))
        self.k, self.v = [], []
        for r, n in enumerate(lengths):
            ids = order[at:at + need[r]]
            self.table[r, :need[r]] = ids
            at += need[r]
            for cache, rows in ((self.k_cache, self.k), (self.v_cache, self.v)):
                x = torch.randn(n, kv_heads, dim, generator=gen, device="cuda").to(t)
                rows.append(x)
                for p in range(need[r]):
                    part = x[p * page:(p + 1) * page]
                    cache[ids[p].long(), :, :part.shape[0]] = part.transpose(0, 1)
        self.n = ints(lengths)

    def run(self, fill=255, stream=None, lse=True):
        self.o = torch.full(self.q.shape, NAN, dtype=self.q.dtype, device="cuda")
        self.lse = torch.full(self.q.shape[:2], NAN, device="cuda")
        self.ws = B.workspace(B.dll_paged_attention_workspace_bytes(self.spec)).fill_(fill)
        B.dll_paged_attention(self.spec, self.q, self.k_cache, self.v_cache, self.table, self.n, self.scale, self.o, self.lse if lse else None,
                              self.ws, stream)
        return self

    def check(self, left_out={}):
        for r in range(len(self.lengths)):
            keep = [t for t in range(self.lengths[r]) if t not in left_out.get(r, ())]
            want = attention_ref.sequence(self.q[r:r + 1], self.k[r][keep], self.v[r][keep], self.scale, False)
            if not keep:
                assert (self.o[r] == 0).all() and torch.isneginf(self.lse[r]).all()
                continue
            ref.check(self.o[r:r + 1], want["o"], f"o of request {r}")
            ref.check(self.lse[r][:, None], want["lse"], f"lse of request {r}")
        return self


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim,page", [
    ([1], 1, 1, 64, 16), ([0], 2, 1, 64, 16), ([5, 0, 17], 4, 2, 128, 16), ([127, 128, 129, 1], 8, 8, 64, 16), ([1000], 16, 4, 128, 16),
    ([33, 600, 0, 0, 31, 2], 8, 1, 96, 20), ([3000, 1], 24, 1, 64, 64), ([70] * 40, 6, 3, 80, 7), ([2049], 5, 1, 256, 100), ([300, 20], 4, 4, 32, 1),
    ([0, 9000, 3], 2, 2, 128, 32), ([4000, 4001], 40, 2, 128, 16), ([1, 2, 3] * 100, 2, 1, 16, 16)], ids=str)
def test_attention(lengths, heads, kv_heads, dim, page, dtype):
    Paged(lengths, heads, kv_heads, dim, page, dtype).run().check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", [1, 4, 7, 20, 33, 65, 100, 127, 200, 255])
def test_head_sizes(dim, dtype):
    Paged([50, 333], 6, 2, dim, 16, dtype, seed=1).run().check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 2.0])
def test_scales(scale, dtype):
    Paged([200, 3], 4, 2, 64, 16, dtype, seed=2, scale=scale).run().check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_pages_that_are_none(dtype):
    """Entries outside the cache leave their keys out, a request all of whose entries are has none; what lies behind a table's room, too."""
    c = Paged([100, 40, 300, 16], 4, 2, 64, 16, dtype, seed=3)
    c.table[0, 2], c.table[0, 6], c.table[2, 0] = -1, c.spec.pages, 1 << 30
    c.table[1, :3] = -5
    c.run().check({0: [*range(32, 48), *range(96, 100)], 1: range(40), 2: range(16)})
    c = Paged([100, 64], 4, 2, 64, 16, dtype, seed=3, columns=7)
    c.n = ints([1 << 30, -3])
    c.table[:] = c.table[0]
    c.k[0], c.v[0], c.lengths = c.k[0][:96], c.v[0][:96], [96, 0]
    c.table[0, 6] = -1   # the last of the seven
    c.run().check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_growing_scores(dtype):
    c = Paged([700], 4, 2, 32, 16, dtype, seed=4)
    for p, id in enumerate(c.table[0, :44].tolist()):
        c.k_cache[id] = (c.k_cache[id].float() * 0.1 + p / 4).to(TYPES[dtype])
    c.k[0] = c.k_cache[c.table[0, :44].long()].transpose(1, 2).reshape(-1, 2, 32)[:700]
    c.q.copy_((c.q.float() * 0.1 + 1).to(c.q.dtype))
    c.run().check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_whatever_the_workspace_holds(dtype):
    c = Paged([1000, 3, 0, 2000], 8, 2, 128, 16, dtype, seed=5).run()
    want = c.o, c.lse
    for fill in (0, 0x7F, 0x7E):
        c.run(fill)
        assert torch.equal(c.o, want[0]) and torch.equal(c.lse, want[1])
    c.run(lse=False)
    assert torch.equal(c.o, want[0]) and torch.isnan(c.lse).all()


def test_shared_pages():
    """Two requests whose tables begin with the same pages."""
    c = Paged([160, 170], 4, 2, 64, 16, "bfloat16", seed=6)
    c.table[1, :5] = c.table[0, :5]
    c.k[1][:80], c.v[1][:80] = c.k[0][:80], c.v[0][:80]
    c.run().check()


def test_two_calls_at_once():
    cases = [Paged([3000, 500], 8, 2, 128, 16, "bfloat16", seed=7 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_cache_of_more_than_31_bits():
    """Elements and bytes of the caches pass 32 bits; only pages at both ends are touched."""
    KV, D, page, pages = 8, 128, 16, 140000
    assert pages * KV * page * D > 1 << 31
    spec = CacheSpec(2, 16, KV, D, pages, page, 20, "bfloat16")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    n = [300, 17]
    caches = [torch.empty(pages, KV, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    free = ints([pages - 1 - i if i % 2 else i for i in range(30)])
    table, starts, slots, state = ints([[-1] * 20] * 2), ints([0] * 3), ints([0] * sum(n)), ints([0, 0])
    B.dll_cache_plan(spec, ints(n), ints(n), free, table, starts, slots, state)
    k, v = (torch.randn(sum(n), KV, D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    B.dll_cache_write(spec, k, v, slots, *caches)
    q = torch.randn(2, 16, D, generator=gen, device="cuda").to(torch.bfloat16)
    o = torch.full_like(q, NAN)
    B.dll_paged_attention(spec, q, *caches, table, ints(n), D ** -0.5, o, ws=B.workspace(B.dll_paged_attention_workspace_bytes(spec)))
    for r, (a, b) in enumerate(((0, 300), (300, 317))):
        ref.check(o[r:r + 1], attention_ref.sequence(q[r:r + 1], k[a:b], v[a:b], D ** -0.5, False)["o"], f"o of request {r}")


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_server(dtype):
    """Prompts through attention and into the cache, then steps of one token: plan, store, attention and a gated block, the steps captured once and
    replayed.  Every step's attention is that of the whole history so far."""
    H, KV, D, page, prompts, steps = 8, 2, 64, 16, [37, 1, 100, 16], 6
    R, width = len(prompts), H * D
    t = TYPES[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    spec = CacheSpec(R, H, KV, D, 40, page, 10, dtype)
    caches = [torch.full((40, KV, page, D), NAN, dtype=t, device="cuda") for _ in range(2)]
    table, starts, state, at = ints([[-1] * 10] * R), ints([0] * (R + 1)), ints([0, 0]), ints([0])
    free, lengths = ints(random.Random(1).sample(range(40), 40)), ints(prompts)
    total = sum(prompts)
    qkv = torch.randn(total, H + 2 * KV, D, generator=gen, device="cuda").to(t)
    q, k, v = qkv.split([H, KV, KV], 1)
    slots = ints([-1] * total)
    B.dll_cache_plan(spec, lengths, lengths, free, table, starts, slots, state, at)
    row = (H + 2 * KV) * D
    prompt = AttentionSpec(total, total, R, H, KV, D, True, dtype, row, row)
    o = torch.full((total, H, D), NAN, dtype=t, device="cuda")
    B.dll_attention_fwd(prompt, q, k, v, starts, starts, D ** -0.5, o, ws=B.workspace(B.dll_attention_fwd_workspace_bytes(prompt)))
    B.dll_cache_write(spec, k, v, slots, *caches)
    ends = starts.tolist()
    keys = [[k[a:b], v[a:b]] for a, b in zip(ends, ends[1:])]
    for r, (a, b) in enumerate(zip(ends, ends[1:])):
        ref.check(o[a:b], attention_ref.sequence(q[a:b], k[a:b], v[a:b], D ** -0.5, True)["o"], f"prompt {r}")

    block = GatedSpec(R, width, 96, "silu", dtype)
    w = [torch.randn(s, generator=gen, device="cuda").to(t) / 16 for s in ((96, width), (96, width), (width, 96))]
    new = torch.empty(R, H + 2 * KV, D, dtype=t, device="cuda")
    qn, kn, vn = torch.empty(R, H, D, dtype=t, device="cuda"), new[:, H:H + KV], new[:, H + KV:]
    one, out, y, step_slots = ints([1] * R), torch.empty(R, H, D, dtype=t, device="cuda"), torch.empty(R, width, dtype=t, device="cuda"), ints([-1] * R)
    ws, ws_block = B.workspace(B.dll_paged_attention_workspace_bytes(spec)), B.workspace(B.dll_gated_fwd_workspace_bytes(block))

    def step():
        lengths.add_(one)
        at.copy_(state[:1])
        qn.copy_(new[:, :H])
        B.dll_cache_plan(spec, lengths, one, free, table, starts, step_slots, state, at)
        B.dll_cache_write(spec, kn, vn, step_slots, *caches)
        B.dll_paged_attention(spec, qn, *caches, table, lengths, D ** -0.5, out, ws=ws)
        B.dll_gated_fwd(block, out.reshape(R, width), *w, y, ws=ws_block)

    graph = None
    for turn in range(steps):
        new.copy_(torch.randn(new.shape, generator=gen, device="cuda").to(t))
        if graph is None and turn == 2:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        torch.cuda.synchronize()
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        assert lengths.tolist() == [n + turn + 1 for n in prompts] and state.tolist()[1] == 0
        for r in range(R):
            keys[r] = [torch.cat((a, b[r:r + 1])) for a, b in zip(keys[r], (kn, vn))]
            ref.check(out[r:r + 1], attention_ref.sequence(new[r:r + 1, :H], *keys[r], D ** -0.5, False)["o"], f"step {turn} of request {r}")
        eager = torch.empty_like(y)
        B.dll_gated_fwd(block, out.reshape(R, width), *w, eager, ws=ws_block)
        assert torch.equal(y, eager)
    held = sum(-(-(n + steps) // page) for n in prompts)
    assert state.tolist() == [held, 0]
