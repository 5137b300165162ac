"""Attention in 64 bits, elementary torch operations only, and how far 32-bit sums and the roundings of an operand type may take a
result from it (the kinds of error as in large_ref.py).

A score's sum of D terms is off by gamma(D) sum |q||k|, its exponent by the roundings of the scale's factor and of the difference;
2^x by EXP relative, and once more for each of the nk / 32 tiles at which a row's running maximum may grow.  Exponentials below 2^-126 vanish.
In bfloat16 p and ds are rounded before they are summed up.
"""
import torch

from large_ref import EXP, U32, gamma, unit

TINY = 2.0 ** -126


def _rows(t):
    return t.double().transpose(0, 1)


def sequence(q, k, v, scale, causal, d_o=None):
    """One sequence: q, d_o [n_q][H][D], k, v [n_k][KV][D] in their own type.  {name: (value, bound)}, lse as [H][n_q]."""
    u, D = unit(q.dtype), q.shape[2]
    (nq, H), (nk, KV) = q.shape[:2], k.shape[:2]
    g = H // KV
    q, k, v = _rows(q), _rows(k).repeat_interleave(g, 0), _rows(v).repeat_interleave(g, 0)
    kT, vT = k.transpose(1, 2), v.transpose(1, 2)
    z = scale * (q @ kT)
    ez = abs(scale) * gamma(D) * (q.abs() @ kT.abs()) + 4 * U32 * z.abs()
    at = torch.arange(max(nq, nk), device=q.device)
    seen = torch.ones(nq, nk, dtype=torch.bool, device=q.device)
    if causal:
        seen = at[None, :nk] <= at[:nq, None] + nk - nq
    empty = ~seen.any(1)
    zm = torch.where(seen, z, -torch.inf)
    top = zm.amax(2, keepdim=True) if nk else torch.full((H, nq, 1), -torch.inf, dtype=torch.float64, device=q.device)
    top = torch.where(torch.isinf(top), 0.0, top)
    e = torch.exp(zm - top)
    lse = top[..., 0] + e.sum(2).log()
    p = torch.where(empty[:, None], 0.0, torch.exp(zm - torch.where(empty, 0.0, lse)[..., None]))
    ep = p * (ez + 4 * U32 * top.abs() + EXP * (1 + nk / 32)) + TINY * seen
    el = (ep.sum(2) + gamma(nk) * p.sum(2))   # of the sum of exponentials, relative, as p sums to 1
    o = p @ v
    eo = (ep + (u + gamma(2 * nk)) * p) @ v.abs() + (el[..., None] + u + 4 * U32) * o.abs()
    out = {"o": (o, eo), "lse": (lse, el + 64 * U32 + 4 * U32 * torch.where(empty, 0.0, lse).abs())}
    if d_o is not None:
        d_o = _rows(d_o)
        dp = d_o @ vT
        delta = (d_o * o).sum(2, keepdim=True)
        edelta = (d_o.abs() * (eo + gamma(D) * o.abs())).sum(2, keepdim=True)
        # rows that see few keys take delta as sum p dp, whose terms are off by p's and dp's errors
        edelta = edelta + (p * gamma(D) * (d_o.abs() @ vT.abs()) + ep * dp.abs() + gamma(nk) * (p * dp).abs()).sum(2, keepdim=True)
        edp = gamma(D) * (d_o.abs() @ vT.abs() + delta.abs()) + edelta
        ep = p * (ez + out["lse"][1][..., None] + 4 * U32 * (z.abs() + torch.where(empty, 0.0, lse)[..., None].abs()) + EXP) + TINY * seen
        ds = p * (dp - delta)
        eds = (p + ep) * edp + ep * (dp - delta).abs() + u * ds.abs()
        ep = ep + u * p

        def product(a, ea, b, terms, factor):
            return factor * (a @ b), abs(factor) * ((ea + gamma(terms) * a.abs()) @ b.abs())

        shared = lambda t: t.reshape(KV, g, nk, D).sum(1)   # noqa: E731
        dq = product(ds, eds, k, nk, scale)
        dk = [shared(t) for t in product(ds.transpose(1, 2), eds.transpose(1, 2), q, nq * g, scale)]
        dv = [shared(t) for t in product(p.transpose(1, 2), ep.transpose(1, 2), d_o, nq * g, 1.0)]
        for name, (value, bound) in (("dq", dq), ("dk", dk), ("dv", dv)):
            out[name] = (value, bound + (u + 2 * U32) * value.abs())
    return {name: t if name == "lse" else (t[0].transpose(0, 1), t[1].transpose(0, 1)) for name, t in out.items()}
