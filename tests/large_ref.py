"""The large-model operators in 64 bits, elementary torch operations only, and how far 32-bit sums and the roundings of
an operand type may take a result from them.

Bounds are elementwise and follow the computation.  A product of K terms summed in 32 bits in any order is off by at most
K * 2^-24 * sum |a||b| (first order); a rounding to type t by half a step, eps(t) / 2 relative; errors of operands pass
through products with the other operand's magnitude and through a function with the bound of its derivative.
Single precision may be multiplied as three bfloat16 parts, x = hi + mid + lo + r with |mid| <= 2^-8 |x|, |lo| <= 2^-16 |x|,
|r| <= 2^-24 |x|: the six products kept leave out mid lo + lo mid + r y + x r', at most 4 * 2^-24 |x||y|, and each term is six
numbers to add, of which five are at most 2^-8 of it: five roundings of the first sums more.  Hence K + 12 for K + 4.
"""
import math

import torch

U32 = 2.0 ** -24


def unit(dtype):
    """Half a step of the type, relative."""
    return torch.finfo(dtype).eps / 2


def gamma(k):
    return (k + 12) * U32


def act(name, a):
    """The gate's activation and its derivative."""
    if name == "identity":
        return a, torch.ones_like(a)
    if name == "relu":
        return a.clamp(min=0), (a > 0).to(a.dtype)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-a))
    if name == "sigmoid":
        return sig, sig * (1 - sig)
    return a * sig, sig * (1 + a * (1 - sig))


# the largest |f'| and |f''| (ReLU's jump is counted where it may happen)
SLOPE = {"identity": 1.0, "sigmoid": 0.25, "relu": 1.0, "silu": 1.1, "gelu": 1.13}
BEND = {"identity": 0.0, "sigmoid": 0.1, "relu": 0.0, "silu": 0.5, "gelu": 0.8}
FUNC = 16 * U32   # of the activation itself, relative to 1 + |a|


def gated(x, wg, wu, wd, gate, dy=None):
    """Results and bounds {name: (value, bound)} of the block; operands in their own type."""
    dtype = x.dtype
    u, T = unit(dtype), x.shape[0]
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    H, D = wg.shape
    a, b = x @ wg.t(), x @ wu.t()
    ea, eb = gamma(D) * (x.abs() @ wg.abs().t()), gamma(D) * (x.abs() @ wu.abs().t())
    f, d = act(gate, a)
    h = f * b
    efun = FUNC * (1 + a.abs())
    eh = (SLOPE[gate] * ea + efun) * b.abs() + f.abs() * eb + u * h.abs()
    y = h @ wd.t()
    out = {"y": (y, (eh + gamma(H) * h.abs()) @ wd.abs().t() + u * y.abs())}
    out["gate_pre"], out["up_pre"] = (a, ea + u * a.abs()), (b, eb + u * b.abs())
    if dy is None:
        return out
    dy = dy.double()
    ea, eb = ea + u * a.abs(), eb + u * b.abs()   # as kept
    eh = (SLOPE[gate] * ea + efun) * (b.abs() + eb) + f.abs() * eb + u * h.abs()
    dh = dy @ wd
    edh = gamma(D) * (dy.abs() @ wd.abs())
    da, db = dh * b * d, dh * f
    ed = BEND[gate] * ea + efun
    if gate == "relu":
        ed = ed + (a.abs() <= ea).double()
    eda = edh * (b * d).abs() + dh.abs() * eb * d.abs() + dh.abs() * (b.abs() + eb) * ed + u * da.abs()
    edb = edh * f.abs() + dh.abs() * (SLOPE[gate] * ea + efun) + u * db.abs()

    def pair(v, e):
        return v, e + u * v.abs()

    out["dx"] = pair(da @ wg + db @ wu, (eda + gamma(2 * H) * da.abs()) @ wg.abs() + (edb + gamma(2 * H) * db.abs()) @ wu.abs())
    out["dw_gate"] = pair(da.t() @ x, (eda + gamma(T) * da.abs()).t() @ x.abs())
    out["dw_up"] = pair(db.t() @ x, (edb + gamma(T) * db.abs()).t() @ x.abs())
    out["dw_down"] = pair(dy.t() @ h, dy.abs().t() @ (eh + gamma(T) * h.abs()))
    return out


EXP = 2.0 ** -17   # of exp(x), relative, down to x = -80 (|x| * 2^-24 * log2 e and the hardware's last digits)


def vocab(x, w, bias, labels, scale=1.0):
    """Results and bounds of loss and gradients; rows whose label lies outside the classes do not count."""
    dtype = x.dtype
    u = unit(dtype)
    V, D = w.shape
    T = x.shape[0]
    rows = ((labels >= 0) & (labels < V)).nonzero()[:, 0]
    n = len(rows)
    lab = labels[rows].long()
    xr, w = x[rows].double(), w.double()
    z = xr @ w.t()
    ez = gamma(D) * (xr.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        ez = ez + torch.where(torch.isinf(z), 0.0, U32 * z.abs())
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    lse = top + e.sum(1, keepdim=True).log()
    p = torch.exp(z - lse)
    elz = (p * ez).sum(1, keepdim=True) + (p * EXP).sum(1, keepdim=True) + 64 * U32 + 2 * U32 * lse.abs()
    at = torch.arange(n, device=x.device)
    each = lse[:, 0] - z[at, lab]
    eeach = elz[:, 0] + ez[at, lab] + 2 * U32 * (lse[:, 0].abs() + z[at, lab].abs())

    def full(v):
        return torch.zeros((T,) + v.shape[1:], dtype=torch.float64, device=x.device).index_copy(0, rows, v)

    zero = torch.zeros(1, dtype=torch.float64, device=x.device)
    out = {"row_loss": (full(each), full(eeach)), "row_lse": (full(lse[:, 0]), full(elz[:, 0])),
           "loss": (each.mean().reshape(1), eeach.mean().reshape(1) + U32 * each.mean().abs()) if n else (zero, zero)}
    if not n:
        dz = torch.zeros_like(z)
        edz = dz
    else:
        g = scale / n
        dz = p * g
        # an exponential below the smallest normal number, 2^-126, becomes 0, as may its product with exp(m_g - lse) <= 1 and
        # with g: whatever the value, each of the two steps takes off less than 2^-126 times g (or 2^-126 where g > 1 is not there)
        edz = dz.abs() * (ez + elz + u + EXP) + 2 * 2.0 ** -126 * max(1.0, abs(g))
        dz[at, lab] -= g
        edz = edz + (u + 4 * U32) * dz.abs() + torch.zeros_like(dz).index_put((at, lab), torch.tensor(4 * U32 * abs(g), dtype=torch.float64, device=x.device))
    dx, dw, db = dz @ w, dz.t() @ xr, dz.sum(0)
    out["dx"] = (full(dx), full((edz + gamma(V) * dz.abs()) @ w.abs() + u * dx.abs()))
    out["dw"] = (dw, (edz + gamma(n) * dz.abs()).t() @ xr.abs() + u * dw.abs())
    out["dbias"] = (db, (edz + gamma(n) * dz.abs()).sum(0) + u * db.abs())
    return out


def check(got, ref, what=""):
    """Every element within its bound."""
    value, bound = ref
    got = got.double().reshape(value.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - value).abs() - bound
    worst = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or over.flatten()[worst] <= 1e-300, (
        f"{what}: element {worst} is {got.flatten()[worst]} for {value.flatten()[worst]}, bound {bound.flatten()[worst]}")
