"""Plain 64-bit implementations of the operators around the layer, each with a bound on how far a kernel's output may be
from it, element by element.

A value rounded to the storage type t is off by at most HALF[t] = finfo(t).eps / 2 of itself.  An fp32 sum of n terms, in any
order, is off by at most n 2^-24 of the sum of the terms' absolute values; a matrix instruction may cut instead of round, so its
sums count 2^-23 per addition.  Every intermediate value carries its bound through the formulas to first order; the second orders
are below a hundredth of the first and are covered by the factor 1.02 at the end.
"""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
SLACK = 1.02


def within(got, ref, bound, name):
    got, ref, bound = got.double().cpu(), ref.double().cpu(), bound.double().cpu() * SLACK + 1e-37
    assert got.shape == ref.shape, name
    off = (got - ref).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst "
                                 f"{float((off / bound).nan_to_num(1e9).max()):.3g} times it at {int((off / bound).nan_to_num(1e9).argmax())}")


def norm_forward(x, residual, weight, eps, dt):
    """s, y and their bounds.  A lane adds at most 64 squares one after the other, then 12 partial sums; 1 / sqrt of it and two
    products: 96 roundings at most, half of those of the sum count (the root)."""
    s = x.double() + (residual.double() if residual is not None else 0)
    r = 1.0 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    y = s * r * weight.double()
    return s, y, s.abs() * (HALF[dt] + U), y.abs() * (HALF[dt] + 96 * U)


def norm_backward(s, weight, dy, dsum, eps, dt):
    """From the stored sum: d_x, d_weight and their bounds."""
    s, w, dy = s.double(), weight.double(), dy.double()
    r = 1.0 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    n, m = s * r, dy * w
    along, mag = (m * n).mean(1, keepdim=True), (m * n).abs().mean(1, keepdim=True)
    g = dsum.double() if dsum is not None else torch.zeros_like(m)
    dx = g + r * (m - n * along)
    bx = HALF[dt] * dx.abs() + 128 * U * (g.abs() + r * (m.abs() + n.abs() * mag))
    dw = (dy * n).sum(0)
    # rows one after the other in a block (at most 768 of them share the rows), 4 wavefronts, 48 + 16 partial sums
    depth = s.shape[0] // 768 + 68 + 96
    return dx, dw, bx, depth * U * (dy * n).abs().sum(0)


def _product(a, b, ea, eb, steps, terms):
    """a b with the bounds of the operands carried through; steps: additions to an accumulator."""
    ref = a @ b
    mag = a.abs() @ b.abs()
    own = (6 if terms == 3 else 1) * steps * 2.0 ** -23 + (2.0 ** -21 if terms == 3 else 0.0)
    e = mag * own
    if ea is not None:
        e = e + ea @ b.abs()
    if eb is not None:
        e = e + a.abs() @ eb
    return ref, e


def gated(x, w, addend, dt, dy=None, dx_addend=None):
    """y, and with dy d_x and the gradients of Wg, Wu, Wd: {name: (reference, bound)}."""
    terms = 1 if dt == torch.bfloat16 else 3
    half = HALF[dt]
    x = x.double()
    Wg, Wu, Wd = (w[n].double() for n in ("Wg", "Wu", "Wd"))
    T, d = x.shape
    H = Wg.shape[1]
    adds = lambda k: k / 8 + 48  # noqa: E731  (an instruction adds 16 products, in pairs at worst; shares and segments on top)
    g, eg = _product(x, Wg, None, None, adds(d), terms)
    u, eu = _product(x, Wu, None, None, adds(d), terms)
    return _gated_tail(x, g, eg, u, eu, Wg, Wu, Wd, addend, dt, half, terms, adds, dy, dx_addend, T, d, H)


def _gated_tail(x, g, eg, u, eu, Wg, Wu, Wd, addend, dt, half, terms, adds, dy, dx_addend, T, d, H):
    sg = torch.sigmoid(g)
    s = g * sg
    slope = sg + s * (1 - sg)              # silu'
    curve = 0.5                            # |silu''| <= 1/2
    # the exponential and the reciprocal: relative 2^-21 with a |g| 2^-23 of the exponent's own rounding
    rel = 2.0 ** -20 + g.abs() * 2.0 ** -23
    es = slope.abs() * eg + s.abs() * rel
    a = s * u
    ea = s.abs() * eu + u.abs() * es + (half + 4 * U) * a.abs()
    f, ef = _product(a, Wd, ea, None, adds(H), terms)
    add = addend.double() if addend is not None else torch.zeros_like(f)
    y = add + f
    out = {"y": (y, ef + half * y.abs() + U * add.abs())}
    if dy is None:
        return out
    dy = dy.double()
    da, eda = _product(dy, Wd.t(), None, None, adds(d), terms)
    du = da * s
    edu = eda * s.abs() + da.abs() * es + (half + 4 * U) * du.abs()
    dg = da * u * slope
    edg = eda * (u * slope).abs() + (da * slope).abs() * eu + (da * u).abs() * (curve * eg + (sg + s.abs()) * rel) + (half + 8 * U) * dg.abs()
    p, ep = _product(dg, Wg.t(), edg, None, adds(H), terms)
    q, eq = _product(du, Wu.t(), edu, None, adds(H), terms)
    add = dx_addend.double() if dx_addend is not None else torch.zeros_like(p)
    dx = add + p + q
    out["d_x"] = (dx, ep + eq + half * dx.abs() + U * (add.abs() + p.abs()))
    for name, l, el, r, er in (("Wg", x, None, dg, edg), ("Wu", x, None, du, edu), ("Wd", a, ea, dy, None)):
        v, e = _product(l.t(), r, None if el is None else el.t(), er, adds(T), terms)
        out[name] = (v, e + half * v.abs())
    return out


def gated_quantized(xq, xs, w, addend):
    x = xq.float().double() * xs.double()[:, None]
    Wg, Wu = ((w[n].float().double() * w[n + "_scale"].double()[:, None]).t() for n in ("Wg", "Wu"))
    T, d = x.shape
    H = Wg.shape[1]
    adds = lambda k: k / 8 + 48  # noqa: E731
    g, eg = _product(x, Wg, None, None, adds(d), 1)
    u, eu = _product(x, Wu, None, None, adds(d), 1)
    eg, eu = eg + 4 * U * g.abs(), eu + 4 * U * u.abs()   # the scales
    return _gated_tail(x, g, eg, u, eu, Wg, Wu, w["Wd"].double(), addend, torch.bfloat16, HALF[torch.bfloat16], 1, adds, None, None, T, d, H)["y"]
