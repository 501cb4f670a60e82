"""Norms on both sides of a block, in 64 bits, with bounds carried through the formulas (the roundings: block_reference.py)."""
import torch

from block_reference import HALF, U

SUM = 128 * U      # a row's sum: a lane's values one after the other, the lanes, up to 16 wavefronts


def _wide(t):
    return None if t is None else t.double().cpu()


def forward(x, post, gate, residual, pre, a, eps, dt):
    """{name: (reference, bound)} of sum, y (if pre), stats; and y's fp32 bound."""
    x, post, gate, residual, pre = map(_wide, (x, post, gate, residual, pre))
    r1 = 1.0 / (x.square().mean(1, keepdim=True) + eps).sqrt() if post is not None else torch.ones(x.shape[0], 1, dtype=torch.float64)
    n = x * r1 * (post if post is not None else 1.0) * (gate if gate is not None else 1.0)
    s = a * residual + n
    es = n.abs() * (SUM + 4 * U) + U * (a * residual).abs() + U * s.abs()
    r2 = 1.0 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    rel = SUM + es.square().mean(1, keepdim=True).sqrt() * r2
    out = {"sum": (s, es + HALF[dt] * s.abs()), "stats": (torch.cat([r1, r2], 1), torch.cat([r1 * SUM, r2 * rel], 1))}
    if pre is not None:
        y = s * r2 * pre
        e = y.abs() * (rel + 4 * U) + (r2 * pre).abs() * es
        out["y"], out["y32"] = (y, e + HALF[dt] * y.abs()), (y, e)
    return out


def backward(x, post, gate, s, pre, stats, dy, dsum, a, dt, token):
    x, post, gate, s, pre, stats, dy, dsum = map(_wide, (x, post, gate, s, pre, stats, dy, dsum))
    T = x.shape[0]
    r1, r2 = stats[:, :1], stats[:, 1:]
    one = torch.ones(x.shape[1], dtype=torch.float64)
    w, g = (post if post is not None else one), (gate if gate is not None else one)
    n2, m2, dsum = s * r2, dy * pre, dsum if dsum is not None else torch.zeros_like(s)
    ds = dsum + r2 * (m2 - n2 * (m2 * n2).mean(1, keepdim=True))
    eds = SUM * (dsum.abs() + r2 * (m2.abs() + n2.abs() * (m2 * n2).abs().mean(1, keepdim=True)))
    n1, m1 = x * r1, ds * g * w
    em1 = (g * w).abs() * eds + 4 * U * m1.abs()
    k = 1.0 if post is not None else 0.0
    mean = k * (m1 * n1).mean(1, keepdim=True)
    emean = k * ((em1 * n1.abs()).mean(1, keepdim=True) + SUM * (m1 * n1).abs().mean(1, keepdim=True))
    dx = r1 * (m1 - n1 * mean)
    out = {"d_x": (dx, HALF[dt] * dx.abs() + r1 * (em1 + n1.abs() * emean + 8 * U * (m1.abs() + n1.abs() * mean.abs())))}
    out["d_residual"] = (a * ds, HALF[dt] * (a * ds).abs() + abs(a) * (eds + U * ds.abs()))
    depth = (T // 256 + 168) * U
    along, ealong = ds * n1, (eds * n1.abs() + 2 * U * (ds * n1).abs())

    def column(v, e):
        return v.sum(0), e.sum(0) + depth * v.abs().sum(0)
    if post is not None:
        out["d_post"] = column(along * g, ealong * g.abs())
    if gate is not None:
        v, e = along * w, ealong * w.abs()
        out["d_gate"] = (v, e + (HALF[dt] + 2 * U) * v.abs()) if token else column(v, e)
    out["d_pre"] = column(dy * n2, 2 * U * (dy * n2).abs())
    return out
