"""A training step through the norms around the layer: the layer between two of them, forward and backward, against differences of the loss, and
captured into one graph while an eager step of the same tensors lives."""
import dataclasses

import pytest
import torch

from common import make_inputs
from paper_2510_04286_amd import workload as wl

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


class Train:
    """Norm -> layer -> norm; the loss is the sum of c * y + e * s of the last norm."""

    def __init__(self, B, T, gate, dtype):
        shape = dataclasses.replace(wl.CONFIGS["tiny"].scaled(T), dtype=dtype)
        s, _, w = make_inputs(shape)
        dt = torch.bfloat16 if dtype == "bf16" else F32
        self.B, self.T, self.d = B, T, s.d
        self.cfg = B.config_of(s)
        w = B.weights_to_device(w, dtype)
        self.w = B.pack(self.cfg, w) if B.slicemoe_packed_bytes(self.cfg) else w
        self.ncfg = B.make_block_norm_config(T, s.d, 1e-5, 0.5, gate, dt)
        g = torch.Generator().manual_seed(T)
        r = lambda *shape, scale=1.0, add=0.0: (torch.randn(*shape, generator=g) * scale + add).to(dt).cuda()  # noqa: E731
        self.token = gate == "token"
        self.leaves = {"x": r(T, s.d, scale=0.3), "residual": r(T, s.d, scale=2.0)}
        for i in "12":
            self.leaves.update({"post" + i: r(s.d, scale=0.2, add=1.0), "pre" + i: r(s.d, scale=0.2, add=1.0),
                                "gate" + i: r(T, s.d) if self.token else r(s.d)})
        self.c, self.e = r(T, s.d), r(T, s.d)
        like = lambda: torch.empty((T, s.d), dtype=dt, device="cuda")  # noqa: E731
        self.s1, self.y1, self.out, self.s2, self.y2, self.d_out, self.d_s1, self.d_y1, self.d_x, self.d_res = (like() for _ in range(10))
        self.st1, self.st2 = (torch.empty((T, 2), device="cuda") for _ in range(2))
        self.ws, self.wgrads = B.alloc_workspace(self.cfg), B.alloc_weight_grads(self.cfg)
        self.bws = torch.empty(max(256, B.slicemoe_backward_workspace_bytes(self.cfg)), dtype=torch.uint8, device="cuda")
        self.nws = torch.empty(max(256, B.slicemoe_block_norm_backward_workspace_bytes(self.ncfg)), dtype=torch.uint8, device="cuda")
        vec = lambda: torch.empty(s.d, device="cuda")  # noqa: E731
        self.grads = {n: vec() for n in ("post1", "pre1", "post2", "pre2")}
        self.grads.update({n: like() if self.token else vec() for n in ("gate1", "gate2")})

    def forward(self):
        B, v = self.B, self.leaves
        B.slicemoe_block_norm(self.ncfg, v["x"], v["post1"], v["gate1"], v["residual"], v["pre1"], self.s1, self.y1, stats=self.st1)
        B.slicemoe_forward(self.cfg, self.y1, self.w, self.out, self.ws)
        B.slicemoe_block_norm(self.ncfg, self.out, v["post2"], v["gate2"], self.s1, v["pre2"], self.s2, self.y2, stats=self.st2)

    def loss(self):
        self.forward()
        return float((self.c.double() * self.y2.double() + self.e.double() * self.s2.double()).sum())

    def step(self):
        B, v, g = self.B, self.leaves, self.grads
        self.forward()
        B.slicemoe_block_norm_backward(self.ncfg, self.out, v["post2"], v["gate2"], self.s2, v["pre2"], self.st2, self.c, self.d_out, self.d_s1,
                                       g["post2"], g["gate2"], g["pre2"], self.nws, d_sum=self.e)
        B.slicemoe_backward(self.cfg, self.y1, self.w, self.ws, self.d_out, self.d_y1, self.wgrads, self.bws)
        B.slicemoe_block_norm_backward(self.ncfg, v["x"], v["post1"], v["gate1"], self.s1, v["pre1"], self.st1, self.d_y1, self.d_x, self.d_res,
                                       g["post1"], g["gate1"], g["pre1"], self.nws, d_sum=self.d_s1)

    def results(self):
        torch.cuda.synchronize()
        return {n: t.clone() for n, t in dict(self.grads, x=self.d_x, residual=self.d_res, y=self.y2, sum=self.s2, **{"W." + n: t for n, t in self.wgrads.items()}).items()}


@pytest.mark.parametrize("gate", ["channel", "token"])
def test_gradients_against_differences(B, gate):
    """Central differences along the last norm's leaves and the layer's output: the function between is smooth there (the router picks experts
    in front of it, so a difference through it may step over a change of picks).

    The loss is taken in 64 bits of y and s in fp32; `base` is the sum of the sizes of what its terms are made of.  A step of eps = 2^-7 along a
    relative change u, |u_i| <= |leaf_i|.  Rounding: each term is off by at most 136 U of its size (a row's sum of up to 128 roundings, 8 more), so
    the difference quotient by 2 * 136 * 2^-24 / (2 * 2^-7) < 2^-9.9 of base.  Third order: two norms behind each other, in each the derivatives of
    1 / rms along a relative change at most 1, 3 and 15 of it, so a term's third derivative stays below 100 of its size: eps^2 / 6 * 100 < 2^-9.9.
    The direction is taken along the gradient's signs, so that what is compared is as large as can be."""
    o = Train(B, 24, gate, "f32")
    o.step()
    got = o.results()
    B_, v, eps = o.B, o.leaves, 2.0 ** -7
    g = torch.Generator().manual_seed(1)
    along = 0.5 * o.s1.double()
    size = along.abs() + (o.s2.double() - along).abs()
    base = float((((o.c * v["pre2"]).double() * o.st2[:, 1:].double()).abs() * size + o.e.double().abs() * size).sum())

    def tail():
        B_.slicemoe_block_norm(o.ncfg, o.out, v["post2"], v["gate2"], o.s1, v["pre2"], o.s2, o.y2)
        return float((o.c.double() * o.y2.double() + o.e.double() * o.s2.double()).sum())

    for name, leaf, grad in (("post2", v["post2"], got["post2"]), ("gate2", v["gate2"], got["gate2"]), ("pre2", v["pre2"], got["pre2"]),
                             ("out", o.out, o.d_out), ("s1", o.s1, o.d_s1)):
        keep, grad = leaf.clone(), grad.double().clone()
        u = torch.rand(leaf.shape, generator=g).cuda() * keep.abs() * grad.sign().float()
        ends = []
        for sign in (1, -1):
            leaf.copy_(keep + sign * eps * u)
            ends.append(tail())
        step = u.double()   # (the rounding of leaf + step, 2^-24 / eps of the leaf, is one of the 8)
        leaf.copy_(keep)
        want, have = (ends[0] - ends[1]) / (2 * eps), float((grad * step).sum())
        assert abs(want - have) <= 2.0 ** -8 * base, (name, want, have)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,gate", [(1, "token"), (200, "channel"), (777, "token")])
def test_captured_while_an_eager_step_lives(B, T, gate, dtype):
    a, b = Train(B, T, gate, dtype), Train(B, T, gate, dtype)
    a.leaves = b.leaves   # the same leaves in an eager and in a captured step
    b.step()
    b.results()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for k in range(4):
        for n, t in b.leaves.items():
            if n in ("x", "residual"):
                t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(k)))
        b.step()
        want = b.results()
        for t in (*a.grads.values(), *a.wgrads.values(), a.d_x, a.d_res, a.y2, a.s2):
            t.zero_()
        graph.replay()
        got = a.results()
        assert all(torch.equal(got[n], want[n]) for n in want), (k, [n for n in want if not torch.equal(got[n], want[n])])
        assert float(torch.randn(1000, device="cuda").sum()) != 0   # the program's own eager work
