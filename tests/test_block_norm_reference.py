"""The backward formulas of the norms on both sides of a block against central differences of the forward one, in 64 bits."""
import pytest
import torch

import block_norm_reference as N


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_formulas_against_differences(gate, post):
    T, d, a, eps = 3, 7, 0.75, 1e-3
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    t = {"x": rnd(T, d), "residual": rnd(T, d), "pre": 1 + 0.3 * rnd(d), "post": 1 + 0.3 * rnd(d) if post else None,
         "gate": {"none": None, "channel": rnd(d), "token": rnd(T, d)}[gate]}
    dy, dsum = rnd(T, d), rnd(T, d)

    def loss(v):
        f = N.forward(v["x"], v["post"], v["gate"], v["residual"], v["pre"], a, eps, torch.float32)
        return float((f["y"][0] * dy).sum() + (f["sum"][0] * dsum).sum())

    f = N.forward(t["x"], t["post"], t["gate"], t["residual"], t["pre"], a, eps, torch.float32)
    got = N.backward(t["x"], t["post"], t["gate"], f["sum"][0], t["pre"], f["stats"][0], dy, dsum, a, torch.float32, gate == "token")
    h = 1e-5
    for name, v in t.items():
        if v is None:
            assert name in ("post", "gate") and "d_" + name not in got
            continue
        diff = torch.zeros_like(v)
        for i in range(v.numel()):
            ends = []
            for sign in (1, -1):
                w = v.clone()
                w.view(-1)[i] += sign * h
                ends.append(loss({**t, name: w}))
            diff.view(-1)[i] = (ends[0] - ends[1]) / (2 * h)
        # central differences: h^2 / 6 of the third derivative (below 1e3 here) and 2^-52 / h of the loss (below 1e2)
        assert float((got["d_" + name][0] - diff).abs().max()) < 1e3 * h * h + 1e2 * 2.0 ** -52 / h, name
