"""RMS norm of rows whose squares leave the range of fp32 on either side, forward, e4m3 and backward, against 64 bits: every finite
row has the norm of the formula, whatever its size."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
NAME = {B16: "bf16", F32: "f32"}
# subnormal values, squares below the smallest number, either side of the smallest mean that is squared as it is (2^-60: 9e-10), ordinary
# ones, either side of the largest square, the largest values
SCALES = [3e-39, 1e-37, 1e-30, 1e-22, 1e-15, 5e-10, 9.4e-10, 2e-9, 1e-4, 1.0, 1e10, 1e17, 1e18, 1e19, 5e19, 1e22, 1e30, 5e37]


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def scaled_rows(T, d, dt, seed=0, off=0):
    """Row t at the scale t + off of the list, and in every third row a single value 1e6 times the others (where the type has it)."""
    g = torch.Generator().manual_seed(seed)
    scale = torch.tensor([SCALES[(t + off) % len(SCALES)] for t in range(T)], dtype=torch.float64)[:, None]
    v = torch.randn(T, d, generator=g, dtype=torch.float64).clamp(-4, 4)
    v = torch.where(v.abs() < 0.05, 0.05, v) * scale
    if d > 3:
        v[::3, 3] = (v[::3, 3] * 1e6).clamp(-3e38, 3e38)
    return v.to(dt).cuda()


def plain_rows(T, d, dt, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, d, generator=g, dtype=torch.float64) * scale).to(dt).cuda()


# every number of pieces per lane and of wavefronts per row, aligned and not
WIDTHS = [1, 7, 64, 257, 768, 1000, 2048, 2051, 4096, 8192, 8201, 16384]


@pytest.mark.parametrize("eps", [0.0, 1e-5, 1e-25, 1e30, 3e38])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(B, d, dt, eps):
    T = 3 * len(SCALES) + 1
    x, r, w = scaled_rows(T, d, dt, 1), scaled_rows(T, d, dt, 2) * 0.25, plain_rows(1, d, dt, 3)[0].contiguous()
    cfg = B.make_norm_config(T, d, eps, NAME[dt])
    for residual in (r, None):
        s, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        q, sc = torch.zeros((T, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.full((T,), 7.0, device="cuda")
        B.slicemoe_add_rmsnorm(cfg, x, residual, w, s, y, y_quantized=q, y_scale=sc)
        rs, ry, bs, by = R.norm_forward(x, residual, w, float(torch.tensor(eps, dtype=F32)), dt)
        R.within(s, rs, bs, "sum")
        R.within(y, ry, by, "y")
        by = ry.abs() * (R.HALF[F32] + 96 * R.U)
        top = ry.abs().amax(1).clamp_min(1e-30)
        R.within(sc, top / 448, (top / 448) * (98 * R.U), "scale")
        step = torch.maximum(2.0 ** -4 * ry.abs(), 2.0 ** -10 * (top / 448)[:, None])
        R.within(q.float().double() * sc.double()[:, None], ry, step * (1 + 2.0 ** -10) + by, "values")


@pytest.mark.parametrize("eps", [0.0, 1e-5, 1e30])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward(B, d, dt, eps):
    """More rows than blocks: rows of every kind follow one another in a block, in either place of its two exchanges."""
    T = 4 * 768 * 2 + 77 if d <= 1024 else 768 * 2 + 77
    s, w = scaled_rows(T, d, dt, 1), plain_rows(1, d, dt, 2)[0].contiguous()
    cfg = B.make_norm_config(T, d, eps, NAME[dt])
    ws = torch.full((B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
    dy, ds = plain_rows(T, d, dt, 3, 1e-6), plain_rows(T, d, dt, 4, 1e-6)
    for dsum in (ds, None):
        dx, dw = torch.full_like(s, 7.0), torch.full((d,), 7.0, device="cuda")
        B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws, d_sum=dsum)
        rx, rw, bx, bw = R.norm_backward(s, w, dy, dsum, float(torch.tensor(eps, dtype=F32)), dt)
        R.within(dx, rx, bx, "d_x")
        R.within(dw, rw, bw, "d_weight")


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [257, 768, 2048, 8192, 16384])
def test_backward_in_place(B, d, dt):
    """d_x in the place of d_y or of d_sum, rows of every kind next to one another."""
    T = 4 * 768 + 77 if d <= 1024 else 768 * 2 + 77
    s, w = scaled_rows(T, d, dt, 1, off=5), plain_rows(1, d, dt, 2)[0].contiguous()
    cfg = B.make_norm_config(T, d, 0.0, NAME[dt])
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dy, ds = plain_rows(T, d, dt, 3, 1e-6), plain_rows(T, d, dt, 4, 1e-6)
    dx, dw = torch.full_like(s, 7.0), torch.empty(d, device="cuda")
    B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws, d_sum=ds)
    for other in ("dy", "dsum"):
        g, e, dw1 = dy.clone(), ds.clone(), torch.empty(d, device="cuda")
        to = g if other == "dy" else e
        B.slicemoe_add_rmsnorm_backward(cfg, s, w, g, to, dw1, ws, d_sum=e)
        assert torch.equal(to, dx) and torch.equal(dw, dw1)


def test_large_gradients_of_large_rows(B):
    """dy w s leaves the range where neither s^2 nor the result does."""
    T, d = 9, 512
    s, w, dy = plain_rows(T, d, F32, 1, 1e16), plain_rows(1, d, F32, 2)[0].contiguous(), plain_rows(T, d, F32, 3, 1e25)
    cfg = B.make_norm_config(T, d, 1e-5, "f32")
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(s), torch.empty(d, device="cuda")
    B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws)
    rx, rw, bx, bw = R.norm_backward(s, w, dy, None, 1e-5, F32)
    R.within(dx, rx, bx, "d_x")
    R.within(dw, rw, bw, "d_weight")


def test_rows_that_are_not_finite(B):
    """An infinity or a NaN spoils its own row (its scale is NaN), and the gradient of the weight."""
    for d in (512, 4096):
        x, w = plain_rows(1600, d, F32, 1), torch.ones(d, device="cuda")
        bad = {2: float("nan"), 3: float("inf"), 900: -float("inf")}
        for t, v in bad.items():
            x[t, 7] = v
        cfg = B.make_norm_config(1600, d, 0.0, "f32")
        y, q, sc = torch.empty_like(x), torch.zeros((1600, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1600, device="cuda")
        B.slicemoe_add_rmsnorm(cfg, x, None, w, None, y, y_quantized=q, y_scale=sc)
        ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
        B.slicemoe_add_rmsnorm_backward(cfg, x, w, y, dx, dw, ws)
        rows = torch.tensor(sorted(bad), device="cuda")
        fine = torch.ones(1600, dtype=torch.bool, device="cuda")
        fine[rows] = False
        assert bool(torch.isnan(sc[rows]).all()) and bool(torch.isnan(y[rows, 7]).all()) and bool(torch.isnan(dx[rows, 7]).all()) and bool(torch.isnan(dw[7]))
        _, ry, _, by = R.norm_forward(x[fine], None, w, 0.0, F32)
        R.within(y[fine], ry, by, "y")
        assert bool(torch.isfinite(sc[fine]).all()) and bool(torch.isfinite(dx[fine]).all())
