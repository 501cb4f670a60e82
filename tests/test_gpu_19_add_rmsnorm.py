"""RMS norm with the residual's addition, its e4m3 rows and its backward pass, against 64 bits."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
NAME = {B16: "bf16", F32: "f32"}


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rows(T, d, dt, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, d, generator=g, dtype=torch.float64) * scale).to(dt).cuda()


def forward(B, x, residual, w, eps, quantize=False, want_y=True, want_sum=True):
    T, d = x.shape
    cfg = B.make_norm_config(T, d, eps, NAME[x.dtype])
    s = torch.full_like(x, 7.0) if want_sum else None
    y = torch.full_like(x, 7.0) if want_y else None
    q = torch.zeros((T, d), dtype=torch.float8_e4m3fn, device="cuda") if quantize else None
    sc = torch.full((T,), 7.0, device="cuda") if quantize else None
    B.slicemoe_add_rmsnorm(cfg, x, residual, w, s, y, y_quantized=q, y_scale=sc)
    torch.cuda.synchronize()
    return s, y, q, sc


# widths: one value, ragged, each number of pieces per lane and of wavefronts per row, the largest
WIDTHS = [1, 3, 8, 33, 64, 257, 512, 768, 1000, 1023, 2048, 4096, 4100, 5000, 8192, 16383, 16384]


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(B, d, dt):
    for T in (1, 5, 67):
        x, r, w = rows(T, d, dt, 1), rows(T, d, dt, 2, 3.0), rows(1, d, dt, 3)[0].contiguous()
        for residual in (r, None):
            s, y, _, _ = forward(B, x, residual, w, 1e-5)
            rs, ry, bs, by = R.norm_forward(x, residual, w, 1e-5, dt)
            R.within(s, rs, bs, "sum")
            R.within(y, ry, by, "y")


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_eight_bits(B, d, dt):
    T = 37
    x, r, w = rows(T, d, dt, 1), rows(T, d, dt, 2, 3.0), rows(1, d, dt, 3)[0].contiguous()
    x[5] = 0
    r[5] = 0
    s, y, q, sc = forward(B, x, r, w, 1e-5, quantize=True)
    _, ry, _, by = R.norm_forward(x, r, w, 1e-5, F32)
    top = ry.abs().amax(1).clamp_min(1e-30)
    R.within(sc, top / 448, (top / 448) * (98 * R.U), "scale")
    # one rounding to e4m3: half a step, 2^-4 of the value, or 2^-10 (half the smallest value) near zero
    step = torch.maximum(2.0 ** -4 * ry.abs(), 2.0 ** -10 * (top / 448)[:, None])
    R.within(q.float().double() * sc.double()[:, None], ry, step * (1 + 2.0 ** -10) + by, "values")
    assert float(q.float().abs().max()) <= 448 and bool((q[5].float() == 0).all()) and float(sc[5]) > 0
    again = forward(B, x, r, w, 1e-5, quantize=True, want_y=False, want_sum=False)
    assert torch.equal(again[2].view(torch.uint8), q.view(torch.uint8)) and torch.equal(again[3], sc)
    assert torch.equal(forward(B, x, r, w, 1e-5)[1], y)   # the same rows with and without them


def test_eight_bits_of_tiny_and_nonfinite_rows(B):
    d = 512
    x = rows(6, d, F32, 4)
    w = torch.ones(d, device="cuda")
    x[0] *= 1e-38
    x[1] = 0
    x[1, 3] = 1e-20
    x[2, 7] = float("nan")
    x[3, 7] = float("inf")
    x[4, 100] = -float("inf")
    _, y, q, sc = forward(B, x, None, w, 0.0, quantize=True)
    assert bool(torch.isfinite(y[5]).all()) and float(sc[5]) > 0
    assert bool(torch.isnan(sc[2:5]).all())                 # a row with a NaN or an infinity
    assert bool(torch.isfinite(y[1]).all() | torch.isnan(y[1]).any())
    s, y, q, sc = forward(B, x, None, w, 1e-5, quantize=True)
    assert bool(torch.isfinite(y[:2]).all()) and bool(torch.isfinite(sc[:2]).all()) and bool((sc[:2] > 0).all())


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward(B, d, dt):
    for T in (1, 6, 131):
        s, w, dy, ds = rows(T, d, dt, 1, 2.0), rows(1, d, dt, 2)[0].contiguous(), rows(T, d, dt, 3, 1e-3), rows(T, d, dt, 4, 1e-3)
        cfg = B.make_norm_config(T, d, 1e-5, NAME[dt])
        ws = torch.full((B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
        for dsum in (ds, None):
            dx, dw = torch.full_like(s, 7.0), torch.full((d,), 7.0, device="cuda")
            B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws, d_sum=dsum)
            rx, rw, bx, bw = R.norm_backward(s, w, dy, dsum, 1e-5, dt)
            R.within(dx, rx, bx, "d_x")
            R.within(dw, rw, bw, "d_weight")


@pytest.mark.parametrize("T,d,dt", [(9001, 768, B16), (20011, 96, F32), (4097, 4096, B16)])
def test_backward_of_many_rows_is_reproducible(B, T, d, dt):
    s, w, dy = rows(T, d, dt, 1, 2.0), rows(1, d, dt, 2)[0].contiguous(), rows(T, d, dt, 3)
    cfg = B.make_norm_config(T, d, 1e-6, NAME[dt])
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(3):
        dx, dw = torch.empty_like(s), torch.empty(d, device="cuda")
        ws.fill_(255)
        B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws)
        if first is None:
            first = (dx, dw)
            rx, rw, bx, bw = R.norm_backward(s, w, dy, None, 1e-6, dt)
            R.within(dx, rx, bx, "d_x")
            R.within(dw, rw, bw, "d_weight")
        assert torch.equal(dx, first[0]) and torch.equal(dw, first[1])


def test_backward_against_differences(B):
    """d/dv of sum(dy * y(s + v)) along random directions, by central differences of the 64-bit formula at the stored sum."""
    T, d = 4, 40
    s, w, dy = rows(T, d, F32, 1), rows(1, d, F32, 2)[0].contiguous(), rows(T, d, F32, 3)
    cfg = B.make_norm_config(T, d, 1e-5, "f32")
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(s), torch.empty(d, device="cuda")
    B.slicemoe_add_rmsnorm_backward(cfg, s, w, dy, dx, dw, ws)

    def loss(s, w):
        return (dy.double() * s * w / (s.square().mean(1, keepdim=True) + 1e-5).sqrt()).sum()

    for seed in range(5):
        v, u = rows(T, d, F32, 10 + seed).double(), rows(1, d, F32, 20 + seed)[0].double()
        h = 1e-5
        num = (loss(s.double() + h * v, w.double()) - loss(s.double() - h * v, w.double())) / (2 * h)
        # differences: third derivatives times h^2 (below 1e-8 here); fp32 gradients: 128 roundings
        assert abs(float(num - (dx.double() * v).sum())) <= 1e-4 * float((dx.double() * v).abs().sum())
        num = (loss(s.double(), w.double() + h * u) - loss(s.double(), w.double() - h * u)) / (2 * h)
        assert abs(float(num - (dw.double() * u).sum())) <= 1e-4 * float((dw.double() * u).abs().sum())


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
def test_outputs_in_place_of_inputs(B, dt):
    T, d = 77, 1000
    x, r, w = rows(T, d, dt, 1), rows(T, d, dt, 2), rows(1, d, dt, 3)[0].contiguous()
    s0, y0, _, _ = forward(B, x, r, w, 1e-5)
    cfg = B.make_norm_config(T, d, 1e-5, NAME[dt])
    a, b = x.clone(), r.clone()
    B.slicemoe_add_rmsnorm(cfg, a, b, w, b, a)   # sum over the residual, y over x
    assert torch.equal(b, s0) and torch.equal(a, y0)
    dy, ds = rows(T, d, dt, 5), rows(T, d, dt, 6)
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dw0, dw1, dx0 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty_like(x)
    B.slicemoe_add_rmsnorm_backward(cfg, s0, w, dy, dx0, dw0, ws, d_sum=ds)
    for other in ("dy", "dsum"):
        g, e = dy.clone(), ds.clone()
        B.slicemoe_add_rmsnorm_backward(cfg, s0, w, g, g if other == "dy" else e, dw1, ws, d_sum=e)
        assert torch.equal(g if other == "dy" else e, dx0) and torch.equal(dw0, dw1)


def test_no_rows(B):
    d = 100
    e = torch.empty((0, d), dtype=B16, device="cuda")
    w = torch.ones(d, dtype=B16, device="cuda")
    cfg = B.make_norm_config(0, d, 1e-5, "bf16")
    B.slicemoe_add_rmsnorm(cfg, e, e, w, e, e)
    dw = torch.full((d,), 7.0, device="cuda")
    ws = torch.empty(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    B.slicemoe_add_rmsnorm_backward(cfg, e, w, e, e, dw, ws)
    assert bool((dw == 0).all())


def test_rows_behind_the_last_are_left_alone(B):
    T, d = 9, 257
    x, w = rows(T + 4, d, B16, 1), rows(1, d, B16, 3)[0].contiguous()
    s, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    B.slicemoe_add_rmsnorm(B.make_norm_config(T, d, 1e-5, "bf16"), x, x, w, s, y)
    assert bool((s[T:] == 7).all()) and bool((y[T:] == 7).all()) and not bool((y[:T] == 7).all())


def test_more_rows_than_one_launch_holds(B):
    """A wavefront per row: 2^26 rows are 2^32 threads.  Rows of one value against the formula in 64 bits, all of them."""
    T, eps = (1 << 26) + 5, 0.25
    cfg = B.make_norm_config(T, 1, eps, "bf16")
    x = torch.empty((T, 1), dtype=B16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    w = torch.full((1,), 1.5, dtype=B16, device="cuda")
    y, s = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    q, sc = torch.zeros((T, 1), dtype=torch.uint8, device="cuda"), torch.full((T,), 7.0, device="cuda")
    B.slicemoe_add_rmsnorm(cfg, x, None, w, s, y)
    B.slicemoe_add_rmsnorm(cfg, x, x, w, None, None, y_quantized=q, y_scale=sc)
    torch.cuda.synchronize()
    assert torch.equal(s, x)
    for a in range(0, T, 1 << 24):
        rows = slice(a, min(T, a + (1 << 24)))
        v = x[rows].double()
        ref = v / (v * v + eps).sqrt() * 1.5
        # storage, and some ten fp32 roundings
        assert bool(((y[rows].double() - ref).abs() <= ref.abs() * (2.0 ** -8 + 10 * 2.0 ** -24)).all())
        ref = 2 * v / (4 * v * v + eps).sqrt() * 1.5
        got = q[rows].view(torch.float8_e4m3fn).float().double() * sc[rows, None].double()
        # its own largest value: 448 of its scale but for fp32 roundings, which may bring the quotient no further than the neighbour's half step
        assert bool(((got - ref).abs() <= ref.abs() * (2.0 ** -4 + 16 * 2.0 ** -24)).all())
