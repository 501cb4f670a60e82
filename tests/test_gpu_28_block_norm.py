"""Norms on both sides of a block's addition to the residual stream, both directions, against 64 bits."""
import pytest
import torch

import block_norm_reference as N
import block_reference as R
import mx_reference as M

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


def inputs(T, d, dt, gate, post=True):
    x, res = rows(T, d, dt, 1, 0.3), rows(T, d, dt, 2, 3.0)
    vec = lambda seed: (1 + 0.3 * rows(1, d, F32, seed)[0]).to(dt).contiguous()  # noqa: E731
    return {"x": x, "post": vec(3) if post else None, "gate": {None: None, "channel": vec(4), "token": rows(T, d, dt, 5)}[gate], "residual": res, "pre": vec(6)}


def forward(B, t, gate, a, eps, want_y=True, want_stats=True, bits=0, pre=True):
    T, d = t["x"].shape
    cfg = B.make_block_norm_config(T, d, eps, a, gate, t["x"].dtype)
    s = torch.full_like(t["x"], 7.0)
    y = torch.full_like(s, 7.0) if want_y else None
    stats = torch.full((T, 2), 7.0, device="cuda") if want_stats else None
    mx = torch.full((B.slicemoe_mx_bytes(B.make_mx_config(T, d, bits)),), 0xA5, dtype=torch.uint8, device="cuda") if bits else None
    B.slicemoe_block_norm(cfg, t["x"], t["post"], t["gate"], t["residual"], t["pre"] if pre else None, s, y, y_mx=mx, y_bits=bits, stats=stats)
    return cfg, s, y, stats, mx


def backward(B, cfg, t, s, stats, dy, dsum):
    T, d = s.shape
    token = cfg.gate == B.SLICEMOE_GATE_TOKEN
    out = {"d_x": torch.full_like(s, 7.0), "d_residual": torch.full_like(s, 7.0), "d_pre": torch.full((d,), 7.0, device="cuda")}
    if t["post"] is not None:
        out["d_post"] = torch.full((d,), 7.0, device="cuda")
    if t["gate"] is not None:
        out["d_gate"] = torch.full_like(s, 7.0) if token else torch.full((d,), 7.0, device="cuda")
    ws = torch.full((max(256, B.slicemoe_block_norm_backward_workspace_bytes(cfg)),), 0xFF, dtype=torch.uint8, device="cuda")
    B.slicemoe_block_norm_backward(cfg, t["x"], t["post"], t["gate"], s, t["pre"], stats, dy, out["d_x"], out["d_residual"], out.get("d_post"),
                                   out.get("d_gate"), out["d_pre"], ws, d_sum=dsum)
    return out


# one value, ragged, each number of pieces per lane and of wavefronts per row, the largest
WIDTHS = [1, 3, 8, 33, 64, 257, 512, 768, 1000, 1023, 2048, 4096, 4100, 5000, 8192, 16383, 16384]


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_both_directions(B, d, dt):
    for T, gate, post, a in ((1, "channel", True, 1.0), (5, "token", True, 0.5), (67, "channel", True, -1.25), (6, None, False, 1.0), (9, "token", False, 2.0)):
        t = inputs(T, d, dt, gate, post)
        cfg, s, y, stats, _ = forward(B, t, gate, a, 1e-5)
        ref = N.forward(t["x"], t["post"], t["gate"], t["residual"], t["pre"], a, 1e-5, dt)
        for name, got in (("sum", s), ("y", y), ("stats", stats)):
            R.within(got, *ref[name], f"{name} {T} {gate} {post}")
        if not post:
            assert bool((stats[:, 0] == 1).all())
        dy = rows(T, d, dt, 8, 0.1)
        for dsum in (rows(T, d, dt, 9, 0.1), None):
            out = backward(B, cfg, t, s, stats, dy, dsum)
            ref = N.backward(t["x"], t["post"], t["gate"], s, t["pre"], stats, dy, dsum, a, dt, gate == "token")
            assert set(out) == set(ref)
            for name in ref:
                R.within(out[name], *ref[name], f"{name} {T} {gate} {post}")
            again = backward(B, cfg, t, s, stats, dy, dsum)
            assert all(torch.equal(again[n], out[n]) for n in out)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(3001, 513), (5000, 768), (2049, 4096)])
def test_many_rows(B, T, d, dt):
    """More rows than resident blocks: column sums over many of them."""
    for gate in ("channel", "token"):
        t = inputs(T, d, dt, gate)
        cfg, s, y, stats, _ = forward(B, t, gate, 0.5, 1e-5)
        ref = N.forward(t["x"], t["post"], t["gate"], t["residual"], t["pre"], 0.5, 1e-5, dt)
        R.within(s, *ref["sum"], "sum")
        R.within(y, *ref["y"], "y")
        dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 0.1)
        out = backward(B, cfg, t, s, stats, dy, dsum)
        for name, r in N.backward(t["x"], t["post"], t["gate"], s, t["pre"], stats, dy, dsum, 0.5, dt, gate == "token").items():
            R.within(out[name], *r, name)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 33, 64, 255, 256, 257, 768, 1000, 2048, 4096, 4100, 8192, 16384])
def test_microscaled_rows(B, d, dt, bits):
    T = 37
    t = inputs(T, d, dt, "channel")
    cfg, s, y, stats, mx = forward(B, t, "channel", 0.5, 1e-5, bits=bits)
    _, s2, _, _, mx2 = forward(B, t, "channel", 0.5, 1e-5, bits=bits, want_y=False, want_stats=False)
    mc = B.make_mx_config(T, d, bits, "f32")
    got = torch.empty((T, d), device="cuda")
    B.slicemoe_mx_dequantize(mc, mx, got)
    ref = N.forward(t["x"], t["post"], t["gate"], t["residual"], t["pre"], 0.5, 1e-5, dt)["y32"]
    want, bound = M.to_mx_within(*ref, bits)
    R.within(got, want, bound, "values")
    plain = forward(B, t, "channel", 0.5, 1e-5)
    assert torch.equal(plain[1], s) and torch.equal(plain[2], y) and torch.equal(s2, s) and torch.equal(mx2, mx)   # with and without them
    if dt == F32:   # of the fp32 row: the conversion of y gives the same bytes in the rows that there are
        other = torch.full_like(mx, 0xA5)
        B.slicemoe_mx_quantize(mc, y, other)
        a, b = torch.empty_like(y), torch.empty_like(y)
        B.slicemoe_mx_dequantize(mc, other, a)
        assert torch.equal(a, got)
        # what is past the last row stays as it was; what is past the last column is zero
        wide = B.make_mx_config(64, -(-d // 256) * 256, bits, "f32")
        b = torch.empty((64, wide.cols), device="cuda")
        B.slicemoe_mx_dequantize(wide, mx, b)
        assert bool((b[:T, d:] == 0).all())
        tiles = mx.numel() // (1024 * bits + 256)
        left = mx[:tiles * 1024 * bits].view(2, -1, 4, 64 * bits // 4, 16)[1]    # the second row of tiles: rows 32 .. 36 are there
        lane = torch.arange(64 * bits // 4, device="cuda") % 32
        assert bool((left[:, :, lane >= T - 32] == 0xA5).all())


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 100, 768, 4096, 16384])
def test_rows_out_of_range(B, d, dt):
    """Rows whose squares leave fp32, before either norm."""
    T = 12
    t = inputs(T, d, dt, "channel")
    big, small = 2.0 ** 100, 2.0 ** -100
    for r, (fx, fr) in enumerate([(big, 1), (small, 1), (1, big), (1, small), (big, big), (small, small), (2.0 ** 120, 0), (2.0 ** -120, 2.0 ** 110)]):
        t["x"][r], t["residual"][r] = (t["x"][r].double() * fx).to(dt), (t["residual"][r].double() * fr).to(dt)
    for eps in (1e-5, 0.0):
        cfg, s, y, stats, _ = forward(B, t, "channel", 0.5, eps)
        ref = N.forward(t["x"], t["post"], t["gate"], t["residual"], t["pre"], 0.5, eps, dt)
        for name, got in (("sum", s), ("y", y), ("stats", stats)):
            R.within(got, *ref[name], name)
        dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 0.1)
        keep = [0, 2, 8, 9, 10, 11] if eps == 0 else list(range(T))    # the others' gradients may leave fp32 with r near 2^100
        u = {k: (v[keep].contiguous() if v is not None and v.dim() == 2 else v) for k, v in t.items()}
        kc = B.make_block_norm_config(len(keep), d, eps, 0.5, "channel", dt)
        args = (s[keep].contiguous(), stats[keep].contiguous(), dy[keep].contiguous(), dsum[keep].contiguous())
        out = backward(B, kc, u, *args)
        ref = N.backward(u["x"], u["post"], u["gate"], args[0], u["pre"], args[1], args[2], args[3], 0.5, dt, False)
        for name in ref:
            R.within(out[name], *ref[name], name)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
def test_rows_that_are_not_finite_stay_apart(B, dt):
    T, d = 9, 300
    t = inputs(T, d, dt, "token")
    _, s0, y0, st0, mx0 = forward(B, t, "token", 1.0, 1e-5, bits=8)
    t["x"][2, 5], t["residual"][4, 7], t["gate"][6, 9] = float("nan"), float("inf"), float("nan")
    cfg, s, y, st, mx = forward(B, t, "token", 1.0, 1e-5, bits=8)
    good = [0, 1, 3, 5, 7, 8]
    assert torch.equal(s[good], s0[good]) and torch.equal(y[good], y0[good]) and torch.equal(st[good], st0[good])
    assert bool(s[2].isnan().all()) and bool(y[2].isnan().all()) and bool(y[4].isnan().any()) and bool(s[6, 9].isnan()) and bool(y[6].isnan().all())
    a = torch.empty((T, d), device="cuda")
    B.slicemoe_mx_dequantize(B.make_mx_config(T, d, 8, "f32"), mx, a)
    assert bool(a[2].isnan().all()) and bool(a[6].isnan().all()) and bool(a[good].isfinite().all())
    dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 0.1)
    out = backward(B, cfg, t, s, st, dy, dsum)
    assert all(bool(out[n][good].isfinite().all()) for n in ("d_x", "d_residual", "d_gate"))


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 257, 768, 4096, 8192])
def test_in_place(B, d, dt):
    T = 70
    t = inputs(T, d, dt, "token")
    cfg, s, y, stats, _ = forward(B, t, "token", 0.5, 1e-5)
    for target in ("x", "residual"):
        u = dict(t, x=t["x"].clone(), residual=t["residual"].clone())
        other = "residual" if target == "x" else "x"
        B.slicemoe_block_norm(cfg, u["x"], u["post"], u["gate"], u["residual"], u["pre"], u[target], u[other])
        assert torch.equal(u[target], s) and torch.equal(u[other], y)
    dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 0.1)
    want = backward(B, cfg, t, s, stats, dy, dsum)
    ws = torch.empty(B.slicemoe_block_norm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    for swap in (False, True):
        g, h = dy.clone(), dsum.clone()
        o = {n: torch.empty_like(v) for n, v in want.items()}
        o["d_x"], o["d_residual"] = (h, g) if swap else (g, h)
        B.slicemoe_block_norm_backward(cfg, t["x"], t["post"], t["gate"], s, t["pre"], stats, g, o["d_x"], o["d_residual"], o["d_post"], o["d_gate"], o["d_pre"],
                                       ws, d_sum=h)
        assert all(torch.equal(o[n], want[n]) for n in want)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [513, 1025, 1537, 2049, 4097, 5001, 8193, 16383])
def test_in_place_without_a_norm_behind(B, d, dt):
    """Rows whose last piece belongs to two wavefronts, with no sum over the row in front of the stores."""
    T = 1031
    t = inputs(T, d, dt, "channel", post=False)
    cfg, s, y, stats, _ = forward(B, t, "channel", 0.5, 1e-5)
    for target in ("x", "residual"):
        u = dict(t, x=t["x"].clone(), residual=t["residual"].clone())
        out = torch.empty_like(s)
        B.slicemoe_block_norm(cfg, u["x"], None, u["gate"], u["residual"], u["pre"], u[target], out)
        assert torch.equal(u[target], s) and torch.equal(out, y)


def test_sum_alone_and_no_rows(B):
    t = inputs(5, 300, B16, "channel")
    _, s, *_ = forward(B, t, "channel", 0.5, 1e-5)
    _, alone, *_ = forward(B, t, "channel", 0.5, 1e-5, want_y=False, pre=False)
    assert torch.equal(alone, s)
    t = inputs(0, 300, B16, "channel")
    cfg, s, y, stats, _ = forward(B, t, "channel", 0.5, 1e-5, bits=4)
    out = backward(B, cfg, t, s, stats, y, None)
    assert all(bool((out[n] == 0).all()) for n in ("d_pre", "d_post", "d_gate"))


def test_offsets_beyond_32_bits(B):
    """A batch of more than 2^32 bytes and 2^31 elements: its last rows are those of a small batch."""
    T, d, last = 150001, 16384, 40
    free, _ = torch.cuda.mem_get_info()
    if free < 40 * 2 ** 30:
        pytest.skip("needs 40 GiB")
    t = inputs(last, d, B16, "channel")
    cfg, s, y, stats, _ = forward(B, t, "channel", 0.5, 1e-5)
    x, res = (torch.zeros((T, d), dtype=B16, device="cuda") for _ in range(2))
    x[-last:], res[-last:] = t["x"], t["residual"]
    x[:-last, 0] = 1
    big = dict(t, x=x, residual=res)
    bc = B.make_block_norm_config(T, d, 1e-5, 0.5, "channel")
    bs, by = torch.empty_like(x), res                       # y in place of the residual
    st = torch.empty((T, 2), device="cuda")
    B.slicemoe_block_norm(bc, big["x"], t["post"], t["gate"], res, t["pre"], bs, by, stats=st)
    assert torch.equal(bs[-last:], s) and torch.equal(by[-last:], y) and torch.equal(st[-last:], stats)


# rows whose last piece belongs to two wavefronts, four or sixteen of them a row
SHARED_PIECE = [513, 1025, 1537, 2049, 4097, 5001, 8193, 16383]


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", SHARED_PIECE)
def test_in_place_of_rows_with_a_shared_piece(B, d, dt):
    """The sum, and y, in the place of the block's output and of the stream: no wavefront's rows are overwritten before it has them."""
    T = 1031
    for gate, post in (("channel", True), ("token", True), (None, False)):
        t = inputs(T, d, dt, gate, post)
        t["x"][::5], t["residual"][::3] = t["x"][::5] * 2.0 ** 70, t["residual"][::3] * 2.0 ** 70      # (some out of the squares' range)
        cfg, s, y, stats, _ = forward(B, t, gate, 0.5, 1e-5)
        for target, other in (("x", "residual"), ("residual", "x")):
            for y_target in (other, None):
                u = dict(t, x=t["x"].clone(), residual=t["residual"].clone())
                out = u[y_target] if y_target else torch.empty_like(s)
                st = torch.empty_like(stats)
                B.slicemoe_block_norm(cfg, u["x"], u["post"], u["gate"], u["residual"], u["pre"], u[target], out, stats=st)
                assert torch.equal(u[target], s) and torch.equal(out, y) and torch.equal(st, stats)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", SHARED_PIECE)
def test_backward_in_place_of_rows_with_a_shared_piece(B, d, dt):
    """The gradients in the place of those that arrive, either way round and each alone."""
    T = 1031
    for gate, post in (("channel", True), ("token", True), (None, False)):
        t = inputs(T, d, dt, gate, post)
        cfg, s, y, stats, _ = forward(B, t, gate, 0.5, 1e-5)
        dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 0.1)
        want = backward(B, cfg, t, s, stats, dy, dsum)
        ws = torch.empty(B.slicemoe_block_norm_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        for dx_at, dr_at in (("dy", "dsum"), ("dsum", "dy"), (None, "dsum"), ("dsum", None), (None, "dy"), ("dy", None)):
            g = {"dy": dy.clone(), "dsum": dsum.clone()}
            o = {n: torch.empty_like(v) for n, v in want.items()}
            o["d_x"], o["d_residual"] = g.get(dx_at, o["d_x"]), g.get(dr_at, o["d_residual"])
            B.slicemoe_block_norm_backward(cfg, t["x"], t["post"], t["gate"], s, t["pre"], stats, g["dy"], o["d_x"], o["d_residual"], o.get("d_post"),
                                           o.get("d_gate"), o["d_pre"], ws, d_sum=g["dsum"])
            assert all(torch.equal(o[n], want[n]) for n in want), (gate, dx_at, dr_at)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [100, 1000, 5000])
def test_gradients_without_a_norm_behind_of_large_values(B, d, dt):
    """d_x is then d_s times the gate, whatever the block's output: the sum of d_s x, which leaves fp32 here, has no part in it."""
    T = 9
    for gate in (None, "token"):
        t = inputs(T, d, dt, gate, post=False)
        t["x"][::2] = t["x"][::2] * 2.0 ** 100
        cfg, s, y, stats, _ = forward(B, t, gate, 0.5, 1e-5)
        dy, dsum = rows(T, d, dt, 8, 0.1), rows(T, d, dt, 9, 2.0 ** 40)
        out = backward(B, cfg, t, s, stats, dy, dsum)
        ref = N.backward(t["x"], None, t["gate"], s, t["pre"], stats, dy, dsum, 0.5, dt, gate == "token")
        for name in ("d_x", "d_residual"):
            assert bool(out[name].isfinite().all())
            R.within(out[name], *ref[name], f"{name} {gate}")
