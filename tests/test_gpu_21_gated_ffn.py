"""Gated feed-forward network, both directions and with 8-bit operands, against 64 bits."""
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


def tensor(shape, seed, scale=1.0, dt=torch.float64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64, device="cuda") * scale).to(dt)


def weights(d, H, dt, seed=0):
    return {"Wg": tensor((d, H), seed + 1, d ** -0.5, dt), "Wu": tensor((d, H), seed + 2, d ** -0.5, dt),
            "Wd": tensor((H, d), seed + 3, H ** -0.5, dt)}


def space(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # (NaN wherever something is read that was not written)


def run(B, T, d, H, dt, backward=True, seed=0, addend=True):
    w = weights(d, H, dt, seed)
    x, add, dy, dadd = (tensor((T, d), seed + 10 + i, s, dt) for i, s in enumerate((1.0, 1.0, 1e-3, 1e-3)))
    if not addend:
        add = dadd = None
    cfg = B.make_gated_config(T, d, H, NAME[dt])
    got = {"y": torch.full((T, d), 7.0, dtype=dt, device="cuda")}
    B.slicemoe_gated_ffn(cfg, x, w, got["y"], space(B.slicemoe_gated_ffn_workspace_bytes(cfg)), addend=add)
    ref = R.gated(x, w, add, dt, dy if backward else None, dadd)
    if backward:
        got["d_x"] = torch.full((T, d), 7.0, dtype=dt, device="cuda")
        got.update({n: torch.full_like(t, 7.0) for n, t in w.items()})
        B.slicemoe_gated_ffn_backward(cfg, x, w, dy, got["d_x"], got, space(B.slicemoe_gated_ffn_backward_workspace_bytes(cfg)), addend=dadd)
    torch.cuda.synchronize()
    for n, (v, e) in ref.items():
        R.within(got[n], v, e, f"{n} at T={T} d={d} H={H} {dt}")
        # and over all elements: every rounding of the path at its largest, independent of one another
        off = float((got[n].double() - v).norm())
        assert off <= 3 * R.HALF[dt] * float(v.norm()) * (1 if dt == B16 else 8), n
    return got


# (T, d, H): one token and one value; ragged everything; whole tiles; each tile size; splits of the contraction
SMALL = [(1, 1, 1), (1, 8, 8), (1, 64, 64), (3, 5, 7), (31, 40, 33), (32, 64, 128), (33, 72, 200), (64, 128, 256), (64, 1000, 520),
         (65, 65, 65), (100, 257, 683), (128, 64, 64), (129, 136, 72), (257, 264, 1032), (300, 512, 96), (1000, 256, 683)]


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d,H", SMALL)
def test_small(B, T, d, H, dt):
    run(B, T, d, H, dt)


@pytest.mark.parametrize("T,d,H", [(4096, 512, 4096), (4099, 520, 4104), (3001, 4096, 2049)])
def test_large_tiles(B, T, d, H):
    run(B, T, d, H, B16)


@pytest.mark.parametrize("T,d,H,dt", [(130, 4096, 64, B16), (65, 2048, 100, B16), (513, 3000, 72, B16), (5, 4096, 128, B16), (300, 2705, 244, F32),
                                      (40, 1000, 33, F32), (1500, 8192, 130, B16)], ids=str)
def test_projections_in_shares(B, T, d, H, dt):
    """Few tiles and a long contraction: both projections, and the backward of the gate, from sums of shares."""
    run(B, T, d, H, dt)


def test_large_tiles_fp32(B):
    run(B, 2051, 300, 6500, F32)


def test_without_addends(B):
    run(B, 77, 96, 200, B16, addend=False)
    run(B, 300, 257, 200, F32, addend=False)


@pytest.mark.parametrize("T,d,H", [(1, 16, 1), (1, 128, 64), (5, 48, 33), (16, 4096, 200), (32, 256, 768), (33, 272, 100), (64, 1024, 2816),
                                   (65, 128, 130), (65, 8192, 64), (300, 4096, 100), (200, 400, 1000), (257, 2048, 96), (4100, 512, 2056)])
def test_eight_bits(B, T, d, H):
    cfg = B.make_gated_config(T, d, H, "bf16")
    w = weights(d, H, B16)
    w["Wg"][:, 0] = 0
    q = B.quantize_gated_weights(cfg, w)
    for n in ("Wg", "Wu"):   # one rounding to e4m3 of w / scale, scale = largest of the column / 448
        top = w[n].double().abs().amax(0).clamp_min(1e-30)
        R.within(q[n + "_scale"], top / 448, (top / 448) * (4 * R.U), n + "_scale")
        step = torch.maximum(2.0 ** -4 * w[n].double().abs(), 2.0 ** -10 * (top / 448)) * (1 + 2.0 ** -10)
        R.within((q[n].float().double() * q[n + "_scale"].double()[:, None]).t(), w[n].double(), step, n)
    x, add = tensor((T, d), 5, 1.0, B16), tensor((T, d), 6, 1.0, B16)
    ncfg = B.make_norm_config(T, d, 1e-5, "bf16")
    xq, xs = torch.empty((T, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, device="cuda")
    B.slicemoe_add_rmsnorm(ncfg, x, None, torch.ones(d, dtype=B16, device="cuda"), None, None, y_quantized=xq, y_scale=xs)
    for addend in (add, None):
        y = torch.full((T, d), 7.0, dtype=B16, device="cuda")
        B.slicemoe_gated_ffn_quantized(cfg, xq, xs, q, y, space(B.slicemoe_gated_ffn_quantized_workspace_bytes(cfg)), addend=addend)
        v, e = R.gated_quantized(xq, xs, q, addend)
        R.within(y, v, e, "y")
        assert float((y.double() - v).norm()) <= 3 * 2.0 ** -8 * float(v.norm())


# rows on either side of a tile of 32 and of the limit; contractions that end inside an eight, inside a share and at both; features that end
# inside a tile and inside four; shares that are empty
@pytest.mark.parametrize("T,d,H", [(1, 7, 129), (2, 4099, 130), (17, 129, 1000), (31, 8, 3), (32, 2048, 127), (33, 1003, 515), (64, 640, 4100),
                                   (200, 1003, 515), (255, 136, 33), (256, 640, 260), (257, 640, 260)])
def test_fp32_of_few_rows(B, T, d, H):
    run(B, T, d, H, F32, backward=False)
    run(B, T, d, H, F32, backward=False, seed=5, addend=False)


def test_fp32_of_few_rows_in_place_and_infinite(B):
    """y in the place of x; an infinity that meets only finite values stays one (nothing is taken apart into terms), next to a padded k."""
    T, d, H = 40, 131, 70
    cfg, w = B.make_gated_config(T, d, H, "f32"), weights(d, H, F32)
    x, ws = tensor((T, d), 9, 1.0, F32), space(B.slicemoe_gated_ffn_workspace_bytes(cfg))
    y = torch.empty_like(x)
    B.slicemoe_gated_ffn(cfg, x, w, y, ws)
    held = x.clone()
    B.slicemoe_gated_ffn(cfg, held, w, held, ws)
    assert torch.equal(held, y)
    w["Wg"][3, 5], w["Wd"][5] = float("inf"), 1.0       # gate 5 of row t is inf with the sign of x[t, 3]
    x[:, 3] = torch.where(torch.arange(T, device="cuda") % 2 == 0, 1.0, 0.5)
    w["Wu"][:, 5] = 0.0
    w["Wu"][3, 5] = 1.0                                  # up 5 is x[t, 3]: hidden 5 is inf, y is inf in all columns
    B.slicemoe_gated_ffn(cfg, x, w, y, ws)
    assert bool((y == float("inf")).all())


# the same for the backward pass, whose limit is 64 rows: contractions over d, over H and over the rows that end inside an eight; edges of the
# 32 and 128 outputs of a wavefront
@pytest.mark.parametrize("T,d,H", [(1, 7, 129), (2, 4099, 130), (9, 130, 131), (17, 129, 1000), (31, 8, 3), (32, 2048, 127), (33, 1003, 515),
                                   (63, 127, 640), (64, 640, 4100), (65, 640, 4100)])
def test_fp32_of_few_rows_backward(B, T, d, H):
    run(B, T, d, H, F32)
    run(B, T, d, H, F32, seed=5, addend=False)
