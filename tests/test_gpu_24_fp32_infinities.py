"""Infinities in the fp32 gated network: infinite, of which sign, or NaN exactly where IEEE arithmetic says, whichever kernel the number
of rows takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, INF = torch.float32, float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def data(T, d, H, exact):
    """exact: values that bf16 holds, whose lower terms are zero."""
    g = torch.Generator().manual_seed(T + d + H)

    def normal(*size):
        v = torch.randn(size, generator=g)
        v = torch.where(v.abs() < 2.0 ** -6, 2.0 ** -6, v)
        return (v.bfloat16().float() if exact else v).cuda()

    return normal(T, d), {"Wg": normal(d, H) * 0.125, "Wu": normal(d, H) * 0.125, "Wd": normal(H, d) * 0.125}, normal(T, d)


def product(a, b):
    """In 64 bits, term by term: no library's way with zeros and infinities."""
    a, b = a.double(), b.double()
    return torch.cat([(a[i:i + 16, :, None] * b[None]).sum(1) for i in range(0, a.shape[0], 16)])


def reference(x, w, dy):
    g, u = product(x, w["Wg"]), product(x, w["Wu"])
    sg = 1 / (1 + torch.exp(-g))
    s = g * sg
    a = s * u
    da = product(dy, w["Wd"].t())
    dg, du = da * u * (sg + s * (1 - sg)), da * s
    return {"y": product(a, w["Wd"]), "d_x": product(dg, w["Wg"].t()) + product(du, w["Wu"].t()), "Wg": product(x.t(), dg),
            "Wu": product(x.t(), du), "Wd": product(a.t(), dy)}


def same_kind(got, ref, name):
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        a, b = kind(got), kind(ref)
        assert torch.equal(a, b), f"{name}: {kind.__name__} at {int((a != b).sum())} of {a.numel()}, first {int((a != b).flatten().int().argmax())}"


def run(B, x, w, dy, backward):
    (T, d), H = x.shape, w["Wg"].shape[1]
    cfg = B.make_gated_config(T, d, H, "f32")
    out = {"y": torch.full_like(x, 7.0)}
    B.slicemoe_gated_ffn(cfg, x, w, out["y"], torch.empty(B.slicemoe_gated_ffn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"))
    if backward:
        out["d_x"] = torch.full_like(x, 7.0)
        out.update({n: torch.full_like(t, 7.0) for n, t in w.items()})
        B.slicemoe_gated_ffn_backward(cfg, x, w, dy, out["d_x"], out, torch.empty(B.slicemoe_gated_ffn_backward_workspace_bytes(cfg), dtype=torch.uint8,
                                                                                  device="cuda"))
    torch.cuda.synchronize()
    return out


def plant(place, x, w, dy):
    if place == "x":
        x[5, 3], x[x.shape[0] - 1, x.shape[1] - 1] = INF, -INF
    elif place == "dy":
        dy[5, 3], dy[dy.shape[0] - 2, 0] = -INF, INF
    elif place == "all x":
        x.fill_(INF)
    else:
        w[place][2, 1], w[place][-1, -1] = INF, -INF


# rows on either side of the limits of the fp32 instruction; widths that end inside a tile and inside eight; a long contraction in shares
@pytest.mark.parametrize("exact", [True, False], ids=["bf16 values", "any values"])
@pytest.mark.parametrize("place", ["x", "Wg", "Wu", "Wd", "dy", "all x"])
@pytest.mark.parametrize("T,d,H", [(64, 72, 100), (65, 72, 100), (256, 33, 71), (257, 33, 71), (300, 128, 96), (300, 1000, 40)])
def test_kinds(B, T, d, H, place, exact):
    x, w, dy = data(T, d, H, exact)
    plant(place, x, w, dy)
    got, ref = run(B, x, w, dy, True), reference(x, w, dy)
    assert place == "dy" or not bool(torch.isfinite(ref["y"]).all())
    for n, v in ref.items():
        same_kind(got[n], v, n)


def test_a_row_is_the_same_kind_in_any_batch(B):
    x, w, dy = data(300, 64, 48, True)
    w["Wg"][3, 5] = INF
    x[17, 9] = -INF
    whole = run(B, x, w, dy, False)["y"]
    for rows in (slice(0, 1), slice(16, 80), slice(0, 150), slice(150, 300)):
        same_kind(run(B, x[rows].contiguous(), w, dy, False)["y"], whole[rows], str(rows))
    assert bool(torch.isinf(whole).any())


def test_a_zero_beside_an_infinity(B):
    """0 x infinity is NaN, and a nonzero value whose lower terms are zero is not a zero."""
    T, d, H = 300, 16, 8
    x, w, dy = data(T, d, H, True)
    w["Wu"][4] = INF
    x[:, 4] = 1.0
    x[7, 4] = 0.0
    x[9, 4] = 2.0 ** -80
    y = run(B, x, w, dy, False)["y"]
    same_kind(y, reference(x, w, dy)["y"], "y")
    assert bool(torch.isnan(y[7]).all())


@pytest.mark.parametrize("T", [40, 300])
def test_any_nan(B, T):
    """Also one whose upper half has the bits of an infinity."""
    x, w, dy = data(T, 72, 40, False)
    x.view(torch.int32)[5, 3] = 0x7f800001
    dy.view(torch.int32)[6, 1] = -0x7fffff   # 0xff800001
    got = run(B, x, w, dy, True)
    assert bool(torch.isnan(got["y"][5]).all()) and bool(torch.isnan(got["d_x"][5:7]).all()) and bool(torch.isnan(got["Wd"][:, 1]).all())
    assert bool(torch.isfinite(got["y"][6:]).all()) and bool(torch.isfinite(got["d_x"][7:]).all())
