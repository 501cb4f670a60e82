"""The gated network at the widths that its configuration ends at, against 64 bits: rows and contractions of 2^20 values."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
MOST = 1 << 20


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rand(shape, seed, scale, dt):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [2, 70])
@pytest.mark.parametrize("d,H", [(MOST, 9), (8, MOST - 1)])
def test_widest(B, T, d, H, dt):
    w = {"Wg": rand((d, H), 1, d ** -0.5, dt), "Wu": rand((d, H), 2, d ** -0.5, dt), "Wd": rand((H, d), 3, H ** -0.5, dt)}
    x, add, dy, dadd = (rand((T, d), 4 + i, 1.0, dt) for i in range(4))
    cfg = B.make_gated_config(T, d, H, dt)
    got = {"y": torch.full_like(x, 7.0), "d_x": torch.full_like(x, 7.0), **{n: torch.full_like(t, 7.0) for n, t in w.items()}}
    B.slicemoe_gated_ffn(cfg, x, w, got["y"], torch.empty(B.slicemoe_gated_ffn_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), addend=add)
    B.slicemoe_gated_ffn_backward(cfg, x, w, dy, got["d_x"], got, torch.empty(B.slicemoe_gated_ffn_backward_workspace_bytes(cfg), dtype=torch.uint8,
                                                                              device="cuda"), addend=dadd)
    for n, (v, e) in R.gated(x, w, add, dt, dy, dadd).items():
        R.within(got[n], v, e, n)


@pytest.mark.parametrize("T", [40, 300])
def test_small_fp32_gradients(B, T):
    """Powers of two down to 2^-104 (values down to some 2^-108) change nothing but the exponents: the backward pass is linear in d_y."""
    d, H = 136, 200
    w = {"Wg": rand((d, H), 1, d ** -0.5, F32), "Wu": rand((d, H), 2, d ** -0.5, F32), "Wd": rand((H, d), 3, H ** -0.5, F32)}
    x, dy = rand((T, d), 4, 1.0, F32), rand((T, d), 5, 1.0, F32)
    ref = R.gated(x, w, None, F32, dy, None)
    cfg = B.make_gated_config(T, d, H, "f32")
    ws = torch.empty(B.slicemoe_gated_ffn_backward_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    for power in (0, 60, 104):
        got = {"d_x": torch.full_like(x, 7.0), **{n: torch.full_like(t, 7.0) for n, t in w.items()}}
        B.slicemoe_gated_ffn_backward(cfg, x, w, dy * 2.0 ** -power, got["d_x"], got, ws)
        for n, v in got.items():
            R.within(v.double() * 2.0 ** power, *ref[n], f"{n} at 2^-{power}")
