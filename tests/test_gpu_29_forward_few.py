"""The layer for a few tokens in one launch: the bits of slicemoe_forward on the matrix-core path, the oracle's values on the other."""
import numpy as np
import pytest
import torch

import oracle
from common import NEAR_TIE, TOL_F32, make_inputs
from paper_2510_04286_amd import workload as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def few(B, cfg, h, w, **kw):
    Ns = cfg.T * cfg.S
    idx = torch.full((Ns, cfg.k), -7, dtype=torch.int32, device="cuda")
    p = torch.full((Ns, cfg.k), -7.0, device="cuda")
    out = torch.full_like(h, 7.0)
    B.slicemoe_forward_few(cfg, h, w, out, topk_idx=idx, topk_p=p, **kw)
    return out, idx, p


def whole(B, cfg, h, w):
    ws, out = B.alloc_workspace(cfg), torch.empty_like(h)
    B.slicemoe_forward(cfg, h, w, out, ws)
    v = B.workspace_views(cfg, ws)
    return out, v["topk_idx"].clone(), v["topk_p"].clone()


SHAPES = [wl.SliceMoEShape(f"{d}_{S}_{E}_{k}_{He}", T=1, d=d, S=S, E=E, k=k, He=He) for d, S, E, k, He in
          [(1024, 16, 32, 2, 256), (4096, 32, 64, 2, 512), (512, 8, 16, 2, 256), (768, 8, 16, 2, 384), (768, 8, 16, 3, 384), (768, 2, 16, 2, 1536),
           (768, 4, 16, 1, 768), (768, 16, 16, 2, 192), (768, 32, 16, 2, 96), (768, 32, 64, 8, 96), (128, 2, 3, 3, 64), (64, 1, 1, 1, 32), (256, 2, 40, 5, 2080),
           (384, 2, 33, 2, 96), (384, 1, 64, 8, 512), (768, 4, 48, 4, 32)]]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.name)
def test_bits_of_the_whole_forward(B, shape):
    most = B.SLICEMOE_FEW_ASSIGNMENTS // (shape.S * shape.k)
    for T in sorted({1, 2, 3, 17, 64, most}):
        if T > most:
            continue
        s, h, w = make_inputs(shape, T)
        cfg = B.config_of(s)
        assert B.slicemoe_uses_mfma(cfg) == 1
        w = B.pack(cfg, B.weights_to_device(w, "bf16"))
        h = B.to_device(h, "bf16")
        want = whole(B, cfg, h, w)
        got = few(B, cfg, h, {"packed": w["packed"]})
        assert all(torch.equal(a, b) for a, b in zip(got, want)), T
        out = h.clone()
        B.slicemoe_forward_few(cfg, out, w, out)      # in place, nothing but the output
        assert torch.equal(out, want[0])


@pytest.mark.parametrize("E", [1, 2, 5, 31, 33])
def test_equal_logits_and_logits_that_are_not_numbers(B, E):
    """Equal logits go to the lower expert; with NaN or infinite hidden states the selection stays in range."""
    for dtype, ds in (("bf16", 64), ("f32", 40)):
        shape = wl.SliceMoEShape("ties", T=6, d=2 * ds, S=2, E=E, k=min(2, E), He=64, dtype=dtype)
        _, h, w = make_inputs(shape)
        w["Wr2"][:] = 0
        w["br2"][:] = 0.25
        cfg = B.config_of(shape)
        wd = B.pack(cfg, B.weights_to_device(w, dtype))
        h = B.to_device(h, dtype)
        out, idx, p = few(B, cfg, h, wd)
        assert bool((idx == torch.arange(cfg.k, device="cuda", dtype=torch.int32)).all()) and torch.allclose(p, torch.full_like(p, 1.0 / E), rtol=1e-5)
        h[1, 3], h[2, 5], h[3, ds + 1] = float("nan"), float("inf"), -float("inf")
        wd = B.pack(cfg, B.weights_to_device(make_inputs(shape)[2], dtype))
        out, idx, p = few(B, cfg, h, wd)
        assert bool(((idx >= 0) & (idx < E)).all()) and bool(out[[0, 4, 5]].isfinite().all())


GENERIC = [wl.SliceMoEShape("f32_tiny", T=16, d=256, S=4, E=8, k=2, He=256, dtype="f32"), wl.SliceMoEShape("f32_odd", T=5, d=21, S=3, E=7, k=3, He=50, dtype="f32"),
           wl.SliceMoEShape("bf16_odd", T=9, d=100, S=2, E=5, k=2, He=70), wl.SliceMoEShape("one", T=1, d=1, S=1, E=1, k=1, He=1, dtype="f32"),
           wl.SliceMoEShape("wide", T=3, d=1200, S=2, E=64, k=8, He=900, dtype="f32"), wl.SliceMoEShape("router", T=4, d=64, S=2, E=9, k=2, He=40, dtype="f32", Hr=100)]


@pytest.mark.parametrize("shape", GENERIC, ids=lambda s: s.name)
def test_other_shapes_against_the_oracle(B, shape):
    s, h, w = make_inputs(shape)
    cfg = B.config_of(s)
    assert B.slicemoe_uses_mfma(cfg) == 0
    hd = B.to_device(h, s.dtype)
    out, idx, p = few(B, cfg, hd, B.weights_to_device(w, s.dtype))
    ref = oracle.forward(h, s.S, s.k, w)
    g = idx.cpu().numpy()
    same = np.all(g == ref["idx"], axis=1)
    lg = oracle.route(h.reshape(-1, s.ds), w["Wr1"], w["br1"], w["Wr2"], w["br2"], s.k, want_logits=True)["logits"].astype(np.float32).astype(np.float64)
    assert np.all(np.take_along_axis(lg, ref["idx"].astype(np.int64), 1) - np.take_along_axis(lg, g.astype(np.int64), 1) < NEAR_TIE) and np.sum(~same) <= 1
    got, want = out.double().cpu().numpy().reshape(-1, s.ds), ref["h_out"].reshape(-1, s.ds)
    rms = np.sqrt(np.mean(want ** 2))
    assert np.abs(got - want)[same].max() <= (TOL_F32 * rms if s.dtype == "f32" else TOL_F32 * rms + 2.0 ** -8 * np.abs(want).max())
    assert np.abs(p.cpu().numpy() - ref["pk"])[same].max() <= 1e-5
    again = few(B, cfg, hd, B.weights_to_device(w, s.dtype))
    assert torch.equal(again[0], out)


def test_generic_arithmetic_by_flag(B):
    """SLICEMOE_FLAG_FORCE_GENERIC: the logical tensors in fp32, also where the matrix cores would do."""
    shape = wl.CONFIGS["lm"].scaled(8)
    s, h, w = make_inputs(shape)
    wd, hd = B.weights_to_device(w, "bf16"), B.to_device(h, "bf16")
    cfg = B.config_of(s, flags=B.SLICEMOE_FLAG_FORCE_GENERIC)
    out, idx, p = few(B, cfg, hd, wd)
    ref = oracle.forward(h, s.S, s.k, w)
    same = np.all(idx.cpu().numpy() == ref["idx"], axis=1)
    assert np.sum(~same) <= 1
    want = ref["h_out"].reshape(-1, s.ds)
    err = np.abs(out.double().cpu().numpy().reshape(-1, s.ds) - want)[same].max()
    assert err <= TOL_F32 * np.sqrt(np.mean(want ** 2)) + 2.0 ** -8 * np.abs(want).max()


def test_no_tokens_and_refusals(B):
    cfg = B.make_config(0, 1024, 16, 2, 32, 256)
    h = torch.empty((0, 1024), dtype=torch.bfloat16, device="cuda")
    w = {"packed": torch.empty(B.slicemoe_packed_bytes(cfg), dtype=torch.uint8, device="cuda")}
    B.slicemoe_forward_few(cfg, h, w, h)
    torch.cuda.synchronize()
    cfg = B.make_config(4, 1024, 16, 2, 32, 256)
    h = torch.zeros((4, 1024), dtype=torch.bfloat16, device="cuda")
    for bad in ({}, {"packed": w["packed"][:-256]}):
        with pytest.raises((B.SliceMoEError, ValueError)):
            B.slicemoe_forward_few(cfg, h, bad, h)
    with pytest.raises(TypeError):
        B.slicemoe_forward_few(cfg, h.float(), w, h)
    with pytest.raises(ValueError):
        B.slicemoe_forward_few(cfg, h[:3], w, h)


@pytest.mark.parametrize("E,k", [(16, 2), (33, 2), (16, 5), (64, 8)])
def test_masked_experts(B, E, k):
    """Experts whose bias is -infinity: the bits of the whole forward while k are left; with fewer the masked ones follow, each once and with probability 0."""
    for left in (E - 1, k, k - 1, 1):
        for dtype in ("bf16", "f32"):
            shape = wl.SliceMoEShape("masked", T=7, d=128, S=2, E=E, k=k, He=64, dtype=dtype)
            _, h, w = make_inputs(shape)
            keep = np.sort(np.random.default_rng(left).permutation(E)[:left])
            masked = np.setdiff1d(np.arange(E), keep)
            w["br2"][masked] = -np.inf
            cfg = B.config_of(shape, flags=0 if dtype == "bf16" else B.SLICEMOE_FLAG_FORCE_GENERIC)
            wd, hd = B.pack(cfg, B.weights_to_device(w, dtype)), B.to_device(h, dtype)
            out, idx, p = few(B, cfg, hd, wd)
            if left >= k and B.slicemoe_uses_mfma(cfg):
                assert all(torch.equal(a, b) for a, b in zip((out, idx, p), whole(B, cfg, hd, wd)))
            got = idx.cpu().numpy()
            assert all(len(set(r)) == k for r in got.tolist())
            assert np.isin(got[:, :min(k, left)], keep).all() and bool(out.isfinite().all())
            assert (got[:, left:] == masked[:max(0, k - left)]).all() and bool((p[:, left:] == 0).all()) and bool((p[:, :left] > 0).all())
