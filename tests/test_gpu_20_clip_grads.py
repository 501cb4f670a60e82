"""Global gradient norm and clipping, against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
HALF = {B16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def tensors(sizes, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale * (1 + i % 5)).to(dt) for i, (n, dt) in enumerate(sizes)]


def clip(B, grads, max_norm, out="new"):
    norm = torch.full((1,), -1.0, device="cuda")
    ws = torch.full((B.slicemoe_clip_grads_workspace_bytes(grads),), 255, dtype=torch.uint8, device="cuda")
    to = [torch.full_like(g, 7.0) for g in grads] if isinstance(out, str) else out
    B.slicemoe_clip_grads(grads, max_norm, norm, ws, out=to)
    torch.cuda.synchronize()
    return float(norm), to


def check(grads, max_norm, norm, out):
    total = sum(float(g.double().square().sum()) for g in grads)
    want = math.sqrt(total)
    assert abs(norm - want) <= want * (2.0 ** -24 + 1e-12)        # 64-bit sums, one rounding
    factor = min(1.0, max_norm / (want + 1e-6)) if want + 1e-6 > 0 else 1.0
    for g, o in zip(grads, out):
        assert o.dtype == g.dtype
        ref = g.double() * factor
        off = (o.double() - ref).abs()
        # the factor's roundings (norm, sum, quotient), the product, the storage; below the smallest normal number the last step is absolute
        assert bool((off <= ref.abs() * (4 * 2.0 ** -24 + HALF[g.dtype]) + 2.0 ** -133).all())


CASES = [
    [(1, F32)],
    [(1, B16), (3, F32), (7, B16), (8, F32)],
    [(4096, F32), (4097, B16), (4095, F32), (0, F32), (100003, B16)],
    [(3_000_001, F32), (17, B16), (5_000_007, B16), (1, F32)],
    [(11 + 37 * i, (F32, B16)[i % 2]) for i in range(203)],     # more than two launches' tables
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9, math.inf])
def test_against_64_bits(B, case, max_norm):
    grads = tensors(CASES[case], case)
    norm, out = clip(B, grads, max_norm)
    check(grads, max_norm, norm, out)
    again = clip(B, grads, max_norm)
    assert again[0] == norm and all(torch.equal(a, b) for a, b in zip(again[1], out))
    held = [g.clone() for g in grads]                           # in place: the same bits
    assert clip(B, held, max_norm, out=held)[0] == norm
    assert all(torch.equal(a, b) for a, b in zip(held, out))
    assert clip(B, grads, max_norm, out=None)[0] == norm        # measured only


def test_any_alignment(B):
    flat, dst = torch.randn(50_000, device="cuda"), torch.zeros(50_000, device="cuda")
    half, hdst = flat.to(B16), torch.zeros(50_000, dtype=B16, device="cuda")
    grads = [flat[1:10_002], flat[10_003:30_000], half[1:9_000], half[9_003:20_000]]
    out = [dst[3:10_004], dst[20_001:39_998], hdst[5:9_004], hdst[9_004:20_001]]
    norm, got = clip(B, grads, 1.0, out=out)
    check(grads, 1.0, norm, got)
    assert float(dst[:3].abs().sum()) == 0 and float(dst[10_004:20_001].abs().sum()) == 0 and float(hdst[20_001:].abs().sum()) == 0


def test_range(B):
    """Squares beyond fp32's range, and gradients below it."""
    for scale in (1e30, 1e-30):
        grads = tensors([(5000, F32), (3000, B16)], 3, scale)
        norm, out = clip(B, grads, 1.0)
        check(grads, 1.0, norm, out)


def test_not_finite(B):
    for bad in (math.nan, math.inf, -math.inf):
        grads = tensors([(500, F32), (300, B16)], 3)
        grads[0][77] = bad
        norm, out = clip(B, grads, 1.0)
        if math.isnan(bad):
            assert math.isnan(norm) and all(bool(torch.isnan(o).all()) for o in out)
        else:
            assert norm == math.inf and bool((out[1] == 0).all()) and bool(torch.isnan(out[0][77]))


def test_nothing(B):
    assert clip(B, [], 1.0) == (0.0, [])
    norm, out = clip(B, tensors([(0, F32), (0, B16)]), 1.0)
    assert norm == 0.0
    norm, out = clip(B, [torch.zeros(1000, device="cuda")], 0.0)   # factor 0 / 1e-6
    assert norm == 0.0 and bool((out[0] == 0).all())


def test_an_infinite_bound_leaves_every_value(B):
    """factor 1 also where the norm is infinite or NaN: copies to the last bit, and the tensors themselves in place."""
    for bad in (math.nan, math.inf):
        grads = tensors([(500, F32), (300, B16)], 3)
        grads[0][77] = bad
        norm, out = clip(B, grads, math.inf)
        assert not math.isfinite(norm)
        for g, o in zip(grads, out):
            fine = torch.isfinite(g)
            assert torch.equal(o[fine], g[fine]) and torch.equal(torch.isnan(o), torch.isnan(g)) and torch.equal(torch.isinf(o), torch.isinf(g))
        held = [g.clone() for g in grads]
        clip(B, held, math.inf, out=held)
        assert all(torch.equal(h.view(torch.uint8), g.view(torch.uint8)) for h, g in zip(held, grads))
