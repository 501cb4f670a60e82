"""Gradient clipping of lists whose chunks' sums are added up once (more than 192 tensors) and in every block, on either side of the
line: the same norm either way, out of place, in place, measured only, and captured."""
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


def tensors(count, empty=0, seed=0):
    """`count` tensors of 1 to some 5000 values, of both types, and empty ones between them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = [torch.randn(1 + (i * 7919) % 4999, generator=g, device="cuda").to((F32, B16)[i % 2]) for i in range(count)]
    for i in range(empty):
        out.insert(i * 3, torch.empty(0, device="cuda"))
    return out


def space(B, grads):
    return torch.full((B.slicemoe_clip_grads_workspace_bytes(grads),), 255, dtype=torch.uint8, device="cuda")


def check(grads, max_norm, norm, out):
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    assert abs(float(norm) - want) <= want * (2.0 ** -24 + 1e-12)
    factor = min(1.0, max_norm / (want + 1e-6))
    for g, o in zip(grads, out):
        ref = g.double() * factor
        assert bool(((o.double() - ref).abs() <= ref.abs() * (4 * 2.0 ** -24 + HALF[g.dtype]) + 2.0 ** -133).all())


@pytest.mark.parametrize("count,empty", [(96, 0), (97, 0), (192, 0), (192, 100), (193, 0), (193, 50), (1000, 0), (9000, 0)])
@pytest.mark.parametrize("max_norm", [0.5, 1e9, math.inf])
def test_either_side(B, count, empty, max_norm):
    grads = tensors(count, empty)
    norm, ws = torch.full((1,), -1.0, device="cuda"), space(B, grads)
    out = [torch.full_like(g, 7.0) for g in grads]
    B.slicemoe_clip_grads(grads, max_norm, norm, ws, out=out)
    check(grads, max_norm, norm, out)
    held, again = [g.clone() for g in grads], torch.full((1,), -1.0, device="cuda")
    B.slicemoe_clip_grads(held, max_norm, again, space(B, held), out=held)
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(held, out))
    only = torch.full((1,), -1.0, device="cuda")
    B.slicemoe_clip_grads(grads, max_norm, only, space(B, grads))
    assert torch.equal(only, norm)


def test_the_same_values_in_few_and_in_many_tensors(B):
    """A chunk never crosses a tensor, so whole chunks of one tensor are the chunks of many: the same sums in the same order."""
    flat = torch.randn(400 * 4096, device="cuda")
    norms = []
    for grads in ([flat], list(flat.split(4096))):
        norm, out = torch.full((1,), -1.0, device="cuda"), [torch.empty_like(g) for g in grads]
        B.slicemoe_clip_grads(grads, 1.0, norm, space(B, grads), out=out)
        norms.append((norm, torch.cat(out)))
    assert torch.equal(norms[0][0], norms[1][0]) and torch.equal(norms[0][1], norms[1][1])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_not_finite(B, bad):
    grads = tensors(300)
    grads[211][0] = bad
    norm, out = torch.zeros(1, device="cuda"), [torch.empty_like(g) for g in grads]
    B.slicemoe_clip_grads(grads, 1.0, norm, space(B, grads), out=out)
    if math.isnan(bad):
        assert math.isnan(float(norm)) and all(bool(torch.isnan(o).all()) for o in out)
    else:
        assert float(norm) == math.inf and bool((out[0] == 0).all()) and bool(torch.isnan(out[211][0]))


def test_captured(B):
    grads, live = tensors(400, seed=1), tensors(400, seed=2)
    norm, out, ws = torch.empty(1, device="cuda"), [torch.empty_like(g) for g in grads], space(B, grads)
    lnorm, lout, lws = torch.empty(1, device="cuda"), [torch.empty_like(g) for g in live], space(B, live)
    B.slicemoe_clip_grads(live, 0.5, lnorm, lws, out=lout)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slicemoe_clip_grads(grads, 0.5, norm, ws, out=out)
    for k in range(3):
        for a, b, c in zip(grads, live, tensors(400, seed=10 + k)):
            a.copy_(c)
            b.copy_(c)
        B.slicemoe_clip_grads(live, 0.5, lnorm, lws, out=lout)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, lnorm) and all(torch.equal(a, b) for a, b in zip(out, lout)), k
