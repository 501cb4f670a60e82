"""Host-side checks of the layer for few tokens, the norms on both sides of a block and the microscaled products: what they refuse before
anything touches the GPU, their sizes and their structs.  No kernel is launched."""
import ctypes
import os

import pytest
import torch

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_04286_amd import build
        build.build()
    return binding


P, ODD, Q, R_, S_ = (ctypes.c_void_p(v) for v in (4096, 4100, 1 << 20, 1 << 21, 1 << 22))   # never dereferenced
NULL = None
BIG = 1 << 40


def by(x):
    return ctypes.byref(x)


def test_structs_and_constants_match_the_header(B):
    assert [ctypes.sizeof(t) for t in (B.slicemoe_block_norm_config, B.slicemoe_mx_config, B.slicemoe_mx_product_config, B.slicemoe_gated_weights_mx)] == [24, 20, 20, 24]
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "slicemoe.h")).read()
    assert f"#define SLICEMOE_FEW_ASSIGNMENTS {B.SLICEMOE_FEW_ASSIGNMENTS}\n" in header
    assert f"SLICEMOE_GATE_NONE = {B.SLICEMOE_GATE_NONE}, SLICEMOE_GATE_CHANNEL = {B.SLICEMOE_GATE_CHANNEL}, SLICEMOE_GATE_TOKEN = {B.SLICEMOE_GATE_TOKEN}" in header


def test_few_refusals(B):
    f, inv, uns = B.lib().slicemoe_forward_few, B.SLICEMOE_ERR_INVALID_ARG, B.SLICEMOE_ERR_UNSUPPORTED
    packed, logical = B.slicemoe_weights(packed=4096), B.slicemoe_weights(*[4096] * 8, None)
    ok, gen = B.make_config(4, 1024, 16, 2, 32, 256), B.make_config(4, 256, 4, 2, 8, 256, "f32")
    few = B.SLICEMOE_FEW_ASSIGNMENTS
    for c in (B.make_config(few // 32 + 1, 1024, 16, 2, 32, 256), B.make_config(4, 1024, 16, 2, 32, 256, capacity_factor=1.25),
              B.make_config(4, 1024, 16, 8, 32, 8192), B.make_config(4, 1024, 16, 2, 65, 256), B.make_config(few // 8 + 1, 256, 4, 2, 8, 256, "f32")):
        assert f(by(c), P, by(packed), Q, NULL, NULL, NULL) == uns
    for c in (B.make_config(-1, 1024, 16, 2, 32, 256), B.make_config(4, 1000, 16, 2, 32, 256), B.make_config(4, 1024, 16, 33, 32, 256)):
        assert f(by(c), P, by(packed), Q, NULL, NULL, NULL) == inv
    for args in [(NULL, by(packed), Q, P, P), (P, NULL, Q, P, P), (P, by(packed), NULL, P, P), (ODD, by(packed), Q, P, P), (P, by(packed), ODD, P, P),
                 (P, by(packed), Q, ctypes.c_void_p(4097), P), (P, by(packed), Q, P, ctypes.c_void_p(4098)), (P, by(logical), Q, P, P),
                 (P, by(B.slicemoe_weights(packed=4112)), Q, P, P)]:
        assert f(by(ok), *args, NULL) == inv, args
    assert f(by(gen), P, by(packed), Q, P, P, NULL) == inv       # fp32 reads the logical tensors
    assert f(by(gen), P, by(B.slicemoe_weights(*[4096] * 7, None, 4096)), Q, P, P, NULL) == inv
    assert f(NULL, P, by(packed), Q, NULL, NULL, NULL) == inv


def test_block_norm_refusals(B):
    f, g = B.lib().slicemoe_block_norm, B.lib().slicemoe_block_norm_backward
    inv, uns, wsp = B.SLICEMOE_ERR_INVALID_ARG, B.SLICEMOE_ERR_UNSUPPORTED, B.SLICEMOE_ERR_WORKSPACE
    size = B.slicemoe_block_norm_backward_workspace_bytes
    cfg = lambda *a, **k: B.make_block_norm_config(*a, **k)  # noqa: E731
    raw = B.slicemoe_block_norm_config
    for c, want in [(cfg(-1, 64), inv), (cfg(4, 0), inv), (cfg(4, 64, -1e-5), inv), (cfg(4, 64, NAN), inv), (cfg(4, 64, INF), inv), (cfg(4, 64, 1e-5, NAN), inv),
                    (cfg(4, 64, 1e-5, -INF), inv), (raw(4, 64, 1e-5, 1.0, 3, 1), inv), (raw(4, 64, 1e-5, 1.0, 1, 2), inv), (cfg(4, 16385), uns)]:
        assert f(by(c), P, P, P, P, P, Q, P, NULL, 0, NULL, NULL) == want
        assert g(by(c), P, P, P, P, P, P, P, P, Q, R_, P, P, P, P, BIG, NULL) == want and size(c) == 0
    ok, token, none = cfg(4, 64), cfg(4, 64, gate="token"), cfg(4, 64, gate=None)
    # x, post, gate, residual, pre, sum, y, y_mx, bits, stats
    for args in [(NULL, P, P, P, P, Q, P, NULL, 0, NULL), (P, P, NULL, P, P, Q, P, NULL, 0, NULL), (P, P, P, NULL, P, Q, P, NULL, 0, NULL),
                 (P, P, P, P, P, NULL, P, NULL, 0, NULL), (P, P, P, P, P, Q, NULL, NULL, 0, NULL), (P, P, P, P, NULL, Q, P, NULL, 0, NULL),
                 (P, P, P, P, NULL, Q, NULL, P, 4, NULL), (P, P, P, P, P, Q, Q, NULL, 0, NULL), (P, P, P, P, P, Q, P, P, 5, NULL), (P, P, P, P, P, Q, P, ctypes.c_void_p(4096 + 16), 4, NULL),
                 (ODD, P, P, P, P, Q, P, NULL, 0, NULL), (P, ODD, P, P, P, Q, P, NULL, 0, NULL), (P, P, ODD, P, P, Q, P, NULL, 0, NULL),
                 (P, P, P, ODD, P, Q, P, NULL, 0, NULL), (P, P, P, P, ODD, Q, P, NULL, 0, NULL), (P, P, P, P, P, ODD, P, NULL, 0, NULL),
                 (P, P, P, P, P, Q, ODD, NULL, 0, NULL), (P, P, P, P, P, Q, P, NULL, 0, ODD)]:
        assert f(by(ok), *args, NULL) == inv, args
    n = [P, R_, S_, Q, ctypes.c_void_p(1 << 23), ctypes.c_void_p(1 << 24), ctypes.c_void_p(1 << 25), ctypes.c_void_p(1 << 26)]
    for a, b in ((5, 1), (5, 2), (5, 4), (6, 1), (6, 2), (6, 4), (6, 5), (7, 0), (7, 1), (7, 2), (7, 3), (7, 4), (7, 5), (7, 6)):   # outputs in the place of what all rows read, or of each other
        assert f(by(token), *[n[b] if i == a else v for i, v in enumerate(n)], 4, NULL, NULL) == inv, (a, b)
    assert f(by(cfg((1 << 30) + 1, 1, gate="token")), *n, 4, NULL, NULL) == uns        # more rows than microscaled values have
    assert f(by(none), P, P, P, P, P, Q, P, NULL, 0, NULL, NULL) == inv      # a gate that the configuration does not have
    # x, post, gate, sum, pre, stats, d_y, d_sum, d_x, d_residual, d_post, d_gate, d_pre
    good = [P, P, Q, P, P, P, P, P, R_, S_, P, Q, P]
    for at in (0, 2, 3, 4, 5, 6, 8, 9, 10, 11, 12):      # (the d_gate of one row too)
        assert g(by(ok), *[NULL if i == at else v for i, v in enumerate(good)], P, BIG, NULL) == inv, at
    for at in range(13):
        assert g(by(ok), *[ctypes.c_void_p(4098) if i == at else v for i, v in enumerate(good)], P, BIG, NULL) == inv, at
    assert g(by(none), *good, P, BIG, NULL) == inv
    for a, b in ((8, 9), (8, 0), (9, 0), (8, 3), (9, 3)):     # outputs in the place of each other or of x and sum
        assert g(by(ok), *[good[b] if i == a else v for i, v in enumerate(good)], P, BIG, NULL) == inv, (a, b)
    t = [P, P, Q, P, P, P, P, P, R_, S_, P, ctypes.c_void_p(1 << 23), P]
    for a, b in ((11, 8), (11, 9), (11, 2), (11, 6), (11, 0), (8, 2), (9, 2)):
        assert g(by(token), *[t[b] if i == a else v for i, v in enumerate(t)], P, BIG, NULL) == inv, (a, b)
    assert g(by(ok), *good, NULL, BIG, NULL) == wsp and g(by(ok), *good, P, size(ok) - 1, NULL) == wsp and g(by(ok), *good, ODD, BIG, NULL) == inv
    last = 0
    for T in (0, 1, 100, 767, 768, 5000, 1 << 20, (1 << 31) - 1):     # a workspace of the largest batch serves the smaller ones
        assert size(cfg(T, 1000)) >= last
        last = size(cfg(T, 1000))


def test_mx_refusals_and_sizes(B):
    L, inv, uns, wsp = B.lib(), B.SLICEMOE_ERR_INVALID_ARG, B.SLICEMOE_ERR_UNSUPPORTED, B.SLICEMOE_ERR_WORKSPACE
    mc = B.make_mx_config
    for c, want in [(mc(-1, 64), inv), (mc(4, 0), inv), (mc(4, 64, 5), inv), (B.slicemoe_mx_config(4, 64, 4, 2, 0), inv), (B.slicemoe_mx_config(4, 64, 4, 1, 2), inv),
                    (mc(4, (1 << 20) + 1), uns), (mc(1 << 30, 1025), uns), (mc((1 << 30) + 1, 1), uns), (mc((1 << 31) - 1, 1), uns)]:
        assert L.slicemoe_mx_quantize(by(c), P, Q, NULL) == want and L.slicemoe_mx_dequantize(by(c), Q, P, NULL) == want and B.slicemoe_mx_bytes(c) == 0
    ok = mc(4, 64)
    for args in [(NULL, Q), (P, NULL), (ODD, Q), (P, ctypes.c_void_p(4096 + 128))]:
        assert L.slicemoe_mx_quantize(by(ok), *args, NULL) == inv
    for args in [(NULL, P), (Q, NULL), (ctypes.c_void_p(4096 + 128), P), (Q, ODD)]:
        assert L.slicemoe_mx_dequantize(by(ok), *args, NULL) == inv
    for rows, cols, bits in ((1, 1, 4), (32, 256, 8), (33, 257, 4), (70, 4096, 8), (0, 5, 4)):
        tiles = -(-rows // 32) * -(-cols // 256)
        assert B.slicemoe_mx_bytes(mc(rows, cols, bits)) == max(256, tiles * (1024 * bits + 256))
    pc, size = B.make_mx_product_config, B.slicemoe_mx_product_workspace_bytes
    f = L.slicemoe_mx_product
    for c, want in [(pc(-1, 64, 64), inv), (pc(4, 0, 64), inv), (pc(4, 64, 0), inv), (pc(4, 64, 64, 3), inv), (B.slicemoe_mx_product_config(4, 64, 64, 4, 2), inv),
                    (pc((1 << 24) + 1, 64, 64), uns), (pc(4, (1 << 20) + 1, 64), uns), (pc(4, 64, (1 << 20) + 1), uns), (pc(1 << 24, 1 << 13, 64), uns), (pc(1 << 24, 64, (1 << 12) + 1), uns)]:
        assert f(by(c), P, P, P, Q, P, BIG, NULL) == want and size(c) == 0
    for bits in (4, 8):     # a workspace of the largest batch serves the smaller ones
        for K, N in ((64, 64), (11008, 4096), (4096, 11008), (512, 100), (3000, 70000)):
            sizes = [size(pc(T, K, N, bits)) for T in (0, 1, 64, 65, 128, 200, 512, 1000, 4096, 100000)]
            assert sizes == sorted(sizes)
    ok = pc(4, 64, 64)
    for args in [(NULL, P, P, Q), (P, NULL, P, Q), (P, P, P, NULL), (ODD, P, P, Q), (P, ODD, P, Q), (P, P, ODD, Q), (P, P, P, ODD)]:
        assert f(by(ok), *args, P, BIG, NULL) == inv, args
    gc, w = B.make_gated_config(4, 64, 32), B.slicemoe_gated_weights_mx(4096, 4096, 4096)
    h, gs = L.slicemoe_gated_ffn_mx, B.slicemoe_gated_ffn_mx_workspace_bytes
    for c, bits, want in [(B.make_gated_config(-1, 64, 32), 4, inv), (B.make_gated_config(4, 0, 32), 4, inv), (gc, 2, inv), (gc, 16, inv),
                          (B.make_gated_config(4, 64, 32, "f32"), 4, uns), (B.make_gated_config((1 << 24) + 1, 64, 32), 8, uns), (B.make_gated_config(1 << 24, 64, 4097), 8, uns)]:
        assert h(by(c), bits, P, by(w), P, Q, P, BIG, NULL) == want and gs(c, bits) == 0
    for args in [(NULL, by(w), P, Q), (P, NULL, P, Q), (P, by(B.slicemoe_gated_weights_mx(4096, 0, 4096)), P, Q), (P, by(w), P, NULL), (ODD, by(w), P, Q),
                 (P, by(B.slicemoe_gated_weights_mx(4096, 4112, 4096)), P, Q), (P, by(w), ODD, Q), (P, by(w), P, ODD)]:
        assert h(by(gc), 4, *args, P, BIG, NULL) == inv
    for bits in (4, 8):
        assert h(by(gc), bits, P, by(w), P, Q, P, gs(gc, bits) - 1, NULL) == wsp and h(by(gc), bits, P, by(w), P, Q, NULL, BIG, NULL) == wsp
        assert h(by(gc), bits, P, by(w), P, Q, ODD, BIG, NULL) == inv


def test_binding_checks_its_arguments(B):
    with pytest.raises(ValueError):
        B.make_block_norm_config(4, 64, gate="row")
    with pytest.raises(ValueError):
        B.make_mx_config(4, 64, 4, "fp16")
    t = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.slicemoe_mx_quantize(B.make_mx_config(4, 64), t, torch.zeros(8192, dtype=torch.uint8))      # host tensors
    with pytest.raises(TypeError):
        B.slicemoe_forward_few(B.make_config(4, 1024, 16, 2, 32, 256), t, {"packed": t}, t)
    with pytest.raises(TypeError):
        B.slicemoe_block_norm(B.make_block_norm_config(4, 64), t, t, t, t, t, t, t)


def test_block_norm_outputs_in_the_place_of_others(B):
    """Only what the header allows; a refusal of the workspace shows that a call was accepted so far (nothing is launched)."""
    f, g, inv, wsp = B.lib().slicemoe_block_norm, B.lib().slicemoe_block_norm_backward, B.SLICEMOE_ERR_INVALID_ARG, B.SLICEMOE_ERR_WORKSPACE
    at = lambda i: ctypes.c_void_p((i + 1) << 20)  # noqa: E731
    # x, post, gate, residual, pre, sum, y, y_mx, bits, stats
    n = [at(i) for i in range(8)] + [4, at(8)]
    for gate in ("channel", "token"):
        c = B.make_block_norm_config(4, 64, gate=gate)
        for other in range(8):
            assert f(by(c), *[n[other] if i == 9 else v for i, v in enumerate(n)], NULL) == inv, other
    # x, post, gate, sum, pre, stats, d_y, d_sum, d_x, d_residual, d_post, d_gate, d_pre
    names = ["x", "post", "gate", "sum", "pre", "stats", "d_y", "d_sum", "d_x", "d_residual", "d_post", "d_gate", "d_pre", "workspace"]
    good = {name: at(i) for i, name in enumerate(names)}
    allowed = {frozenset(p) for p in (("d_x", "d_y"), ("d_x", "d_sum"), ("d_residual", "d_y"), ("d_residual", "d_sum"))}
    outputs = names[8:]
    for gate in ("channel", "token"):
        c = B.make_block_norm_config(4, 64, gate=gate)

        def call(p, size):
            return g(by(c), *[p[name] for name in names], size, NULL)
        assert call(good, 0) == wsp
        for o in outputs:
            for other in names:
                if other != o and frozenset((o, other)) not in allowed:
                    assert call({**good, o: good[other]}, BIG) == inv, (gate, o, other)
                    assert call({**good, other: good[o]}, BIG) == inv, (gate, o, other)
        for o, other in (("d_x", "d_y"), ("d_x", "d_sum"), ("d_residual", "d_y"), ("d_residual", "d_sum")):
            assert call({**good, o: good[other]}, 0) == wsp
    # what the configuration does not have is not written and may be anything
    c = B.make_block_norm_config(4, 64, gate=None)
    p = {**good, "gate": NULL, "post": NULL, "d_gate": good["x"], "d_post": good["x"]}
    assert g(by(c), *[p[name] for name in names], 0, NULL) == wsp
