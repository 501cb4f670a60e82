"""The operators around the layer as a program uses them: together in a training step of a block, captured into a graph, on other
streams, in place, at their largest offsets, next to memory that must not be read."""
import pytest
import torch

import block_reference as R
from paper_2510_04286_amd import workload as wl

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
NAME = {B16: "bf16", F32: "f32"}


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rand(shape, seed, scale=1.0, dt=B16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def space(n):
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


class Gated:
    """One network's tensors and calls."""

    def __init__(self, B, T, d, H, dt=B16, seed=0):
        self.B, self.dt, self.cfg = B, dt, B.make_gated_config(T, d, H, NAME[dt])
        self.w = {"Wg": rand((d, H), seed + 1, d ** -0.5, dt), "Wu": rand((d, H), seed + 2, d ** -0.5, dt), "Wd": rand((H, d), seed + 3, H ** -0.5, dt)}
        self.x, self.add, self.dy, self.dadd = (rand((T, d), seed + 4 + i, 1.0, dt) for i in range(4))
        self.ws, self.bws = space(B.slicemoe_gated_ffn_workspace_bytes(self.cfg)), space(B.slicemoe_gated_ffn_backward_workspace_bytes(self.cfg))
        self.y, self.dx = torch.full_like(self.x, 7.0), torch.full_like(self.x, 7.0)
        self.g = {n: torch.full_like(t, 7.0) for n, t in self.w.items()}

    def run(self, stream=None):
        self.B.slicemoe_gated_ffn(self.cfg, self.x, self.w, self.y, self.ws, addend=self.add, stream=stream)
        self.B.slicemoe_gated_ffn_backward(self.cfg, self.x, self.w, self.dy, self.dx, self.g, self.bws, addend=self.dadd, stream=stream)

    def out(self):
        return [t.clone() for t in (self.y, self.dx, self.g["Wg"], self.g["Wu"], self.g["Wd"])]


def test_a_training_step_of_a_block(B):
    """Norm, the SliceMoE layer, the network beside it, their backward passes, and the clipping of every gradient.  The layer has tests of
    its own: its outputs stand in the references as they are."""
    shape = wl.CONFIGS["lm"].scaled(300)
    T, d, H = shape.T, shape.d, 1408
    cfg, ncfg, gcfg = B.config_of(shape), B.make_norm_config(T, d, 1e-5, "bf16"), B.make_gated_config(T, d, H, "bf16")
    w = B.pack(cfg, B.weights_to_device(wl.make_weights(shape), shape.dtype))
    gw = {"Wg": rand((d, H), 1, d ** -0.5), "Wu": rand((d, H), 2, d ** -0.5), "Wd": rand((H, d), 3, H ** -0.5)}
    nw = (1 + 0.1 * rand((d,), 4, 1.0, F32)).to(B16)
    branch, stream, d_out, d_stream = rand((T, d), 5), rand((T, d), 6, 3.0), rand((T, d), 7, 1e-2), rand((T, d), 8, 1e-2)
    s, n, h, y = (torch.empty_like(branch) for _ in range(4))
    d_h, d_n, d_s = (torch.empty_like(branch) for _ in range(3))
    ws, bws, gws, gbws, nws = (space(k) for k in (B.slicemoe_workspace_bytes(cfg), B.slicemoe_backward_workspace_bytes(cfg),
                                                  B.slicemoe_gated_ffn_workspace_bytes(gcfg), B.slicemoe_gated_ffn_backward_workspace_bytes(gcfg),
                                                  B.slicemoe_add_rmsnorm_backward_workspace_bytes(ncfg)))
    grads, ggrads, d_nw = B.alloc_weight_grads(cfg), {k: torch.empty_like(t) for k, t in gw.items()}, torch.empty(d, device="cuda")
    norm = torch.empty(1, device="cuda")

    def step():
        B.slicemoe_add_rmsnorm(ncfg, branch, stream, nw, s, n)
        B.slicemoe_forward(cfg, n, w, h, ws)
        B.slicemoe_gated_ffn(gcfg, n, gw, y, gws, addend=h)
        B.slicemoe_backward(cfg, n, w, ws, d_out, d_h, grads, bws)
        B.slicemoe_gated_ffn_backward(gcfg, n, gw, d_out, d_n, ggrads, gbws, addend=d_h)
        B.slicemoe_add_rmsnorm_backward(ncfg, s, nw, d_n, d_s, d_nw, nws, d_sum=d_stream)
        every = [*grads.values(), *ggrads.values(), d_nw]
        held = [t.clone() for t in every]
        B.slicemoe_clip_grads(every, 0.01, norm, cws, out=every)
        return held, every

    cws = space(B.slicemoe_clip_grads_workspace_bytes([*grads.values(), *ggrads.values(), d_nw]))
    held, every = step()
    rs, rn, bs, bn = R.norm_forward(branch, stream, nw, 1e-5, B16)
    R.within(s, rs, bs, "sum")
    R.within(n, rn, bn, "norm")
    for name, (v, e) in R.gated(n, gw, h, B16, d_out, d_h).items():
        got = {"y": y, "d_x": d_n}.get(name)
        R.within(held[8 + list(ggrads).index(name)] if got is None else got, v, e, name)
    rx, rw, bx, bw = R.norm_backward(s, nw, d_n, d_stream, 1e-5, B16)
    R.within(d_s, rx, bx, "d_s")
    R.within(held[-1], rw, bw, "d_weight")
    total = sum(float(t.double().square().sum()) for t in held) ** 0.5
    assert abs(float(norm) - total) <= total * 2.0 ** -23 and total > 0.01
    for a, b in zip(every, held):
        ref = b.double() * (0.01 / (total + 1e-6))
        assert bool(((a.double() - ref).abs() <= ref.abs() * (R.HALF[a.dtype] + 2.0 ** -21) + 1e-37).all())
    first = [t.clone() for t in (y, d_s, *every)]
    step()
    assert all(torch.equal(a, b) for a, b in zip(first, (y, d_s, *every)))


@pytest.mark.parametrize("T,dt", [(5, B16), (50, B16), (300, B16), (3000, B16), (77, F32)], ids=str)
def test_captured_into_a_graph(B, T, dt):
    d, H = (520, 1000) if T < 1000 else (512, 2048)
    net, live = Gated(B, T, d, H, dt), Gated(B, T, d, H, dt)
    ncfg = B.make_norm_config(T, d, 1e-5, NAME[dt])
    s, n, dnx, dw, nws = (torch.empty_like(net.x), torch.empty_like(net.x), torch.empty_like(net.x), torch.empty(d, device="cuda"),
                          space(B.slicemoe_add_rmsnorm_backward_workspace_bytes(ncfg)))
    weight, norm = rand((d,), 30, 1.0, dt), torch.empty(1, device="cuda")
    out = [torch.empty_like(t) for t in net.g.values()]
    cws = space(B.slicemoe_clip_grads_workspace_bytes(list(net.g.values())))

    def body(o):
        B.slicemoe_add_rmsnorm(ncfg, o.x, o.add, weight, s, n)
        o.run()
        B.slicemoe_add_rmsnorm_backward(ncfg, s, weight, o.dx, dnx, dw, nws, d_sum=o.dy)
        B.slicemoe_clip_grads(list(o.g.values()), 0.5, norm, cws, out=out)

    def results(o):
        torch.cuda.synchronize()
        return o.out() + [t.clone() for t in (s, n, dnx, dw, norm, *out)]

    body(live)   # (kernels are loaded before the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(net)
    for k in range(4):
        for o in (net, live):
            for i, t in enumerate((o.x, o.add, o.dy, o.dadd)):
                t.copy_(rand(t.shape, 100 * k + i, 1.0, dt))
        body(live)
        want = results(live)
        graph.replay()
        got = results(net)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        assert float(torch.randn(1000, device="cuda").sum()) != 0   # the program's own eager work


def test_two_graphs_and_two_streams_at_once(B):
    """Calls that overlap in time, each with a workspace of its own, on streams that are not the current one."""
    nets = [Gated(B, 200 + 77 * i, 512, 1408, seed=50 * i) for i in range(2)]
    want = []
    for o in nets:
        o.run()
        torch.cuda.synchronize()
        want.append(o.out())
    streams = [torch.cuda.Stream() for _ in nets]
    for _ in range(3):
        for o in nets:
            for t in (o.y, o.dx, *o.g.values()):
                t.zero_()
        torch.cuda.synchronize()
        for o, st in zip(nets, streams):
            o.run(stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(nets, want) for a, b in zip(o.out(), w))
    graphs = []
    for o in nets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o.run()
        graphs.append(g)
    for _ in range(3):
        for o in nets:
            for t in (o.y, o.dx, *o.g.values()):
                t.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(nets, want) for a, b in zip(o.out(), w))


@pytest.mark.parametrize("T,d,H,dt", [(40, 200, 300, B16), (300, 257, 100, B16), (1000, 512, 1408, B16), (70, 96, 100, F32)], ids=str)
def test_gated_outputs_in_place_of_inputs(B, T, d, H, dt):
    o = Gated(B, T, d, H, dt)
    o.run()
    want = o.out()
    for target in ("x", "add"):
        x, add = o.x.clone(), o.add.clone()
        to = x if target == "x" else add
        B.slicemoe_gated_ffn(o.cfg, x, o.w, to, o.ws, addend=add)
        assert torch.equal(to, want[0])
    for target in ("dy", "dadd"):
        dy, dadd = o.dy.clone(), o.dadd.clone()
        to = dy if target == "dy" else dadd
        B.slicemoe_gated_ffn_backward(o.cfg, o.x, o.w, dy, to, o.g, o.bws, addend=dadd)
        assert all(torch.equal(a, b) for a, b in zip([to, *o.g.values()], want[1:]))


def test_a_workspace_of_a_larger_batch(B):
    """The buffers of the largest batch serve the smaller ones, with the same results."""
    big = Gated(B, 2000, 264, 520)
    for T in (1, 33, 64, 65, 300, 1024):
        o = Gated(B, T, 264, 520, seed=T)
        o.run()
        want = o.out()
        o.ws, o.bws = big.ws, big.bws
        o.run()
        assert all(torch.equal(a, b) for a, b in zip(o.out(), want))


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
def test_no_tokens(B, dt):
    o = Gated(B, 0, 72, 100, dt)
    o.run()
    torch.cuda.synchronize()
    assert all(bool((g == 0).all()) for g in o.g.values())


@pytest.mark.parametrize("T,d,H,dt", [(3, 40, 33, B16), (33, 72, 100, B16), (130, 264, 200, B16), (517, 1000, 1304, B16), (70, 100, 50, F32)], ids=str)
def test_nothing_beyond_the_arrays_is_read_or_written(B, T, d, H, dt):
    """Every array in the middle of one filled with NaN, or with a mark where it is an output."""
    o = Gated(B, T, d, H, dt)
    o.run()
    want = o.out()

    def inside(t, fill):
        pad = 64 * 1024
        whole = torch.full((t.numel() + 2 * pad,), fill, dtype=t.dtype, device="cuda")
        mid = whole[pad:pad + t.numel()].view(t.shape)
        mid.copy_(t)
        return mid, whole

    wholes = []
    for n in ("x", "add", "dy", "dadd"):
        setattr(o, n, inside(getattr(o, n), float("nan"))[0])
    o.w = {n: inside(t, float("nan"))[0] for n, t in o.w.items()}
    for n in ("y", "dx"):
        t, whole = inside(getattr(o, n), 5.0)
        setattr(o, n, t)
        wholes.append((t, whole))
    for n in list(o.g):
        o.g[n], whole = inside(o.g[n], 5.0)
        wholes.append((o.g[n], whole))
    o.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(o.out(), want))
    for t, whole in wholes:
        pad = (whole.numel() - t.numel()) // 2
        assert bool((whole[:pad] == 5).all()) and bool((whole[pad + t.numel():] == 5).all())
    x, sc = inside(o.x.detach().clone(), float("nan"))[0], torch.empty(T, device="cuda")
    cfg = B.make_norm_config(T, d, 1e-5, NAME[dt])
    weight = inside(rand((d,), 3, 1.0, dt), float("nan"))[0]
    s, n = inside(x, 5.0), inside(x, 5.0)
    q = torch.full((T * d + 512,), 1.0, device="cuda").to(torch.float8_e4m3fn)
    B.slicemoe_add_rmsnorm(cfg, x, o.add, weight, s[0], n[0], y_quantized=q[256:256 + T * d].view(T, d), y_scale=sc)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(n[0]).all()) and bool((q[:256].float() == 1).all()) and bool((q[256 + T * d:].float() == 1).all())
    for t, whole in (s, n):
        assert bool((whole[:64 * 1024] == 5).all()) and bool((whole[64 * 1024 + t.numel():] == 5).all())


@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 700])
def test_a_row_that_is_not_finite_stays_alone(B, T, dt):
    o = Gated(B, T, 264, 300, dt)
    o.run()
    want = o.out()
    for bad in (float("nan"), float("inf")):
        keep = o.x.clone()
        o.x[7, 3] = bad
        o.run()
        torch.cuda.synchronize()
        others = torch.arange(T, device="cuda") != 7
        assert torch.equal(o.y[others], want[0][others]) and torch.equal(o.dx[others], want[1][others])
        assert not bool(torch.isfinite(o.y[7]).all()) and not bool(torch.isfinite(o.g["Wg"]).all())
        o.x.copy_(keep)
    o.run()
    assert all(torch.equal(a, b) for a, b in zip(o.out(), want))


def test_saturated_gates(B):
    """Gates far from zero: silu(g) = g or -0, no overflow of the exponential."""
    T, d, H = 64, 64, 64
    for dt in (B16, F32):
        for rows in (T, 200):
            x = torch.ones((rows, d), dtype=dt, device="cuda")
            w = {"Wg": torch.full((d, H), 30.0, dtype=dt, device="cuda"), "Wu": torch.full((d, H), 1.0, dtype=dt, device="cuda"),
                 "Wd": torch.full((H, d), 1.0 / 64, dtype=dt, device="cuda")}
            w["Wg"][:, 1::2] = -30.0
            cfg = B.make_gated_config(rows, d, H, NAME[dt])
            y, dx, g = torch.empty_like(x), torch.empty_like(x), {n: torch.empty_like(t) for n, t in w.items()}
            B.slicemoe_gated_ffn(cfg, x, w, y, space(B.slicemoe_gated_ffn_workspace_bytes(cfg)))
            B.slicemoe_gated_ffn_backward(cfg, x, w, x, dx, g, space(B.slicemoe_gated_ffn_backward_workspace_bytes(cfg)))
            for name, (v, e) in R.gated(x, w, None, dt, x, None).items():
                R.within({"y": y, "d_x": dx}.get(name, g.get(name)), v, e, name)


def test_offsets_beyond_32_bits(B):
    """Arrays of more than 2^32 bytes and 2^31 elements: the last rows, and a contraction over all of them."""
    T, d = 560_000, 4096
    cfg = B.make_norm_config(T, d, 1e-5, "bf16")
    x, w = torch.empty((T, d), dtype=B16, device="cuda"), rand((d,), 1)
    x[: T // 2].normal_()
    x[T // 2:].normal_()
    s, y = torch.empty_like(x), torch.empty_like(x)
    B.slicemoe_add_rmsnorm(cfg, x, x, w, s, y)
    for rows in (slice(0, 3), slice(T - 3, T), slice(524_280, 524_295)):
        rs, ry, bs, by = R.norm_forward(x[rows], x[rows], w, 1e-5, B16)
        R.within(s[rows], rs, bs, "sum")
        R.within(y[rows], ry, by, "y")
    dw = torch.empty(d, device="cuda")
    B.slicemoe_add_rmsnorm_backward(cfg, s, w, y, x, dw, space(B.slicemoe_add_rmsnorm_backward_workspace_bytes(cfg)))
    rx, _, bx, _ = R.norm_backward(s[-3:], w, y[-3:], None, 1e-5, B16)
    R.within(x[-3:], rx, bx, "d_x")
    del s, x
    norm = torch.empty(1, device="cuda")
    y.fill_(1.0)
    y[-1, -1] = -3.0
    B.slicemoe_clip_grads([y], 1.0, norm, space(B.slicemoe_clip_grads_workspace_bytes([y])), out=[y])
    want = (T * d - 1 + 9) ** 0.5
    assert abs(float(norm) - want) <= want * 2.0 ** -23
    assert abs(float(y[-1, -1]) * want + 3) <= 3 * 2.0 ** -7 and abs(float(y[T // 2, 5]) * want - 1) <= 2.0 ** -7
    del y
    torch.cuda.empty_cache()
    T, d, H = 1_100_000, 2048, 40
    gcfg = B.make_gated_config(T, d, H, "bf16")
    gw = {"Wg": rand((d, H), 1, d ** -0.5), "Wu": rand((d, H), 2, d ** -0.5), "Wd": rand((H, d), 3, H ** -0.5)}
    x = torch.empty((T, d), dtype=B16, device="cuda").normal_()
    y = torch.empty_like(x)
    B.slicemoe_gated_ffn(gcfg, x, gw, y, torch.empty(B.slicemoe_gated_ffn_workspace_bytes(gcfg), dtype=torch.uint8, device="cuda"), addend=x)
    dx, g = torch.empty_like(x), {n: torch.empty_like(t) for n, t in gw.items()}
    B.slicemoe_gated_ffn_backward(gcfg, x, gw, y, dx, g, torch.empty(B.slicemoe_gated_ffn_backward_workspace_bytes(gcfg), dtype=torch.uint8, device="cuda"))
    last = slice(T - 40, T)
    ref = R.gated(x[last], gw, x[last], B16, y[last], None)
    R.within(y[last], *ref["y"], "y")
    R.within(dx[last], *ref["d_x"], "d_x")
    # all rows: dWg in 64 bits, chunk by chunk
    Wg, Wu, Wd = (gw[n].double() for n in ("Wg", "Wu", "Wd"))
    want = torch.zeros((d, H), dtype=torch.float64, device="cuda")
    for a in range(0, T, 100_000):
        xc, yc = x[a:a + 100_000].double(), y[a:a + 100_000].double()
        gate, up = xc @ Wg, xc @ Wu
        sg = torch.sigmoid(gate)
        want += xc.t() @ ((yc @ Wd.t()) * up * (sg + gate * sg * (1 - sg)))
    # the rounding of dg to bf16, 2^-8 of each of 1.1 million terms of either sign, and of the result
    assert float((g["Wg"].double() - want).norm()) <= 3 * 2.0 ** -8 * float(want.norm())


def test_arrays_of_another_device_are_refused(B, monkeypatch):
    """With another device current, kernels would reach for this one's memory from there: every call ends in the binding.  (The current
    device is what the binding is told; nothing is launched.)"""
    o = Gated(B, 40, 64, 96)
    ncfg, v = B.make_norm_config(40, 64), torch.empty(64, device="cuda")
    nws, norm = space(B.slicemoe_add_rmsnorm_backward_workspace_bytes(ncfg)), torch.full((1,), 7.0, device="cuda")
    q8 = B.quantize_gated_weights(o.cfg, o.w)
    x8, sc = torch.zeros((40, 64), dtype=torch.float8_e4m3fn, device="cuda"), torch.ones(40, device="cuda")
    cws = space(B.slicemoe_clip_grads_workspace_bytes([o.x]))
    before = [t.clone() for t in (*o.out(), norm, v)]
    held = torch.cuda.current_stream()
    calls = [lambda: B.slicemoe_add_rmsnorm(ncfg, o.x, None, o.w["Wg"][0], None, o.y), o.run, lambda: o.run(held),
             lambda: B.slicemoe_add_rmsnorm_backward(ncfg, o.x, o.w["Wg"][0], o.dy, o.dx, v, nws),
             lambda: B.slicemoe_gated_ffn_backward(o.cfg, o.x, o.w, o.dy, o.dx, o.g, o.bws),
             lambda: B.slicemoe_gated_ffn_quantized(o.cfg, x8, sc, q8, o.y, o.ws), lambda: B.quantize_gated_weights(o.cfg, o.w),
             lambda: B.slicemoe_clip_grads([o.x], 1.0, norm, cws), lambda: B.slicemoe_clip_grads([], 1.0, norm, cws)]
    with monkeypatch.context() as m:
        m.setattr(B, "_device", lambda: 1)
        for call in calls:
            with pytest.raises(ValueError, match="current device is 1"):
                call()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((*o.out(), norm, v), before))
    for call in calls[:1] + calls[3:]:
        call()   # the same calls where they belong
    torch.cuda.synchronize()


def test_few_fp32_rows_captured(B):
    test_captured_into_a_graph(B, 50, F32)


@pytest.mark.parametrize("T,d,H", [(40, 131, 70), (64, 300, 257)])
def test_few_fp32_rows_in_place(B, T, d, H):
    test_gated_outputs_in_place_of_inputs(B, T, d, H, F32)


@pytest.mark.parametrize("T,d,H", [(1, 9, 5), (33, 71, 101), (64, 136, 259)])
def test_few_fp32_rows_next_to_memory_that_must_not_be_read(B, T, d, H):
    test_nothing_beyond_the_arrays_is_read_or_written(B, T, d, H, F32)
