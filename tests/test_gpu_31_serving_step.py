"""The layer for few tokens, the norms around it and the microscaled network as a program uses them: a decoding step of all of them, captured and
replayed, on other streams, two at once, next to memory that is not theirs, and past 32-bit offsets."""
import pytest
import torch

import block_norm_reference as N
import block_reference as R
import mx_reference as M
from common import make_inputs
from paper_2510_04286_amd import workload as wl

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rand(shape, seed, scale=1.0, dt=B16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dt).cuda()


def space(n):
    return torch.full((max(256, n),), 0xFF, dtype=torch.uint8, device="cuda")


class Step:
    """h = norm of the stream behind a block; stream: its sum.  Then layer and network on h, their sum into the next norm."""

    def __init__(self, B, T, bits, gate="channel", layer="lm", seed=0):
        shape = wl.CONFIGS[layer].scaled(T)
        s, _, w = make_inputs(shape)
        self.B, self.T, self.d, self.H, self.bits = B, T, s.d, 700, bits
        self.cfg = B.config_of(s)
        self.w = {"packed": B.pack(self.cfg, B.weights_to_device(w, "bf16"))["packed"]}
        d, H = self.d, self.H
        self.net = B.quantize_gated_weights_mx({"Wg": rand((d, H), 1, d ** -0.5), "Wu": rand((d, H), 2, d ** -0.5), "Wd": rand((H, d), 3, H ** -0.5)})
        self.ncfg, self.gcfg = B.make_block_norm_config(T, d, 1e-5, 0.75, gate), B.make_gated_config(T, d, H)
        self.branch, self.stream = rand((T, d), seed + 4, 0.3), rand((T, d), seed + 5, 2.0)
        self.gate = {None: None, "channel": rand((d,), 6), "token": rand((T, d), 7)}[gate]
        self.post, self.pre = rand((d,), 8, 0.1) + 1, rand((d,), 9, 0.1) + 1
        self.h, self.sum, self.out, self.last, self.y = (torch.empty_like(self.branch) for _ in range(5))
        self.mx = space(B.slicemoe_mx_bytes(B.make_mx_config(T, d, bits)))
        self.ws = space(B.slicemoe_gated_ffn_mx_workspace_bytes(self.gcfg, bits))
        self.idx = torch.empty((T * s.S, s.k), dtype=torch.int32, device="cuda")
        self.p = torch.empty((T * s.S, s.k), device="cuda")

    def run(self, stream=None):
        B = self.B
        B.slicemoe_block_norm(self.ncfg, self.branch, self.post, self.gate, self.stream, self.pre, self.sum, self.h, y_mx=self.mx, y_bits=self.bits, stream=stream)
        B.slicemoe_forward_few(self.cfg, self.h, self.w, self.out, topk_idx=self.idx, topk_p=self.p, stream=stream)
        B.slicemoe_gated_ffn_mx(self.gcfg, self.bits, self.mx, self.net, self.out, self.ws, addend=self.out, stream=stream)
        B.slicemoe_block_norm(self.ncfg, self.out, self.post, self.gate, self.sum, self.pre, self.last, self.y, stream=stream)

    def outputs(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.sum, self.h, self.idx, self.p, self.out, self.last, self.y)]

    def wipe(self):
        for t in (self.sum, self.h, self.idx, self.p, self.out, self.last, self.y):
            t.zero_()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T,gate", [(1, "channel"), (5, "token"), (16, None), (33, "channel"), (64, "token")])
def test_a_decoding_step(B, T, gate, bits):
    """Each operator's output from the ones that went into it, against the plain forms."""
    o = Step(B, T, bits, gate)
    o.run()
    s, h, idx, p, out, last, y = o.outputs()
    ref = N.forward(o.branch, o.post, o.gate, o.stream, o.pre, 0.75, 1e-5, B16)
    R.within(s, *ref["sum"], "sum")
    R.within(h, *ref["y"], "h")
    ws, layer = B.alloc_workspace(o.cfg), torch.empty_like(h)
    _, _, w = make_inputs(wl.CONFIGS["lm"].scaled(T))
    whole = B.pack(o.cfg, B.weights_to_device(w, "bf16"))
    B.slicemoe_forward(o.cfg, h, whole, layer, ws)
    rows = torch.empty((T, o.d), dtype=F32, device="cuda")
    B.slicemoe_mx_dequantize(B.make_mx_config(T, o.d, o.bits, "f32"), o.mx, rows)
    vals = []
    for n, (r, c) in (("Wg", (o.H, o.d)), ("Wu", (o.H, o.d)), ("Wd", (o.d, o.H))):
        v = torch.empty((r, c), dtype=F32, device="cuda")
        B.slicemoe_mx_dequantize(B.make_mx_config(r, c, 4, "f32"), o.net[n], v)
        vals.append(v.double().cpu())
    R.within(out, *M.gated(rows.double().cpu(), *vals, layer, bits), "layer and network")
    ref = N.forward(out, o.post, o.gate, s, o.pre, 0.75, 1e-5, B16)
    R.within(last, *ref["sum"], "next sum")
    R.within(y, *ref["y"], "next y")


@pytest.mark.parametrize("T,bits", [(1, 8), (16, 4), (40, 8), (64, 4)])
def test_captured_into_a_graph(B, T, bits):
    net, live = Step(B, T, bits), Step(B, T, bits)
    live.run()   # (kernels are loaded before the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.run()
    for k in range(4):
        for o in (net, live):
            o.branch.copy_(rand(o.branch.shape, 100 + k, 0.3))
            o.stream.copy_(rand(o.stream.shape, 200 + k, 2.0))
        live.run()
        want = live.outputs()
        net.wipe()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(net.outputs(), want)), k
        assert float(torch.randn(1000, device="cuda").sum()) != 0   # the program's own eager work


@pytest.mark.parametrize("T,bits", [(300, 8), (700, 4)])
def test_products_captured_into_a_graph(B, T, bits):
    """Prompts: shares of the contraction and their addition too."""
    d, H = 512, 5000
    w = B.quantize_gated_weights_mx({"Wg": rand((d, H), 1, d ** -0.5), "Wu": rand((d, H), 2, d ** -0.5), "Wd": rand((H, d), 3, H ** -0.5)})
    cfg, xc = B.make_gated_config(T, d, H), B.make_mx_config(T, d, bits)
    sets = []
    for _ in range(2):
        x = rand((T, d), 4)
        sets.append((x, space(B.slicemoe_mx_bytes(xc)), torch.empty_like(x), space(B.slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits))))

    def run(x, mx, y, ws):
        B.slicemoe_mx_quantize(xc, x, mx)
        B.slicemoe_gated_ffn_mx(cfg, bits, mx, w, y, ws, addend=x)

    run(*sets[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*sets[0])
    for k in range(4):
        for x, *_ in sets:
            x.copy_(rand((T, d), 50 + k))
        run(*sets[1])
        sets[0][2].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(sets[0][2], sets[1][2]), k
        assert float(torch.randn(1000, device="cuda").sum()) != 0


def test_two_at_once_on_other_streams(B):
    nets = [Step(B, 40 + 13 * i, 4 * (i + 1), seed=50 * i) for i in range(2)]
    want = []
    for o in nets:
        o.run()
        want.append(o.outputs())
    streams = [torch.cuda.Stream() for _ in nets]
    for _ in range(3):
        for o in nets:
            o.wipe()
        torch.cuda.synchronize()
        for o, st in zip(nets, streams):
            o.run(stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(nets, want) for a, b in zip(o.outputs(), w))
    graphs = []
    for o in nets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o.run()
        graphs.append(g)
    for _ in range(3):
        for o in nets:
            o.wipe()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(nets, want) for a, b in zip(o.outputs(), w))


def inside(t, fill):
    """t in the middle of a longer array filled with `fill`; the array."""
    pad = 64 * 1024
    whole = torch.full((t.numel() + 2 * pad,), fill, dtype=t.dtype, device="cuda")
    mid = whole[pad:pad + t.numel()].view(t.shape)
    mid.copy_(t)
    return mid, whole


def untouched(pairs):
    for t, whole in pairs:
        pad = (whole.numel() - t.numel()) // 2
        assert bool((whole[:pad] == whole[0]).all()) and bool((whole[pad + t.numel():] == whole[0]).all())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T", [1, 7, 33, 64])
def test_nothing_beyond_the_arrays_is_read_or_written(B, T, bits):
    o = Step(B, T, bits, "token")
    o.run()
    want = o.outputs()
    for n in ("branch", "stream", "gate", "post", "pre"):
        setattr(o, n, inside(getattr(o, n), float("nan"))[0])
    o.w = {"packed": inside(o.w["packed"], 0xFF)[0]}
    o.net = {n: inside(t, 0xFF)[0] for n, t in o.net.items()}
    pairs = []
    for n, fill in (("h", 5.0), ("sum", 5.0), ("out", 5.0), ("last", 5.0), ("y", 5.0), ("mx", 0xFF), ("ws", 0xFF), ("idx", 7), ("p", 7.0)):
        t, whole = inside(getattr(o, n), fill)
        setattr(o, n, t)
        pairs.append((t, whole))
    o.run()
    assert all(torch.equal(a, b) for a, b in zip(o.outputs(), want))
    untouched(pairs)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T,K,N,dt", [(3, 40, 33, B16), (70, 300, 129, B16), (130, 2600, 264, B16), (300, 700, 1000, F32), (517, 1000, 520, B16), (70, 100, 50, F32)], ids=str)
def test_products_stay_within_their_arrays(B, T, K, N, dt, bits):
    x, w, add = rand((T, K), 1, 1.0, dt), rand((N, K), 2, 0.2, dt), rand((T, N), 3, 1.0, dt)
    cfg = B.make_mx_product_config(T, K, N, bits, dt)
    xc = B.make_mx_config(T, K, bits, dt)
    xm, wm, y = space(B.slicemoe_mx_bytes(xc)), B.quantize_mx(w, 4), torch.empty_like(add)
    ws = space(B.slicemoe_mx_product_workspace_bytes(cfg))

    def run():
        B.slicemoe_mx_quantize(xc, x, xm)
        B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=add)
        torch.cuda.synchronize()
        return y.clone()

    want = run()
    pairs = []
    x, add, wm = inside(x, float("nan"))[0], inside(add, float("nan"))[0], inside(wm, 0xFF)[0]
    for name, fill in (("xm", 0xFF), ("ws", 0xFF), ("y", 5.0)):
        pairs.append(inside(locals()[name], fill))
    xm, ws, y = (p[0] for p in pairs)
    assert torch.equal(run(), want)
    untouched(pairs)
    back, whole = inside(torch.empty_like(x), 5.0)
    B.slicemoe_mx_dequantize(xc, xm, back)
    torch.cuda.synchronize()
    untouched([(back, whole)])


def test_a_workspace_of_a_larger_batch(B):
    d, H = 520, 3000
    w = B.quantize_gated_weights_mx({"Wg": rand((d, H), 1, d ** -0.5), "Wu": rand((d, H), 2, d ** -0.5), "Wd": rand((H, d), 3, H ** -0.5)})
    for bits in (4, 8):
        big = space(B.slicemoe_gated_ffn_mx_workspace_bytes(B.make_gated_config(2000, d, H), bits))
        for T in (1, 33, 64, 65, 200, 513, 1024):
            x, cfg = rand((T, d), T), B.make_gated_config(T, d, H)
            xm, got = B.quantize_mx(x, bits), []
            for ws in (big, space(B.slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits))):
                y = torch.empty_like(x)
                B.slicemoe_gated_ffn_mx(cfg, bits, xm, w, y, ws, addend=x)
                got.append(y)
            assert torch.equal(*got)


def test_offsets_beyond_32_bits(B):
    """Packed rows and results of more than 2^32 bytes: the last rows are those of a small batch."""
    free, _ = torch.cuda.mem_get_info()
    if free < 80 * 2 ** 30:
        pytest.skip("needs 80 GiB")
    last, cols = 48, 20000
    rows = 2 ** 32 // cols + 1000
    rows += -rows % 32
    small = rand((last, cols), 1)
    for bits in (8, 4):
        big = torch.zeros((rows, cols), dtype=B16, device="cuda")
        big[-last:] = small
        mx = B.quantize_mx(big, bits)
        back = torch.full_like(big, 7.0)
        B.slicemoe_mx_dequantize(B.make_mx_config(rows, cols, bits), mx, back)
        want = torch.empty_like(small)
        sm = B.quantize_mx(small, bits)
        B.slicemoe_mx_dequantize(B.make_mx_config(last, cols, bits), sm, want)
        assert torch.equal(back[-last:], want) and bool((back[:64] == 0).all()) and bool((back[rows // 2:rows // 2 + 64] == 0).all())
        del back, big
        wm = B.quantize_mx(rand((40, cols), 2, 0.1), 4)
        y = torch.empty((rows, 40), dtype=B16, device="cuda")
        B.slicemoe_mx_product(B.make_mx_product_config(rows, cols, 40, bits), mx, wm, y, space(B.slicemoe_mx_product_workspace_bytes(B.make_mx_product_config(rows, cols, 40, bits))))
        ref, bound = M.product(M.to_mx(small, bits), M.to_mx(rand((40, cols), 2, 0.1), 4), None, B16, bits)
        R.within(y[-last:], ref, bound, "y")
        assert bool((y[:-last] == 0).all())
        del y, mx
    # results past 2^32 bytes
    T, K, N = 2 ** 31 // 8192 + 500, 64, 8192
    x, w = rand((last, K), 3), rand((N, K), 4, 0.2)
    big = torch.zeros((T, K), dtype=B16, device="cuda")
    big[-last:] = x
    cfg = B.make_mx_product_config(T, K, N, 4)
    y = torch.empty((T, N), dtype=B16, device="cuda")
    B.slicemoe_mx_product(cfg, B.quantize_mx(big, 4), B.quantize_mx(w, 4), y, space(B.slicemoe_mx_product_workspace_bytes(cfg)))
    ref, bound = M.product(M.to_mx(x, 4), M.to_mx(w, 4), None, B16, 4)
    R.within(y[-last:], ref, bound, "y")
    assert bool((y[:100] == 0).all()) and bool((y[-last - 100:-last] == 0).all())


def test_tensors_of_another_kind_are_refused(B):
    o = Step(B, 3, 8)
    with pytest.raises(ValueError):
        B.slicemoe_block_norm(o.ncfg, o.branch.t(), o.post, o.gate, o.stream, o.pre, o.sum, o.h)
    with pytest.raises(TypeError):
        B.slicemoe_block_norm(o.ncfg, o.branch.float(), o.post, o.gate, o.stream, o.pre, o.sum, o.h)
    with pytest.raises(TypeError):
        B.slicemoe_block_norm(o.ncfg, o.branch.cpu(), o.post, o.gate, o.stream, o.pre, o.sum, o.h)
    with pytest.raises(ValueError):
        B.slicemoe_gated_ffn_mx(o.gcfg, 8, o.mx[:-256], o.net, o.out, o.ws)
    with pytest.raises(ValueError):
        B.slicemoe_gated_ffn_mx(o.gcfg, 8, o.mx, dict(o.net, Wd=o.net["Wd"][:-1]), o.out, o.ws)
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_gated_ffn_mx(o.gcfg, 6, o.mx, o.net, o.out, o.ws)
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_gated_ffn_mx(o.gcfg, 8, o.mx, o.net, o.out, o.ws[:256])
    with pytest.raises(B.SliceMoEError):
        B.slicemoe_forward_few(B.make_config(65, 512, 8, 2, 16, 256), rand((65, 512), 1), o.w, torch.empty((65, 512), dtype=B16, device="cuda"))
