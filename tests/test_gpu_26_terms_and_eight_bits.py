"""The gated network's two other forms as a program uses them: fp32 rows beyond the limits of the fp32 instruction (products of bf16
terms) and 8-bit operands.  Captured into a graph, on another stream, in place, next to memory that must not be read, with rows that are
not finite, and at offsets beyond 32 bits."""
import pytest
import torch

import block_reference as R

pytestmark = pytest.mark.gpu

B16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
PAD = 64 * 1024


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rand(shape, seed, scale=1.0, dt=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def space(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def inside(t, fill=None):
    """t in the middle of an array of `fill` (NaN where none is given), and that array as bytes."""
    whole = torch.empty(t.numel() + 2 * PAD, dtype=t.dtype, device="cuda")
    if fill is not None:
        whole.fill_(fill)
    elif t.dtype == F8:
        whole.view(torch.uint8).fill_(0x7f)
    else:
        whole.fill_(float("nan"))
    mid = whole[PAD:PAD + t.numel()].view(t.shape)
    mid.copy_(t)
    return mid, whole


def untouched(mid, whole, fill):
    rest = torch.cat([whole[:PAD], whole[PAD + mid.numel():]])
    return bool((rest == fill).all())


class Terms:
    """fp32, both directions."""

    def __init__(self, B, T, d, H, seed=0):
        self.B, self.cfg = B, B.make_gated_config(T, d, H, "f32")
        self.w = {"Wg": rand((d, H), seed + 1, d ** -0.5), "Wu": rand((d, H), seed + 2, d ** -0.5), "Wd": rand((H, d), seed + 3, H ** -0.5)}
        self.x, self.add, self.dy, self.dadd = (rand((T, d), seed + 4 + i) for i in range(4))
        self.ws, self.bws = space(B.slicemoe_gated_ffn_workspace_bytes(self.cfg)), space(B.slicemoe_gated_ffn_backward_workspace_bytes(self.cfg))
        self.y, self.dx = torch.full_like(self.x, 7.0), torch.full_like(self.x, 7.0)
        self.g = {n: torch.full_like(t, 7.0) for n, t in self.w.items()}

    def run(self, stream=None):
        self.B.slicemoe_gated_ffn(self.cfg, self.x, self.w, self.y, self.ws, addend=self.add, stream=stream)
        self.B.slicemoe_gated_ffn_backward(self.cfg, self.x, self.w, self.dy, self.dx, self.g, self.bws, addend=self.dadd, stream=stream)

    def inputs(self):
        return [self.x, self.add, self.dy, self.dadd]

    def out(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.y, self.dx, *self.g.values())]

    def refill(self, seed):
        for i, t in enumerate(self.inputs()):
            t.copy_(rand(t.shape, seed + i))


class Eight:
    """8-bit operands; the rows come from the norm."""

    def __init__(self, B, T, d, H, seed=0):
        self.B, self.cfg, self.ncfg = B, B.make_gated_config(T, d, H, "bf16"), B.make_norm_config(T, d, 1e-5, "bf16")
        w = {"Wg": rand((d, H), seed + 1, d ** -0.5, B16), "Wu": rand((d, H), seed + 2, d ** -0.5, B16), "Wd": rand((H, d), seed + 3, H ** -0.5, B16)}
        self.q = B.quantize_gated_weights(self.cfg, w)
        self.nw = 1 + rand((d,), seed + 6, 0.1).to(B16)
        self.x, self.add = rand((T, d), seed + 4, 1.0, B16), rand((T, d), seed + 5, 1.0, B16)
        self.xq, self.xs = torch.empty((T, d), dtype=F8, device="cuda"), torch.empty(T, device="cuda")
        self.ws, self.y = space(B.slicemoe_gated_ffn_quantized_workspace_bytes(self.cfg)), torch.full_like(self.x, 7.0)

    def norm(self, stream=None):
        self.B.slicemoe_add_rmsnorm(self.ncfg, self.x, None, self.nw, None, None, y_quantized=self.xq, y_scale=self.xs, stream=stream)

    def network(self, stream=None):
        self.B.slicemoe_gated_ffn_quantized(self.cfg, self.xq, self.xs, self.q, self.y, self.ws, addend=self.add, stream=stream)

    def run(self, stream=None):
        self.norm(stream)
        self.network(stream)

    def out(self):
        torch.cuda.synchronize()
        return [self.xq.view(torch.uint8).clone(), self.xs.clone(), self.y.clone()]

    def refill(self, seed):
        for i, t in enumerate((self.x, self.add)):
            t.copy_(rand(t.shape, seed + i, 1.0, B16))


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


TERMS = [(65, 136, 100), (257, 101, 130), (300, 257, 101), (700, 512, 260)]
EIGHT = [(T, d, H) for T, d, H in ((1, 16, 33), (31, 272, 101), (32, 272, 1), (33, 16, 101), (63, 272, 33), (64, 16, 1), (65, 272, 101), (300, 144, 515))]
ALL = [(Terms, s) for s in TERMS] + [(Eight, s) for s in EIGHT]
IDS = [f"{k.__name__}-{s[0]}-{s[1]}-{s[2]}" for k, s in ALL]


@pytest.mark.parametrize("kind,size", ALL, ids=IDS)
def test_captured(B, kind, size):
    net, live = kind(B, *size), kind(B, *size)
    live.run()   # (kernels are loaded before the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.run()
    for k in range(4):
        for o in (net, live):
            o.refill(100 * k)
        live.run()
        want = live.out()
        graph.replay()
        assert same(net.out(), want), k
        assert float(torch.randn(1000, device="cuda").sum()) != 0   # the program's own eager work


@pytest.mark.parametrize("kind,size", ALL, ids=IDS)
def test_on_another_stream(B, kind, size):
    net, other, side = kind(B, *size), kind(B, *size), torch.cuda.Stream()
    net.run()
    want = net.out()
    other.run(stream=side)
    assert same(other.out(), want)


@pytest.mark.parametrize("T,d,H", TERMS)
def test_terms_in_place(B, T, d, H):
    net = Terms(B, T, d, H)
    net.run()
    want = net.out()
    for target in range(2):
        x, add = net.x.clone(), net.add.clone()
        to = (x, add)[target]
        B.slicemoe_gated_ffn(net.cfg, x, net.w, to, net.ws, addend=add)
        assert torch.equal(to, want[0])
        dy, dadd = net.dy.clone(), net.dadd.clone()
        to = (dy, dadd)[target]
        B.slicemoe_gated_ffn_backward(net.cfg, net.x, net.w, dy, to, net.g, net.bws, addend=dadd)
        assert same([to, *net.g.values()], want[1:])


@pytest.mark.parametrize("T,d,H", EIGHT)
def test_eight_bits_in_place(B, T, d, H):
    net = Eight(B, T, d, H)
    net.run()
    want = net.out()[2]
    net.y = net.add
    net.network()
    assert torch.equal(net.out()[2], want)


@pytest.mark.parametrize("T,d,H", TERMS)
def test_terms_next_to_memory_that_must_not_be_read(B, T, d, H):
    net = Terms(B, T, d, H)
    net.run()
    want = net.out()
    for n in ("x", "add", "dy", "dadd"):
        setattr(net, n, inside(getattr(net, n))[0])
    net.w = {n: inside(t)[0] for n, t in net.w.items()}
    outs = {n: inside(getattr(net, n), 5.0) for n in ("y", "dx")}
    net.y, net.dx = outs["y"][0], outs["dx"][0]
    for n in list(net.g):
        outs[n] = inside(net.g[n], 5.0)
        net.g[n] = outs[n][0]
    net.run()
    assert same(net.out(), want) and all(untouched(m, w, 5.0) for m, w in outs.values())


@pytest.mark.parametrize("T,d,H", EIGHT)
def test_eight_bits_next_to_memory_that_must_not_be_read(B, T, d, H):
    net = Eight(B, T, d, H)
    net.run()
    want = net.out()
    v, e = R.gated_quantized(net.xq, net.xs, net.q, net.add)
    R.within(net.y, v, e, "y")
    net.q = {n: inside(t)[0] for n, t in net.q.items()}
    net.x, net.add, net.nw = (inside(t)[0] for t in (net.x, net.add, net.nw))
    (net.xq, rows), (net.xs, scales) = inside(net.xq), inside(net.xs)   # (NaN around what the norm writes and the network reads)
    net.y, whole = inside(net.y, 5.0)
    net.run()
    assert same(net.out(), want) and untouched(net.y, whole, 5.0)
    assert bool(scales[:PAD].isnan().all()) and bool(scales[PAD + T:].isnan().all())
    raw = rows.view(torch.uint8)
    assert bool((raw[:PAD] == 0x7f).all()) and bool((raw[PAD + T * d:] == 0x7f).all())


@pytest.mark.parametrize("T,d,H", [s for s in EIGHT if s[0] > 8])
def test_eight_bits_a_row_that_is_not_finite_stays_alone(B, T, d, H):
    net = Eight(B, T, d, H)
    net.run()
    want = net.out()[2]
    for bad in (float("nan"), float("inf")):
        keep = net.x.clone()
        net.x[7, 3] = bad
        net.run()
        got = net.out()[2]
        rows = torch.arange(T, device="cuda") != 7
        assert torch.equal(got[rows], want[rows]) and bool(torch.isnan(got[7]).all())
        net.x.copy_(keep)


def test_eight_bits_at_offsets_beyond_32_bits(B):
    """Rows of 4.5 GB, outputs of 9: the first rows, the last, and those around byte 2^32 and element 2^32."""
    T, d, H = 1_100_000, 4096, 24
    w = {"Wg": rand((d, H), 1, d ** -0.5, B16), "Wu": rand((d, H), 2, d ** -0.5, B16), "Wd": rand((H, d), 3, H ** -0.5, B16)}
    cfg, ncfg = B.make_gated_config(T, d, H, "bf16"), B.make_norm_config(T, d, 1e-5, "bf16")
    q = B.quantize_gated_weights(cfg, w)
    x = torch.empty((T, d), dtype=B16, device="cuda")
    x[: T // 2].normal_()
    x[T // 2:].normal_()
    xq, xs = torch.empty((T, d), dtype=F8, device="cuda"), torch.empty(T, device="cuda")
    B.slicemoe_add_rmsnorm(ncfg, x, None, torch.ones(d, dtype=B16, device="cuda"), None, None, y_quantized=xq, y_scale=xs)
    y = torch.full_like(x, 7.0)
    B.slicemoe_gated_ffn_quantized(cfg, xq, xs, q, y, torch.empty(B.slicemoe_gated_ffn_quantized_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), addend=x)
    at = 2 ** 32 // d
    for rows in (slice(0, 5), slice(at // 2 - 5, at // 2 + 5), slice(at - 5, at + 5), slice(T - 40, T)):
        _, ry, _, by = R.norm_forward(x[rows], None, torch.ones(d, device="cuda"), 1e-5, F32)
        top = ry.abs().amax(1)
        R.within(xs[rows], top / 448, (top / 448) * (98 * R.U), "scale")
        step = torch.maximum(2.0 ** -4 * ry.abs(), 2.0 ** -10 * (top / 448)[:, None])
        R.within(xq[rows].float().double() * xs[rows].double()[:, None], ry, step * (1 + 2.0 ** -10) + by, "values")
        v, e = R.gated_quantized(xq[rows], xs[rows], q, x[rows])
        R.within(y[rows], v, e, "y")
