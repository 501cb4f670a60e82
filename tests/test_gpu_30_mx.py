"""Microscaled values: conversion, products and the gated network on them, against 64 bits."""
import pytest
import torch

import block_reference as R
import mx_reference as M

pytestmark = pytest.mark.gpu

B16, F32 = torch.bfloat16, torch.float32
NAME = {B16: "bf16", F32: "f32"}


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    assert torch.cuda.is_available()
    return binding


def rand(shape, seed, dt, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dt).cuda()


def pack(B, t, bits, transposed=False):
    """The packed matrix, in a buffer that held something else."""
    rows, cols = t.shape[::-1] if transposed else t.shape
    cfg = B.make_mx_config(rows, cols, bits, NAME[t.dtype], transposed)
    mx = torch.full((B.slicemoe_mx_bytes(cfg),), 0xA5, dtype=torch.uint8, device="cuda")
    B.slicemoe_mx_quantize(cfg, t.contiguous(), mx)
    return cfg, mx


def unpack(B, cfg, mx):
    out = torch.empty((cfg.cols, cfg.rows) if cfg.transposed else (cfg.rows, cfg.cols), dtype=F32, device="cuda")
    wide = B.make_mx_config(cfg.rows, cfg.cols, cfg.bits, "f32", bool(cfg.transposed))
    B.slicemoe_mx_dequantize(wide, mx, out)
    return out


def from_layout(mx, rows, cols, bits):
    """Values and scale bytes by the layout that the header states."""
    mx = mx.cpu()
    tk = -(-cols // 256)
    tiles = -(-rows // 32) * tk
    r, c = torch.meshgrid(torch.arange(rows), torch.arange(cols), indexing="ij")
    tile, i, b = (r // 32) * tk + c // 256, r % 32, c // 32 % 8
    ks, h, p = b // 2, b % 2, 16 * (c // 4 % 2) + 4 * (c // 8 % 4) + c % 4
    if bits == 4:
        byte = mx[tile * 4096 + 1024 * ks + 16 * (i + 32 * h) + p // 2].long()
        code = torch.where(p % 2 == 1, byte >> 4, byte & 15)
        v = M.GRID[4][code & 7] * torch.where(code & 8 > 0, -1.0, 1.0).double()
    else:
        v = mx[tile * 8192 + 2048 * ks + 1024 * h + 16 * (i + 32 * (p // 16)) + p % 16].view(torch.float8_e4m3fn).double()
    scale = mx[tiles * 1024 * bits + tile * 256 + 4 * (i + 32 * h) + ks].long()
    return v * torch.where(scale == 255, float("nan"), torch.exp2((scale - 127).double())), scale


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (32, 256), (33, 257), (31, 255), (70, 1000), (257, 513), (5, 4099), (200, 768)])
def test_values_are_the_nearest(B, rows, cols, dt, bits):
    """Bit for bit: magnitudes over many powers of two, ties, blocks of zeros."""
    x = rand((rows, cols), rows + cols, F32) * torch.exp2(torch.randint(-20, 20, (rows, cols), generator=torch.Generator().manual_seed(1)).float()).cuda()
    ties = torch.randint(-24, 25, (rows, cols), generator=torch.Generator().manual_seed(2)).float().cuda() / 4     # every grid value, and the middles
    x = torch.where(torch.arange(rows, device="cuda")[:, None] % 3 == 1, ties, x).to(dt)
    x[rows // 2, : min(32, cols)] = 0
    cfg, mx = pack(B, x, bits)
    ref = M.to_mx(x, bits)
    got, scale = from_layout(mx, rows, cols, bits)
    assert torch.equal(got, ref)
    assert torch.equal(unpack(B, cfg, mx).double().cpu(), ref)
    cfg_t, mx_t = pack(B, x.t().contiguous(), bits, transposed=True)
    assert torch.equal(mx_t, mx)
    assert torch.equal(unpack(B, cfg_t, mx_t).t().double().cpu(), ref)
    if dt == B16:
        out = torch.empty_like(x)
        B.slicemoe_mx_dequantize(cfg, mx, out)
        assert torch.equal(out.double().cpu(), ref)
    # a second pass changes nothing: the values stand for themselves
    assert torch.equal(M.to_mx(ref, bits), ref)
    # past the last column: zeros
    tk = -(-cols // 256)
    whole, _ = from_layout(mx, rows, tk * 256, bits)
    assert bool((whole[:, cols:] == 0).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_ends_of_the_range(B, bits):
    """The smallest and largest numbers, infinities and NaN."""
    x = torch.zeros((8, 64), device="cuda")
    x[0, 3] = 2.0 ** -149
    x[1, 3] = 2.0 ** -126
    x[2, :32] = 3.0e38
    x[3, 5] = float("inf")
    x[4, 40] = float("nan")
    x[5, 7] = -float("inf")
    x[6] = 2.0 ** -127 * 6
    x[6, 9] = 2.0 ** -128
    cfg, mx = pack(B, x, bits)
    got, scale = from_layout(mx, 8, 64, bits)
    fine = [0, 1, 6, 7]
    assert torch.equal(got[fine], M.to_mx(x[fine], bits))
    assert bool(got[2, :32].isfinite().all()) and float((got[2, :32] / 3.0e38 - 1).abs().max()) <= (0.25 if bits == 4 else 2.0 ** -4)
    for r, c in ((3, 0), (4, 32), (5, 0)):      # the block is NaN, the row's other one is not
        assert bool(got[r, c:c + 32].isnan().all()) and bool((got[r, 32 - c:64 - c] == 0).all())
        assert bool((scale[r, c:c + 32] == 255).all())


SHAPES = [(1, 1, 1), (1, 33, 7), (2, 256, 64), (16, 300, 129), (31, 1000, 96), (33, 257, 100), (64, 512, 256), (65, 513, 255), (100, 2000, 333), (128, 64, 40),
          (200, 768, 1000), (257, 511, 257), (300, 1025, 513), (513, 1300, 130), (130, 5000, 264), (257, 2816, 500), (1025, 4096, 130), (4100, 2048, 2050),
          (1, 1, 4097), (17, 300, 4200), (40, 513, 4096), (64, 257, 5003), (16, 4500, 4100), (8200, 300, 1100)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_product(B, T, K, N, dt, bits):
    x, w, add = rand((T, K), 1, dt), rand((N, K), 2, dt, 0.2), rand((T, N), 3, dt)
    cfg = B.make_mx_product_config(T, K, N, bits, NAME[dt])
    (_, xm), (_, wm) = pack(B, x, bits), pack(B, w, 4)
    ws = torch.empty(max(256, B.slicemoe_mx_product_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    for addend in (add, None):
        y = torch.full((T, N), 7.0, dtype=dt, device="cuda")
        B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=addend)
        ref, bound = M.product(M.to_mx(x, bits), M.to_mx(w, 4), addend, dt, bits)
        R.within(y, ref, bound, "y")
    y = add.clone()
    B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=y)      # in place of the addend
    ref, bound = M.product(M.to_mx(x, bits), M.to_mx(w, 4), add, dt, bits)
    R.within(y, ref, bound, "y in place")
    again = add.clone()
    B.slicemoe_mx_product(cfg, xm, wm, again, ws, addend=again)
    assert torch.equal(again, y)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T,d,H", [(1, 1, 1), (1, 40, 33), (2, 256, 256), (16, 512, 1000), (31, 300, 257), (33, 257, 96), (64, 1024, 300), (65, 768, 513), (129, 200, 1100),
                                   (256, 1000, 2047), (300, 513, 100), (520, 264, 800), (20, 300, 8300), (48, 300, 8300), (64, 2100, 8200), (4100, 300, 1100)])
def test_gated_network(B, T, d, H, bits):
    x, add = rand((T, d), 1, B16), rand((T, d), 2, B16)
    w = {"Wg": rand((d, H), 3, B16, d ** -0.5), "Wu": rand((d, H), 4, B16, d ** -0.5), "Wd": rand((H, d), 5, B16, H ** -0.5)}
    packed = B.quantize_gated_weights_mx(w)
    cfg = B.make_gated_config(T, d, H)
    ws = torch.full((B.slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits),), 0xFF, dtype=torch.uint8, device="cuda")
    _, xm = pack(B, x, bits)
    Wg, Wu, Wd = (M.to_mx(w[n].t(), 4) for n in ("Wg", "Wu", "Wd"))
    for addend in (add, None):
        y = torch.full_like(x, 7.0)
        B.slicemoe_gated_ffn_mx(cfg, bits, xm, packed, y, ws, addend=addend)
        ref, bound = M.gated(M.to_mx(x, bits), Wg, Wu, Wd, addend, bits)
        R.within(y, ref, bound, "y")
    y = add.clone()
    B.slicemoe_gated_ffn_mx(cfg, bits, xm, packed, y, ws, addend=y)
    first = torch.empty_like(x)
    B.slicemoe_gated_ffn_mx(cfg, bits, xm, packed, first, ws, addend=add)
    assert torch.equal(y, first)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T", [5, 40, 300])
def test_rows_stay_apart(B, T, bits):
    """A row that holds a NaN is NaN, the others are what they were; rows past the last one in the packed matrices may hold anything."""
    d, H = 300, 200
    x = rand((T, d), 1, B16)
    w = {"Wg": rand((d, H), 3, B16, d ** -0.5), "Wu": rand((d, H), 4, B16, d ** -0.5), "Wd": rand((H, d), 5, B16, H ** -0.5)}
    packed, cfg = B.quantize_gated_weights_mx(w), B.make_gated_config(T, d, H)
    ws = torch.full((B.slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(xm, pw):
        y = torch.empty_like(x)
        B.slicemoe_gated_ffn_mx(cfg, bits, xm, pw, y, ws)
        return y

    _, xm = pack(B, x, bits)
    want = run(xm, packed)
    bad = x.clone()
    bad[T // 2, 7] = float("nan")
    got = run(pack(B, bad, bits)[1], packed)
    keep = torch.arange(T, device="cuda") != T // 2
    assert bool(got[T // 2].isnan().all()) and torch.equal(got[keep], want[keep])

    def spoil(mx, rows, cols, b):
        """0xFF where the rows past the last one lie: NaN scales and values."""
        mx = mx.clone()
        tk = -(-cols // 256)
        tiles = -(-rows // 32) * tk
        for t in range((rows // 32) * tk, tiles):
            for i in range(rows % 32, 32) if rows % 32 else ():
                for h in range(2):
                    for ks in range(4):
                        if b == 4:
                            at = t * 4096 + 1024 * ks + 16 * (i + 32 * h)
                        else:
                            at = t * 8192 + 2048 * ks + 16 * (i + 32 * h)
                            mx[at + 1024:at + 1040] = 0xFF
                        mx[at:at + 16] = 0xFF
                        mx[tiles * 1024 * b + t * 256 + 4 * (i + 32 * h) + ks] = 0xFF
        return mx

    got = run(spoil(xm, T, d, bits), {"Wg": spoil(packed["Wg"], H, d, 4), "Wu": spoil(packed["Wu"], H, d, 4), "Wd": spoil(packed["Wd"], d, H, 4)})
    assert torch.equal(got, want)


def test_no_rows(B):
    for bits in (4, 8):
        cfg, gc = B.make_mx_config(0, 70, bits), B.make_gated_config(0, 70, 50)
        mx = torch.empty(B.slicemoe_mx_bytes(cfg), dtype=torch.uint8, device="cuda")
        none = torch.empty((0, 70), dtype=B16, device="cuda")
        B.slicemoe_mx_quantize(cfg, none, mx)
        B.slicemoe_mx_dequantize(cfg, mx, none)
        w = B.quantize_gated_weights_mx({"Wg": rand((70, 50), 1, B16), "Wu": rand((70, 50), 2, B16), "Wd": rand((50, 70), 3, B16)})
        ws = torch.empty(B.slicemoe_gated_ffn_mx_workspace_bytes(gc, bits), dtype=torch.uint8, device="cuda")
        B.slicemoe_gated_ffn_mx(gc, bits, mx, w, none, ws)
    torch.cuda.synchronize()


# many tiles over a long contraction: by the measured costs of both tiles these take 256 x 256, whatever the bits; the last tile of either side is a ragged one
LARGE = [(4090, 2900, 4000), (4000, 2900, 4090)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [B16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", LARGE)
def test_large_product(B, T, K, N, dt, bits):
    """Every result, with an addend (elsewhere and in place) and without, whole pieces of a row and not."""
    x, w, add = rand((T, K), 1, dt), rand((N, K), 2, dt, 0.2), rand((T, N), 3, dt)
    cfg = B.make_mx_product_config(T, K, N, bits, NAME[dt])
    (_, xm), (_, wm) = pack(B, x, bits), pack(B, w, 4)
    ws = torch.empty(max(256, B.slicemoe_mx_product_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    vx, vw = M.to_mx(x, bits), M.to_mx(w, 4)
    guard = torch.full((T + 2, N), 7.0, dtype=dt, device="cuda")      # whole rows on both sides that must stay
    for addend in (None, add):
        y = guard[1:-1] if N % 8 == 0 else torch.full((T, N), 7.0, dtype=dt, device="cuda")
        B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=addend)
        R.within(y, *M.product(vx, vw, addend, dt, bits), "y")
    assert bool((guard[0] == 7).all()) and bool((guard[-1] == 7).all())
    first = y.clone()
    y = add.clone()
    B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=y)
    assert torch.equal(y, first)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("T,d,H", [(4000, 4000, 4090), (3990, 3990, 4060)])
def test_large_network(B, T, d, H, bits):
    """Every seventh row against 64 bits, and those of the last tile.  A row's bits are the same wherever in the batch it is: the batch moved on by one to
    six rows shows every row's place."""
    x, add = rand((T, d), 1, B16), rand((T, d), 2, B16)
    w = {"Wg": rand((d, H), 3, B16, d ** -0.5), "Wu": rand((d, H), 4, B16, d ** -0.5), "Wd": rand((H, d), 5, B16, H ** -0.5)}
    packed, cfg = B.quantize_gated_weights_mx(w), B.make_gated_config(T, d, H)
    ws = torch.full((B.slicemoe_gated_ffn_mx_workspace_bytes(cfg, bits),), 0xFF, dtype=torch.uint8, device="cuda")
    _, xm = pack(B, x, bits)
    y = torch.full_like(x, 7.0)
    B.slicemoe_gated_ffn_mx(cfg, bits, xm, packed, y, ws, addend=add)
    pick = torch.cat([torch.arange(0, T - 160, 7), torch.arange(T - 160, T)])
    Wg, Wu, Wd = (M.to_mx(w[n].t(), 4) for n in ("Wg", "Wu", "Wd"))
    R.within(y[pick.cuda()], *M.gated(M.to_mx(x.cpu()[pick], bits), Wg, Wu, Wd, add.cpu()[pick], bits), "y")
    in_place = add.clone()
    B.slicemoe_gated_ffn_mx(cfg, bits, xm, packed, in_place, ws, addend=in_place)
    assert torch.equal(in_place, y)
    for by in range(1, 7):
        moved = torch.empty_like(x)
        B.slicemoe_gated_ffn_mx(cfg, bits, pack(B, x.roll(by, 0), bits)[1], packed, moved, ws, addend=add.roll(by, 0))
        assert torch.equal(moved, y.roll(by, 0))


# every kernel: few rows with 16 and with 32 features a block, tiles, shares of the contraction, large tiles
IN_PARTS = [(1, 64, 5), (16, 300, 129), (33, 513, 200), (64, 1000, 96), (16, 4500, 4200), (50, 257, 5003), (66, 2000, 300), (257, 511, 257), (2000, 700, 520), (1100, 256, 4100),
            (4090, 2900, 4000)]


@pytest.mark.parametrize("T,K,N", IN_PARTS)
def test_eight_bit_rows_in_fp32_storage_are_exact(B, T, K, N):
    """Products and sums of which each, in any order, is an fp32 number: large products that cancel beside small ones 2^-17 of their size.  Rows and
    weights are microscaled values already; a row's result in fp32 storage is the exact one."""
    gen = torch.Generator().manual_seed(T + K + N)
    blocks = -(-K // 32)
    x = torch.randint(-15, 16, (T, blocks, 32), generator=gen).double() / 64          # products with weights: multiples of 2^-7, below 2
    w = torch.randint(-2, 3, (N, blocks, 32), generator=gen).double() / 2
    place = torch.randint(0, 32, (blocks,), generator=gen)
    at = torch.arange(blocks)
    sign = torch.where(at % 2 == 0, 1.0, -1.0).double()
    x[:, at, place], w[:, at, place] = 448.0, 6.0 * sign                              # +- 2688 by turns
    x, w = x.flatten(1)[:, :K], w.flatten(1)[:, :K]
    y = torch.empty((T, N), device="cuda")
    (_, xm), (_, wm) = pack(B, x.float().cuda(), 8), pack(B, w.float().cuda(), 4)
    assert torch.equal(M.to_mx(x, 8), x) and torch.equal(M.to_mx(w, 4), w)
    cfg = B.make_mx_product_config(T, K, N, 8, "f32")
    ws = torch.empty(max(256, B.slicemoe_mx_product_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    B.slicemoe_mx_product(cfg, xm, wm, y, ws)
    # a sum of any of the products is a multiple of 2^-7 and below half of the large ones and all of the small ones together: 24 bits
    exact = 2688 * ((blocks + 1) // 2) + 0.25 * K < 2.0 ** 17
    want = x @ w.t()
    if exact:
        assert torch.equal(y.double().cpu(), want)
    R.within(y, *M.product_in_parts(x, w, None), "y")


@pytest.mark.parametrize("T,K,N", IN_PARTS)
def test_eight_bit_rows_in_fp32_storage(B, T, K, N):
    x, w, add = rand((T, K), 1, F32), rand((N, K), 2, F32, 0.2), rand((T, N), 3, F32)
    cfg = B.make_mx_product_config(T, K, N, 8, "f32")
    (_, xm), (_, wm) = pack(B, x, 8), pack(B, w, 4)
    ws = torch.empty(max(256, B.slicemoe_mx_product_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    vx, vw = M.to_mx(x, 8), M.to_mx(w, 4)
    for addend in (add, None):
        y = torch.full((T, N), 7.0, device="cuda")
        B.slicemoe_mx_product(cfg, xm, wm, y, ws, addend=addend)
        R.within(y, *M.product_in_parts(vx, vw, addend), "y")
