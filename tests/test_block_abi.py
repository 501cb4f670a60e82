"""Host-side checks of the entry points around the layer (norm, gated feed-forward network, gradient clipping): what they refuse
before anything touches the GPU, their workspace sizes and their structs.  No kernel is launched."""
import ctypes
import math
import os

import pytest

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2510_04286_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_04286_amd import build
        build.build()
    return binding


P, ODD, Q = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(1 << 20)   # never dereferenced
NULL = None
BIG = 1 << 40


def by(x):
    return ctypes.byref(x)


def test_struct_sizes(B):
    assert [ctypes.sizeof(t) for t in (B.slicemoe_norm_config, B.slicemoe_gated_config, B.slicemoe_gated_weights, B.slicemoe_gated_weight_grads,
                                       B.slicemoe_gated_weights_quantized, B.slicemoe_grad)] == [16, 16, 24, 24, 40, 32]
    import struct
    assert struct.calcsize(B._GRAD_FIELDS) == 32


def norm_cfgs(B):
    bad = [B.make_norm_config(-1, 64), B.make_norm_config(4, 0), B.make_norm_config(4, 64, -1e-5), B.make_norm_config(4, 64, NAN),
           B.make_norm_config(4, 64, INF), B.slicemoe_norm_config(4, 64, 1e-5, 2)]
    return bad, [B.make_norm_config(4, 16385)]


def test_norm_refusals(B):
    L, ok = B.lib(), B.make_norm_config(4, 64)
    f = L.slicemoe_add_rmsnorm
    bad, unsupported = norm_cfgs(B)
    for c in bad:
        assert f(by(c), P, P, P, P, P, NULL, NULL, NULL) == B.SLICEMOE_ERR_INVALID_ARG
        assert B.slicemoe_add_rmsnorm_backward_workspace_bytes(c) == 0
    for c in unsupported:
        assert f(by(c), P, P, P, P, P, NULL, NULL, NULL) == B.SLICEMOE_ERR_UNSUPPORTED
        assert B.slicemoe_add_rmsnorm_backward_workspace_bytes(c) == 0
    assert f(NULL, P, P, P, P, P, NULL, NULL, NULL) == B.SLICEMOE_ERR_INVALID_ARG
    for args in [(NULL, P, P, P, P, NULL, NULL), (P, P, NULL, P, P, NULL, NULL), (P, P, P, P, NULL, NULL, NULL),   # x, weight, no output
                 (P, P, P, P, P, P, NULL),                                                                        # values without a scale
                 (ODD, P, P, P, Q, NULL, NULL), (P, ODD, P, P, Q, NULL, NULL), (P, P, ODD, P, Q, NULL, NULL),
                 (P, P, P, ODD, Q, NULL, NULL), (P, P, P, P, ODD, NULL, NULL), (P, P, P, P, Q, ODD, P),
                 (P, P, P, P, Q, Q, ctypes.c_void_p(4097)), (P, P, P, Q, Q, NULL, NULL)]:                          # sum and y the same array
        assert f(by(ok), *args, NULL) == B.SLICEMOE_ERR_INVALID_ARG, args
    g = L.slicemoe_add_rmsnorm_backward
    assert g(by(ok), P, P, P, P, Q, P, P, 16, NULL) == B.SLICEMOE_ERR_WORKSPACE
    assert g(by(ok), P, P, P, P, Q, P, NULL, BIG, NULL) == B.SLICEMOE_ERR_WORKSPACE
    assert g(by(ok), P, P, P, P, Q, P, ODD, BIG, NULL) == B.SLICEMOE_ERR_INVALID_ARG
    for args in [(NULL, P, P, P, Q, P), (P, NULL, P, P, Q, P), (P, P, NULL, P, Q, P), (P, P, P, P, NULL, P), (P, P, P, P, Q, NULL),
                 (P, P, P, P, P, P), (ODD, P, P, P, Q, P), (P, P, P, ODD, Q, P), (P, P, P, P, Q, ctypes.c_void_p(4098))]:
        assert g(by(ok), *args, P, BIG, NULL) == B.SLICEMOE_ERR_INVALID_ARG, args


def test_gated_refusals(B):
    L, ok = B.lib(), B.make_gated_config(4, 64, 32)
    w, none = B.slicemoe_gated_weights(4096, 4096, 4096), B.slicemoe_gated_weights()
    sizes = (B.slicemoe_gated_ffn_workspace_bytes, B.slicemoe_gated_ffn_backward_workspace_bytes, B.slicemoe_gated_ffn_quantized_workspace_bytes)
    fwd, bwd, qnt, pack = L.slicemoe_gated_ffn, L.slicemoe_gated_ffn_backward, L.slicemoe_gated_ffn_quantized, L.slicemoe_gated_ffn_quantize_weights
    gr = B.slicemoe_gated_weight_grads(8192, 8192, 8192)
    qw = B.slicemoe_gated_weights_quantized(4096, 4096, 4096, 4096, 4096)

    def all_of(c, want):
        assert fwd(by(c), P, by(w), P, P, P, BIG, NULL) == want
        assert bwd(by(c), P, by(w), P, P, P, by(gr), P, BIG, NULL) == want
        assert qnt(by(c), P, P, by(qw), P, P, P, BIG, NULL) == want
        assert pack(by(c), by(w), P, P, P, P, NULL) == want
        assert all(s(c) == 0 for s in sizes)

    for c in [B.make_gated_config(-1, 64, 32), B.make_gated_config(4, 0, 32), B.make_gated_config(4, 64, 0), B.slicemoe_gated_config(4, 64, 32, 7)]:
        all_of(c, B.SLICEMOE_ERR_INVALID_ARG)
    for c in [B.make_gated_config(1 << 30, 64, 32), B.make_gated_config(4, (1 << 20) + 1, 32), B.make_gated_config(4, 64, (1 << 20) + 1),
              B.make_gated_config((1 << 30) - 1, 64, 1 << 20)]:
        all_of(c, B.SLICEMOE_ERR_UNSUPPORTED)
    for c in [B.make_gated_config(4, 64, 32, "f32"), B.make_gated_config(4, 72, 32)]:   # 8-bit operands: bf16 storage, whole 16-byte rows
        assert qnt(by(c), P, P, by(qw), P, P, P, BIG, NULL) == B.SLICEMOE_ERR_UNSUPPORTED and sizes[2](c) == 0
        assert pack(by(c), by(w), P, P, P, P, NULL) == B.SLICEMOE_ERR_UNSUPPORTED
        assert sizes[0](c) > 0 and sizes[1](c) > 0
    inv, wsp = B.SLICEMOE_ERR_INVALID_ARG, B.SLICEMOE_ERR_WORKSPACE
    for args in [(NULL, by(w), P, P), (P, NULL, P, P), (P, by(none), P, P), (P, by(w), P, NULL), (ODD, by(w), P, P), (P, by(w), ODD, P),
                 (P, by(w), P, ODD), (P, by(B.slicemoe_gated_weights(4096, 4100, 4096)), P, P)]:
        assert fwd(by(ok), *args, P, BIG, NULL) == inv
    assert fwd(by(ok), P, by(w), P, P, NULL, BIG, NULL) == wsp and fwd(by(ok), P, by(w), P, P, P, sizes[0](ok) - 1, NULL) == wsp
    assert fwd(by(ok), P, by(w), P, P, ODD, BIG, NULL) == inv
    half = B.slicemoe_gated_weight_grads(8192, None, 8192)
    for args in [(NULL, by(w), P, P, P, by(gr)), (P, by(w), NULL, P, P, by(gr)), (P, by(w), P, P, NULL, by(gr)), (P, by(w), P, P, P, NULL),
                 (P, by(w), P, P, P, by(half)), (P, by(w), ODD, P, P, by(gr)), (P, by(w), P, P, ODD, by(gr)),
                 (P, by(w), P, P, P, by(B.slicemoe_gated_weight_grads(8192, 8196, 8192)))]:
        assert bwd(by(ok), *args, P, BIG, NULL) == inv
    assert bwd(by(ok), P, by(w), P, P, P, by(gr), P, sizes[1](ok) - 1, NULL) == wsp
    for args in [(NULL, P, by(qw), P, P), (P, NULL, by(qw), P, P), (P, P, NULL, P, P), (P, P, by(B.slicemoe_gated_weights_quantized()), P, P),
                 (P, P, by(qw), P, NULL), (ODD, P, by(qw), P, P), (P, ctypes.c_void_p(4097), by(qw), P, P)]:
        assert qnt(by(ok), *args, P, BIG, NULL) == inv
    assert qnt(by(ok), P, P, by(qw), P, P, P, sizes[2](ok) - 1, NULL) == wsp
    assert pack(by(ok), by(w), NULL, P, P, P, NULL) == inv and pack(by(ok), by(w), P, P, P, ctypes.c_void_p(4098), NULL) == inv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspaces_never_fall_as_the_batch_grows(B, dtype):
    for d, H in ((64, 64), (768, 2048), (1024, 2816), (257, 683), (4096, 11008), (16, 1)):
        last = [0, 0, 0, 0]
        for T in (0, 1, 7, 31, 32, 33, 63, 64, 65, 100, 128, 129, 255, 256, 257, 512, 1000, 2047, 4096, 8191, 16384, 65536):
            c = B.make_gated_config(T, d, H, dtype)
            now = [B.slicemoe_gated_ffn_workspace_bytes(c), B.slicemoe_gated_ffn_backward_workspace_bytes(c),
                   B.slicemoe_gated_ffn_quantized_workspace_bytes(c), B.slicemoe_add_rmsnorm_backward_workspace_bytes(B.make_norm_config(T, d, 1e-5, dtype))]
            assert all(a <= b for a, b in zip(last, now)), (d, H, T)
            assert all(n % 256 == 0 for n in now) and now[0] > 0 and now[1] > 0 and now[3] > 0
            last = now
    big = B.slicemoe_gated_ffn_workspace_bytes(B.make_gated_config(1 << 20, 4096, 11008))   # beyond 32 bits
    assert big >= (1 << 20) * 11008 * 2


def grads(B, *items):
    arr = (B.slicemoe_grad * max(1, len(items)))()
    for a, (g, o, n, dt) in zip(arr, items):
        a.grad, a.out, a.n, a.dtype = g, o, n, dt
    return arr, len(items)


def test_clip_refusals(B):
    L = B.lib()

    def call(items, max_norm=1.0, norm=P, ws=P, room=BIG):
        arr, n = grads(B, *items)
        return L.slicemoe_clip_grads(arr, n, max_norm, norm, ws, room, NULL)

    inv = B.SLICEMOE_ERR_INVALID_ARG
    one = (4096, 4096, 16, 0)
    for bad in [(4096, 4096, -1, 0), (4096, 4096, 16, 2), (None, None, 16, 0), (4098, 4098, 16, 0), (4097, 4097, 16, 1), (4096, 8193, 16, 1)]:
        assert call([bad]) == inv
        arr, n = grads(B, bad)
        assert L.slicemoe_clip_grads_workspace_bytes(arr, n) == 0
    for m in (-1.0, NAN, -INF):
        assert call([one], max_norm=m) == inv
    assert call([one], norm=NULL) == inv and call([one], norm=ctypes.c_void_p(4098)) == inv
    assert call([one], ws=NULL) == B.SLICEMOE_ERR_WORKSPACE and call([one], room=8) == B.SLICEMOE_ERR_WORKSPACE
    assert call([one], ws=ODD) == inv
    assert L.slicemoe_clip_grads(NULL, 1, 1.0, P, P, BIG, NULL) == inv and L.slicemoe_clip_grads(NULL, -1, 1.0, P, P, BIG, NULL) == inv
    # overlaps: the same tensor twice, an output inside another tensor, an output over its own input in part
    for items in ([one, one], [(4096, None, 16, 0), (4096, 4096, 16, 0)], [(4096, 8192, 16, 0), (16384, 8252, 16, 0)], [(4096, 4100, 16, 0)],
                  [(4096, 65536, 1024, 1), (6000, 131072, 8, 0), (262144, 6140, 1, 0)], [(4096, 8192, 16, 0), (8192, None, 16, 0)]):
        assert call(items) == inv, items
    assert L.slicemoe_clip_grads_workspace_bytes(NULL, 0) > 0
    arr, n = grads(B, (4096, None, 10 ** 12, 0), (4096, None, 1, 0))
    assert L.slicemoe_clip_grads_workspace_bytes(arr, n) == 0   # more than the sums' table is made for
    for n in (0, 1, 4096, 10 ** 9):
        arr, k = grads(B, (4096, None, n, 0))
        assert 0 < L.slicemoe_clip_grads_workspace_bytes(arr, k) <= 8 * 16384


def test_binding_refuses_host_tensors_and_wrong_types(B):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.slicemoe_add_rmsnorm(B.make_norm_config(4, 64), x, None, x[0], None, x)
    with pytest.raises(TypeError):
        B.slicemoe_clip_grads_workspace_bytes([torch.zeros(4)])
    with pytest.raises(TypeError):
        B.slicemoe_clip_grads_workspace_bytes([None])
    assert math.isinf(INF)


def test_the_longest_batch(B):
    """The contraction over the rows counts bytes, and a step of 128 beyond them, in a signed 32-bit number."""
    sizes = (B.slicemoe_gated_ffn_workspace_bytes, B.slicemoe_gated_ffn_backward_workspace_bytes, B.slicemoe_gated_ffn_quantized_workspace_bytes)
    assert 2 * (1 << 29) + 128 < 1 << 31
    for size in sizes:
        # the hidden rows at least, T x 64 bf16 values; nothing else forward, whose contractions of one step have no shares
        assert size(B.make_gated_config(1 << 29, 16, 8)) >= (1 << 29) * 64 * 2
        for T in ((1 << 29) + 1, (1 << 30) - 1):
            assert size(B.make_gated_config(T, 16, 8)) == 0
    c = B.make_gated_config((1 << 30) - 1, 16, 8)
    w = B.slicemoe_gated_weights(4096, 4096, 4096)
    assert B.lib().slicemoe_gated_ffn(by(c), P, by(w), P, P, P, BIG, NULL) == B.SLICEMOE_ERR_UNSUPPORTED


class OnDevice:
    """A tensor's face: what the binding asks of one."""
    is_cuda = True

    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


def test_binding_refuses_a_stream_of_another_device(B, monkeypatch):
    class Stream:
        cuda_stream, device_index = 4096, 1
    assert B._stream_on(1, Stream()) == 4096
    with pytest.raises(ValueError, match="device 1"):
        B._stream_on(0, Stream())
    import torch
    monkeypatch.setattr(B.torch, "Tensor", OnDevice)
    with pytest.raises(ValueError, match="is on device 1, the current device is 0"):
        B._ptr(OnDevice(1), None, None, "x", 0)
    assert isinstance(OnDevice(1), torch.Tensor)


def test_quantized_weights_are_made_where_the_weights_are(B, monkeypatch):
    import torch
    made = {}

    def pack(cfg, w, Wg, Wg_scale, Wu, Wu_scale, stream=None):
        made.update(Wg=Wg, Wg_scale=Wg_scale, Wu=Wu, Wu_scale=Wu_scale)
    monkeypatch.setattr(B, "slicemoe_gated_ffn_quantize_weights", pack)
    w = {n: torch.empty((16, 8) if n != "Wd" else (8, 16), dtype=torch.bfloat16, device="meta") for n in ("Wg", "Wu", "Wd")}
    q = B.quantize_gated_weights(B.make_gated_config(4, 16, 8), w)
    assert sorted(made) == ["Wg", "Wg_scale", "Wu", "Wu_scale"] and all(q[n] is t and t.device.type == "meta" for n, t in made.items())
    assert q["Wd"] is w["Wd"] and B.quantize_gated_weights(B.make_gated_config(4, 16, 8), w, device="cpu")["Wg"].device.type == "cpu"


def test_storage_types_by_name(B):
    import torch
    for make in (lambda t: B.make_norm_config(4, 16, 1e-5, t), lambda t: B.make_gated_config(4, 16, 8, t)):
        assert all(make(t).dtype == B.SLICEMOE_BF16 for t in ("bf16", "bfloat16", torch.bfloat16, B.SLICEMOE_BF16))
        assert all(make(t).dtype == B.SLICEMOE_F32 for t in ("f32", "fp32", "float32", torch.float32, B.SLICEMOE_F32))
        for t in ("fp16", "BF16", torch.float16, torch.float64, torch.float8_e4m3fn, 2, -1, None, ["bf16"]):
            with pytest.raises(ValueError, match="dtype must be"):
                make(t)


@pytest.mark.parametrize("dtype,narrow", [("bf16", 1024), ("f32", 512)])
def test_backward_blocks_of_wide_rows(B, dtype, narrow):
    """A row of partial weight gradients per block: four rows a block where they go side by side, but a row each, up to one block per CU,
    where a block takes one after the other."""
    def blocks(T, d):
        return B.slicemoe_add_rmsnorm_backward_workspace_bytes(B.make_norm_config(T, d, 1e-5, dtype)) // (4 * d)
    for d, wide in ((narrow, False), (64, False), (2 * narrow, True), (16384, True)):
        assert [blocks(T, d) for T in (0, 1, 5, 100, 256)] == ([1, 1, 5, 100, 256] if wide else [1, 1, 2, 25, 64])
        assert [blocks(T, d) for T in (500, 1024)] == ([256, 256] if wide else [125, 256])
        assert [blocks(T, d) for T in (1025, 3071, 10 ** 6, 2 ** 31 - 1)] == [257, 768, 768, 768]


NO_MEMORY = """
import ctypes, resource, sys
class Grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]
L = ctypes.CDLL(sys.argv[1])
f = L.slicemoe_clip_grads
f.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
lists = []
for count in (512, 513, 1 << 20):   # each ends with its first tensor once more: refused, whatever memory there is, before anything is launched
    a = (Grad * count)()
    for i in range(count):
        a[i].grad = a[i].out = (1 << 20) + 4096 * (i % (count - 1))
        a[i].n = 4
    lists.append((a, count))
def call(a, count):
    return f(ctypes.addressof(a), count, 1.0, 4096, 1 << 20, 1 << 40, None)
print([call(*l) for l in lists])
pages = int(open("/proc/self/statm").read().split()[0])
resource.setrlimit(resource.RLIMIT_AS, (pages * 4096 + (8 << 20),) * 2)
print([call(*l) for l in lists])
"""


def test_lists_are_checked_without_memory(B):
    """Up to 512 tensors on the stack; a longer list that finds no memory is an error, not an exception through the C boundary."""
    import subprocess
    import sys
    out = subprocess.run([sys.executable, "-c", NO_MEMORY, B.LIB_PATH], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    inv, hip = B.SLICEMOE_ERR_INVALID_ARG, 4
    assert out.stdout.split("\n")[:2] == [str([inv, inv, inv]), str([inv, inv, hip])]
