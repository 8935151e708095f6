"""CPU-side checks of the microscaled operators and of gradient clipping: refusals before any CUDA call (no context, no GPU), sizes, and what the
binding refuses by shape, type and device."""
import ctypes

import pytest
import torch

from paper_1602_02830_b200 import binding, build

P = 0x1000          # never dereferenced: every call below is refused, or only sizes things
INVALID, ALIGNMENT = -1, -2
BF = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def host():
    """A context without a device, for the parts of the binding that only look at shapes: CPU tensors are on its device, -1."""
    build.build()
    c = object.__new__(binding.Context)
    c.device, c._device, c._raw, c._h = -1, torch.device("cpu"), 0, None
    c._here = lambda: True
    return c


def mx(**k):
    return binding.MxDesc(*({"format": 0, "rows": 4, "cols": 64, "values": P, "scales": P} | k).values())


def linear(**k):
    return ctypes.byref(binding.MxLinearDesc(*({"dtype": 3, "act": 1, "W": mx(rows=32), "bias": P} | k).values()))


def gated(**k):
    return ctypes.byref(binding.MxGatedDesc(*({"dtype": 1, "act": 4, "Wg": mx(rows=32), "Wu": mx(rows=32)} | k).values()))


BAD = [({"format": 2}, INVALID), ({"format": -1}, INVALID), ({"rows": -1}, INVALID), ({"cols": 1 << 31}, INVALID), ({"values": None}, INVALID),
       ({"scales": None}, INVALID), ({"values": P + 16}, ALIGNMENT), ({"scales": P + 8}, ALIGNMENT)]


@pytest.mark.parametrize("format,cols,pitch", [(0, 1, 128), (0, 128, 128), (0, 129, 256), (1, 1, 64), (1, 128, 64), (1, 1011, 512), (0, 0, 0), (2, 64, 0), (0, -1, 0)])
def test_pitches(lib, format, cols, pitch):
    assert lib.bnn_mx_ld(format, cols) == pitch


@pytest.mark.parametrize("rows,cols,size", [(1, 1, 512), (128, 128, 512), (129, 128, 1024), (128, 129, 1024), (1000, 1011, 8 * 8 * 512), (0, 64, 0), (64, 0, 0), (-1, 4, 0),
                                            (0x7fff0000, 0x7fff0000, 0x7fff0000 // 128 * (0x7fff0000 // 128) * 512)])
def test_scale_bytes(lib, rows, cols, size):
    assert lib.bnn_mx_scale_bytes(rows, cols) == size


@pytest.mark.parametrize("k,want", BAD + [({}, INVALID)])
def test_matrices(lib, k, want):
    q = ctypes.byref(mx(**k))
    assert lib.bnn_mx_quantize(None, 3, P, 64, q, None, 0) == want              # {}: only the missing context is left to refuse
    assert lib.bnn_mx_values(None, q, 3, P, 64) == want
    w = mx(**({"rows": 32} | k))
    assert lib.bnn_mx_linear(None, linear(W=w), ctypes.byref(mx()), None, 0, P, 32, None, 0, None) == want
    assert lib.bnn_mx_gated(None, gated(Wg=w, Wu=w), ctypes.byref(mx()), P, 32, None, 0, None) == want
    assert lib.bnn_mx_linear(None, linear(), q, None, 0, P, 32, None, 0, None) == want


def test_quantize_arguments(lib):
    q = ctypes.byref(mx())
    assert lib.bnn_mx_quantize(None, 2, P, 64, q, None, 0) == INVALID           # signed bytes are no source
    assert lib.bnn_mx_quantize(None, 3, P, 63, q, None, 0) == INVALID
    assert lib.bnn_mx_quantize(None, 3, None, 64, q, None, 0) == INVALID
    assert lib.bnn_mx_quantize(None, 3, P + 1, 64, q, None, 0) == ALIGNMENT
    assert lib.bnn_mx_quantize(None, 0, P, 64, q, P + 2, 64) == ALIGNMENT
    assert lib.bnn_mx_quantize(None, 3, P, 64, q, P, 63) == INVALID
    assert lib.bnn_mx_quantize(None, 3, P, 64, None, None, 0) == INVALID
    assert lib.bnn_mx_values(None, q, 3, None, 64) == INVALID and lib.bnn_mx_values(None, q, 7, P, 64) == INVALID


def test_norm_arguments(lib):
    norm = lambda **k: ctypes.byref(binding.BlockNormDesc(*({"dtype": 3, "kind": 0, "D": 64, "eps": 1e-6, "alpha": 1.0, "post": 0, "pre": 1, "post_weight": None,  # noqa: E731
                                                             "post_shift": None, "pre_weight": P, "pre_shift": None, "gate": None, "ld_gate": 0, "rows_per_gate": 1} | k).values()))
    call = lambda d, q, M=4, represented=None: lib.bnn_block_norm_mx(None, d, P, 64, P, 64, M, P, 64, q and ctypes.byref(q), represented, 64, None)  # noqa: E731
    assert call(norm(), mx()) == INVALID                                        # only the context is missing
    assert call(norm(), None) == INVALID and call(norm(pre=0), mx()) == INVALID
    assert call(norm(), mx(rows=5)) == INVALID and call(norm(), mx(cols=63)) == INVALID
    assert call(norm(), mx(), represented=P + 1) == ALIGNMENT and call(norm(), mx(values=P + 4)) == ALIGNMENT


def test_product_arguments(lib):
    x = ctypes.byref(mx())
    call = lambda d, x=x, r=None, y=P, ldy=32, pre=None, q=None: lib.bnn_mx_linear(None, d, x, r, 32, y, ldy, pre, 32, q and ctypes.byref(q))  # noqa: E731
    assert call(linear()) == INVALID                                            # only the context is missing
    assert call(linear(dtype=0)) == INVALID and call(linear(act=7)) == INVALID and call(linear(bias=P + 1)) == ALIGNMENT
    assert call(linear(), x=ctypes.byref(mx(cols=96))) == INVALID               # another inner size
    assert call(linear(), x=ctypes.byref(mx(format=1))) == INVALID              # 4-bit inputs with 8-bit weights
    assert call(linear(), y=None) == INVALID and call(linear(), ldy=31) == INVALID and call(linear(), r=P + 1) == ALIGNMENT and call(linear(), pre=P + 2) == ALIGNMENT
    out = mx(cols=32)
    assert call(linear(), q=out) == INVALID                                     # both y and y_mx
    assert call(linear(), y=None, q=out, r=P) == INVALID and call(linear(), y=None, q=out, pre=P) == INVALID
    assert call(linear(), y=None, q=mx(cols=31)) == INVALID and call(linear(), y=None, q=mx(cols=32, values=P + 8)) == ALIGNMENT
    both = lambda **k: lib.bnn_mx_gated(None, gated(**k), x, P, 32, None, 0, None)  # noqa: E731
    assert both() == INVALID and both(Wu=mx(rows=31)) == INVALID and both(Wu=mx(rows=32, format=1)) == INVALID and both(act=9) == INVALID and both(dtype=2) == INVALID


def test_clip_arguments(lib):
    def call(entries=((P, P, 8, 0),), max_norm=1.0, eps=1e-6, norm=P, count=None):
        a = (binding.Gradient * max(1, len(entries)))(*[binding.Gradient(*e) for e in entries])
        return lib.bnn_clip_gradients(None, a, len(entries) if count is None else count, max_norm, eps, norm)
    assert call() == INVALID                                                    # only the context is missing
    assert call(max_norm=-1.0) == INVALID and call(max_norm=float("nan")) == INVALID and call(eps=-1e-6) == INVALID and call(norm=None) == INVALID and call(norm=P + 1) == ALIGNMENT
    assert call(((P, P, -1, 0),)) == INVALID and call(((P, P, 8, 2),)) == INVALID and call(((None, P, 8, 0),)) == INVALID and call(((P, None, 8, 0),)) == INVALID
    assert call(((P + 2, P, 8, 0),)) == ALIGNMENT and call(((P, P + 1, 8, 3),)) == ALIGNMENT and call(count=-1) == INVALID
    assert lib.bnn_clip_workspace_bytes(-1) == 0 and 0 < lib.bnn_clip_workspace_bytes(0) <= lib.bnn_clip_workspace_bytes(5000)


def test_binding_refuses_by_shape_and_type(host):
    x = torch.zeros(4, 64, dtype=BF)
    q, w, w4, other = host.make_mx(4, 64, "e4m3"), host.make_mx(32, 64, "e4m3"), host.make_mx(32, 64, "e2m1"), host.make_mx(32, 96, "e4m3")
    norm, flat = host.make_block_norm(64, BF), host.make_block_norm(64, BF, pre=False)
    layer, glu = host.make_mx_linear(w), host.make_mx_gated(w, w)
    q4, q64, w64 = host.make_mx(4, 64, "e2m1"), host.make_mx(4, 64), host.make_mx(64, 64)
    square, layer64 = host.make_mx_gated(w64, w64), host.make_mx_linear(w64)
    for call, match in [
        (lambda: host.make_mx(4, 64, "e5m2"), "format"), (lambda: host.make_mx(-1, 64), "rows, cols"),
        (lambda: host.mx_quantize(x.int()), "x:"), (lambda: host.mx_quantize(x, "e2m1", out=q), "format"), (lambda: host.mx_quantize(x, out=w), "out:"),
        (lambda: host.mx_quantize(x, out=q, values=x.float()), "values:"), (lambda: host.mx_quantize(x.t(), out=q), "x:|out:"), (lambda: host.mx_quantize(x, out=x), "out:"),
        (lambda: host.mx_values(x), "q:"), (lambda: host.mx_values(q, torch.int8), "dtype"), (lambda: host.mx_values(q, BF, out=x.float()), "out:"),
        (lambda: host.block_norm_mx(flat, x), "layer:"), (lambda: host.block_norm_mx(norm, x, out=w), "out:"), (lambda: host.block_norm_mx(norm, x, format="e2m1", out=q), "format"),
        (lambda: host.make_mx_linear(x), "weights:"), (lambda: host.make_mx_linear(w, dtype=torch.float32), "dtype"), (lambda: host.make_mx_linear(w, act="tanh"), "act"),
        (lambda: host.make_mx_linear(w, torch.zeros(31, dtype=BF)), "bias"), (lambda: host.make_mx_gated(w, w4), "weights:"), (lambda: host.make_mx_gated(w, other), "weights:"),
        (lambda: host.mx_linear(glu, q), "layer:"), (lambda: host.mx_gated(layer, q), "layer:"), (lambda: host.mx_linear(layer, x), "x:"), (lambda: host.mx_linear(layer, q4), "e2m1"),
        (lambda: host.mx_linear(host.make_mx_linear(other), q), "x:"), (lambda: host.mx_linear(layer, q, out=host.make_mx(4, 31)), "out:"),
        (lambda: host.mx_linear(layer, q, x[:, :32], out=host.make_mx(4, 32)), "without residual"), (lambda: host.mx_linear(layer, q, pre=torch.zeros(4, 32, dtype=BF)), "pre:"),
        (lambda: host.mx_gated(glu, q, pre=torch.zeros(2, 4, 31)), "pre:"), (lambda: host.mx_gated(glu, q, pre=torch.zeros(2, 4, 32), out=host.make_mx(4, 32)), "without residual"),
        (lambda: host.mx_gated(square, q64, out=q64), "must not be x"), (lambda: host.mx_linear(layer64, q64, out=q64), "must not be x"),
    ]:
        with pytest.raises(ValueError, match=match):
            call()


def test_binding_refuses_gradients(host):
    t = torch.zeros(4, 6)
    for call, match in [
        (lambda: host.make_gradients([t.int()]), "tensors"), (lambda: host.make_gradients([t.t()]), "tensors"), (lambda: host.make_gradients([t], [t.half()]), "out"),
        (lambda: host.make_gradients([t], []), "out"), (lambda: host.make_gradients([t], [torch.zeros(6, 4)]), "out"), (lambda: host.make_gradients([t, t]), "share memory"),
        (lambda: host.make_gradients([t, t[2:]]), "share memory"), (lambda: host.make_gradients([t[:2]], [t[1:3]]), "share memory"),
        (lambda: host.clip_gradients(host.make_gradients([t]), -1.0), "max_norm"), (lambda: host.clip_gradients(host.make_gradients([t]), 1.0, eps=float("nan")), "max_norm"),
    ]:
        with pytest.raises(ValueError, match=match):
            call()
    assert len(host.make_gradients([t[:2], t[2:], t[:0]]).tensors) == 3          # neighbours and empty tensors are fine


def test_handles_of_another_device_are_refused(host):
    """Only addresses reach the library: on another device they would be read as that device's memory."""
    other = object.__new__(binding.Context)
    other.device = 0
    other._here = lambda: True
    q, w, x = host.make_mx(4, 64), host.make_mx(32, 64), torch.zeros(4, 64, dtype=BF)
    layer, glu, grads = host.make_mx_linear(w), host.make_mx_gated(w, w), host.make_gradients([x])
    for call in (lambda: other.mx_linear(layer, q), lambda: other.mx_gated(glu, q), lambda: other.mx_values(q), lambda: other.make_mx_linear(w),
                 lambda: other.make_mx_gated(w, w), lambda: other.clip_gradients(grads, 1.0), lambda: other.mx_quantize(x, out=q)):
        with pytest.raises(ValueError, match="on cuda:|on cpu"):
            call()
