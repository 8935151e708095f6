"""A microscaled result that shares memory with an input of the same call is refused at the C entry points: it would be overwritten while other tiles still read it.  The context
here is a block of zeros: a call that is not refused gets as far as asking for a device, which this machine has not."""
import ctypes

import pytest
import torch

from paper_1602_02830_b200 import binding, build

INVALID, BF = -1, 3
X, XS, W, WS, U, US, Q, QS = (0x10000000 * i for i in range(1, 9))      # never dereferenced
M = K = N = 256
V, S = M * 256, 2 * 2 * 512                                             # bytes of the elements (e4m3) and of the scales of each

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses are not memory: only where no call can reach a device")


@pytest.fixture(scope="module")
def call():
    build.build()
    L, ctx = binding.lib(), ctypes.create_string_buffer(4096)
    mx = lambda v, s, fmt=0: binding.MxDesc(fmt, M, K, v, s)  # noqa: E731
    ref = ctypes.byref

    def linear(q, bias=None):
        return L.bnn_mx_linear(ctx, ref(binding.MxLinearDesc(BF, 0, mx(W, WS), bias)), ref(mx(X, XS)), None, 0, None, 0, None, 0, ref(mx(*q)))

    def gated(q):
        return L.bnn_mx_gated(ctx, ref(binding.MxGatedDesc(BF, 4, mx(W, WS), mx(U, US))), ref(mx(X, XS)), None, 0, None, 0, ref(mx(*q)))

    def quantize(q, x=X, represented=None, ld=K):
        return L.bnn_mx_quantize(ctx, BF, x, ld, ref(mx(*q)), represented, K)

    def values(q, out):
        return L.bnn_mx_values(ctx, ref(mx(*q)), BF, out, K)

    def norm(q, stream=US, represented=None):
        d = binding.BlockNormDesc(BF, 0, K, 1e-6, 1.0, 0, 1, None, None, None, None, None, 0, 1)
        return L.bnn_block_norm_mx(ctx, ref(d), X, K, W, K, M, stream, K, ref(mx(*q)), represented, K, None)

    return linear, gated, quantize, values, norm


@pytest.mark.parametrize("v,s", [(X, QS), (X + 32, QS), (X + V - 32, QS), (X - 32, QS), (X - V + 32, QS), (Q, XS), (Q, XS + S - 16), (Q, X + 512), (XS - 64, QS),
                                 (W, QS), (W + V - 32, QS), (Q, WS - S + 16)])
def test_products_refuse_a_result_on_their_operands(call, v, s):
    linear, gated = call[:2]
    assert linear((v, s)) == INVALID and gated((v, s)) == INVALID


def test_products_refuse_more(call):
    linear, gated = call[:2]
    assert gated((U + 64, QS)) == INVALID and gated((Q, US)) == INVALID
    assert linear((Q, QS), bias=Q + 64) == INVALID and linear((Q, QS), bias=QS - 2 * N + 2) == INVALID


@pytest.mark.parametrize("v,s", [(Q, QS), (X + V, QS), (X - V, QS), (Q, XS + S), (Q, XS - S), (W + V, U - S)])
def test_neighbours_are_not_refused(call, v, s):
    linear, gated = call[:2]
    assert linear((v, s)) not in (0, INVALID) and gated((v, s)) not in (0, INVALID)


def test_rows_and_their_microscaled_form(call):
    quantize, values, norm = call[2:]
    rows = 2 * M * K                                                    # bytes in 16 bits
    for v in (X, X + rows - 32, X - V + 32):
        assert quantize((v, QS)) == INVALID and norm((v, QS)) == INVALID and values((v, QS), X) == INVALID
        assert quantize((v, QS), x=W, represented=X) == INVALID and norm((v + W - X, QS)) == INVALID and norm((v + U - X, QS), stream=U, represented=None) == INVALID
        assert norm((v + U - X, QS), represented=U) == INVALID
    assert quantize((Q, X + rows - 16)) == INVALID
    assert quantize((X + rows, QS)) not in (0, INVALID) and quantize((X - V, QS)) not in (0, INVALID) and quantize((X + rows, QS), ld=K + 8) == INVALID
    assert norm((X + rows, QS)) not in (0, INVALID) and values((X + rows, QS), X) not in (0, INVALID)
    assert quantize((Q, QS), x=X, represented=X) not in (0, INVALID)    # onto the source itself is fine
