"""CPU-side checks of the real-valued operators' C entry points: every refusal comes before any CUDA call (no context, no GPU)."""
import ctypes

import pytest

from paper_1602_02830_b200 import binding, build

P = 0x1000          # never dereferenced: every call below is refused, or only sizes things


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def linear(**k):
    f = {"dtype": 3, "act": 1, "K": 64, "N": 32, "W": P, "ldw": 64, "bias": P} | k
    return ctypes.byref(binding.LinearDesc(*f.values()))


def gated(**k):
    f = {"dtype": 1, "act": 4, "K": 64, "N": 32, "Wg": P, "ldg": 64, "Wu": P, "ldu": 64} | k
    return ctypes.byref(binding.GatedDesc(*f.values()))


def norm(**k):
    f = {"dtype": 0, "kind": 0, "D": 64, "eps": 1e-6, "alpha": 1.0, "post": 1, "pre": 1, "post_weight": P, "post_shift": None, "pre_weight": P,
         "pre_shift": None, "gate": P, "ld_gate": 64, "rows_per_gate": 4} | k
    return ctypes.byref(binding.BlockNormDesc(*f.values()))


INVALID, ALIGNMENT = -1, -2


@pytest.mark.parametrize("k,want", [({"dtype": 0}, INVALID), ({"dtype": 2}, INVALID), ({"dtype": 9}, INVALID), ({"act": 7}, INVALID), ({"act": -1}, INVALID),
                                    ({"K": -1}, INVALID), ({"N": 1 << 31}, INVALID), ({"W": None}, INVALID), ({"ldw": 63}, INVALID),
                                    ({"W": P + 1}, ALIGNMENT), ({"bias": P + 1}, ALIGNMENT), ({}, INVALID)])
def test_linear_descriptors(lib, k, want):
    call = lambda d: lib.bnn_linear(None, d, P, 64, 4, None, 0, P, 32, None, 0)  # noqa: E731
    assert call(linear(**k)) == want                     # {}: only the missing context is left to refuse
    assert lib.bnn_linear_backward(None, linear(**k), P, 32, P, 64, 4, None, 0, P, 64, P, 64, P if k.get("bias", P) else None) == want
    assert (lib.bnn_linear_workspace_bytes(linear(**k), 4, 1, 1) > 0) == (not k)


def test_linear_arguments(lib):
    d = linear()
    assert lib.bnn_linear(None, None, P, 64, 4, None, 0, P, 32, None, 0) == INVALID
    assert lib.bnn_linear(None, d, P, 64, -1, None, 0, P, 32, None, 0) == INVALID
    assert lib.bnn_linear(None, d, P + 1, 64, 4, None, 0, P, 32, None, 0) == ALIGNMENT
    assert lib.bnn_linear(None, d, P, 64, 4, P + 1, 32, P, 32, None, 0) == ALIGNMENT
    assert lib.bnn_linear(None, d, P, 64, 4, None, 0, P, 32, P + 2, 32) == ALIGNMENT
    assert lib.bnn_linear(None, d, P, 64, 4, None, 0, P, 31, None, 0) == INVALID
    assert lib.bnn_linear_backward(None, linear(bias=None), P, 32, P, 64, 4, None, 0, P, 64, P, 64, P) == INVALID


@pytest.mark.parametrize("k,want", [({"dtype": 0}, INVALID), ({"act": 7}, INVALID), ({"Wu": None}, INVALID), ({"ldu": 2}, INVALID), ({"Wg": P + 1}, ALIGNMENT), ({}, INVALID)])
def test_gated_descriptors(lib, k, want):
    assert lib.bnn_gated(None, gated(**k), P, 64, 4, P, 32, None, 0) == want
    assert lib.bnn_gated_backward(None, gated(**k), P, 32, P, 64, 4, None, 0, P, 64, P, 64, P, 64) == want
    assert (lib.bnn_gated_workspace_bytes(gated(**k), 4, 1, 1) > 0) == (not k)


@pytest.mark.parametrize("k,want", [({"dtype": 2}, INVALID), ({"kind": 2}, INVALID), ({"D": 0}, INVALID), ({"D": 32769}, INVALID), ({"eps": -1.0}, INVALID),
                                    ({"eps": float("nan")}, INVALID), ({"post": 2}, INVALID), ({"pre": -1}, INVALID), ({"rows_per_gate": 0}, INVALID),
                                    ({"pre_weight": P + 2}, ALIGNMENT), ({"gate": P + 2}, ALIGNMENT), ({"ld_gate": 3, "rows_per_gate": 1}, INVALID), ({}, INVALID)])
def test_norm_descriptors(lib, k, want):
    g = binding.BlockNormGrads(P, 64, P, 64, P, None, P, None, P, 64)
    assert lib.bnn_block_norm(None, norm(**k), P, 64, P, 64, 4, P, 64, P, 64, P) == want
    assert lib.bnn_block_norm_backward(None, norm(**k), P, 64, P, 64, P, 64, P, 64, P, 4, ctypes.byref(g)) == want
    assert (lib.bnn_block_norm_workspace_bytes(norm(**k), 4) > 0) == (not k)


def test_norm_arguments(lib):
    g = binding.BlockNormGrads(P, 64, P, 64, P, None, P, None, P, 64)
    back = lambda d, g, block=P, stats=P, dn=P: lib.bnn_block_norm_backward(None, d, P, 64, dn, 64, P, 64, block, 64, stats, 4, g and ctypes.byref(g))  # noqa: E731
    assert lib.bnn_block_norm(None, norm(), P, 64, None, 0, 4, P, 64, P, 64, P) == INVALID        # post and gate without a block
    assert lib.bnn_block_norm(None, norm(pre=0), P, 64, P, 64, 4, P, 64, P, 64, P) == INVALID     # normed without pre
    assert lib.bnn_block_norm(None, norm(), P + 2, 64, P, 64, 4, P, 64, P, 64, P) == ALIGNMENT
    assert lib.bnn_block_norm(None, norm(), P, 64, P, 64, 4, P, 64, P, 64, P + 2) == ALIGNMENT
    assert back(norm(), None) == INVALID
    assert back(norm(), g, stats=None) == INVALID
    assert back(norm(gate=None), g) == INVALID                                                    # dgate without a gate
    assert back(norm(post=0), g) == INVALID                                                       # dpost_weight without post
    assert back(norm(pre=0), g) == INVALID


def test_dropout_arguments(lib):
    call = lambda dtype=0, x=P, ldx=8, y=P, rows=2, cols=8, p=0.5: lib.bnn_dropout(None, dtype, x, ldx, None, 0, y, 8, rows, cols, p, 1, 2)  # noqa: E731
    assert call() == INVALID and call(dtype=2) == INVALID and call(dtype=5) == INVALID
    assert call(rows=-1) == INVALID and call(cols=1 << 31) == INVALID and call(x=None) == INVALID and call(ldx=7) == INVALID
    assert call(p=-0.1) == INVALID and call(p=1.01) == INVALID and call(p=float("nan")) == INVALID
    assert call(x=P + 2) == ALIGNMENT and call(dtype=3, y=P + 1) == ALIGNMENT
