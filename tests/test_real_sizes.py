"""CPU-side checks of what the real-valued operators ask for before they launch anything."""
import os
import subprocess
import sys

import pytest
import torch

from paper_1602_02830_b200 import binding, build

BF = torch.bfloat16


@pytest.fixture(scope="module")
def host():
    """A context without a device, for the parts of the binding that only look at shapes: CPU tensors are on its device, -1."""
    build.build()
    c = object.__new__(binding.Context)
    c.device = -1
    return c


@pytest.mark.parametrize("act", ("none", "gelu"))
@pytest.mark.parametrize("M,N,K", [(64, 1011, 512), (512, 1010, 1024), (64, 1016, 512), (1, 1011, 512), (0, 3, 8)])
def test_linear_workspace_without_dy_is_that_of_contiguous_rows(host, M, N, K, act):
    layer = host.make_linear(torch.zeros(N, K, dtype=BF), torch.zeros(N, dtype=BF), act)
    x, dy = torch.zeros(M, K, dtype=BF), torch.zeros(M, N, dtype=BF)
    copied = act == "none" and M > 1 and N % 8 != 0             # dy is an operand, its rows are not whole 16-byte groups
    size = lambda aligned: int(binding.lib().bnn_linear_workspace_bytes(layer.ref, M, 1, aligned))  # noqa: E731
    assert host.linear_workspace_bytes(layer, x, backward=True) == size(0 if copied else 1)
    if act == "none":
        assert host.linear_workspace_bytes(layer, x, backward=True) == host.linear_workspace_bytes(layer, x, backward=True, dy=dy)
    assert host.linear_workspace_bytes(layer, x) == int(binding.lib().bnn_linear_workspace_bytes(layer.ref, M, 0, 1))


FAR = r"""
import ctypes
from paper_1602_02830_b200 import binding
P = 0x1000
for M in (1, 2, 7, 300, 0x7fff0000):
    for far in (M, 0x7fffffff, (1 << 62) + 1, (1 << 63) - 2, (1 << 63) - 1):
        d = ctypes.byref(binding.BlockNormDesc(3, 0, 64, 1e-6, 1.0, 0, 1, None, None, None, None, P, 64, far))
        print(M, far, binding.lib().bnn_block_norm_workspace_bytes(d, M), binding.lib().bnn_block_norm(None, d, P, 64, P, 64, M, P, 64, None, 0, None), flush=True)
"""


def test_one_gate_row_may_cover_more_rows_than_there_are():
    """rows_per_gate >= M means one gate row, whatever the number; in a process of its own, which an overflow would end."""
    build.build()
    run = subprocess.run([sys.executable, "-c", FAR], capture_output=True, text=True, cwd=os.path.dirname(build.HERE))
    assert run.returncode == 0, f"ended by {run.returncode} after\n{run.stdout}{run.stderr}"
    seen = {}
    for line in run.stdout.splitlines():
        M, far, *answer = line.split()
        assert seen.setdefault(M, answer) == answer, line
    assert len(seen) == 5


def test_layers_of_another_device_are_refused(host):
    """Only the addresses of a layer's tensors reach the library: on another device they would be read as that device's memory."""
    other = object.__new__(binding.Context)
    other.device = 0
    t = torch.zeros(4, 8, dtype=BF)
    linear, gated, norm = host.make_linear(t), host.make_gated(t, t), host.make_block_norm(8, BF, pre_weight=t[0])
    for call in (lambda: other.linear(linear, t), lambda: other.linear_backward(linear, t[:, :4], t), lambda: other.gated(gated, t),
                 lambda: other.gated_backward(gated, t[:, :4], t), lambda: other.block_norm(norm, t), lambda: other.block_norm_backward(norm, t, t, t)):
        with pytest.raises(ValueError, match="layer: its tensors are on"):
            call()
