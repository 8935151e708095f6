"""CPU-side checks of what the real-valued operators ask for before they launch anything."""
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
