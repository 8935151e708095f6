"""Edges of the real-valued operators on the GPU."""
import pytest
import torch

import real_reference as ref
from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def normal(seed, *shape, dtype=BF, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=g).to(dtype)


@pytest.mark.parametrize("M,N,K", [(64, 1011, 512), (512, 1010, 1024), (3, 9, 8)])
@pytest.mark.parametrize("bias", (True, False), ids=("bias", "plain"))
def test_linear_backward_in_the_workspace_asked_for(ctx, M, N, K, bias):
    """x and W in whole 16-byte groups, contiguous dy not: a layer without activation copies dy."""
    x, W, dy = normal(1, M, K), normal(2, N, K, scale=K ** -0.5), normal(3, M, N)
    b = normal(4, N) if bias else None
    layer = ctx.make_linear(W, b)
    n = ctx.linear_workspace_bytes(layer, x, backward=True)
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n] if n else None)
    want = ref.linear(x, W, b, None, "none", dy)
    for key, t in zip(("dx", "dW", "db"), ctx.linear_backward(layer, dy, x)):
        if t is not None:
            ref.check(t, *want[key], key)
    ctx.device_status()
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)
