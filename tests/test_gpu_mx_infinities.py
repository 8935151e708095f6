"""Pre-activations that are infinite, NaN or near the largest number: every activation follows its formula as it stands (z Phi(z) of minus infinity is NaN), for any number of rows
and in the layers of 16 bits alike."""
import math

import pytest
import torch

from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
INF, NAN = math.inf, math.nan
LIMITS = {  # act: values at +inf, -inf, and at a large finite z > 0 and -z
    "none": (INF, -INF, 1, -1), "relu": (INF, 0.0, 1, 0.0), "gelu": (INF, NAN, 1, 0.0), "gelu_tanh": (INF, NAN, 1, 0.0), "silu": (INF, NAN, 1, 0.0), "sigmoid": (1.0, 0.0, None, None),
    "htanh": (1.0, -1.0, None, None)}


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(torch.nan_to_num(a, 0.0, 1e9, -1e9), torch.nan_to_num(b, 0.0, 1e9, -1e9))


@pytest.mark.parametrize("act", LIMITS)
@pytest.mark.parametrize("dtype", (BF, HF), ids=("bf16", "f16"))
@pytest.mark.parametrize("M,N", [(1, 160), (4, 352), (1024, 1024), (3000, 2080), (2500, 2331)])
def test_activations_at_the_ends(ctx, M, N, dtype, act):
    big = 1e38 if dtype is BF else 6e4
    ends = [INF, -INF, NAN, big, -big]
    g = torch.Generator(device="cuda").manual_seed(M)
    x, W = torch.randn(M, 128, device="cuda", generator=g).to(dtype), (torch.randn(N, 128, device="cuda", generator=g) / 11).to(dtype)
    b = torch.zeros(N, device="cuda", dtype=dtype)
    at = torch.arange(3, N, 32, device="cuda")[:N // 32 // 2 * 2 : 2]                 # a column of every other block
    which = torch.arange(len(at), device="cuda") % 5
    b[at] = torch.tensor(ends, device="cuda").to(dtype)[which]
    layer = ctx.make_mx_linear(ctx.mx_quantize(W), b, act, dtype=dtype)
    q, pre = ctx.mx_quantize(x), ctx.empty(M, N, dtype=torch.float32)
    up, down, lp, ln = LIMITS[act]
    big = float(torch.tensor(big).to(dtype))
    want = torch.tensor([up, down, NAN, up if lp is None else big, down if lp is None else ln * big], device="cuda").to(dtype)[which].expand(M, -1)
    sixteen = ctx.linear(ctx.make_linear(W, b, act), x)
    for y in (ctx.mx_linear(layer, q), ctx.mx_linear(layer, q, pre=pre), sixteen):
        assert same(y[:, at], want), (act, y[0, at[:5]].tolist())
        rest = torch.ones(N, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert y[:, rest].isfinite().all()
    assert same(pre[:, at[which < 3]], torch.tensor(ends, device="cuda")[which[which < 3]].expand(M, -1))
    # a microscaled result: the block of an infinity or a NaN is NaN, the others are not
    v = ctx.mx_values(ctx.mx_linear(layer, q, out=ctx.make_mx(M, N)))
    bad = ~want[0].isfinite()
    for c, nan in zip((at // 32).tolist(), bad.tolist()):
        block = v[:, 32 * c:32 * c + 32]
        assert block.isnan().all() if nan else block.isfinite().all()
    ctx.device_status()
