"""The residual of microscaled products: with operands of zeros every output is its own element of the residual, whatever way it takes - whole sectors, pieces through
shared memory, whole and half-width tiles, one accumulator and both, ahead of the sums or beside kept pre-activations."""
import pytest
import torch

from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


SHAPES = [  # M, N, columns between rows, elements before the first
    (4096, 4096, 0, 0), (4096, 4096, 16, 16), (4000, 4080, 8, 8), (4001, 4094, 2, 2), (4097, 3999, 1, 0), (4096, 4000, 0, 1), (5000, 2336, 0, 0),
    (1024, 1024, 0, 0), (1000, 1030, 2, 0), (1100, 1111, 1, 1), (20000, 130, 0, 0), (300, 30000, 0, 0), (7, 1000, 0, 0), (150, 333, 1, 0),
]


@pytest.mark.parametrize("dtype", (BF, HF), ids=("bf16", "f16"))
@pytest.mark.parametrize("xf,wf", (("e4m3", "e2m1"), ("e2m1", "e2m1")))
@pytest.mark.parametrize("M,N,pad,lead", SHAPES)
def test_every_output_has_its_own_element(ctx, M, N, pad, lead, xf, wf, dtype):
    x, w = ctx.mx_quantize(torch.zeros(M, 128, dtype=BF, device="cuda"), xf), ctx.mx_quantize(torch.zeros(N, 128, dtype=BF, device="cuda"), wf)
    i, j = torch.arange(M, device="cuda")[:, None], torch.arange(N, device="cuda")[None, :]

    def room(t):
        buf = torch.full((lead + M * (N + pad) + 64,), 77.0, dtype=t, device="cuda")
        return buf[lead:lead + M * (N + pad)].view(M, N + pad)[:, :N]

    r, y, pre = room(dtype), room(dtype), room(torch.float32)
    for act in ("none", "gelu"):
        layer = ctx.make_mx_linear(w, None, act, dtype=dtype)
        for part in (i % 256 + 0 * j, i // 256 + 0 * j, j % 256 + 0 * i, j // 256 + 0 * i):        # whole numbers up to 256: exact in both types
            r.copy_(part)
            for keeps in (False, True):
                y.fill_(-1.0), pre.fill_(5.0)
                ctx.mx_linear(layer, x, r, out=y, pre=pre if keeps else None)
                off = y != r
                assert not off.any(), f"act {act}, pre {keeps}: {int(off.sum())} outputs have another element, first {off.nonzero()[0].tolist()}"
                assert not keeps or (pre == 0).all()
            inplace = room(dtype)
            inplace.copy_(part)
            ctx.mx_linear(layer, x, inplace, out=inplace)
            assert torch.equal(inplace, r)
    ctx.device_status()
