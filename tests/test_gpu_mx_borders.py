"""Norms with a microscaled result beside the borders of two elements and of two shared exponents: the side is that of the unrounded value."""
import pytest
import torch

import mx_reference as mx
from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
FORMATS = ("e4m3", "e2m1")
EPS = 2.0 ** -20
# rows, columns, whether a block is added: one slot a thread, a ragged width, a whole team without optional parts, four slots behind predicates, widths off the 16-byte rule
SHAPES = [(1, 32768, False), (3, 4096, True), (2, 1000, True), (300, 4096, True), (300, 4096, False), (300, 4104, True), (300, 1011, True), (2, 20001, False)]


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def aim(target, shift):
    """One row s of small whole numbers, whose squares float32 adds up without an error, and float32 weights w with s w r beside `target` (float64), up to `shift`
    units of the weight apart; the values s w r in 64 bits, where they are told from the target by 2^-40, thirty-two times what 64 bits lose and the kernel's two floats may."""
    D = target.numel()
    j = torch.arange(D, device="cuda")
    s = (1 + j * 7 % 13).double() * torch.where(j % 3 == 0, -1.0, 1.0)
    r = 1 / (s.pow(2).mean() + EPS).sqrt()
    w = (target / (s * r)).float()
    for k in range(shift):
        w = torch.where(j % 7 == 2 * k + 1, torch.nextafter(w, 2 * w), torch.where(j % 7 == 2 * k + 2, torch.nextafter(w, 0 * w), w))
    v = s * w.double() * r
    return s, w, v, (v - target).abs() > 2.0 ** -40 * target.abs()


def normed(ctx, s, w, M, block, fmt):
    x = s.float().expand(M, -1).contiguous()
    layer = ctx.make_block_norm(s.numel(), torch.float32, eps=EPS, pre_weight=w)
    return ctx.block_norm_mx(layer, x, torch.zeros_like(x) if block else None, format=fmt)[1]


@pytest.mark.parametrize("shift", (0, 2))
@pytest.mark.parametrize("M,D,block", SHAPES)
@pytest.mark.parametrize("fmt", FORMATS)
def test_elements_beside_every_border(ctx, fmt, M, D, block, shift):
    """All borders of the format, those of its smallest elements (e4m3 below 2^-6; e2m1 0.25 and 0.75) among them."""
    t = mx.table(fmt).cuda()
    mid = (t[1:] + t[:-1]) / 2
    j = torch.arange(D, device="cuda")
    b = j // 32
    scale = torch.exp2((b % 17 - 8).double())
    target = scale * torch.where(j % 2 == 0, 1.0, -1.0) * mid[(j + b) % len(mid)]
    target = torch.where(j % 32 == 0, scale * 1.5 * 2.0 ** mx.EMAX[fmt], target)          # sets the block's exponent, beside no border
    s, w, v, sure = aim(target, shift)
    want = mx.quantize(v[None], fmt)[0].cpu()
    got = mx.read(normed(ctx, s, w, M, block, fmt))[0]
    sure = sure.cpu()
    assert sure.sum() > 0.99 * D
    off = (got != want) & sure
    assert not off.any(), f"{int(off.sum())} of {int(sure.sum()) * M} elements on the other side, first {off.nonzero()[0].tolist()}"


@pytest.mark.parametrize("shift", (0, 2))
@pytest.mark.parametrize("M,D,block", SHAPES)
@pytest.mark.parametrize("fmt", FORMATS)
def test_largest_values_beside_a_power_of_two(ctx, fmt, M, D, block, shift):
    """The block's exponent is that of its unrounded largest value: just below 2^k it is one less, and the largest value saturates."""
    j = torch.arange(D, device="cuda")
    b = j // 32
    target = torch.exp2((b % 23 - 11).double()) * torch.where(j % 32 == b % 32, 1.0, torch.where(j % 5 == 0, -0.3, 0.37))
    target = torch.where((j % 32 == (b + 5) % 32) & (b % 2 == 0), -torch.exp2((b % 23 - 11).double()), target)      # two of them in every other block
    s, w, v, sure = aim(target, shift)
    q = normed(ctx, s, w, M, block, fmt)
    got, _, scales = mx.read(q)
    X = mx.exponent(mx.blocks(v[None]).abs().amax(2), fmt).cpu()
    blocks = mx.blocks(torch.where(sure, 0.0, 1.0)[None]).amax(2).cpu() == 0
    assert blocks.sum() > 0.9 * blocks.numel()
    off = ((scales - 127 != X) & blocks)
    assert not off.any(), f"{int(off.sum())} of {int(blocks.sum()) * M} exponents off, first {off.nonzero()[0].tolist()}"
    if D % 32 == 0:
        inside = blocks.repeat_interleave(32, 1)
        assert torch.equal(got[inside.expand(M, -1)], mx.quantize(v[None], fmt).cpu().expand(M, -1)[inside.expand(M, -1)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", (1, 128, 1000, 4096))
def test_values_on_a_border(ctx, fmt, D):
    """Rows of one value without eps: the norm is the weight itself, a power of two or a border, and stays on it."""
    t = mx.table(fmt).cuda()
    mid = torch.cat([t[1:], (t[1:] + t[:-1]) / 2])
    for c in (1.0, 3.0, -7.0, 1.7, 100.3, 2.0 ** -30, 3e10):
        x = torch.full((2, D), c, device="cuda")
        w = mid[torch.arange(D, device="cuda") % len(mid)].float()
        w[::32] = 2.0 ** mx.EMAX[fmt] * (1 if D % 128 else 1.5)
        layer = ctx.make_block_norm(D, torch.float32, eps=0.0, pre_weight=w)
        got = mx.read(ctx.block_norm_mx(layer, x, format=fmt)[1])[0]
        want = mx.quantize(torch.sign(x.double()) * w.double(), fmt).cpu()
        assert torch.equal(got, want), (c, int((got != want).sum()))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", (1e-25, 1e-18, 1e-10, 1.0, 1e10, 1e18, 1e30, 1e35))
def test_rows_of_any_size(ctx, fmt, size):
    """float32 rows whose squares float32 does not hold: every element is that of the 64-bit result (one in 2^35 values is closer to a border than the kernel can tell)."""
    g = torch.Generator(device="cuda").manual_seed(int(abs(torch.tensor(size).log10())) + 1)
    x, w = torch.randn(40, 1032, device="cuda", generator=g) * size, 1 + torch.randn(1032, device="cuda", generator=g) / 5
    for eps in (0.0, 2.0 ** -20):
        layer = ctx.make_block_norm(1032, torch.float32, eps=eps, pre_weight=w)
        v = x.double() / (x.double().pow(2).mean(1, keepdim=True) + eps).sqrt() * w.double()
        assert torch.equal(mx.read(ctx.block_norm_mx(layer, x, format=fmt)[1])[0], mx.quantize(v, fmt).cpu()), eps


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", (64, 1000, 4096))
def test_rows_that_are_not_finite_or_zero(ctx, fmt, D):
    x = torch.randn(5, D, device="cuda")
    x[0, 5], x[1, 40], x[2], x[3, D - 1] = float("inf"), float("nan"), 0.0, -float("inf")
    w = torch.ones(D, device="cuda")
    q = ctx.block_norm_mx(ctx.make_block_norm(D, torch.float32, eps=1e-6, pre_weight=w), x, format=fmt)[1]
    v = x.double() / (x.double().pow(2).mean(1, keepdim=True) + float(torch.tensor(1e-6))).sqrt()
    want = mx.quantize(v, fmt).cpu()
    got = mx.read(q)[0]
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(torch.nan_to_num(got, 0.0), torch.nan_to_num(want, 0.0))
    assert got[0].isnan().sum() == 32 and got[1].isnan().all() and (got[2] == 0).all()
