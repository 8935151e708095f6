"""The norm of all gradients together and their clipping on the GPU against 64 bits."""
import math

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


def lend(ctx, n):
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n])
    return ws


def make(seed, sizes, types, scale=0.02, lead=0):
    """Contiguous tensors of these sizes; lead: elements before each in its own buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        buf = torch.full((lead + n + 40,), 77.0, dtype=t, device="cuda")
        buf[lead:lead + n] = torch.empty(n, device="cuda").normal_(0, scale, generator=g).to(t)
        out.append(buf[lead:lead + n])
    return out


def exact_norm(tensors):
    top = max([float(t.double().abs().max()) for t in tensors if t.numel()] + [0.0])
    return top * math.sqrt(math.fsum(float((t.double() / top).pow(2).sum()) for t in tensors if t.numel())) if top else 0.0


# 2^-19: float32 sums of 32 squares (32 additions and the squares, 33 half units); the rest in float64, and half a unit of the float32 norm
NORM_ERR = 33 * 2.0 ** -24 + 2.0 ** -24


def check(ctx, tensors, out, max_norm, eps=1e-6):
    norm = exact_norm(tensors)
    factor = min(1.0, max_norm / (norm + eps)) if norm + eps else 1.0
    before = [t.clone() for t in tensors]
    G = ctx.make_gradients(tensors, out)
    n = ctx.clip_workspace_bytes(G)
    ws = lend(ctx, n)
    got = ctx.clip_gradients(G, max_norm, eps)
    assert got.shape == () and got.dtype is FF and abs(float(got) - norm) <= NORM_ERR * norm + 1e-45
    for b, t, o in zip(before, tensors, tensors if out is None else out):
        want = b.double() * factor
        # the factor's own error is the norm's and its rounding; one rounding of the product
        ref.check(o, want, (NORM_ERR + 2.0 ** -23) * want.abs() + ref.UNIT[o.dtype] * want.abs() * (1 + 2.0 ** -20) + ref.TINY[o.dtype], "clipped")
        if out is not None:
            assert torch.equal(b, t), "an input was written"
        buf = o.untyped_storage()
        around = torch.empty(0, dtype=o.dtype, device="cuda").set_(buf)
        at = o.storage_offset()
        assert (around[:at] == 77).all() and (around[at + o.numel():] == 77).all(), "written around a tensor"
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)


SETS = [  # sizes, types, lead
    ([1], [FF], 0), ([0, 5, 0], [BF], 0), ([7, 8, 9, 31, 32, 33], [FF, BF, HF], 0), ([333 * 1011] * 3 + [333, 1011], [FF], 0), ([8191, 8192, 8193, 16384], [BF, FF], 0),
    ([8195, 40000, 3], [BF, HF, FF], 1), ([70001, 12345], [BF], 3), ([1 << 20, 100], [HF, FF], 5), ([3000000], [BF], 0), ([17] * 24, [BF], 0), ([17] * 25, [FF, BF], 0),
    ([100 + i % 7 for i in range(1000)], [BF, FF], 0), ([50 + i % 11 for i in range(2300)], [BF, FF, HF], 1), ([1 << 24, 5, 1 << 22], [BF, FF], 0),
]


@pytest.mark.parametrize("max_norm", (0.5, 1e9))
@pytest.mark.parametrize("inplace", (True, False), ids=("in place", "apart"))
@pytest.mark.parametrize("case", range(len(SETS)))
def test_clip(ctx, case, inplace, max_norm):
    sizes, types, lead = SETS[case]
    tensors = make(case, sizes, types, scale=1.0 if sum(sizes) < 1000 else 0.02, lead=lead)
    out = None
    if not inplace:
        out = make(case + 100, sizes, types, lead=lead if case % 2 else (lead + 1) % 4)      # on the tensors' footing, and on another
    check(ctx, tensors, out, max_norm)


@pytest.mark.parametrize("scale", (1e-30, 1e-18, 1e18, 1e25))
def test_squares_beyond_float32(ctx, scale):
    check(ctx, make(5, [1000, 50000], [FF, BF], scale=scale), None, scale, eps=0.0)


def test_not_clipped_is_untouched_and_zero_is_fine(ctx):
    t = make(1, [5000, 77], [BF, FF])
    before = [x.clone() for x in t]
    lend(ctx, 1 << 16)
    ctx.clip_gradients(ctx.make_gradients(t), 1e9)
    assert all(torch.equal(a, b) for a, b in zip(t, before))
    z = [torch.zeros(1000, device="cuda")]
    for eps in (0.0, 1e-6):
        assert float(ctx.clip_gradients(ctx.make_gradients(z), 0.0, eps=eps)) == 0.0 and (z[0] == 0).all()
    assert float(ctx.clip_gradients(ctx.make_gradients([]), 1.0)) == 0.0
    ctx.clip_gradients(ctx.make_gradients(t), 0.0)
    assert all((x == 0).all() for x in t)
    ctx.set_workspace(None)


def test_not_finite_follows_the_formula(ctx):
    lend(ctx, 1 << 16)
    t = make(2, [100, 20000], [FF, BF])
    t[1][7] = float("inf")
    assert float(ctx.clip_gradients(ctx.make_gradients(t), 1.0)) == math.inf
    assert (t[0] == 0).all() and t[1][7].isnan() and t[1].isnan().sum() == 1 and (torch.nan_to_num(t[1].float(), 0.0) == 0).all()
    t = make(2, [100, 20000], [FF, BF])
    t[0][3] = float("nan")
    assert math.isnan(float(ctx.clip_gradients(ctx.make_gradients(t), 1.0)))
    assert all(x.isnan().all() for x in t)
    ctx.set_workspace(None)


def test_the_same_call_gives_the_same_bits_and_needs_its_workspace(ctx):
    t = make(3, [123456, 1 << 21, 999], [BF, FF])
    out = [torch.empty_like(x) for x in t]
    G = ctx.make_gradients(t, out)
    ctx.set_workspace(None)
    with pytest.raises(binding.BnnError, match="workspace"):
        ctx.clip_gradients(G, 1.0)
    lend(ctx, ctx.clip_workspace_bytes(G))
    a = ctx.clip_gradients(G, 1.0).clone()
    first = [x.clone() for x in out]
    for _ in range(3):
        assert torch.equal(ctx.clip_gradients(G, 1.0), a) and all(torch.equal(x, y) for x, y in zip(out, first))
    side = torch.cuda.Stream()                                       # captured, and replayed on new gradients
    c = binding.Context(0, side)
    ws = torch.empty(c.clip_workspace_bytes(G), dtype=torch.uint8, device="cuda")
    c.set_workspace(ws)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.clip_gradients(G, 1.0)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            n = c.clip_gradients(G, 1.0)
        for x in t:
            x.mul_(3.0)
        graph.replay()
        side.synchronize()
    assert abs(float(n) - exact_norm(t)) <= NORM_ERR * float(n)
    ctx.set_workspace(None)
    c.set_workspace(None)
    del graph
    c.close()
