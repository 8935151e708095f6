"""The few-bit operators run together: a stack of gated layers served from microscaled weights, and a training step of the 16-bit stack with its
gradients clipped together, both against 64 bits."""
import math

import pytest
import torch

import mx_reference as mx
import real_reference as ref
from paper_1602_02830_b200 import binding, build, nets

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def parts(M, D, F, dtype):
    g = torch.Generator(device="cuda").manual_seed(M + D)

    def mk(*shape, scale=1.0, shift=0.0):
        return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=g).to(dtype)

    layers = [{"Wg": mk(F, D, scale=D ** -0.5), "Wu": mk(F, D, scale=D ** -0.5), "Wd": mk(D, F, scale=F ** -0.5), "gate": mk(D, scale=0.1, shift=0.5),
               "post_weight": mk(D, scale=0.1, shift=1.0), "next_weight": mk(D, scale=0.1, shift=1.0)} for _ in range(2)]
    return mk, layers, mk(D, scale=0.1, shift=1.0), mk(M, D)


@pytest.mark.parametrize("M,D,F,dtype,wf,xf", [(1, 256, 700, BF, "e2m1", "e4m3"), (37, 104, 264, HF, "e4m3", "e4m3"), (300, 512, 1032, BF, "e2m1", "e2m1"), (600, 320, 512, BF, "e2m1", "e4m3")])
def test_feed_forward_mx(M, D, F, dtype, wf, xf):
    build.build()
    ctx = binding.Context(0)
    _, layers, first, x = parts(M, D, F, dtype)
    net = nets.prepare_feed_forward_mx(ctx, layers, first, weights=wf, activations=xf)
    stream, normed = nets.feed_forward_mx(ctx, net, x)
    ctx.device_status()

    def norm(v, w):
        return v / (v.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * w.double()

    s = x.double()
    n = mx.quantize(norm(s, first), xf)
    for i, L in enumerate(layers):
        Wg, Wu, Wd = (mx.quantize(L[k].double(), wf) for k in ("Wg", "Wu", "Wd"))
        h = mx.quantize(ref.act(n @ Wg.T, "silu") * (n @ Wu.T), xf)
        s = s + L["gate"].double() * norm(h @ Wd.T, L["post_weight"])
        n = norm(s, L["next_weight"])
        if i + 1 < len(layers):
            n = mx.quantize(n, xf)
    # Roundings to 16 bits: four in each layer.  A rounding of the block or the stream by half a unit moves a value across a border of two elements, half a
    # step (at most 2^-4 or 2^-2 of the value) apart, with probability unit / step: in the 2-norm sqrt(unit step) of the values, once per quantised matrix that
    # such a value enters (the second layer's norm and h, as the first layer's inputs are the same on both sides up to float32).
    unit, step = ref.UNIT[dtype], 2.0 ** -4 if xf == "e4m3" else 2.0 ** -2
    bound = 8 * unit + 2 * 2 * math.sqrt(unit * step)
    for t, w in ((stream, s), (normed, n)):
        assert float((t.double() - w).norm() / w.norm()) <= bound
    one = nets.feed_forward_mx(ctx, net, x[:1])                    # a single token agrees with the batch
    assert float((one[0].double() - stream[:1].double()).norm() / stream[:1].double().norm()) <= bound
    ctx.close()


def test_training_step_with_clipped_gradients():
    build.build()
    ctx = binding.Context(0)
    M, D, F, dtype = 70, 128, 264, BF
    mk, layers, first, x = parts(M, D, F, dtype)
    ds, dn = mk(M, D), mk(M, D)
    net = nets.prepare_feed_forward(ctx, layers, first)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws)
    keep = []
    nets.feed_forward(ctx, net, x, keep=keep)
    _, head, grads = nets.feed_forward_backward(ctx, net, keep, ds, dn)
    tensors = nets.feed_forward_gradients(head, grads)
    assert len(tensors) == 13
    before = [t.clone() for t in tensors]
    G = ctx.make_gradients(tensors)
    assert ctx.clip_workspace_bytes(G) <= ws.numel()
    norm = ctx.clip_gradients(G, 1.0)
    want = math.sqrt(math.fsum(float(t.double().pow(2).sum()) for t in before))
    assert want > 1 and abs(float(norm) - want) <= 2.0 ** -18 * want
    for t, b in zip(tensors, before):
        w = b.double() / (want + 1e-6)
        assert ((t.double() - w).abs() <= (ref.UNIT[dtype] + 2.0 ** -17) * w.abs() + 1e-38).all()
    # the updated weights, microscaled again, serve the next forward pass; the values they stand for are what a straight-through step trains on
    W = layers[0]["Wd"] - 0.1 * grads[0]["dWd"]
    values = torch.empty_like(W)
    q = ctx.mx_quantize(W, "e2m1", values=values)
    h = ctx.mx_quantize(mk(M, F), "e4m3")
    y = ctx.mx_linear(ctx.make_mx_linear(q), h)
    ref.check(y, *mx.linear(ctx.mx_values(h).double(), values.double(), None, None, "none", dtype)["y"], "y")
    ctx.set_workspace(None)
    ctx.close()
