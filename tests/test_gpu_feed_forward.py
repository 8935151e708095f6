"""A stack of gated feed-forward layers run with the real-valued operators together, forward and backward, against the same
stack in 64 bits."""
import pytest
import torch

import real_reference as ref
from paper_1602_02830_b200 import binding, build, nets

pytestmark = pytest.mark.gpu


def stack64(x, first, layers, masks, act, p):
    def norm(v, w):
        return v / (v.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * w
    s, n = x, norm(x, first)
    for L, mask in zip(layers, masks):
        b = (ref.act(n @ L["Wg"].T, act) * (n @ L["Wu"].T)) @ L["Wd"].T
        if mask is not None:
            b = b * mask / (1 - p)
        s = s + L["gate"] * norm(b, L["post_weight"])
        n = norm(s, L["next_weight"])
    return s, n


@pytest.mark.parametrize("M,D,F,dtype,p", [(1, 256, 700, torch.bfloat16, 0.0), (37, 104, 264, torch.float16, 0.25), (300, 512, 1032, torch.bfloat16, 0.1)])
def test_feed_forward_stack(M, D, F, dtype, p):
    build.build()
    ctx = binding.Context(0)
    g = torch.Generator(device="cuda").manual_seed(M)

    def mk(*shape, scale=1.0, shift=0.0):
        return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=g).to(dtype)

    layers = [{"Wg": mk(F, D, scale=D ** -0.5), "Wu": mk(F, D, scale=D ** -0.5), "Wd": mk(D, F, scale=F ** -0.5), "gate": mk(D, scale=0.1, shift=0.5),
               "post_weight": mk(D, scale=0.1, shift=1.0), "next_weight": mk(D, scale=0.1, shift=1.0)} for _ in range(2)]
    first, x, ds, dn = mk(D, scale=0.1, shift=1.0), mk(M, D), mk(M, D), mk(M, D)
    net = nets.prepare_feed_forward(ctx, layers, first, drop=p)
    ws = torch.empty(max(256, nets.feed_forward_workspace_bytes(ctx, net, x, backward=True)), dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws)
    keep = []
    stream, normed = nets.feed_forward(ctx, net, x, seed=77, keep=keep)
    dx, dfirst, grads = nets.feed_forward_backward(ctx, net, keep, ds, dn, seed=77)
    ctx.device_status()
    masks = [ref.kept(M, D, p, 77, i).cuda().double() if p else None for i in range(2)]
    big = [{k: v.double().requires_grad_(True) for k, v in L.items()} for L in layers]
    X, W0 = x.double().requires_grad_(True), first.double().requires_grad_(True)
    s64, n64 = stack64(X, W0, big, masks, "silu", p)
    flat = [X, W0] + [L[k] for L in big for k in ("Wg", "Wu", "Wd", "gate", "post_weight", "next_weight")]
    want = torch.autograd.grad([s64, n64], flat, [ds.double(), dn.double()])
    got = [dx, dfirst["dpre_weight"]] + [t for q in grads for t in (q["dWg"], q["dWu"], q["dWd"], q["dgate"], q["dpost_weight"], q["dpre_weight"])]
    # every path has at most 24 roundings to 16 bits (two layers, twelve each way), independent of one another: in the 2-norm
    # their relative sizes add up to at most 24 half units, amplified at most twice by the norms' divisions
    for t, w in [(stream, s64.detach()), (normed, n64.detach()), *zip(got, want)]:
        assert float((t.double() - w).norm() / w.norm()) <= 48 * ref.UNIT[dtype]
    one = nets.feed_forward(ctx, net, x[:1])                       # the form for a single token agrees with the batch
    if not p:
        assert float((one[0].double() - stream[:1].double()).norm() / stream[:1].double().norm()) <= 24 * ref.UNIT[dtype]
    ctx.set_workspace(None)
    ctx.close()
