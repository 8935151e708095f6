"""Uploading a network to the GPU through the C ABI: weights are sign-packed by bnn_pack_signs,
BatchNorm + Sign is folded into integer thresholds by bnn_fold_batchnorm, and the layer list is laid
out as the descriptor bnn_mlp_forward takes.  Everything numeric happens inside the library calls."""
from __future__ import annotations

import numpy as np
import torch

from . import binding


def _dev(ctx, a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    if dtype is not None:
        t = t.to(dtype)
    return t.to(f"cuda:{ctx.device}")


def pack_weight(ctx, W: np.ndarray) -> torch.Tensor:
    """K x N int8 +-1 host matrix -> packed N x K device operand."""
    return ctx.pack_signs(_dev(ctx, W, torch.int8), pack_along=1)


def fold(ctx, bn: dict, x_max: int):
    thr, flip = binding.fold_batchnorm(*(torch.from_numpy(np.asarray(bn[k])) for k in ("gamma", "beta", "mean", "var")),
                                       bn["eps"], x_max)
    return thr.to(f"cuda:{ctx.device}"), flip.to(f"cuda:{ctx.device}")


def prepare_mlp(ctx, weights, bns, expand_weights: bool = True):
    """Algorithm 4's inputs (binary weights W^b and BatchNorm parameters theta) -> device layer list.
    With expand_weights the hidden layers' weights are also stored as +-1 bytes (bnn_expand_signs) once, so the
    tensor-core engine does not have to expand them on every forward call."""
    layers = []
    L = len(weights)
    for k, (W, bn) in enumerate(zip(weights, bns)):
        K, N = W.shape
        d = {"Wp": pack_weight(ctx, W), "K": K, "N": N}
        if k < L - 1:
            d["thr"], d["flip"] = fold(ctx, bn, 255 * K if k == 0 else K)
            if expand_weights:
                # the first layer multiplies bytes by bytes; the others can run on either operand width
                d["W8"] = ctx.expand_signs(d["Wp"], N, K)
                if k > 0:
                    d["W4"] = ctx.expand_signs_f4(d["Wp"], N, K)
        else:
            for name in ("gamma", "beta", "mean", "var"):
                d[name] = _dev(ctx, bn[name], torch.float32)
            d["eps"] = bn["eps"]
        layers.append(d)
    desc, keep = ctx.make_mlp_desc(layers)
    return {"layers": layers, "desc": desc, "_keep": keep}


def prepare_convnet(ctx, layers, expand_weights: bool = True):
    """Conv layer list {wgt: Cout x 3 x 3 x Cin, bn, pool} -> packed device weights and folded thresholds
    (and, with expand_weights, the weights as +-1 bytes and, where used, 4-bit nibbles for the tensor-core engine)."""
    out = []
    for i, L in enumerate(layers):
        wgt = L["wgt"]
        Cout, _, _, Cin = wgt.shape
        flat = wgt.reshape(Cout, 9 * Cin)                      # [n][tap*Cin + c]
        if i == 0 and 9 * Cin <= 32:
            Wp = ctx.pack_signs(_dev(ctx, flat, torch.int8), pack_along=0)[:, 0].contiguous()
            x_max = 255 * 9 * Cin
        else:
            Wp = ctx.pack_signs(_dev(ctx, flat, torch.int8), pack_along=0)[:, :9 * Cin // 32].contiguous()
            x_max = 9 * Cin
        thr, flip = fold(ctx, L["bn"], x_max)
        d = {"Wp": Wp, "Cin": Cin, "Cout": Cout, "pool": bool(L.get("pool")), "thr": thr, "flip": flip}
        if expand_weights:
            # the same bits viewed as Cout rows of 9*Cin: re-pack with a legal leading dimension, then expand
            rows = ctx.pack_signs(_dev(ctx, flat, torch.int8), pack_along=0)
            d["W8"] = ctx.expand_signs(rows, Cout, 9 * Cin)
            if i > 0 and Cin % 128 == 0:                       # layers the library may run on 4-bit operands
                d["W4"] = ctx.expand_signs_f4(rows, Cout, 9 * Cin)
        out.append(d)
    return out


def convnet_output_shape(net, B: int, H: int, W: int):
    for L in net:
        if L["pool"]:
            H, W = H // 2, W // 2
    return (B, H, W, binding.words(net[-1]["Cout"]))


def convnet_forward(ctx, net, X_u8: torch.Tensor, keep_all: bool = False):
    """X_u8: B x H x W x C uint8 on the device.  One bnn_binary_conv2d call per layer; returns the packed
    output of the last layer (or of every layer)."""
    B, H, W, _ = X_u8.shape
    act = X_u8
    outs = []
    for L in net:
        act, _ = ctx.binary_conv2d(act, B, H, W, L["Cin"], L["Wp"], L["Cout"], pool=L["pool"], thr=L["thr"],
                                   flip=L["flip"])
        if L["pool"]:
            H, W = H // 2, W // 2
        if keep_all:
            outs.append(act)
    return outs if keep_all else act


def convnet_workspace_bytes(ctx, net, B: int, H: int, W: int) -> int:
    """Largest workspace any layer of `net` asks for on the tensor-core engine (0 if none qualifies)."""
    need = 0
    for L in net:
        need = max(need, ctx.conv_workspace_bytes(B, H, W, L["Cin"], L["Cout"], L["pool"]))
        if L["pool"]:
            H, W = H // 2, W // 2
    return need


def prepare_feed_forward(ctx, layers, first_weight=None, act: str = "silu", kind: str = "rms", eps: float = 1e-6, alpha: float = 1.0,
                         drop: float = 0.0):
    """Device weights of a stack of gated feed-forward layers (dicts with Wg, Wu [F, D], Wd [D, F] and optionally gate [D],
    post_weight [D] and next_weight [D], the scale of the norm in front of the following layer) -> handles of the real-valued operators.
    Layer i:  stream += gate * Norm(dropout((act(n Wg^T) * (n Wu^T)) Wd^T)),  n = Norm(stream)."""
    D, dtype = layers[0]["Wd"].shape[0], layers[0]["Wd"].dtype
    net = {"first": ctx.make_block_norm(D, dtype, kind=kind, eps=eps, pre_weight=first_weight), "layers": [], "drop": drop, "act": act}
    for L in layers:
        net["layers"].append({
            "up": ctx.make_gated(L["Wg"], L["Wu"], act), "down": ctx.make_linear(L["Wd"]),
            "norm": ctx.make_block_norm(D, dtype, kind=kind, eps=eps, alpha=alpha, gate=L.get("gate"), post=L.get("post_weight") is not None,
                                        post_weight=L.get("post_weight"), pre_weight=L.get("next_weight"))})
    return net


def feed_forward_workspace_bytes(ctx, net, x, backward: bool = False) -> int:
    """Workspace for feed_forward on rows like x, and for feed_forward_backward."""
    need = 0
    for L in net["layers"]:
        h = torch.empty(x.shape[0], L["up"].outer, dtype=x.dtype, device=x.device)
        need = max(need, ctx.gated_workspace_bytes(L["up"], x, backward), ctx.linear_workspace_bytes(L["down"], h, backward),
                   ctx.block_norm_workspace_bytes(L["norm"], x.shape[0]) if backward else 0)
    return max(need, ctx.block_norm_workspace_bytes(net["first"], x.shape[0]) if backward else 0)


def feed_forward(ctx, net, x, seed: int | None = None, keep: list | None = None):
    """x [M, D] through the stack: (stream, normed) after the last layer; one row is the form for a single token.  A layer is three or
    four calls (gated, linear, dropout, block_norm) of 5 to 10 us on the host each, more than a small layer takes for one row: capture the calls in a CUDA graph there.
    seed: trains with dropout (one offset per layer); keep: a list that receives what feed_forward_backward needs."""
    def stats():
        return ctx.empty(x.shape[0], 4, dtype=torch.float32) if keep is not None else None

    st = stats()
    stream, n = ctx.block_norm(net["first"], x, stats=st)
    if keep is not None:
        keep.append((x, st))
    for i, L in enumerate(net["layers"]):
        pre = ctx.empty(2, x.shape[0], L["up"].outer, dtype=torch.float32) if keep is not None else None
        h = ctx.gated(L["up"], n, pre=pre)
        block = ctx.linear(L["down"], h)
        if seed is not None and net["drop"] > 0:
            ctx.dropout(block, net["drop"], seed, i, out=block)
        st = stats()
        if keep is not None:
            keep.append((n, pre, h, stream, block, st))
        stream, n = ctx.block_norm(L["norm"], stream, block, stats=st)
    return stream, n


def feed_forward_backward(ctx, net, keep, dstream=None, dnormed=None, seed: int | None = None):
    """Gradients of feed_forward (with the same seed) from those of its two results: (dx, first norm's gradients, a dict per
    layer with dWg, dWu, dWd and the norm's dgate, dpost_weight, dpre_weight)."""
    grads = []
    for i in reversed(range(len(net["layers"]))):
        L, (n, pre, h, stream, block, st) = net["layers"][i], keep[i + 1]
        g = ctx.block_norm_backward(L["norm"], dstream, dnormed, stream, block, st)
        dstream, dblock = g["dx"], g["dblock"]
        if seed is not None and net["drop"] > 0:
            ctx.dropout(dblock, net["drop"], seed, i, out=dblock)
        dh, g["dWd"], _ = ctx.linear_backward(L["down"], dblock, h)
        dnormed, g["dWg"], g["dWu"] = ctx.gated_backward(L["up"], dh, n, pre)
        grads.insert(0, g)
    x, st = keep[0]
    first = ctx.block_norm_backward(net["first"], dstream, dnormed, x, stats=st)
    return first["dx"], first, grads


def feed_forward_gradients(first, grads) -> list:
    """The tensors of feed_forward_backward's parameter gradients, for Context.make_gradients: their norm is taken, and clipped, together."""
    names = ("dWg", "dWu", "dWd", "dgate", "dpost_weight", "dpre_weight")
    return [t for t in [first["dpre_weight"]] + [g[n] for g in grads for n in names] if t is not None]


def prepare_feed_forward_mx(ctx, layers, first_weight=None, act: str = "silu", kind: str = "rms", eps: float = 1e-6, alpha: float = 1.0,
                            weights: str = "e2m1", activations: str = "e4m3"):
    """The stack of prepare_feed_forward (same dicts) for serving in few bits: weights microscaled once, norms and gated projections with
    microscaled results.  weights, activations: formats; e2m1 activations go with e2m1 weights."""
    D, dtype = layers[0]["Wd"].shape[0], layers[0]["Wd"].dtype
    net = {"first": ctx.make_block_norm(D, dtype, kind=kind, eps=eps, pre_weight=first_weight), "layers": [], "format": activations}
    for L in layers:
        Wg, Wu, Wd = (ctx.mx_quantize(L[n], weights) for n in ("Wg", "Wu", "Wd"))
        net["layers"].append({
            "up": ctx.make_mx_gated(Wg, Wu, act, dtype=dtype), "down": ctx.make_mx_linear(Wd, dtype=dtype),
            "norm": ctx.make_block_norm(D, dtype, kind=kind, eps=eps, alpha=alpha, gate=L.get("gate"), post=L.get("post_weight") is not None,
                                        post_weight=L.get("post_weight"), pre_weight=L.get("next_weight"))})
    return net


def feed_forward_mx(ctx, net, x):
    """x [M, D] through the stack: (stream, normed) after the last layer, both of x's type.  A layer is three calls: gated projections with a microscaled
    result, the projection back, and the norms that tie it to the stream, whose result for the next layer is microscaled."""
    stream, n = ctx.block_norm_mx(net["first"], x, format=net["format"])
    for i, L in enumerate(net["layers"]):
        h = ctx.mx_gated(L["up"], n, out=ctx.make_mx(x.shape[0], L["up"].outer, net["format"]))
        block = ctx.mx_linear(L["down"], h)
        if i + 1 < len(net["layers"]):
            stream, n = ctx.block_norm_mx(L["norm"], stream, block, format=net["format"])
        else:
            stream, n = ctx.block_norm(L["norm"], stream, block)
    return stream, n
