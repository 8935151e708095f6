"""Microscaled matrices in 64 bits, from the format's definition: the elements as a table, the nearest one by search; their layout in memory
byte by byte; and the products of represented values with the error model of real_reference.py."""
import math

import torch

import real_reference as ref

EMAX = {"e4m3": 8, "e2m1": 2}


def table(fmt):
    """The magnitudes in the order of their codes (e4m3: without the code for NaN)."""
    bits, bias, codes = (3, 7, 127) if fmt == "e4m3" else (1, 1, 8)
    out = []
    for c in range(codes):
        e, m = c >> bits, c & ((1 << bits) - 1)
        out.append(m * 2.0 ** (1 - bias - bits) if e == 0 else (1 + m / (1 << bits)) * 2.0 ** (e - bias))
    return torch.tensor(out, dtype=torch.float64)


def exponent(amax, fmt):
    """The shared exponent of blocks with these largest magnitudes (float64)."""
    f = torch.frexp(amax)[1] - 1
    return torch.where(amax > 0, f - EMAX[fmt], torch.full_like(f, -127)).clamp(-127, 127)


def codes_at(v, X, fmt):
    """Codes of the elements nearest to v 2^-X, even codes on ties, the largest beyond it; sign apart."""
    t = table(fmt).to(v.device)
    size = v.abs() * torch.exp2(-X.double())
    hi = torch.searchsorted(t, size.contiguous()).clamp(max=len(t) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = t[hi] - size, size - t[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def values_at(v, X, fmt):
    return torch.sign(v) * table(fmt).to(v.device)[codes_at(v, X, fmt)] * torch.exp2(X.double())


def blocks(v):
    M, K = v.shape
    return torch.nn.functional.pad(v, (0, -K % 32)).reshape(M, -1, 32)


def quantize(v, fmt):
    """What the microscaled form of the rows v (float64) stands for."""
    b = blocks(v)
    amax = b.abs().amax(2, keepdim=True)
    out = values_at(torch.nan_to_num(b, 0.0, 0.0, 0.0), exponent(torch.where(amax.isfinite(), amax, 0.0), fmt), fmt)
    return torch.where(amax.isfinite(), out, math.nan).reshape(v.shape[0], -1)[:, :v.shape[1]]


def read(q):
    """What an MxMatrix stands for, from its bytes: (values [rows, cols], values of the padding, scale bytes [rows, blocks])."""
    M, K = q.rows, q.cols
    raw, scales = q.values.cpu().long(), q.scales.cpu().long()
    if q.format == "e2m1":
        c = torch.stack((raw & 15, raw >> 4), 2).reshape(M, -1)
        sign, mag = c >> 3, c & 7
    else:
        c = raw
        sign, mag = c >> 7, c & 127
    t = torch.cat([table(q.format), torch.tensor([math.nan], dtype=torch.float64)])
    groups = -(-K // 128)
    r, b = torch.arange(M)[:, None], torch.arange(groups * 4)[None, :]
    s = scales[((r // 128) * groups + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4]
    X = torch.where(s == 255, math.nan, torch.exp2((s - 127).double())).repeat_interleave(32, 1)
    v = torch.where(sign == 1, -1.0, 1.0) * t[mag] * X
    return v[:, :K], c[:, K:], s[:, : -(-K // 32)]


def accept(got, v, err, fmt, what):
    """Whether `got` is what the microscaled form of some matrix within `err` of v stands for: for each block with the exponent of a largest magnitude
    within reach, every element between those of v - err and v + err."""
    b, e, g = blocks(v), blocks(err), blocks(got.double())
    hi, lo = (b.abs() + e).amax(2, keepdim=True), (b.abs() - e).clamp(min=0).amax(2, keepdim=True)
    fine = torch.zeros(b.shape[:2], dtype=torch.bool, device=v.device)
    for X in (exponent(lo, fmt), exponent(hi, fmt)):
        fine |= ((g >= values_at(b - e, X, fmt)) & (g <= values_at(b + e, X, fmt))).all(2)
    assert fine.all(), f"{what}: {int((~fine).sum())} of {fine.numel()} blocks are not those of any matrix within the bound, first {(~fine).nonzero()[0].tolist()}"


def linear(x, W, bias, residual, act, dtype):
    """{output: (value, bound)} of the dense layer of represented values x, W (float64), results of `dtype`; "raw": y before its rounding."""
    b = torch.zeros(W.shape[0], dtype=torch.float64, device=x.device) if bias is None else bias.double()
    z = x @ W.T + b
    ez = ref.gamma(x.shape[1]) * (x.abs() @ W.abs().T + b.abs())
    y, ey = ref.act(z, act), ref.act_bound(z, ez, act)
    if residual is not None:
        y = residual.double() + y
        ey = ey + 2.0 ** -23 * (residual.double().abs() + y.abs())
    return {"y": (y, ref.rounded(y, ey, dtype)), "raw": (y, ey), "pre": (z, ez + 1e-30)}


def gated(x, Wg, Wu, act, dtype):
    g, u = x @ Wg.T, x @ Wu.T
    k = ref.gamma(x.shape[1])
    eg, eu = k * (x.abs() @ Wg.abs().T), k * (x.abs() @ Wu.abs().T)
    a, ea = ref.act(g, act), ref.act_bound(g, eg, act)
    h = a * u
    eh = ea * (u.abs() + eu) + (a.abs() + ea) * eu + 2.0 ** -22 * h.abs()
    return {"h": (h, ref.rounded(h, eh, dtype)), "raw": (h, eh), "g": (g, eg + 1e-30), "u": (u, eu + 1e-30)}
