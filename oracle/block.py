"""A residual block's operators from their formulas, in 64 bits (torch double tensors, on the
CPU or the GPU), with the sums of magnitudes that error bounds need."""
import math

import torch


def checkpoint(x):
    """8-bit checkpoint of x (rows x cols): its bytes (codes, then exponents) and the values
    that they stand for."""
    x = x.double()
    rows, cols = x.shape
    wide = -(-cols // 32) * 32
    v = torch.zeros(rows, wide, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, wide // 32, 32)
    number = torch.isfinite(v)
    top = torch.where(number, v.abs(), torch.zeros_like(v)).amax(2)
    e = torch.frexp(top).exponent - 1            # 2^e <= top < 2^(e + 1)
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp_min(-119)
    step = torch.exp2((e - 6).double())[:, :, None]
    q = torch.round(v / step).clamp(-127, 127)   # halves to even
    codes = torch.where(number, q, torch.full_like(q, -128)).to(torch.int8)
    value = torch.where(number, q * step, torch.full_like(q, math.nan))
    packed = torch.cat([codes.reshape(-1).view(torch.uint8), (e + 127).to(torch.uint8).reshape(-1)])
    return packed, value.view(rows, wide)[:, :cols].contiguous()


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """y, mean, rstd of each row."""
    x = x.double()
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight.double()
    return (y if bias is None else y + bias.double()), mean, rstd


def layer_norm_grad(dy, x, mean, rstd, weight=None, add=None):
    """A dict: dx, dweight, dbias, and what bounds need: g, xh, s1, s2 (the means), the means
    of the terms' magnitudes a1, a2, and the columns' sums of them aw, ab."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    g = dy if weight is None else dy * weight.double()
    s1, s2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - s1 - xh * s2)
    if add is not None:
        dx = dx + add.double()
    return {"dx": dx, "dweight": (dy * xh).sum(0), "dbias": dy.sum(0), "g": g, "xh": xh, "s1": s1,
            "s2": s2, "a1": g.abs().mean(1, keepdim=True),
            "a2": (g * xh).abs().mean(1, keepdim=True), "aw": (dy * xh).abs().sum(0),
            "ab": dy.abs().sum(0)}


def act(z, kind):
    return z if kind == "none" else z.clamp_min(0) if kind == "relu" else \
        z * torch.special.ndtr(z)


def slope(z, kind):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).to(z.dtype)
    # z times the density: 0 at infinities
    far = z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.special.ndtr(z) + torch.where(torch.isinf(z), torch.zeros_like(z), far)


def linear(x, w, bias=None, residual=None, kind="none"):
    """y, z and the sums of the products' magnitudes."""
    x, w = x.double(), w.double()
    z = x @ w.t()
    if bias is not None:
        z = z + bias.double()
    y = act(z, kind)
    return (y if residual is None else y + residual.double()), z, x.abs() @ w.abs().t()


def linear_grad(dy, x, w, z=None, kind="none"):
    """A dict: dz, dx, dw, dbias, and the sums of magnitudes ax, aw, ab."""
    dz = dy.double()
    if kind != "none":
        dz = dz * slope(z.double(), kind)
    o = {"dz": dz, "dbias": dz.sum(0), "ab": dz.abs().sum(0)}
    if w is not None:
        o["dx"], o["ax"] = dz @ w.double(), dz.abs() @ w.double().abs()
    if x is not None:
        t = dz.t().contiguous()
        o["dw"], o["aw"] = t @ x.double(), t.abs() @ x.double().abs()
    return o
