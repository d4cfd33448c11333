"""Softmax cross entropy of a linear head and its gradients, from the formulas, in 64 bits
(torch double tensors, on the CPU or the GPU), with what error bounds need."""
import torch


def xent(h, w, target, weight=None, scale=1.0, mean=True):
    """h: T x H, w: V x H, target: T whole numbers, weight: T or None. Returns a dict:
    loss, lse (T), totals (2), dh (T x H), dw (V x H), and the sums of the products'
    magnitudes: la (T; the largest over the classes), dha, dwa."""
    v = w.shape[0]
    h, w = h.double(), w.double()
    live = (target >= 0) & (target < v)
    wt = torch.ones(h.shape[0], dtype=torch.float64, device=h.device) if weight is None \
        else weight.double()
    live &= wt != 0
    wt = torch.where(live, wt, torch.zeros_like(wt))
    h = torch.where(live[:, None], h, torch.zeros_like(h))
    at = target.long().clamp(0, v - 1)[:, None]
    z = h @ w.t()
    lse = torch.logsumexp(z, 1)
    zero = torch.zeros_like(lse)
    nll = lse - z.gather(1, at)[:, 0]
    loss = torch.where(live, wt * nll, zero)
    total = wt.sum()
    r = scale * wt
    if mean:
        r = r / total if float(total) != 0 else torch.zeros_like(r)
    p = torch.exp(z - lse[:, None])
    g = p.scatter_add(1, at, -torch.ones_like(at, dtype=torch.float64))
    # p - 1 of a likely target, without cancellation
    g.scatter_(1, at, torch.expm1(-nll)[:, None])
    g = torch.where(live[:, None], g * r[:, None], torch.zeros_like(g))
    return {"loss": loss, "lse": torch.where(live, lse, zero),
            "totals": torch.stack([loss.sum(), total]), "dh": g @ w, "dw": g.t() @ h,
            "la": (h.abs() @ w.abs().t()).amax(1), "dha": g.abs() @ w.abs(),
            "dwa": g.abs().t() @ h.abs(), "live": live, "r": r}
