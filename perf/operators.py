"""Training operators of a classification head: their cases and plain forms.

Two operators, as a program that trains with this library calls them:

  dropout   y = residual + keep * x / q and its gradient, the mask drawn from a
            counter-based generator (Philox 4x32, 7 rounds) and stored nowhere;
  xent      softmax cross entropy of a linear head: per-row losses from features
            and the head's weights ("fwd"), or these with the loss-scaled
            gradients of both ("grad"); rows whose target lies outside the
            classes are masked.

Definition of the mask. Element i = row * cols + col takes the 16-bit half i % 2
(0: the low one) of word (i % 8) / 2 of the Philox block with the counter
(i / 8 mod 2^32, i / 2^35, step, site) and the key (seed mod 2^32, seed / 2^32); it is
kept where that number is below t = round((1 - p) * 65536), and kept elements are
multiplied by 65536 / t.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = 0xFFFFFFFF
MAX_ELEMS = 16384 * 4096                  # of a drawn dropout
MAX_FLOPS = 6.0 * 8192 * 4096 * 131072    # of a drawn loss with its gradients


# ---- the cases ---------------------------------------------------------------
def _drop(name, kind, rows, cols, x_ld, y_ld, z_ld, dtype, p):
    """kind: "fwd", "fwd_residual", "bwd_gate"; z: the residual or the gate."""
    return {"name": name, "op": "dropout", "kind": kind, "rows": rows, "cols": cols,
            "x_ld": x_ld, "y_ld": y_ld, "z_ld": z_ld, "dtype": dtype, "p": p}


def _xent(name, kind, rows, hidden, vocab, dtype, masked, h_ld=0, weights=False, mean=True,
          scale=1.0):
    """masked: share of rows without a target; h_ld: row stride of h (0: dense)."""
    return {"name": name, "op": "xent", "kind": kind, "rows": rows, "hidden": hidden,
            "vocab": vocab, "dtype": dtype, "masked": masked, "h_ld": h_ld,
            "weights": weights, "mean": mean, "scale": scale}


def listed():
    return [
        # a few rows of activations: launch latency
        _drop("dropout_small", "fwd", 32, 1024, 1024, 1024, 0, "f16", 0.5),
        # a dense block's layer output (growth rate 256) in its wide buffer, after the ReLU
        _drop("dropout_slice", "fwd", 65536, 256, 1024, 1024, 0, "f16", 0.5),
        # its gradient: out of the wide gradient buffer, gated by the ReLU, dense
        _drop("dropout_slice_grad", "bwd_gate", 65536, 256, 1280, 256, 1024, "f16", 0.5),
        # a sublayer's output added to its residual stream, large batch
        _drop("dropout_residual", "fwd_residual", 16384, 4096, 4096, 4096, 4096, "bf16", 0.1),
        # fp32 features whose width nothing divides
        _drop("dropout_ragged", "fwd", 8191, 1023, 1030, 1023, 0, "f32", 0.2),
        # one row scored: latency
        _xent("xent_one", "fwd", 1, 512, 8192, "bf16", 0.0),
        # a few rows scored against a large vocabulary: the weights are read once
        _xent("xent_few", "fwd", 48, 2048, 65536, "bf16", 0.0),
        # validation loss of a batch
        _xent("xent_eval", "fwd", 4096, 2048, 32768, "f16", 0.1),
        # pixel classes over the dense network's last features, unlabelled pixels masked
        _xent("xent_pixels", "grad", 65536, 512, 12, "f16", 0.1, scale=32768.0),
        # an ordinary training step, fp16 with its loss scale
        _xent("xent_step", "grad", 2048, 1024, 32000, "f16", 0.05, scale=32768.0),
        # nothing divides anything; weighted rows, a third masked, rows of a wider buffer
        _xent("xent_ragged", "grad", 1531, 777, 10007, "bf16", 0.33, h_ld=800, weights=True,
              mean=False, scale=0.01),
        # the largest step: a long batch, a large vocabulary
        _xent("xent_large", "grad", 8192, 4096, 131072, "bf16", 0.05),
    ]


def _between(rng, lo, hi):
    """A whole number, its logarithm spread evenly over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: half of them multiples of 64 (of 8 below 128), the others any number."""
    n = _between(rng, lo, hi)
    if rng.random() < 0.5:
        unit = 64 if n >= 128 else 8
        n = min(hi, max(lo, n // unit * unit))
    return n


def draw(rng):
    if rng.random() < 0.4:
        kind = rng.choice(["fwd", "fwd_residual", "bwd_gate"])
        cols = _width(rng, 16, 8192)
        rows = _between(rng, 1, max(1, MAX_ELEMS // cols))
        unit = 8 if cols % 8 == 0 else 1
        lds = [cols + unit * rng.choice([0, 0, rng.randint(1, 64)]) for _ in range(3)]
        # wide buffers stay within the largest dense one
        rows = min(rows, max(1, MAX_ELEMS // max(lds)))
        return dict(_drop("", kind, rows, cols, lds[0], lds[1], 0 if kind == "fwd" else lds[2],
                          rng.choice(["f16", "bf16", "f32"]), rng.choice([0.1, 0.2, 0.5])))
    kind = rng.choice(["fwd", "grad", "grad"])
    if rng.random() < 0.3:     # pixel classes
        hidden, vocab = _width(rng, 16, 1024), _between(rng, 2, 150)
        rows = _between(rng, 1024, 262144)
    else:                      # a vocabulary
        hidden, vocab = _width(rng, 64, 4096), _width(rng, 512, 131072)
        rows = _between(rng, 1, 8192)
    rows = min(rows, max(1, int(MAX_FLOPS / (6.0 * hidden * vocab))))
    dtype = rng.choice(["f16", "bf16"])
    h_ld = hidden + (rng.randint(1, 64) if rng.random() < 0.3 else 0)
    mean = rng.random() < 0.7
    scale = (32768.0 if dtype == "f16" else 1.0) * (1.0 if mean else 1.0 / rows)
    return _xent("", kind, rows, hidden, vocab, dtype, rng.choice([0.0, 0.05, 0.3]), h_ld=h_ld,
                 weights=rng.random() < 0.3, mean=mean, scale=scale)


def work(case):
    if case["op"] == "dropout":
        size = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["cols"]
        return {"bytes": n * size * (2 if case["kind"] == "fwd" else 3), "flops": 2 * n}
    # masked rows cost their target, their loss and, with gradients, their zeros
    t, h, v = case["rows"], case["hidden"], case["vocab"]
    live = t * (1.0 - case["masked"])
    grad = case["kind"] == "grad"
    b = 2 * live * h + 2 * v * h + t * (4 + 8) + (4 * t if case["weights"] else 0)
    if grad:
        b += 2 * t * h + 2 * v * h
    return {"bytes": b, "flops": (6.0 if grad else 2.0) * live * h * v}


# ---- inputs ------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(t, ld):
    """t's rows in a wider buffer (ld 0 or t's width: as it is)."""
    if ld in (0, t.shape[1]):
        return t.contiguous()
    wide = torch.zeros(t.shape[0], ld, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _prepare_dropout(case, seed):
    g = _gen(seed)
    rows, cols, dt = case["rows"], case["cols"], DT[case["dtype"]]
    n = lambda: torch.randn(rows, cols, generator=g, device=DEV)
    # forward: features after a ReLU, or a sublayer's output; backward: a gradient
    x = n()
    if case["kind"] == "fwd":
        x = x.clamp_min(0)
    z = None
    if case["kind"] == "fwd_residual":
        z = n()
    elif case["kind"] == "bwd_gate":   # the forward output: half positive, half of that kept
        z = torch.where(torch.rand(rows, cols, generator=g, device=DEV) < 0.5, n().clamp_min(0),
                        torch.zeros((), device=DEV))
    st = {"case": case, "x": _rows(x.to(dt), case["x_ld"]),
          "z": None if z is None else _rows(z.to(dt), case["z_ld"]),
          "seed": 0x9E3779B97F4A7C15 ^ seed, "site": 3 + seed % 5, "step": 1000 + seed % 7,
          "step_count": torch.tensor([seed % 11], dtype=torch.int32, device=DEV)}
    if own:
        import paper_1909_11150_amd as fg
        st["desc"] = fg.DropoutDesc.make(
            rows, cols, case["p"], st["seed"], site=st["site"], step=st["step"],
            dtype=fg.dtype_of(st["x"]), x_ld=case["x_ld"], y_ld=case["y_ld"], z_ld=case["z_ld"])
        st["y"] = _rows(torch.zeros(rows, cols, dtype=dt, device=DEV), case["y_ld"])
    return st


def _prepare_xent(case, seed):
    g = _gen(seed)
    t, h, v, dt = case["rows"], case["hidden"], case["vocab"], DT[case["dtype"]]
    w = torch.randn(v, h, generator=g, device=DEV) / math.sqrt(h)
    # few classes are frequent; the features lean towards their row's class by an amount
    # of their own, so that its probability lies anywhere between chance and almost one
    u = torch.rand(t, generator=g, device=DEV)
    target = (v * u * u).to(torch.int32).clamp_(0, v - 1)
    lean = (3.0 + math.log(v)) * torch.rand(t, 1, generator=g, device=DEV)
    x = torch.randn(t, h, generator=g, device=DEV) + lean * w[target.long()]
    off = torch.rand(t, generator=g, device=DEV) < case["masked"]
    target = torch.where(off, torch.full_like(target, -100), target)
    # what stands in masked rows is anything
    x = torch.where(off[:, None], torch.full_like(x, math.nan), x)
    st = {"case": case, "h": _rows(x.to(dt), case["h_ld"]), "w": w.to(dt).contiguous(),
          "target": target, "weight": None}
    if case["weights"]:
        st["weight"] = torch.rand(t, generator=g, device=DEV) * 2.0
    if own:
        import paper_1909_11150_amd as fg
        e = lambda *s: torch.empty(*s, dtype=dt, device=DEV)
        f = lambda *s: torch.empty(*s, dtype=torch.float32, device=DEV)
        d = fg.XentDesc.make(t, h, v, dtype=fg.dtype_of(st["h"]), h_ld=case["h_ld"],
                             mean=case["mean"], scale=case["scale"])
        grad = case["kind"] == "grad"
        st.update(desc=d, loss=f(t), lse=f(t),
                  totals=f(2),
                  ws=torch.empty(max(16, fg.linear_xent_workspace_bytes(d, grad)),
                                 dtype=torch.uint8, device=DEV))
        if grad:
            st.update(dh=e(t, h), dw=e(v, h),
                      flag=torch.zeros(1, dtype=torch.int32, device=DEV))
    return st


def prepare(case, seed):
    return _prepare_dropout(case, seed) if case["op"] == "dropout" else _prepare_xent(case, seed)


# ---- plain forms -------------------------------------------------------------
def _mul32(a, m):
    """High and low 32 bits of a * m; a: int64 tensor below 2^32, m a number."""
    lo = a * (m & 0xFFFF)
    hi = a * (m >> 16) + (lo >> 16)
    return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)


def _kept(n, seed, step, site, threshold):
    """Truth value for each of n elements."""
    b = torch.arange((n + 7) // 8, dtype=torch.int64, device=DEV)
    c0, c1 = b & LOW, b >> 32
    c2, c3 = step + torch.zeros_like(b), torch.full_like(b, site)
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(7):
        h0, l0 = _mul32(c0, M0)
        h1, l1 = _mul32(c2, M1)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    words = torch.stack([c0, c1, c2, c3], dim=1)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=2)
    return (halves < threshold).view(-1)[:n]


def _plain_dropout(st):
    case = st["case"]
    rows, cols = case["rows"], case["cols"]
    thr = round((1.0 - case["p"]) * 65536)
    step = (st["step"] + st["step_count"].long()) & LOW
    keep = _kept(rows * cols, st["seed"], step, st["site"], thr).view(rows, cols)
    if case["kind"] == "bwd_gate":
        keep = keep & (st["z"] > 0)
    zero = torch.zeros((), device=DEV)
    y = torch.where(keep, st["x"].float() * (65536.0 / thr), zero)
    if case["kind"] == "fwd_residual":
        y = st["z"].float() + y
    return y.to(DT[case["dtype"]])


def _plain_xent(st):
    case = st["case"]
    dt = DT[case["dtype"]]
    v = case["vocab"]
    target = st["target"].long()
    live = (target >= 0) & (target < v)
    h = torch.where(live[:, None], st["h"].float(), torch.zeros((), device=DEV))
    w = st["w"].float()
    weight = live.float() if st["weight"] is None else st["weight"] * live
    at = target.clamp(0, v - 1)[:, None]
    logits = h @ w.t()
    top = logits.max(dim=1, keepdim=True).values
    e = (logits - top).exp_()
    total = e.sum(dim=1, keepdim=True)
    lse = top + total.log()
    loss = weight * (lse - logits.gather(1, at))[:, 0]
    lse = torch.where(live, lse[:, 0], torch.zeros((), device=DEV))
    totals = torch.stack([loss.sum(), weight.sum()])
    if case["kind"] == "fwd":
        return loss, lse, totals
    del logits
    r = case["scale"] * weight
    if case["mean"]:
        r = torch.where(totals[1] != 0, r / totals[1], torch.zeros((), device=DEV))
    g = e.div_(total)
    g.scatter_add_(1, at, torch.full_like(top, -1.0))
    g.mul_(r[:, None])
    dh = (g @ w).to(dt)
    dw = (g.t() @ h).to(dt)
    flag = (~torch.isfinite(dw)).any().to(torch.int32)[None]
    return loss, lse, totals, dh, dw, flag


def _own_dropout(st):
    import paper_1909_11150_amd as fg
    case = st["case"]
    if case["kind"] == "bwd_gate":
        fg.dropout_bwd(st["desc"], st["x"], st["y"], gate=st["z"], step_count=st["step_count"])
    else:
        fg.dropout_fwd(st["desc"], st["x"], st["y"], residual=st["z"],
                       step_count=st["step_count"])
    return st["y"]


def _own_xent(st):
    import paper_1909_11150_amd as fg
    out = (st["loss"], st["lse"], st["totals"])
    kw = dict(lse=st["lse"], totals=st["totals"], weight=st["weight"], ws=st["ws"])
    if st["case"]["kind"] == "fwd":
        fg.linear_xent_fwd(st["desc"], st["h"], st["w"], st["target"], st["loss"], **kw)
        return out
    fg.linear_xent_grad(st["desc"], st["h"], st["w"], st["target"], st["loss"], st["dh"],
                        st["dw"], found_nonfinite=st["flag"], **kw)
    return out + (st["dh"], st["dw"], st["flag"])


def run(state):
    if state["case"]["op"] == "dropout":
        return _own_dropout(state) if own else _plain_dropout(state)
    return _own_xent(state) if own else _plain_xent(state)


# ---- values in 64 bits -------------------------------------------------------
def _exact_dropout(case, st):
    rows, cols = case["rows"], case["cols"]
    u = np.uint64
    mask, s32, s16 = u(LOW), u(32), u(16)
    n = rows * cols
    x0 = np.arange(-(-n // 8), dtype=np.uint64)
    x1 = x0 >> s32
    x0 = x0 & mask
    step = (st["step"] + int(st["step_count"].item())) & LOW
    x2, x3 = np.full_like(x0, step), np.full_like(x0, st["site"])
    for r in range(7):
        k0 = u(((st["seed"] & LOW) + r * W0) & LOW)
        k1 = u(((st["seed"] >> 32) + r * W1) & LOW)
        p, q = x0 * u(M0), x2 * u(M1)
        x0, x1, x2, x3 = (q >> s32) ^ x1 ^ k0, q & mask, (p >> s32) ^ x3 ^ k1, p & mask
    out = np.empty((x0.size, 8), dtype=np.uint16)
    for j, word in enumerate((x0, x1, x2, x3)):
        out[:, 2 * j] = word & u(0xFFFF)
        out[:, 2 * j + 1] = word >> s16
    threshold = round((1.0 - case["p"]) * 65536)
    keep = (out.reshape(-1)[:n] < threshold).reshape(rows, cols)
    x = st["x"].double().cpu().numpy()
    if case["kind"] == "bwd_gate":
        keep &= st["z"].float().cpu().numpy() > 0
    y = np.where(keep, x * (65536.0 / threshold), 0.0)
    if case["kind"] == "fwd_residual":
        y += st["z"].double().cpu().numpy()
    return torch.from_numpy(y)


def _exact_xent(case, st):
    rows, hidden, v = case["rows"], case["hidden"], case["vocab"]
    w = st["w"].double()
    weight = torch.ones(rows, dtype=torch.float64, device=DEV) if st["weight"] is None \
        else st["weight"].double()
    live = torch.nonzero((st["target"] >= 0) & (st["target"] < v))[:, 0]
    weight = weight[live]
    loss = torch.zeros(rows, dtype=torch.float64, device=DEV)
    lse = torch.zeros_like(loss)
    dh = torch.zeros(rows, hidden, dtype=torch.float64, device=DEV)
    dw = torch.zeros(v, hidden, dtype=torch.float64, device=DEV)
    factor = case["scale"]
    if case["mean"]:
        whole = float(weight.sum())
        factor = factor / whole if whole else 0.0
    piece = max(1, (1 << 28) // v)     # rows at a time: 2 GiB of logits
    for i in range(0, live.numel(), piece):
        at = live[i:i + piece]
        wt = weight[i:i + piece]
        x = st["h"][at].double()
        y = st["target"][at].long()
        one = torch.arange(at.numel(), device=DEV)
        z = x @ w.t()
        l = torch.logsumexp(z, dim=1)
        lse[at] = l
        loss[at] = wt * (l - z[one, y])
        if case["kind"] == "grad":
            z.sub_(l[:, None]).exp_()
            z[one, y] -= 1.0
            z.mul_((factor * wt)[:, None])
            dh[at] = z @ w
            dw.add_(z.t() @ x)
    totals = torch.stack([loss.sum(), weight.sum()])
    if case["kind"] == "fwd":
        return loss, lse, totals
    return loss, lse, totals, dh, dw, None


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return _exact_dropout(case, st) if case["op"] == "dropout" else _exact_xent(case, st)
