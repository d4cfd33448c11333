"""linear_xent_fwd and linear_xent_grad against the formulas in 64 bits: every type, sizes
from one row and two classes on, widths, strides and class counts that nothing divides,
masked rows that hold anything, weights, several pieces of rows, values at the ends of the
range, refusals on the device side (nothing), graphs and streams.

Bounds, derived from the arithmetic (u = 2^-24; v = the storage type's half unit in the
last place, 2^-11 or 2^-8), elementwise:
  logits   products of 16-bit values are exact; the fp32 sum over H runs in steps of 16:
           |dl| <= 4 (H/16 + 16) u sum |h w|
  lse      the largest |dl|, the exponentials' and the sum's relative error (at most 300 u:
           64 additions in a lane, joins, 2 u each for the exponentials), and roundings
           of lse itself (4 u |lse|)
  loss     |w| times the errors of lse and of the target's logit
  G        relative: v (its rounding) + 2^-11 (the fp16 numerators) + twice the logits' and
           lse's errors; the target's entry r (p - 1) also moves by r p (dl + dlse), whatever
           is left of it; below the smallest normal: 2^-39 of the largest
  dh, dw   the sum of |G||W| (|G||h|) times G's error and 4 (n/16 + 64) u for the sum,
           plus the store's rounding v |x| and half its smallest subnormal number.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_1909_11150_amd as fg
from oracle.xent import xent

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def inputs(t, h, v, dt, seed, masked=0.2, weights=False, gain=1.0, h_ld=0, w_ld=0):
    rng = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))
    w = f(v, h) / np.sqrt(h)
    target = torch.from_numpy((v * rng.random(t) ** 2).astype(np.int32)).clamp_(0, v - 1)
    lean = torch.from_numpy(rng.random((t, 1)).astype(np.float32)) * (3 + np.log(v))
    x = (f(t, h) + lean * w[target.long()]) * gain
    off = torch.from_numpy(rng.random(t) < masked)
    x[off] = float("nan")
    bad = torch.from_numpy(rng.choice(np.array([-100, -1, v, v + 5, 2 ** 31 - 1, -2 ** 31],
                                               dtype=np.int64), t)).to(torch.int32)
    target = torch.where(off, bad, target)

    def rows(a, ld):
        ld = ld or a.shape[1]
        b = torch.full((a.shape[0], ld), float("nan"), dtype=TYPES[dt])
        b[:, :a.shape[1]] = a.to(TYPES[dt])
        return b.cuda()[:, :a.shape[1]]
    wt = torch.from_numpy(rng.uniform(-1, 2, t).astype(np.float32)) if weights else None
    return rows(x, h_ld), rows(w, w_ld), target.cuda(), wt.cuda() if weights else None


def call(h, w, target, weight, grad=True, mean=True, scale=1.0, dh=True, dw=True, stream=None,
         dh_ld=0, dw_ld=0):
    t, hid = h.shape
    v = w.shape[0]
    ld = lambda a: 0 if a.is_contiguous() else a.stride(0)
    d = fg.XentDesc.make(t, hid, v, dtype=fg.dtype_of(h), mean=mean, scale=scale, h_ld=ld(h),
                         w_ld=ld(w), dh_ld=dh_ld, dw_ld=dw_ld)
    need = fg.linear_xent_workspace_bytes(d, grad)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN wherever read
    f = lambda n: torch.full((n,), 7.0, device="cuda")
    out = {"loss": f(t), "lse": f(t), "totals": f(2)}
    kw = dict(lse=out["lse"], totals=out["totals"], weight=weight, ws=ws, stream=stream)
    if not grad:
        fg.linear_xent_fwd(d, h, w, target, out["loss"], **kw)
        return out
    wide = lambda n, ld: torch.full((n, ld or hid), 3.0, dtype=h.dtype, device="cuda")
    a = wide(t, dh_ld) if dh else None
    b = wide(v, dw_ld) if dw else None
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    fg.linear_xent_grad(d, h, w, target, out["loss"], None if a is None else a[:, :hid],
                        None if b is None else b[:, :hid], found_nonfinite=flag, **kw)
    for x in (a, b):   # columns beside a row's are left alone
        if x is not None and x.shape[1] > hid:
            assert bool((x[:, hid:] == 3).all())
    out.update(flag=flag, dh=None if a is None else a[:, :hid],
               dw=None if b is None else b[:, :hid])
    return out


def check(out, h, w, target, weight, dt, mean=True, scale=1.0, gpu_oracle=False):
    dev = (lambda x: x) if gpu_oracle else (lambda x: x.cpu())
    opt = lambda x: None if x is None else dev(x)
    H, V, T = h.shape[1], w.shape[0], h.shape[0]
    o = xent(dev(h), dev(w), dev(target), opt(weight), scale, mean)
    wt = torch.ones(T, dtype=torch.float64) if weight is None else weight.double().cpu()
    wt = torch.where(o["live"], wt.to(o["loss"].device), torch.zeros_like(o["loss"]))
    dl = 4 * (H / 16 + 16) * U * o["la"]
    dlse = dl + 300 * U + 4 * U * (o["lse"].abs() + 32)
    dloss = wt.abs() * (dl + dlse) + 2 * U * o["loss"].abs()

    def near(name, got, want, bound):
        got = dev(got).double()
        err = (got - want).abs()
        assert bool(torch.isfinite(got).all()), name
        worst = (err / bound.clamp_min(1e-300)).max() if err.numel() else 0
        print(f"{name}: {float(worst):.3f} of the bound", flush=True)
        assert bool((err <= bound).all()), f"{name}: {float(worst):.3f} of the bound"

    near("lse", out["lse"], o["lse"], torch.where(o["live"], dlse, torch.zeros_like(dlse)))
    near("loss", out["loss"], o["loss"], torch.where(o["live"], dloss, torch.zeros_like(dlse)))
    # summed in 64 bits from the fp32 losses, rounded once
    sums = torch.stack([dloss.sum() + U * o["loss"].abs().sum(), U * wt.abs().sum() * 2])
    near("totals", out["totals"], o["totals"], sums + 1e-30)
    if "dh" not in out:
        return o
    dg = HALF[dt] + 2.0 ** -11 + 2 * (dl + dlse) + 16 * U     # per row, relative
    floor = 2.0 ** -39 * o["r"].abs().max()
    tot = U if not mean else 4 * U
    moved = o["r"].abs() * (dl + dlse) * o["live"]
    at = dev(target).long().clamp(0, V - 1)
    if out["dh"] is not None:
        b = o["dha"] * (dg[:, None] + 4 * (V / 16 + 64) * U + tot) + \
            floor * dev(w).double().abs().sum(0) + moved[:, None] * dev(w).double().abs()[at]
        b = b * (1 + HALF[dt]) + HALF[dt] * o["dh"].abs() + TINY[dt]
        near("dh", out["dh"], o["dh"], torch.where(o["live"][:, None], b, torch.zeros_like(b)))
    if out["dw"] is not None:
        hl = torch.where(o["live"][:, None], dev(h).double(), torch.zeros_like(dev(h).double()))
        b = o["dwa"] * (dg.max() + 4 * (T / 16 + 64) * U + tot) + floor * hl.abs().sum(0)
        b = b.index_add(0, at, moved[:, None] * hl.abs())
        near("dw", out["dw"], o["dw"], b * (1 + HALF[dt]) + HALF[dt] * o["dw"].abs() + TINY[dt])
        assert int(out["flag"]) == 0
    return o


# rows, hidden, classes
SIZES = [(1, 1, 1), (1, 8, 2), (2, 5, 3), (1, 64, 513), (17, 64, 64), (63, 40, 130), (64, 128, 257),
         (65, 72, 1000), (130, 33, 300), (300, 257, 77), (257, 520, 1025), (700, 96, 12),
         (1030, 64, 5), (3, 1000, 2049), (129, 64, 4100)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradients_match_the_formulas(dt, size):
    print(dt, size, flush=True)
    x = inputs(*size, dt, seed=sum(size))
    scale = 4096.0 if dt == "f16" else 1.0
    check(call(*x, scale=scale), *x, dt, scale=scale)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("size", [(1, 64, 2), (5, 24, 1000), (200, 129, 700), (1, 512, 5000)],
                         ids=str)
def test_losses_alone(dt, size):
    x = inputs(*size, dt, seed=1)
    check(call(*x, grad=False), *x, dt)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("mean", [False, True])
def test_weights_and_strides(dt, mean):
    """Weighted rows (some negative, some 0), every tensor in a wider buffer whose other
    columns hold NaN."""
    h, w, t, wt = inputs(333, 104, 419, dt, 5, weights=True, h_ld=136, w_ld=112)
    wt[::7] = 0.0
    out = call(h, w, t, wt, mean=mean, scale=64.0, dh_ld=110, dw_ld=120)
    check(out, h, w, t, wt, dt, mean=mean, scale=64.0)
    assert float(out["loss"][::7].abs().sum()) == 0 and float(out["dh"][::7].abs().sum()) == 0


@pytest.mark.parametrize("dt", TYPES)
def test_odd_strides_and_addresses(dt):
    """Rows that no 16-byte access fits: odd strides, addresses off by an element."""
    h, w, t, wt = inputs(70, 48, 90, dt, 6, h_ld=51, w_ld=53)
    one = lambda x: torch.cat([x.new_zeros(1), x.reshape(-1)])[1:].view(x.shape)
    h, w1 = one(h), one(w)
    assert h.data_ptr() % 16 == w1.data_ptr() % 16 == 2
    out = call(h, w, t, wt, dh_ld=49, dw_ld=51)
    check(out, h, w, t, wt, dt)
    check(call(h, w1, t, wt), h, w1, t, wt, dt)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hidden", [7, 8, 9, 12, 15, 31, 65, 66, 127, 131])
def test_any_width(dt, hidden):
    """Widths around a chunk of 8 and a stage of 64, rows followed by NaN."""
    for t, v, ld in ((40, 300, 0), (150, 50, hidden + 3)):
        print(dt, hidden, t, v, ld, flush=True)
        x = inputs(t, hidden, v, dt, hidden, h_ld=ld, w_ld=ld)
        x[1][v // 2:, 0] = 4.0      # a neighbour's first element is not to be taken in
        check(call(*x, scale=64.0, dw_ld=ld), *x, dt, scale=64.0)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows", [64, 65, 127, 200, 256, 257])
def test_rows_around_those_kept_in_place(dt, rows):
    """Rows that stay where they are, and that are copied first, with and without weights,
    from no masked row to nothing else, in narrow rows too."""
    for hidden, classes, share, weights in ((88, 513, 0.3, True), (3, 300, 0.1, False),
                                            (200, 1000, 0.0, True), (64, 400, 1.0, True),
                                            (72, 290, 0.98, False)):
        print(dt, rows, hidden, classes, share, flush=True)
        x = inputs(rows, hidden, classes, dt, rows, masked=share, weights=weights, h_ld=hidden + 5)
        check(call(*x, scale=64.0), *x, dt, scale=64.0)
        check(call(*x, mean=False, grad=False), *x, dt, mean=False)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("classes", [9, 40, 90, 200])
def test_many_pixels(dt, classes):
    """More tiles of rows than every workgroup adds the counts of, and about as many."""
    for rows, share in ((70_001, 0.3), (140_000, 1.0), (65_536, 0.1), (65_537, 0.1),
                        (32_768, 0.2), (32_769, 0.2)):
        print(dt, classes, rows, share, flush=True)
        x = inputs(rows, 24, classes, dt, rows, masked=share)
        check(call(*x, scale=64.0), *x, dt, scale=64.0, gpu_oracle=True)
        check(call(*x, grad=False), *x, dt, gpu_oracle=True)


@pytest.mark.parametrize("share", [0.0, 0.97, 1.0])
def test_masked_shares(share):
    """From no masked row to nothing else."""
    x = inputs(600, 64, 200, "bf16", 8, masked=share)
    out = call(*x)
    check(out, *x, "bf16")
    if share == 1.0:
        for k in ("loss", "lse", "totals", "dh", "dw"):
            assert float(out[k].float().abs().sum()) == 0


def test_one_gradient_only():
    x = inputs(100, 64, 150, "f16", 9)
    both = call(*x, scale=1024.0)
    a, b = call(*x, dw=False, scale=1024.0), call(*x, dh=False, scale=1024.0)
    assert torch.equal(a["dh"], both["dh"]) and torch.equal(b["dw"], both["dw"])
    assert a["dw"] is None and b["dh"] is None


def test_no_rows():
    """Totals and dw are written, and nothing else is asked for."""
    w = torch.randn(40, 24, device="cuda").half()
    d = fg.XentDesc.make(0, 24, 40)
    ws = torch.empty(fg.linear_xent_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    tot, dw = torch.ones(2, device="cuda"), torch.ones_like(w)
    st = fg.lib().linear_xent_grad(ctypes.byref(d), None, w.data_ptr(), None, None, None, None,
                                   tot.data_ptr(), None, dw.data_ptr(), None, ws.data_ptr(),
                                   ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == fg.FG_OK
    assert float(tot.abs().sum()) == 0 and float(dw.float().abs().sum()) == 0


@pytest.mark.parametrize("dt", TYPES)
def test_far_apart_logits(dt):
    """Logits of hundreds: probabilities of 0 and 1, and p - 1 of a sure target."""
    x = inputs(200, 64, 300, dt, 10, gain=12.0)
    check(call(*x), *x, dt)


def test_impossible_classes_and_non_numbers():
    """Classes at -inf have probability 0 (a whole tile of them too); NaN and +inf logits
    make their rows' losses NaN and raise the flag, other rows' losses stay."""
    h = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1.0
    w = torch.randn(700, 64, device="cuda").bfloat16()
    w[:, 0] = 0.25
    w[300:, 0] = float("-inf")
    w[:, 1:] = 0
    t = torch.tensor([3, 299, 0, 77], dtype=torch.int32, device="cuda")
    out = call(h, w, t, None, grad=False)
    assert torch.allclose(out["loss"].cpu(), torch.full((4,), float(np.log(300))), rtol=1e-6)
    t[1] = 600      # an impossible target: an infinite loss
    out = call(h, w, t, None, grad=False)
    assert out["loss"][1].item() == float("inf")
    h2, w2, t2, _ = inputs(70, 64, 200, "bf16", 3, masked=0.0)
    ref = call(h2, w2, t2, None)
    h2[5, 3] = float("nan")
    h2[9, 7] = float("inf")
    out = call(h2, w2, t2, None)
    nan = torch.isnan(out["loss"]).cpu()
    assert nan[5] and nan[9] and int(nan.sum()) == 2
    keep = ~nan
    assert torch.equal(out["loss"].cpu()[keep], ref["loss"].cpu()[keep])
    assert torch.equal(torch.isnan(out["dh"].float()).any(1).cpu(), nan)
    assert torch.isnan(out["totals"][0]) and int(out["flag"]) == 1


def test_overflow_raises_the_flag():
    """Gradients past fp16's range are infinities, and the flag tells."""
    x = inputs(64, 64, 32, "f16", 4, masked=0.0)
    out = call(*x, scale=1e8)
    assert int(out["flag"]) == 1 and bool(torch.isinf(out["dw"]).any())
    assert int(call(*x, scale=1.0)["flag"]) == 0


@pytest.mark.parametrize("dt", TYPES)
def test_large_tiles(dt):
    """Sizes that run the largest tiles and long sums, ragged ends included; checked
    against 64 bits on the GPU."""
    for size in ((2100, 520, 9000), (4097, 264, 2500), (96, 1024, 33000), (40000, 128, 19)):
        print(dt, size, flush=True)
        x = inputs(*size, dt, 11, masked=0.1)
        check(call(*x, scale=512.0), *x, dt, scale=512.0, gpu_oracle=True)


def test_several_pieces():
    """More rows than one piece of numerators holds (1 GiB): dw adds up over pieces."""
    t, h, v = 5000, 64, 131072 + 40
    d = fg.XentDesc.make(t, h, v, dtype=fg.BF16)
    assert 2 * t * v > 1 << 30
    x = inputs(t, h, v, "bf16", 12, masked=0.3)
    out = call(*x)
    check(out, *x, "bf16", gpu_oracle=True)
    again = call(*x)
    for k in ("loss", "lse", "totals", "dh", "dw"):
        assert torch.equal(out[k], again[k]), k


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    x = inputs(500, 128, 3000, "f16", 13)
    ref = call(*x, scale=256.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = call(*x, scale=256.0)
    s.synchronize()
    for k in ("loss", "lse", "totals", "dh", "dw"):
        assert torch.equal(ref[k], other[k]), k
    h, w, t, _ = x
    d = fg.XentDesc.make(500, 128, 3000, scale=256.0)
    ws = torch.empty(fg.linear_xent_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    loss, dh, dw = torch.empty(500, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        fg.linear_xent_grad(d, h, w, t, loss, dh, dw, ws=ws)
    for k in range(3):
        for a in (loss, dh, dw):
            a.zero_()
        g.replay()
        torch.cuda.synchronize()
        for name, a in (("loss", loss), ("dh", dh), ("dw", dw)):
            assert torch.equal(a, ref[name]), (k, name)


def test_gradients_against_differences():
    """The gradients the kernels return against differences of the losses they return:
    a step along the gradient itself, bf16 inputs stepped by whole units."""
    h, w, t, _ = inputs(64, 64, 200, "f16", 14, masked=0.0)
    out = call(h, w, t, None, mean=False)
    for x, g in ((h, out["dh"]), (w, out["dw"])):
        step = torch.sign(g.float()) * 2.0 ** -7
        up, down = (x.float() + step).half(), (x.float() - step).half()
        real = (up.float() - down.float()).double()      # the step the rounding left
        a = (up, w) if x is h else (h, up)
        b = (down, w) if x is h else (h, down)
        f1 = call(*a, t, None, grad=False)["loss"].double().sum()
        f0 = call(*b, t, None, grad=False)["loss"].double().sum()
        want = (real * g.double()).sum()
        # the difference's error is of third order in the step; the gradient's 2^-11
        assert abs(float(f1 - f0 - want)) <= 0.02 * abs(float(want)), (float(f1 - f0), float(want))


def test_offsets_beyond_32_bits_in_rows():
    """Features and their gradients of more than 2^32 bytes, few classes: rows at both ends
    against 64 bits, the weights' gradient against a sum over pieces."""
    t, h, v = 1_100_003, 2048, 11
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(t, h, generator=g, device="cuda", dtype=torch.bfloat16)
    w = (torch.randn(v, h, generator=g, device="cuda") / 45).bfloat16()
    target = torch.randint(-1, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    out = call(x, w, target, None, mean=False)
    n = 0
    dw = torch.zeros(v, h, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(dw)
    for i in range(0, t, 50_000):
        sl = slice(i, min(t, i + 50_000))
        o = xent(x[sl], w, target[sl], None, 1.0, False)
        dw += o["dw"]
        bound += o["dwa"]
        n += int(o["live"].sum())
        if i in (0, 1_100_000):
            part = {k: out[k][sl] for k in ("loss", "lse", "dh")}
            part.update(totals=o["totals"], dw=None, flag=out["flag"])
            check(part, x[sl], w, target[sl], None, "bf16", mean=False, gpu_oracle=True)
    assert float(out["totals"][1]) == n
    # roundings of G, of the fp32 sums of a million rows (in parts), of the store
    err = (out["dw"].double() - dw).abs()
    assert bool((err <= bound * (2.0 ** -8 + 2.0 ** -11 + 4 * (t / 16 + 64) * U)
                 + 2.0 ** -8 * dw.abs()).all())


def test_offsets_beyond_32_bits_in_classes():
    """Weights and their gradient of more than 2^32 bytes: classes at both ends."""
    t, h, v = 9, 1024, 2_200_001
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.empty(v, h, dtype=torch.float16, device="cuda")
    for i in range(0, v, 1 << 18):
        k = min(v, i + (1 << 18)) - i
        w[i:i + k] = torch.randn(k, h, generator=g, device="cuda").half() / 32
    x = torch.randn(t, h, generator=g, device="cuda").half()
    target = torch.tensor([0, v - 1, -1, v, 5, v - 2, 1 << 21, 77, v // 2], dtype=torch.int32,
                          device="cuda")
    out = call(x, w, target, None, scale=1024.0)
    live = (target >= 0) & (target < v)
    z = torch.cat([x.double() @ w[i:i + (1 << 18)].double().t() for i in range(0, v, 1 << 18)], 1)
    lse = torch.logsumexp(z, 1)
    at = target.long().clamp(0, v - 1)[:, None]
    nll = torch.where(live, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    # logits of 64 fp32 steps of magnitude below 30, and 300 units of the sum
    assert float((out["loss"].double() - nll).abs().max()) <= 1e-4
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, at, -torch.ones_like(nll)[:, None])
    p *= (live * (1024.0 / float(live.sum())))[:, None]
    for sl in (slice(0, 300), slice(v - 300, v), slice((1 << 21) - 5, (1 << 21) + 5)):
        want = p[:, sl].t() @ x.double()
        mag = p[:, sl].abs().t() @ x.double().abs()
        err = (out["dw"][sl].double() - want).abs()
        assert bool((err <= mag * (2.0 ** -10 + 4e-4) + 2.0 ** -11 * want.abs() + 2.0 ** -24).all())
    dh = sum(p[:, i:i + (1 << 18)] @ w[i:i + (1 << 18)].double() for i in range(0, v, 1 << 18))
    mag = sum(p[:, i:i + (1 << 18)].abs() @ w[i:i + (1 << 18)].double().abs()
              for i in range(0, v, 1 << 18))
    # probabilities of 1 / v: their fp16 values keep all bits (2^15 / v > 2^-14)
    assert bool(((out["dh"].double() - dh).abs() <= mag * 2e-3 + 2.0 ** -11 * dh.abs()
                 + 2.0 ** -24).all())


def test_offsets_beyond_32_bits_in_numerators():
    """One piece of more than 2^32 bytes of numerators (less than fp32 sums of the weights'
    gradient would add): rows at both ends, and the gradient of some classes over all rows."""
    t, h, v = 5376, 2048, 400_000
    assert 2 * t * v > 1 << 32 and 2 * t * v <= (1 << 30) + 4 * v * h
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(t, h, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.empty(v, h, dtype=torch.bfloat16, device="cuda")
    for i in range(0, v, 50_000):
        w[i:i + 50_000] = torch.randn(50_000, h, generator=g, device="cuda").bfloat16() / 32
    target = torch.randint(-20_000, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    pick = torch.tensor([0, 1, 255, 256, 199_999, v - 1], device="cuda")
    target[::97] = pick[torch.arange(len(target[::97]), device="cuda") % 6].int()
    d = fg.XentDesc.make(t, h, v, dtype=fg.BF16)
    need = fg.linear_xent_workspace_bytes(d, True)
    # one piece and no fp32 sums of dw (3.3 GB); parts of dh, rows and tiles' sums below 1 GiB
    assert 2 * t * v < need < 2 * t * v + (1 << 30)
    out = call(x, w, target, None, mean=False)
    for sl in (slice(0, 6), slice(t - 10, t)):
        part = {k: out[k][sl] for k in ("loss", "lse", "dh")}
        part.update(totals=xent(x[sl], w, target[sl], None, 1.0, False)["totals"], dw=None)
        check(part, x[sl], w, target[sl], None, "bf16", mean=False, gpu_oracle=True)
    xd, wd = x.double(), w[pick].double()
    lse = out["lse"].double()[:, None]
    hot = (target[:, None] == pick).double()
    r = ((target >= 0).double())[:, None]
    G = r * (torch.exp(xd @ wd.t() - lse) - hot)
    dl = 4 * (h / 16 + 16) * U * (xd.abs() @ wd.abs().t()).max()
    dlse = dl + 300 * U + 4 * U * (lse.abs().max() + 32)
    # as in check(); twice the error of lse, which the values here take from the output
    dg = 2.0 ** -8 + 2.0 ** -11 + 2 * (dl + 2 * dlse) + 16 * U
    b = G.abs().t() @ xd.abs() * (dg + 4 * (t / 16 + 64) * U + U) + \
        2.0 ** -39 * xd.abs().sum(0) + (r * hot * (dl + 2 * dlse)).t() @ xd.abs()
    want = G.t() @ xd
    b = b * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + TINY["bf16"]
    err = (out["dw"][pick].double() - want).abs()
    print(f"dw: {float((err / b).max()):.3f} of the bound")
    assert bool((err <= b).all())


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("size", [(1, 64, 2000), (48, 96, 3000), (200, 64, 500), (900, 64, 300),
                                  (9000, 64, 300), (3000, 40, 12), (70_000, 24, 100)], ids=str)
def test_graph_replays_of_every_path(size, grad):
    """Tickets, counts and marks are made anew by each replay, whatever the workspace holds,
    and whatever the targets have become."""
    t, h, v = size
    x = inputs(t, h, v, "f16", 21)
    d = fg.XentDesc.make(t, h, v, scale=64.0)
    ws = torch.full((fg.linear_xent_workspace_bytes(d, grad),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    f = lambda *s: torch.zeros(*s, device="cuda")
    loss, lse, totals = f(t), f(t), f(2)
    dh, dw = torch.zeros_like(x[0]), torch.zeros_like(x[1])
    target = x[2].clone()
    args = (d, x[0], x[1], target, loss)
    kw = dict(lse=lse, totals=totals, ws=ws)
    run = (lambda: fg.linear_xent_grad(*args, dh, dw, **kw)) if grad else \
        (lambda: fg.linear_xent_fwd(*args, **kw))
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run()
    for k in range(3):
        target.copy_(x[2])
        target[k::5] = -1
        ref = call(x[0], x[1], target, None, grad=grad, scale=64.0)
        ws.fill_(255 - k)
        for a in (loss, lse, totals, dh, dw):
            a.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        got = dict(loss=loss, lse=lse, totals=totals, **(dict(dh=dh, dw=dw) if grad else {}))
        for name, a in got.items():
            assert torch.equal(a, ref[name]), (k, name)


# One tile of rows: each tile of classes begins its sums elsewhere. Widths of up to 40 stages
# of 64 that 8 does not divide (and some that it does), classes in more tiles than stages.
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hidden", [193, 257, 333, 381, 384, 777, 1001, 1037, 2047, 2048, 2500])
def test_few_rows_of_any_width(dt, hidden):
    """Losses and gradients of 1 to 128 rows, dense and in wider buffers."""
    for classes, ld in ((513, 0), (10007, hidden + 5)):
        h, w, t, _ = inputs(128, hidden, classes, dt, hidden, h_ld=ld, w_ld=ld)
        t[0], h[0] = classes - 1, h[0].nan_to_num()       # a call of one row has a live one
        for rows in (1, 3, 48, 64, 65, 100, 128):
            print(dt, hidden, classes, rows, flush=True)
            x = (h[:rows], w, t[:rows], None)
            check(call(*x, scale=64.0), *x, dt, scale=64.0, gpu_oracle=True)
            check(call(*x, grad=False), *x, dt, gpu_oracle=True)


@pytest.mark.parametrize("dt", TYPES)
def test_few_rows_of_an_odd_width_and_many_classes(dt):
    """Hundreds of tiles of classes, each starting stage many times."""
    for rows, hidden, classes in ((48, 2047, 65536), (3, 2500, 21696), (10, 381, 51219),
                                  (100, 777, 50000)):
        print(dt, rows, hidden, classes, flush=True)
        x = inputs(rows, hidden, classes, dt, rows)
        check(call(*x, scale=64.0), *x, dt, scale=64.0, gpu_oracle=True)


def test_equal_classes_have_equal_logits_in_every_tile():
    """Every row of the weights the same, of small whole numbers, whose sums are exact: the
    losses are log(classes), whichever tile a class is in."""
    rng = np.random.default_rng(1)
    for rows, hidden in ((1, 777), (64, 2047), (128, 333)):
        h = torch.from_numpy(rng.integers(-3, 4, (rows, hidden)).astype(np.float32)).half().cuda()
        one = torch.from_numpy(rng.integers(-1, 2, hidden).astype(np.float32)).half().cuda()
        w = one.expand(20000, hidden).contiguous()
        t = torch.arange(rows, dtype=torch.int32, device="cuda") * 150
        out = call(h, w, t, None, grad=False)
        logit = h.double() @ one.double()
        # the roundings of lse (and of the loss's difference): 4 units of its magnitude, and
        # 300 of the sum of exponentials
        bound = 300 * U + 8 * U * (logit.abs() + 32)
        err = (out["loss"].double() - float(np.log(20000))).abs()
        print(rows, hidden, float((err / bound).max()), flush=True)
        assert bool((err <= bound).all())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("size", [(40, 64, 300), (200, 64, 300), (900, 64, 300), (300, 64, 12),
                                  (70_000, 24, 40)], ids=str)
def test_weights_below_the_normal_range(dt, size):
    """Weights of 2^-140 times eighths: a mean's gradients are those of the eighths, bit for
    bit, since every factor that a common power of two changes is exact; so are the sum's with
    a scale that takes the power back."""
    h, w, t, _ = inputs(*size, dt, 17)
    rng = np.random.default_rng(18)
    wt = torch.from_numpy(rng.integers(1, 17, size[0]).astype(np.float32) / 8).cuda()
    wt[::9] = 0.0
    tiny = wt * 2.0 ** -140
    assert float(tiny[1]) > 0
    for mean, scale, back in ((True, 64.0, 1.0), (False, 0.5, 2.0 ** 140)):
        ref = call(h, w, t, wt, mean=mean, scale=scale)
        check(ref, h, w, t, wt, dt, mean=mean, scale=scale, gpu_oracle=True)
        out = call(h, w, t, tiny, mean=mean, scale=scale * back)
        assert int(out["flag"]) == 0
        for k in ("lse", "dh", "dw"):
            assert torch.equal(out[k], ref[k]), (mean, k)
        # losses are rounded to the subnormal grid, 2^-149
        err = (out["loss"].double() - ref["loss"].double() * 2.0 ** -140).abs()
        assert float(err.max()) <= 2.0 ** -149


@pytest.mark.parametrize("v", [11, 257])
def test_most_rows(v):
    """One row less than the largest number refused: rows at both ends, and the counts."""
    t = (1 << 28) - 1
    w = torch.linspace(-2, 2, v, device="cuda").half()[:, None].contiguous()
    h = torch.ones(t, 1, dtype=torch.float16, device="cuda")
    h[1::2] = -0.5
    target = torch.full((t,), 7, dtype=torch.int32, device="cuda")
    target[::4] = -1
    target[-1] = v - 1
    d = fg.XentDesc.make(t, 1, v)
    ws = torch.empty(fg.linear_xent_workspace_bytes(d, False), dtype=torch.uint8, device="cuda")
    loss, totals = torch.full((t,), 7.0, device="cuda"), torch.empty(2, device="cuda")
    fg.linear_xent_fwd(d, h, w, target, loss, totals=totals, ws=ws)
    n = 4096
    for sl in (slice(0, n), slice(t // 2, t // 2 + n), slice(t - n, t)):
        o = xent(h[sl], w, target[sl])
        # as in check(): logits 4 * 16 * 2 units, the sum 300, lse (below 8) 4 * 40
        assert float((loss[sl].double() - o["loss"]).abs().max()) <= 588 * U
    assert float(totals[1]) == float(np.float32(t - (t + 3) // 4))
