"""The dense network with dropout after its dense layers and a head of pixel classes: one
step against the oracle network with the same masks, masks that change with the step and
only with it, streams, gradient groups, and training that learns."""
import numpy as np
import pytest
import torch

import paper_1909_11150_amd as fg
import synth
from gpu_util import chain_parity, dev, host
from oracle import dense_net as DN
from oracle import dropout as D
from oracle.xent import xent
from paper_1909_11150_amd.densenet import DenseNet

pytestmark = pytest.mark.gpu

S, CLASSES, SEED = 2.0 ** 12, 5, 0x123456789ABCDEF


def _net(p=0.5, loss="xent", **kw):
    layers = synth.densenet_layers(n=1, h=32, c_in=32, c0=32, growth=32, levels=2,
                                   per_block=2, classes=CLASSES if loss == "xent" else 1)
    x = synth.diffraction_like(1, 32, 32, seed=0)
    w = synth.he_weights(layers, seed=1)
    return layers, x, w, DenseNet(layers, w, x, loss_scale=S, loss=loss, dropout=p, seed=SEED,
                                  **kw)


def _target():
    t = np.random.default_rng(2).integers(0, CLASSES, 32 * 32).astype(np.int32)
    t[::9] = -100       # unlabelled
    return t


def _masks(layers, p, step):
    """Kept elements and factor of every dense layer."""
    out = {}
    for i, L in enumerate(layers):
        if L.name[0] in "DBU" and "." in L.name:
            n = int(np.prod(L.y_shape))
            out[L.name] = (D.keep(n, SEED, step, i, p).reshape(L.y_shape),
                           float(np.float32(65536) / np.float32(D.threshold(p))))
    return out


def _gpu_forward(net):
    """The stored forward tensors, keyed as the oracle network's."""
    view = lambda s: host(net._view(s))
    fw = {name: host(a) for name, a in net.act.items()}
    lv, per = net.levels, net.per
    for d in range(1, lv + 1):
        fw[f"in:TU{d}"] = host(net.NF["B" if d == lv else f"U{d + 1}"])
        fw[f"skip{d}"] = fw[f"Z:D{d}:{per}"] = view(net.inp[f"TD{d}"])
    for blk in net._blocks():
        for l in range(1, per + 1):
            fw[f"Z:{blk}:{l - 1}"] = view(net.inp[f"{blk}.{l}"])
        if not blk.startswith("D"):
            fw[f"Z:{blk}:{per}"] = np.concatenate([fw[f"Z:{blk}:{per - 1}"],
                                                   fw[f"{blk}.{per}"]], axis=-1)
    return fw


@pytest.mark.parametrize("p", [0.5, 0.2])
def test_step_matches_the_oracle_network(p):
    layers, x, w, net = _net(p)
    net.step_count.fill_(3)
    t = _target()
    net.step(dev(t))
    torch.cuda.synchronize()
    masks = _masks(layers, p, 3)
    factor = masks["D1.1"][1]
    f16 = DN.forward(layers, x, w, drop=masks)
    f64 = DN.forward(layers, x, w, store_fp16=False, drop=masks)
    fw = _gpu_forward(net)
    for name, (keep, _) in masks.items():
        assert not fw[name][~keep].any(), name
    for L in layers[:-1]:
        chain_parity(fw[L.name], f16[L.name], f64[L.name], None, f"{L.name} act")
    # the head's losses and gradients from the GPU's own features
    nf = net.NF["U1"]
    o = xent(nf.cpu().view(-1, nf.shape[3]), torch.from_numpy(w[-1]).view(CLASSES, -1),
             torch.from_numpy(t), None, S, True)
    live = o["live"].numpy()
    loss = host(net.pixel_loss)
    assert not loss[~live].any() and (~live).sum() == len(t[::9])
    # fp32 sums over 64 features: a few 2^-24 of logits of magnitude below 16
    np.testing.assert_allclose(loss, o["loss"].numpy(), rtol=0, atol=1e-4)
    np.testing.assert_allclose(host(net.totals), o["totals"].numpy(), rtol=1e-5)
    dnf = host(net.dNF["U1"])
    chain_parity(dnf.reshape(-1, nf.shape[3]), o["dh"].numpy().astype(np.float16),
                 o["dh"].numpy(), None, "head dx")
    chain_parity(host(net.dw["F1x1"]).reshape(CLASSES, -1), o["dw"].numpy().astype(np.float16),
                 o["dw"].numpy(), None, "head dW")
    # the rest of the backward pass from the GPU's own tensors
    dW16, dX16 = DN.backward(layers, fw, x, w, None, factor=factor, dnf=dnf)
    dW64, dX64 = DN.backward(layers, fw, x, w, None, store_fp16=False, factor=factor, dnf=dnf)
    for L in layers[:-1]:
        chain_parity(host(net.dw[L.name]), dW16[L.name], dW64[L.name], None, f"{L.name} dW")
    chain_parity(host(net.dX), dX16, dX64, None, "dX")


def test_masks_follow_the_step_count():
    _, _, _, net = _net()
    t = dev(_target())
    runs = []
    for step in (0, 1, 0):
        net.step_count.fill_(step)
        net.step(t)
        runs.append({k: host(v).copy() for k, v in net.dw.items()})
    assert all(np.array_equal(runs[0][k].view(np.uint16), runs[2][k].view(np.uint16))
               for k in runs[0])
    assert not np.array_equal(runs[0]["C0"], runs[1]["C0"])


def test_dropout_with_the_huber_head():
    """The two options do not depend on each other."""
    layers, x, w, net = _net(loss="huber")
    net.step(dev(synth.smooth_target(1, 32, seed=4)))
    torch.cuda.synchronize()
    fw = _gpu_forward(net)
    for name, (keep, _) in _masks(layers, 0.5, 0).items():
        assert not fw[name][~keep].any(), name
    assert np.isfinite(host(net.dX).astype(np.float32)).all()


@pytest.mark.parametrize("groups", [False, True])
def test_streams_match_one_stream(groups):
    _, _, _, net = _net(group_cap_bytes=48 * 1024 if groups else None)
    t = dev(_target())
    want = None
    for streams in (1, 2, 3):
        prog = net.program(t, streams=streams)
        for _ in range(2):
            prog.run()
        torch.cuda.synchronize()
        got = {k: host(v).copy() for k, v in net.dw.items()}
        if groups:
            got.update({f"m{k}": host(v).copy() for k, v in net.master.items()})
            assert not host(net.flags).any()
        got["loss"] = host(net.pixel_loss).copy()
        if want is None:
            want = got
        for k in want:
            assert np.array_equal(want[k], got[k]), (streams, k)


def test_program_checks_the_target():
    _, _, _, net = _net()
    with pytest.raises(ValueError, match="int32"):
        net.program(dev(_target().astype(np.int64)))
    with pytest.raises(ValueError, match="int32"):
        net.program(dev(_target()[:100]))
    with pytest.raises(ValueError, match="huber or xent"):
        _net(loss="l1")


def test_training_learns():
    from examples.pixel_classes import train
    first, last = train(steps=40, say=lambda *_: None)
    assert last < 0.6 * first, (first, last)
