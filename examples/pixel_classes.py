"""Trains a small FC-DenseNet to classify pixels: dropout after its dense layers, a softmax
cross entropy head, gradient groups, an adaptive loss scale and the layer-wise Adam update,
all through the library.

    python examples/pixel_classes.py [steps]

Pixels carry the class of the blob that they lie in; a tenth of them is unlabelled.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1909_11150_amd as fg
import synth
from paper_1909_11150_amd.densenet import DenseNet


def images(n, h, c, classes, seed):
    """Images of blobs, a noisy channel pattern per class, and each pixel's class."""
    rng = np.random.default_rng(seed)
    yy, xx = np.mgrid[:h, :h]
    label = np.zeros((n, h, h), np.int32)
    for i in range(n):
        for _ in range(12):
            cy, cx, r = rng.integers(0, h, 2).tolist() + [rng.integers(h // 10, h // 4)]
            label[i][(yy - cy) ** 2 + (xx - cx) ** 2 < r * r] = rng.integers(0, classes)
    pattern = np.random.default_rng(99).standard_normal((classes, c))
    x = pattern[label] + 1.5 * rng.standard_normal((n, h, h, c))
    label[rng.random(label.shape) < 0.1] = -1
    return x.astype(np.float16), label


def train(steps=100, n=2, h=32, c=32, classes=5, dropout=0.2, lr=2e-3, device="cuda", say=print):
    """Mean loss of the first and of the last five steps."""
    layers = synth.densenet_layers(n=n, h=h, c_in=c, c0=32, growth=32, levels=2, per_block=2,
                                   classes=classes)
    x, t = images(n, h, c, classes, seed=0)
    scale = fg.LossScaleState(scale=2.0 ** 15, clean=0, interval=200, s_min=1.0, s_max=2.0 ** 24)
    step_count = torch.zeros(1, dtype=torch.int32, device=device)
    net = DenseNet(layers, synth.he_weights(layers, seed=1), x, device=device, loss="xent",
                   loss_scale=scale.scale, dropout=dropout, seed=7, step_count=step_count,
                   group_cap_bytes=1 << 20)
    names = [L.name for L in layers]
    w16 = [net.w[k] for k in names]
    w32 = [w.float() for w in w16]
    m, v = ([torch.zeros_like(w) for w in w32] for _ in range(2))
    tensors = fg.opt_tensors(w32, w16, m, v, [net.master[k] for k in names])
    ws = torch.empty(fg.lars_adam_workspace_bytes(tensors), dtype=torch.uint8, device=device)
    target = torch.from_numpy(t).to(device)
    prog = net.program(target)
    losses = []
    for step in range(steps):
        new, label = images(n, h, c, classes, seed=step)
        net.x.copy_(torch.from_numpy(new))
        target.copy_(torch.from_numpy(label))
        prog.run()
        fg.lars_adam_update(tensors, lr, net.flags, step_count, ws)
        total, pixels = net.totals.tolist()
        losses.append(total / pixels)
        if not fg.loss_scale_update(scale, bool(net.flags.any())):
            say(f"step {step}: overflow, loss scale now {scale.scale:g}")
        prog.set_loss_scale(scale.scale)
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.4f}, loss scale {scale.scale:g}")
    return float(np.mean(losses[:5])), float(np.mean(losses[-5:]))


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 100)
