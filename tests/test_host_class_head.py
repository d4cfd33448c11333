"""The dense network's class head and dropout as prepared calls, without a GPU: the calls
that replace the Huber head and the gated copies, their order and dependencies, and that
without the options nothing changes."""
import ctypes

import pytest
import torch

import paper_1909_11150_amd as fg
import synth
from paper_1909_11150_amd.densenet import DenseNet
from test_host_programs import no_cuda  # noqa: F401


def _net(loss, dropout, **kw):
    layers = synth.densenet_layers(n=1, h=32, c_in=32, c0=32, growth=32, levels=2, per_block=2,
                                   classes=5 if loss == "xent" else 1)
    w = [torch.zeros(L.w_shape, dtype=torch.float16) for L in layers]
    x = torch.zeros(layers[0].x_shape, dtype=torch.float16)
    t = torch.zeros(1, 32, 32, dtype=torch.int32 if loss == "xent" else torch.float32)
    return DenseNet(layers, w, x, device="cpu", loss=loss, dropout=dropout, **kw), t


@pytest.mark.parametrize("streams", [1, 2, 3])
def test_dropout_replaces_the_gated_copies(no_cuda, streams):  # noqa: F811
    plain, t = _net("huber", 0.0)
    a = [c.label for c in plain.program(t, streams=streams).calls]
    net, t = _net("huber", 0.5)
    prog = net.program(t, streams=streams)
    b = [c.label for c in prog.calls]
    assert [x for x in b if not x.endswith(".drop")] == a
    idx = {c.label: i for i, c in enumerate(prog.calls)}
    sites = set()
    for name in (L.name for L in net.layers if "." in L.name):
        f, g = (prog.calls[idx[f"{name}.{k}"]] for k in ("drop", "dy"))
        assert idx[f"{name}.drop"] == idx[f"{name}.fwd"] + 1
        df, dg = (ctypes.cast(c.args[0], ctypes.POINTER(fg.DropoutDesc))[0] for c in (f, g))
        assert (df.site, df.seed, df.rows, df.cols) == (dg.site, dg.seed, dg.rows, dg.cols)
        assert f.args[1] == f.args[3] == g.args[2]    # in place; the gate is its output
        sites.add(df.site)
        # copies of a layer's output follow its dropout
        if f"{name}.new" in idx and streams == 3:
            assert idx[f"{name}.drop"] in prog.calls[idx[f"{name}.new"]].deps
    assert len(sites) == len([x for x in b if x.endswith(".drop")])


def test_class_head_is_one_call(no_cuda):  # noqa: F811
    net, t = _net("xent", 0.0, group_cap_bytes=48 * 1024)
    prog = net.program(t, streams=2)
    labels = [c.label for c in prog.calls]
    assert "F1x1.xent" in labels and not {"F1x1.fwd", "head_grad", "F1x1.dW", "F1x1.dx"} & set(labels)
    assert "F1x1" not in net.out
    # its kernel gradient is on the main stream: every group call comes after it, by order
    # or by an event
    i = labels.index("F1x1.xent")
    pack = next(c for c in prog.calls if c.label == "G0.pack")
    assert prog.calls[i].sid == 0 and pack.sid == 1
    first = next(c for c in prog.calls if c.sid == 1 and c.label.endswith((".dW", ".pack")))
    assert first.deps and min(first.deps) >= i
    prog.set_loss_scale(64.0)
    assert net.xent.scale == 64.0


def test_options_are_checked(no_cuda):  # noqa: F811
    with pytest.raises(ValueError, match="huber or xent"):
        _net("l2", 0.0)
    net, t = _net("xent", 0.0)
    with pytest.raises(ValueError, match="int32"):
        net.program(t.long())


@pytest.mark.parametrize("classes,kernel", [(5, "xent_classes_kernel"), (256, "xent_classes_kernel"),
                                            (257, "xent_logits_kernel")])
def test_class_head_names_the_kernel_it_launches(no_cuda, classes, kernel):  # noqa: F811
    layers = synth.densenet_layers(n=1, h=32, c_in=32, c0=32, growth=32, levels=2, per_block=2,
                                   classes=classes)
    w = [torch.zeros(L.w_shape, dtype=torch.float16) for L in layers]
    net = DenseNet(layers, w, torch.zeros(layers[0].x_shape, dtype=torch.float16), device="cpu",
                   loss="xent")
    calls = net.program(torch.zeros(1, 32, 32, dtype=torch.int32)).calls
    assert [c.kernel for c in calls if c.label == "F1x1.xent"] == [kernel]


def test_addresses_that_kernels_read_are_on_the_device(no_cuda):  # noqa: F811
    """A step count or a target of another type or device is refused, not read."""
    for bad in (torch.zeros(1, dtype=torch.int64), torch.zeros(1), torch.zeros(0, dtype=torch.int32),
                torch.zeros(1, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError, match="step_count"):
            _net("huber", 0.5, step_count=bad)
    _net("huber", 0.5, step_count=torch.zeros(1, dtype=torch.int32))
    net, t = _net("xent", 0.0)
    with pytest.raises(ValueError, match="int32"):
        net.program(t.to("meta"))
