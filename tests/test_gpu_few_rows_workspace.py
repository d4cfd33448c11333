"""linear_fwd of few rows without a workspace: its kernel splits no sums over workgroups, only
widths below 8 are copied. The same bits as with the workspace that a training step brings."""
import math

import pytest
import torch

import paper_1909_11150_amd as fg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [fg.ACT_NONE, fg.ACT_GELU])
@pytest.mark.parametrize("shape", [(24, 4096, 4096), (1, 2048, 520), (64, 8000, 24),
                                   (32, 512, 8200), (1, 5001, 40), (64, 8, 8192)], ids=str)
def test_no_workspace(shape, act):
    rows, k, m = shape
    n = lambda *s: torch.randn(*s, device="cuda").half()
    x, w, b = n(rows, k), (n(m, k) / math.sqrt(k)).half(), n(m)
    d = fg.LinearDesc.make(rows, k, m, act=act)
    y, y2, z, z2 = (n(rows, m) for _ in range(4))
    kept = act != fg.ACT_NONE
    if not kept:
        assert fg.linear_workspace_bytes(d, False) == 0
    fg.linear_fwd(d, x, w, y, bias=b, z=z if kept else None)
    ws = torch.empty(fg.linear_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    fg.linear_fwd(d, x, w, y2, bias=b, z=z2 if kept else None, ws=ws)
    assert torch.equal(y, y2) and (not kept or torch.equal(z, z2))
    want = x.double() @ w.double().t() + b.double()
    if kept:
        want = want * torch.special.ndtr(want)
    # (test_gpu_linear.py holds this kernel to its bounds: here that it is the one that ran)
    assert float((y.double() - want).norm() / want.norm()) <= 2.0 ** -11


def test_narrow_layers_need_their_copies_alone():
    rows, k, m = 33, 5, 40
    x, w = (torch.randn(s, k, device="cuda").half() for s in (rows, m))
    y = torch.empty(rows, m, dtype=torch.float16, device="cuda")
    need = 768 + 768         # 40 rows of w, 33 of x, by 16 bytes
    for act in (fg.ACT_NONE, fg.ACT_RELU):
        d = fg.LinearDesc.make(rows, k, m, act=act)
        whole = torch.full((need + 256,), 99, dtype=torch.uint8, device="cuda")
        fg.linear_fwd(d, x, w, y, ws=whole[:need])
        assert bool((whole[need:] == 99).all())
        want = x.double() @ w.double().t()
        want = want.clamp_min(0) if act else want
        assert torch.allclose(y.double(), want, rtol=2.0 ** -10, atol=1e-5)
        with pytest.raises(fg.FgError):
            fg.linear_fwd(d, x, w, y, ws=whole[:need - 1])
    # a checkpoint of z is the tiles': what a long sum's parts need is still asked for
    d = fg.LinearDesc.make(64, 8000, 24, act=fg.ACT_GELU)
    x, w = (torch.randn(s, 8000, device="cuda").half() for s in (64, 24))
    y = torch.empty(64, 24, dtype=torch.float16, device="cuda")
    packed = torch.empty(fg.act8_bytes(64, 24), dtype=torch.uint8, device="cuda")
    assert fg.linear_workspace_bytes(d, False) > 0
    with pytest.raises(fg.FgError):
        fg.linear_fwd(d, x, w, y, packed_z=packed)
