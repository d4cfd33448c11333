"""A pre-norm residual block, forward and backward, as a program runs it: layer norm, a linear
layer with gelu, one back onto the residual stream; everything that the backward pass reads
is kept in 8 bits. Each call is held to the 64-bit formula on the inputs that it got."""
import math

import pytest
import torch

import paper_1909_11150_amd as fg
from oracle import block as B
from test_gpu_linear import check_grads, check_packed, check_y
from test_gpu_norm import EPS, check_bwd, check_fwd

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


class Block:
    def __init__(self, rows, width, inner, dt):
        t = TYPES[dt]
        g = torch.Generator(device="cuda").manual_seed(rows + width)
        n = lambda *s: torch.randn(*s, generator=g, device="cuda")
        e = lambda *s: torch.empty(*s, dtype=t, device="cuda")
        u8 = lambda k: torch.empty(max(16, k), dtype=torch.uint8, device="cuda")
        self.t, self.x, self.dy = t, n(rows, width).to(t), n(rows, width).to(t)
        self.g, self.b = (1 + 0.1 * n(width)).to(t), (0.1 * n(width)).to(t)
        self.w1, self.b1 = (n(inner, width) / math.sqrt(width)).to(t), (0.1 * n(inner)).to(t)
        self.w2, self.b2 = (n(width, inner) / math.sqrt(inner)).to(t), (0.1 * n(width)).to(t)
        code = fg.dtype_of(self.x)
        self.norm = fg.NormDesc.make(rows, width, eps=EPS, dtype=code)
        self.lin1 = fg.LinearDesc.make(rows, width, inner, dtype=code, act=fg.ACT_GELU)
        self.lin2 = fg.LinearDesc.make(rows, inner, width, dtype=code)
        self.keep = fg.Act8Desc.make(rows, width, dtype=code)
        self.keep2 = fg.Act8Desc.make(rows, inner, dtype=code)
        kept = lambda c: u8(fg.act8_bytes(rows, c))
        self.px, self.pu, self.pz, self.pa = kept(width), kept(width), kept(inner), kept(inner)
        self.stats = torch.empty(rows, 2, device="cuda")
        self.u, self.a, self.y = e(rows, width), e(rows, inner), e(rows, width)
        self.da, self.du, self.dx = e(rows, inner), e(rows, width), e(rows, width)
        self.grads = [torch.empty_like(v) for v in (self.g, self.b, self.w1, self.b1, self.w2,
                                                    self.b2)]
        self.flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = u8(max(fg.layer_norm_workspace_bytes(self.norm),
                         *(fg.linear_workspace_bytes(d, k) for d in (self.lin1, self.lin2)
                           for k in (0, 1))))

    def forward(self):
        fg.layer_norm_fwd(self.norm, self.x, self.u, weight=self.g, bias=self.b,
                          stats=self.stats, packed=self.px)
        fg.act8_pack(self.keep, self.u, self.pu)
        fg.linear_fwd(self.lin1, self.u, self.w1, self.a, bias=self.b1, packed_z=self.pz,
                      ws=self.ws)
        fg.act8_pack(self.keep2, self.a, self.pa)
        fg.linear_fwd(self.lin2, self.a, self.w2, self.y, bias=self.b2, residual=self.x,
                      ws=self.ws)

    def backward(self):
        dg, db, dw1, db1, dw2, db2 = self.grads
        fg.linear_bwd(self.lin2, self.dy, packed_x=self.pa, w=self.w2, dx=self.da, dw=dw2,
                      dbias=db2, found_nonfinite=self.flag, ws=self.ws)
        fg.linear_bwd(self.lin1, self.da, packed_x=self.pu, w=self.w1, packed_z=self.pz,
                      dx=self.du, dw=dw1, dbias=db1, found_nonfinite=self.flag, ws=self.ws)
        fg.layer_norm_bwd(self.norm, self.du, self.stats, packed=self.px, weight=self.g,
                          add=self.dy, dx=self.dx, dweight=dg, dbias=db,
                          found_nonfinite=self.flag, ws=self.ws)

    def check(self):
        t = self.t
        dg, db, dw1, db1, dw2, db2 = self.grads
        rows = self.x.shape[0]
        check_fwd(self.x, self.g, self.b, self.u, self.stats, t)
        z, tz = check_y(self.a, self.u, self.w1, self.b1, None, "gelu", t)
        check_packed(self.pz, z, tz)
        check_y(self.y, self.a, self.w2, self.b2, self.x, "none", t)
        kept = {}
        for name, v in (("x", self.x), ("u", self.u), ("a", self.a)):
            want, kept[name] = B.checkpoint(v)
            assert torch.equal(getattr(self, "p" + name), want)
        zk = torch.empty(z.shape, device="cuda")
        fg.act8_unpack(fg.Act8Desc.make(rows, z.shape[1], dtype=fg.F32), self.pz, zk)
        check_grads(self.dy, kept["a"], self.w2, None, "none", t, self.da, dw2, db2)
        check_grads(self.da, kept["u"], self.w1, zk, "gelu", t, self.du, dw1, db1)
        o = B.layer_norm_grad(self.du, kept["x"], self.stats[:, 0], self.stats[:, 1], self.g,
                              self.dy)
        check_bwd(o, self.dx, dg, db, rows, self.stats[:, 1], self.dy, t)
        assert int(self.flag) == 0


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("shape", [(1, 64, 256), (77, 100, 391), (1024, 256, 1024)], ids=str)
def test_forward_and_backward(dt, shape):
    b = Block(*shape, dt)
    b.forward()
    b.backward()
    b.check()


def test_captured_with_one_workspace():
    """The whole step in a graph, replayed with new inputs."""
    b = Block(300, 128, 512, "f16")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            b.forward()
            b.backward()
    for k in range(3):
        b.x.copy_(torch.randn(b.x.shape) * (1 + k))
        b.dy.copy_(torch.randn(b.dy.shape))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        b.check()


def test_gradient_of_the_whole_block():
    """Against autograd in 64 bits through the exact block: what 8 bits of x, u, z and a cost.
    A code is off by half a step of at most 2^-6 of its group's largest value, some 2.5 times
    the values' size, a uniform error of 2.5 * 2^-6 / sqrt(12) = 1.1% of it; dw takes in one
    such factor, z's slope another: 3% in norm, with the 16-bit roundings."""
    b = Block(512, 192, 640, "f16")
    b.forward()
    b.backward()
    leaf = [v.double().requires_grad_() for v in (b.x, b.g, b.b, b.w1, b.b1, b.w2, b.b2)]
    x, g, bb, w1, b1, w2, b2 = leaf
    u = torch.nn.functional.layer_norm(x, (192,), g, bb, EPS)
    z = u @ w1.t() + b1
    y = x + (z * torch.special.ndtr(z)) @ w2.t() + b2
    (y * b.dy.double()).sum().backward()
    for got, want in zip([b.dx] + b.grads, leaf):
        off = float((got.double() - want.grad).norm() / want.grad.norm())
        assert off <= 0.03, off
