"""act8_pack and act8_unpack byte for byte against the definition in 64 bits: every type,
widths and strides that nothing divides, groups of zeros, of the largest and smallest
values, infinities and NaN, guards around the outputs, offsets past 32 bits, graphs."""
import numpy as np
import pytest
import torch

import paper_1909_11150_amd as fg
from oracle import block as B

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# rows, cols, stride, elements before the first
SHAPES = [(1, 1, 1, 0), (3, 7, 9, 1), (2, 8, 8, 0), (5, 31, 31, 3), (4, 32, 32, 0), (7, 33, 40, 5),
          (64, 256, 1024, 0), (33, 129, 129, 1), (2, 4099, 4100, 2), (1031, 40, 40, 0),
          (300, 1000, 1000, 0)]


def buffer(rows, cols, ld, dt, lead=0, seed=0, scale=1.0):
    """(view of rows x cols, the whole buffer); the rows' groups are of unlike magnitude."""
    g = torch.Generator().manual_seed(seed + rows * 7 + cols)
    t = torch.randn(rows * ld + lead, generator=g) * scale
    t = t * torch.exp2(torch.randint(-6, 6, ((t.numel() + 15) // 16,), generator=g)
                       .float()).repeat_interleave(16)[:t.numel()]
    t = t.to(dt).cuda()
    return t[lead:].view(rows, ld)[:, :cols], t


def pack(x, ld=0, guard=64):
    rows, cols = x.shape
    n = fg.act8_bytes(rows, cols)
    p = torch.full((n + guard,), 77, dtype=torch.uint8, device="cuda")
    fg.act8_pack(fg.Act8Desc.make(rows, cols, dtype=fg.dtype_of(x), x_ld=ld), x, p)
    assert bool((p[n:] == 77).all())
    return p[:n]


def same(got, want):
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan].double(), want[~nan].double())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bytes_and_values(dt, shape):
    rows, cols, ld, lead = shape
    x, _ = buffer(rows, cols, ld, TYPES[dt], lead)
    want, value = B.checkpoint(x.cpu())
    packed = pack(x, ld)
    assert torch.equal(packed.cpu(), want)
    y, whole = buffer(rows, cols, ld, TYPES[dt], lead, seed=5)
    before = whole.cpu()
    fg.act8_unpack(fg.Act8Desc.make(rows, cols, dtype=fg.dtype_of(x), x_ld=ld), packed, y)
    same(y.cpu(), value)        # exact in every type: nothing is rounded
    after = whole.cpu()
    after[lead:].view(rows, ld)[:, :cols] = before[lead:].view(rows, ld)[:, :cols]
    assert torch.equal(after, before)


@pytest.mark.parametrize("dt", TYPES)
def test_extremes(dt):
    """Zeros, subnormal groups, the type's largest values, halves, infinities and NaN."""
    t = TYPES[dt]
    f = torch.finfo(t)
    x = torch.zeros(12, 64)
    x[1, 5] = f.tiny / 4
    x[2] = torch.linspace(-1, 1, 64) * f.tiny
    x[3] = torch.linspace(-1, 1, 64) * f.max
    x[4] = (torch.arange(64) - 32 + 0.5) * 2.0 ** -3
    x[5] = torch.randn(64)
    x[5, 3], x[5, 40] = float("inf"), float("nan")
    x[6] = float("-inf")
    x[7] = float("nan")
    x[8] = -f.max
    x[9] = 1.0
    x[9, 0] = 127.75
    x[10] = 2.0 ** -119 if t is not torch.float16 else 2.0 ** -24
    x[11, ::2] = -0.0
    x = x.to(t).cuda()
    want, value = B.checkpoint(x.cpu())
    packed = pack(x)
    assert torch.equal(packed.cpu(), want)
    y = torch.empty_like(x)
    fg.act8_unpack(fg.Act8Desc.make(12, 64, dtype=fg.dtype_of(x)), packed, y)
    same(y.cpu(), value)
    assert torch.isfinite(y[3]).all() and torch.isfinite(y[8]).all()


def test_unpacked_into_another_type_rounds_once():
    x, _ = buffer(50, 100, 100, torch.float32, scale=0.01)
    packed, value = pack(x), B.checkpoint(x.cpu())[1]
    for t in (torch.float16, torch.bfloat16):
        y = torch.empty(50, 100, dtype=t, device="cuda")
        fg.act8_unpack(fg.Act8Desc.make(50, 100, dtype=fg.dtype_of(y)), packed, y)
        assert torch.equal(y.cpu(), value.float().to(t))     # (fp32 holds the values)


def test_slice_of_its_own_buffer_and_other_stream():
    """Unpacking into the columns beside what was packed; a stream that is not torch's."""
    _, whole = buffer(130, 256, 256, torch.float16)
    whole = whole.view(130, 256)
    before = whole.cpu()
    d = fg.Act8Desc.make(130, 96, x_ld=256)
    packed = torch.empty(fg.act8_bytes(130, 96), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fg.act8_pack(d, whole[:, :96], packed, stream=s.cuda_stream)
    fg.act8_unpack(d, packed, whole[:, 96:192], stream=s.cuda_stream)
    s.synchronize()
    after = whole.cpu()
    same(after[:, 96:192], B.checkpoint(before[:, :96])[1])
    assert torch.equal(after[:, :96], before[:, :96])
    assert torch.equal(after[:, 192:], before[:, 192:])


def test_replays_of_a_graph():
    x, _ = buffer(64, 200, 200, torch.bfloat16)
    y = torch.empty_like(x)
    packed = torch.empty(fg.act8_bytes(64, 200), dtype=torch.uint8, device="cuda")
    d = fg.Act8Desc.make(64, 200, dtype=fg.BF16)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            fg.act8_pack(d, x, packed)
            fg.act8_unpack(d, packed, y)
    for k in range(3):
        x.copy_(torch.randn(64, 200) * 10.0 ** k)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        same(y.cpu(), B.checkpoint(x.cpu())[1])


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes of input: the first and the last rows."""
    rows, cols = (1 << 31) // 1000 + 5, 1000
    x = torch.empty(rows, cols, dtype=torch.float16, device="cuda").normal_()
    packed = torch.empty(fg.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    fg.act8_pack(fg.Act8Desc.make(rows, cols), x, packed)
    wide = 1024
    for r in (0, rows - 4):
        want, value = B.checkpoint(x[r:r + 4].cpu())
        assert torch.equal(packed[r * wide:(r + 4) * wide].cpu(), want[:4 * wide])
        e = rows * wide + r * 32
        assert torch.equal(packed[e:e + 128].cpu(), want[4 * wide:])
    y = torch.empty_like(x)
    fg.act8_unpack(fg.Act8Desc.make(rows, cols), packed, y)
    for r in (0, rows // 2, rows - 4):
        same(y[r:r + 4].cpu(), B.checkpoint(x[r:r + 4].cpu())[1])
