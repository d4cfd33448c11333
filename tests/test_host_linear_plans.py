"""Plans of linear layers: a training step over as many layers as the table has places finds each
layer's plans of both passes again, and the sizes asked for depend on the descriptor alone."""
import ctypes
import random
import time

import paper_1909_11150_amd as fg


def layers(n):
    return [fg.LinearDesc.make(1000 + k, 512, 1024, act=fg.ACT_GELU) for k in range(n)]


def sizes(descs):
    f = fg.lib().fg_linear_workspace_bytes
    return [(f(ctypes.byref(d), 0), f(ctypes.byref(d), 1)) for d in descs]


def test_a_step_over_32_layers_looks_at_every_tile_once():
    def layer_us(n):
        f, refs = fg.lib().fg_linear_workspace_bytes, [ctypes.byref(d) for d in layers(n)]
        best = 1e9
        for k in range(80):
            t = time.perf_counter()
            for r in refs:
                f(r, 0)
                f(r, 1)
            if k >= 3:      # what is kept by then
                best = min(best, time.perf_counter() - t)
        return best / n * 1e6
    # 0.9 us a layer, nearly all of it the two calls; 4.5 where each one plans anew
    few, many = layer_us(4), layer_us(32)
    assert many <= 2.5 * few, (few, many)


def test_sizes_do_not_depend_on_what_was_asked_before():
    descs = layers(100)
    want = [sizes([d])[0] for d in descs]
    order = list(range(100)) * 2
    random.Random(5).shuffle(order)
    assert [sizes([descs[k]])[0] for k in order] == [want[k] for k in order]
    # gradients first, then forward, of layers not asked for yet
    f = fg.lib().fg_linear_workspace_bytes
    for d in layers(140)[100:]:
        grad = f(ctypes.byref(d), 1)
        assert (f(ctypes.byref(d), 0), grad) == sizes([d])[0]


def test_a_workspace_that_is_needed_is_insisted_on():
    """Of a width below 8, whose padded copies every call makes, and of a long sum's parts."""
    at = lambda k: 0x1000000 * (k + 1)      # never dereferenced
    for rows, k, m, packed in ((64, 7, 24, None), (3, 1, 24, None), (500, 5, 9000, at(4)),
                               (64, 8000, 24, at(4))):
        d = fg.LinearDesc.make(rows, k, m, act=fg.ACT_GELU)
        need = fg.linear_workspace_bytes(d, False)
        assert need > 0
        for ws, n in ((None, need), (at(5), need - 1), (at(5) + 8, need), (at(5), 0)):
            assert fg.lib().linear_fwd(ctypes.byref(d), at(0), at(1), None, None, at(2), None,
                                       packed, ws, n, None) == fg.FG_EWORKSPACE
