"""hb_linear_q4 against the oracle, bit for bit: sizes around every tile, group sizes, odd inputs, any numbers of the ring."""
import numpy as np
import pytest
import torch

import decode_util as du
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000011


def _check(rng, rows, inputs, outputs, group, frac=18, sigma=1.0, big=False):
    x, weight, scales = du.layer(rng, rows, inputs, outputs, group, frac, sigma, big)
    o0, o1, bits = hb.hb_linear_q4(*du.gpu(*x, weight, scales), group, frac, SEED)
    want = decode.linear(*x, weight, scales, group, frac, SEED)
    assert bits == 64 * rows * outputs
    for got, w in zip((o0, o1), want):
        assert got.shape == (rows, outputs)
        bad = np.argwhere(du.host(got) != w)
        assert not len(bad), "%d of %d differ, first at %s" % (len(bad), w.size, bad[0])


@pytest.mark.parametrize("group", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("inputs", [1, 2, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 512, 1000, 1025, 2117])
def test_inputs_and_groups(inputs, group):
    _check(np.random.default_rng(inputs * 1000 + group), 2, inputs, 37, group)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 33, 64, 65])
def test_rows(rows):
    _check(np.random.default_rng(rows), rows, 320, 70, 64)


@pytest.mark.parametrize("outputs", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 1000, 4100])
def test_outputs(outputs):
    rng = np.random.default_rng(outputs)
    _check(rng, 1, 384, outputs, 128)
    _check(rng, 3, 160, outputs, 32)


@pytest.mark.parametrize("inputs,outputs,group", [(4096, 4096, 128), (4096, 300, 64), (11008, 520, 128), (16384, 48, 32), (5000, 2048, 4096), (300, 16384, 100 * 32)])
def test_layers(inputs, outputs, group):
    rng = np.random.default_rng(inputs + outputs)
    _check(rng, 1, inputs, outputs, group, 20)
    _check(rng, 6, inputs, min(outputs, 520), group, 20)


@pytest.mark.parametrize("rows,inputs,outputs,group", [(257, 130, 1100, 128), (300, 517, 1011, 256), (261, 33, 1025, 128), (257, 130, 1100, 32),
                                                      (259, 310, 1031, 64), (1, 700, 16500, 32), (1, 1301, 16390, 64)])
def test_many_rows_and_outputs(rows, inputs, outputs, group):
    _check(np.random.default_rng(rows + outputs), rows, inputs, outputs, group)


@pytest.mark.parametrize("frac", [1, 7, 31])
@pytest.mark.parametrize("rows,inputs,outputs,group", [(1, 517, 40, 32), (4, 640, 33, 128), (20, 256, 64, 64)])
def test_any_number_of_the_ring(rows, inputs, outputs, group, frac):
    """Inputs over all 64 bits, scales over all of int32: every carry between digits; and the extremes."""
    rng = np.random.default_rng(frac)
    _check(rng, rows, inputs, outputs, group, frac, None, True)
    x, weight, scales = du.layer(rng, rows, inputs, outputs, group, frac, None, True)
    edge = np.array([0, -1, 1, -(1 << 63), (1 << 63) - 1, 0x8080808080808080 - (1 << 64), 0x7F7F7F7F7F7F7F7F, 128, -128, 127], dtype=np.int64)
    x = [edge[rng.integers(0, len(edge), v.shape)] for v in x]
    weight[:] = rng.choice(np.array([0x88, 0x77, 0x78, 0x87, 0x0F], dtype=np.uint8), weight.shape)
    scales[:] = rng.choice(np.array([-2**31, 2**31 - 1, 0, -1]), scales.shape)
    want = decode.linear(*x, weight, scales, group, frac, SEED)
    got = hb.hb_linear_q4(*du.gpu(*x, weight, scales), group, frac, SEED)
    assert all(np.array_equal(du.host(g), w) for g, w in zip(got, want))


@pytest.mark.parametrize("rows,inputs,outputs,group", [(1, 511, 40, 32), (3, 640, 33, 128), (17, 1026, 130, 64)])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5, 8])
def test_buffers_anywhere(rows, inputs, outputs, group, shift):
    """Weights at any byte, scales at any four, shares at any eight; nothing around any buffer is written."""
    rng = np.random.default_rng(shift)
    x, weight, scales = du.layer(rng, rows, inputs, outputs, group, 18)
    frames = [du.framed(a, before=b, after=11, fill=f) for a, b, f in ((x[0], 1 + shift, -5), (x[1], 2 + shift, -5), (weight, 16 + shift, 0xA5), (scales, 4 + shift, -77))]
    outs = [du.framed(np.zeros((rows, outputs), dtype=np.int64), before=1 + shift, after=600) for _ in range(2)]
    hb.hb_linear_q4(*(v for _, v in frames), group, 18, SEED, *(v for _, v in outs))
    for (whole, view), want in zip(outs, decode.linear(*x, weight, scales, group, 18, SEED)):
        assert np.array_equal(du.host(view), want) and du.frame_intact(whole, want.size, 1 + shift)
    for (whole, view), a in zip(frames, (*x, weight, scales)):
        assert np.array_equal(du.host(view), a)


def test_leading_shapes_and_nothing_to_do():
    rng = np.random.default_rng(1)
    x, weight, scales = du.layer(rng, 6, 64, 10, 32, 18)
    w, s = du.gpu(weight, scales)
    want = decode.linear(*x, weight, scales, 32, 18, SEED)
    o0, o1, _ = hb.hb_linear_q4(*(t.view(2, 3, 64) for t in du.gpu(*x)), w, s, 32, 18, SEED)
    assert o0.shape == (2, 3, 10) and np.array_equal(du.host(o0).reshape(6, 10), want[0])
    one = [t[2] for t in du.gpu(*x)]
    o0, _, bits = hb.hb_linear_q4(*one, w, s, 32, 18, SEED)
    assert o0.shape == (10,) and bits == 640
    empty = torch.empty((0, 64), dtype=torch.int64, device=du.DEV)
    o0, o1, bits = hb.hb_linear_q4(empty, empty, w, s, 32, 18, SEED)
    assert o0.shape == (0, 10) and bits == 0
    o0, _, bits = hb.hb_linear_q4(*du.gpu(*x), w[:0], s[:0], 32, 18, SEED)
    assert o0.shape == (6, 0) and bits == 0


def test_refusals():
    rng = np.random.default_rng(2)
    x, weight, scales = du.layer(rng, 4, 64, 64, 32, 18)
    x0, x1, w, s = du.gpu(*x, weight, scales)
    out = [torch.full((4, 64), 5, dtype=torch.int64, device=du.DEV) for _ in range(2)]
    for args, kind in (((x0, x1, w, s, 32, 0), hb.HbError), ((x0, x1, w, s, 32, 32), hb.HbError), ((x0, x1, w, s, 48, 18), hb.HbError),
                       ((x0, x1, w, s, 0, 18), ValueError), ((x0, x1, w, s, -32, 18), ValueError), ((x0, x1, w, s, 64, 18), ValueError),
                       ((x0, x1[:3], w, s, 32, 18), ValueError), ((x0.to(torch.int32), x1, w, s, 32, 18), TypeError),
                       ((x0, x1, w.to(torch.int8), s, 32, 18), TypeError), ((x0, x1, w, s.float(), 32, 18), TypeError),
                       ((x0.cpu(), x1, w, s, 32, 18), TypeError), ((x0, x1, w[:, :31], s, 32, 18), TypeError),
                       ((x0, x1, w[:, :31].contiguous(), s, 32, 18), ValueError), ((x0.t(), x1, w, s, 32, 18), TypeError)):
        with pytest.raises(kind):
            hb.hb_linear_q4(*args, SEED, *out)
    for outs in ((x0, out[1]), (out[0], out[0]), (out[0], x1)):              # in place, the same twice
        with pytest.raises(hb.HbError) as e:
            hb.hb_linear_q4(x0, x1, w, s, 32, 18, SEED, *outs)
        assert e.value.status == hb.HB_EINVAL
    call = [x0.data_ptr(), x1.data_ptr(), 4, 64, 64, w.data_ptr(), s.data_ptr(), 32, 18, SEED, out[0].data_ptr(), out[1].data_ptr(), None, None]

    def status(at, value):
        return hb.raw("hb_linear_q4", *(value if i == at else v for i, v in enumerate(call)))
    assert [status(i, None) for i in (0, 1, 5, 6, 10, 11)] == [hb.HB_EINVAL] * 6
    assert [status(i, call[i] + 4) for i in (0, 1, 10, 11)] == [hb.HB_EALIGN] * 4 and status(6, call[6] + 2) == hb.HB_EALIGN
    assert status(3, 0) == status(2, 1 << 25) == status(3, 1 << 25) == status(4, 1 << 25) == hb.HB_EINVAL
    assert status(2, 1 << 22) == hb.HB_EINVAL                                # beyond the buffers
    host = np.zeros((4, 64), dtype=np.int64)
    assert status(0, host.ctypes.data) == hb.HB_EINVAL
    torch.cuda.synchronize()
    assert all(bool((t == 5).all()) for t in out)
    assert hb.raw("hb_linear_q4", *call) == hb.HB_OK                          # opened_bits and the stream may be null
