"""What the decoder operators refuse, and what they answer, without a GPU: sizes, null pointers, host memory, the binding's checks."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2309_04875_amd import hb

SEED = 7


def _cache(pages=4, heads=2, page=8, dim=16, keys=8, values=16, seeds=24):
    return hb.hb_cache(keys, values, seeds, pages, heads, page, dim)


def _workspace(batch, q_heads, max_len, **cache):
    return hb.raw("hb_attention_workspace_bytes", ctypes.byref(_cache(**cache)), batch, q_heads, max_len)


def test_workspace_sizes():
    assert _workspace(1, 2, 100) > 16 * 2 * 100
    assert _workspace(0, 2, 100) == _workspace(0, 2, 0) == 0                     # of nothing
    sizes = [_workspace(3, 4, n) for n in (0, 1, 63, 64, 65, 1000, 100000, 1 << 25)]
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
    for bad in ((1, 3, 10), (1, 1, 10), (1, 0, 10), (1, -2, 10), (65536, 2, 10), (1, 2, (1 << 27) + 1), (60000, 4, 1 << 26)):
        assert _workspace(*bad) == 0, bad
    for cache in (dict(dim=15), dict(dim=0), dict(dim=258), dict(heads=0), dict(page=0), dict(page=65537), dict(pages=1 << 31), dict(pages=1 << 30, page=65536, dim=256)):
        assert _workspace(1, 2, 10, **cache) == 0, cache
    assert hb.raw("hb_attention_workspace_bytes", None, 1, 2, 10) == 0


def test_refusals_without_memory():
    """Every pointer here is one that no GPU knows: what is wrong with the numbers is found first, then the memory."""
    host = np.zeros(1 << 12, dtype=np.int64)
    at = host.ctypes.data
    at += -at % 256

    def linear(rows=1, inputs=32, out=16, group=32, frac=16, x0=at, weight=at, scales=at, out0=at):
        return hb.raw("hb_linear_q4", x0, at, rows, inputs, out, weight, scales, group, frac, SEED, out0, at, None, None)
    for bad in (dict(group=0), dict(group=-32), dict(group=33), dict(frac=0), dict(frac=32), dict(inputs=0), dict(inputs=(1 << 17) + 1), dict(rows=1 << 25),
                dict(out=1 << 25), dict(x0=None), dict(weight=None), dict(scales=None), dict(out0=None), dict()):
        assert linear(**bad) == hb.HB_EINVAL, bad
    assert linear(x0=at + 4) == linear(scales=at + 2) == hb.HB_EALIGN
    bits = ctypes.c_uint64(9)
    assert hb.raw("hb_linear_q4", None, None, 0, 32, 16, None, None, 32, 16, SEED, None, None, ctypes.byref(bits), None) == hb.HB_OK and bits.value == 0

    def append(cache=None, tokens=2, rows=4, rot=8, frac=16, q_heads=2, k0=at):
        cache = ctypes.byref(cache or _cache(keys=at, values=at, seeds=at))
        return hb.raw("hb_cache_append", cache, k0, at, at, at, tokens, at, at, at, at, rows, rot, frac, at, at, q_heads, 1, SEED, at, at, None, None)
    for bad in (dict(rot=7), dict(rot=-2), dict(rot=18), dict(frac=0), dict(frac=31), dict(q_heads=-1), dict(q_heads=65537), dict(tokens=1 << 25), dict(rows=0),
                dict(rows=1 << 31), dict(k0=None), dict(cache=_cache(dim=14, heads=0)), dict(cache=_cache(keys=None)), dict()):
        assert append(**bad) == hb.HB_EINVAL, bad
    assert append(k0=at + 4) == hb.HB_EALIGN
    assert append(tokens=0) == hb.HB_OK and append(tokens=0, rows=0) == hb.HB_OK

    def attention(cache=None, batch=1, q_heads=2, width=2, max_len=10, k=12, m=20, room=1 << 14, workspace=at):
        cache = ctypes.byref(cache or _cache(keys=at, values=at, seeds=at))
        return hb.raw("hb_attention", cache, at, at, batch, q_heads, at, width, at, max_len, k, m, SEED, at, at, workspace, room, None, None)
    for bad in (dict(q_heads=3), dict(width=1), dict(max_len=17), dict(k=20), dict(k=-1), dict(m=65), dict(room=100), dict(workspace=None), dict(batch=65536),
                dict(cache=_cache(dim=1)), dict()):
        assert attention(**bad) == hb.HB_EINVAL, bad
    assert attention(workspace=at + 128) == hb.HB_EALIGN
    assert attention(batch=0) == hb.HB_OK and attention(batch=0, max_len=0, width=0) == hb.HB_OK
    assert not host.any()


def test_the_binding_refuses():
    x = torch.zeros((2, 32), dtype=torch.int64)
    w, s = torch.zeros((16, 16), dtype=torch.uint8), torch.zeros((16, 1), dtype=torch.int32)
    for args in ((x, x, w, s, 32, 16), (None, x, w, s, 32, 16), (x, x, None, s, 32, 16)):
        with pytest.raises(TypeError):
            hb.hb_linear_q4(*args, SEED)
    with pytest.raises(ValueError):
        hb.hb_linear_q4(x, x, w, s, 0, 16, SEED)
    with pytest.raises(ValueError):
        hb.hb_linear_q4(x[:, :0], x[:, :0], w, s, 32, 16, SEED)
    with pytest.raises(TypeError):
        hb.Cache(torch.zeros((1, 1, 1, 2), dtype=torch.int64), torch.zeros((1, 1, 1, 2), dtype=torch.int64), torch.zeros(1, dtype=torch.int64))
    for call in (lambda: hb.hb_cache_append(None, *[x] * 4, x, None, None, None, 16, SEED), lambda: hb.hb_attention(None, x, x, x, x, 1, 12, 20, SEED),
                 lambda: hb.hb_attention_workspace_bytes(None, 1, 2, 10)):
        with pytest.raises(TypeError):
            call()
