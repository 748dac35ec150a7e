"""Numbers that an int does not hold are refused by the decoder operators, on both paths of the binding: C would get their lower 32 bits."""
import pytest
import torch

import decode_util as du
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x23090487500000A1
LARGE = [1 << 32, -(1 << 32), 1 << 64, 1 << 80]


def _tensors(*shapes):
    return [torch.zeros(s, dtype=torch.int64, device=du.DEV) for s in shapes]


@pytest.mark.parametrize("native", [True, False])
def test_numbers_out_of_range(native, monkeypatch):
    hb.load()
    if not native:
        monkeypatch.setattr(hb, "_native", hb._NotThere)
    cache = hb.Cache(*_tensors((3, 2, 4, 8), (3, 2, 4, 8), (3,)))
    kv, q, out = _tensors(*[(2, 2, 8)] * 4), _tensors(*[(2, 4, 8)] * 2), _tensors(*[(2, 4, 8)] * 2)
    slots = torch.arange(2, device=du.DEV)
    x, y = _tensors((2, 32), (2, 32)), _tensors((2, 16), (2, 16))
    weight = torch.zeros((16, 16), dtype=torch.uint8, device=du.DEV)
    scales, table, lens = (torch.zeros(s, dtype=torch.int32, device=du.DEV) for s in ((16, 1), (2, 3), (2,)))
    room = torch.zeros(hb.hb_attention_workspace_bytes(cache, 2, 4, 12), dtype=torch.uint8, device=du.DEV)
    for t in (*out, *y):
        t.fill_(5)

    def linear(group=32, frac=18):
        return hb.hb_linear_q4(*x, weight, scales, group, frac, SEED, *y)

    def append(frac=18, q_mul=1):
        return hb.hb_cache_append(cache, *kv, slots, None, None, None, frac, SEED, *q, q_mul, *out)

    def attention(k=12, m=20, max_len=12):
        return hb.hb_attention(cache, *q, table, lens, max_len, k, m, SEED, *out, room)
    for by in LARGE:
        for call, name, good in ((linear, "group", 32), (linear, "frac", 18), (append, "frac", 18), (append, "q_mul", 5), (attention, "k", 12), (attention, "m", 20)):
            with pytest.raises(ValueError):
                call(**{name: good + by})
    for value in ((1 << 31), (1 << 31) + 5, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            append(q_mul=value)
    for value in ((1 << 64) + 12, 12 - (1 << 64)):
        with pytest.raises(ValueError):
            attention(max_len=value)
    torch.cuda.synchronize()
    assert all(bool((t == 5).all()) for t in (*out, *y))
    for value in ((1 << 31) - 1, -(1 << 31)):
        append(q_mul=value)
    linear()
    attention()
