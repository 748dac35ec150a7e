"""One workspace, of the greatest step, serves every smaller one (no GPU)."""
import ctypes

import pytest

from paper_2309_04875_amd import hb


def _bytes(batch, q_heads, max_len, heads, dim):
    cache = hb.hb_cache(8, 16, 24, 4, heads, 8, dim)
    return hb.raw("hb_attention_workspace_bytes", ctypes.byref(cache), batch, q_heads, max_len)


CONFIGS = [(8, 32, 128), (8, 8, 64), (1, 8, 256), (1, 1, 2), (2, 12, 80), (12, 12, 80), (1, 64, 128), (256, 256, 2), (300, 600, 2), (4096, 4096, 2)]


@pytest.mark.parametrize("heads,q_heads,dim", CONFIGS)
def test_a_larger_batch_or_length_never_needs_less(heads, q_heads, dim):
    batches = sorted({1, 2, 3, 4, 7, 8, 15, 16, 31, 32, 33, 63, 64, 65, 66, 100, 127, 128, 129, 200, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 4000})
    lengths = sorted({1, 2, 63, 64, 65, 127, 128, 129, 192, 193, 255, 256, 257, 512, 513, 767, 768, 769, 1000, 1024, 1025, 2048, 4095, 4096, 4097, 8192, 8193,
                      16384, 32768, 100000})
    sizes = [[_bytes(b, q_heads, n, heads, dim) for n in lengths] for b in batches]
    for i, row in enumerate(sizes):
        here = [n for n in row if n != 0]                            # (0: batch x q_heads x max_len beyond HB_MAX_ELEMENTS)
        assert here == sorted(here) and row == here + [0] * (len(row) - len(here)), batches[i]
        assert len(here) >= sum(batches[i] * q_heads * n <= 1 << 40 for n in lengths)
        assert i == 0 or all(a <= b for a, b in zip(sizes[i - 1], here)), batches[i]


def test_little_more_than_the_scores():
    """What is asked for beyond the scores' shares: no more than the pieces' sums of a few hundred sequences."""
    for heads, q_heads, dim in CONFIGS:
        for batch, max_len in ((1, 4096), (8, 4096), (64, 1000), (128, 4096)):
            scores = 16 * batch * q_heads * max_len
            assert _bytes(batch, q_heads, max_len, heads, dim) <= scores + 1024 + 16 * q_heads * dim * (batch + -(-1024 // heads))
