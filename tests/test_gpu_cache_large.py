"""hb_cache_append on more tokens than one grid takes: 2^24, the most of a call, with 129 query heads of two dimensions."""
import numpy as np
import pytest
import torch

import decode_util as du
from oracle import decode
from paper_2309_04875_amd import hb
from plan_util import plan

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000071


def test_as_many_tokens_as_there_may_be():
    tokens, q_heads, frac, q_mul = 1 << 24, 129, 18, 185364
    page = 1 << 16
    one = plan().append_tokens(1, q_heads)                           # tokens of one launch
    assert one < tokens
    rng = np.random.default_rng(1)
    seeds = du.uniform(rng, tokens // page)
    keys, values = (torch.zeros((tokens // page, 1, page, 2), dtype=torch.int64, device=du.DEV) for _ in range(2))
    slots = torch.arange(tokens, device=du.DEV)
    shares = [(torch.arange(2 * tokens, device=du.DEV) * (2 * i + 1) + i).view(tokens, 1, 2) for i in range(4)]           # k0, k1, v0, v1
    q = [torch.full((tokens, q_heads, 2), i - 5, dtype=torch.int64, device=du.DEV) for i in range(2)]
    o0, o1, bits = hb.hb_cache_append(hb.Cache(keys, values, du.gpu(seeds)), *shares, slots, None, None, None, frac, SEED, *q, q_mul, *q)
    assert o0 is q[0] and o1 is q[1] and bits == 64 * tokens * (4 + 2 * q_heads)
    # both sides of the first launch's end, the ends, and some between
    at = np.unique(np.concatenate([np.arange(3), tokens - 1 - np.arange(3), one + np.arange(-300, 300), rng.integers(0, tokens, 20000)]))
    at = at[at < tokens]
    rows = torch.from_numpy(at).to(du.DEV)
    start = decode.word(SEED, 1)
    i = 2 * tokens + (at[:, None, None] * q_heads + np.arange(q_heads)[:, None]) * 2 + np.arange(2)
    with np.errstate(over="ignore"):
        y = [np.full(i.shape, (j - 5) * q_mul, dtype=np.int64).view(np.uint64) for j in range(2)]
        want = decode.truncate(*y, frac, start, 4 * i)
        for got, w in zip((o0, o1), want):
            assert np.array_equal(du.host(got[rows]), w.view(np.int64))
        e = 2 * ((at % page)[:, None] * 2 + np.arange(2))
        for number, (store, s0, s1) in enumerate(((keys, *shares[:2]), (values, *shares[2:]))):
            masks = decode.words(du.host(torch.from_numpy(seeds)).view(np.uint64)[at // page], np.full(len(at), number))[:, None]
            a, b = (du.host(s[rows]).view(np.uint64)[:, 0] for s in (s0, s1))
            assert np.array_equal(du.host(store.view(tokens, 2)[rows]).view(np.uint64), (a - decode.words(masks, e)) + (b - decode.words(masks, e + 1)))
    # every token has been answered: none is left as it was
    assert not bool((o0[:, 0, 0] == -5).any())
    del q, o0, o1, keys, values, shares
    torch.cuda.empty_cache()
