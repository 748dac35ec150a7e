"""hb_attention on a workspace that was reserved for a larger step."""
import numpy as np
import pytest
import torch

import decode_util as du
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000081


@pytest.mark.parametrize("heads,q_heads,dim,batch,max_len,steps", [(1, 8, 16, 65, 256, [(65, 256), (64, 256), (64, 250), (33, 129), (1, 256)]),
                                                                   (8, 8, 8, 128, 200, [(128, 200), (127, 200), (127, 150), (2, 64)]),
                                                                   (1, 8, 18, 200, 769, [(200, 768), (3, 769)])])
def test_smaller_steps_in_one_workspace(heads, q_heads, dim, batch, max_len, steps):
    rng = np.random.default_rng(dim)
    page = 16
    pages, table = du.paged(rng, batch, max_len, page)
    keys, values, seeds = du.filled_cache(rng, pages, heads, page, dim)
    q = du.shares(rng, 0.3, batch, q_heads, dim)
    lens = rng.integers(0, 40, batch).astype(np.int32)
    lens[:2] = max_len, max_len - 1
    cache = hb.Cache(*du.gpu(keys, values, seeds))
    need = hb.hb_attention_workspace_bytes(cache, batch, q_heads, max_len)
    room = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device=du.DEV)
    for b, n in steps:
        got = hb.hb_attention(cache, *du.gpu(*(a[:b] for a in q), table[:b], lens[:b]), n, 12, 20, SEED, workspace=room[256: 256 + need])
        want = decode.attention(keys, values, seeds, [a[:b] for a in q], table[:b], lens[:b], n, 12, 20, SEED)
        for g, w in zip(got, want):
            assert np.array_equal(du.host(g), w), (b, n)
    assert bool((room[:256] == 0x5A).all()) and bool((room[256 + need:] == 0x5A).all())
