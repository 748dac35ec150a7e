"""The native short cuts of the decoder operators against the general path (a call with its stream given, or with outputs left out): same results."""
import numpy as np
import pytest
import torch

import decode_util as du
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000041


def _calls():
    rng = np.random.default_rng(4)
    x, weight, scales = du.layer(rng, 3, 200, 70, 64, 18)
    lin = (*du.gpu(*x, weight, scales), 64, 18, SEED)
    pages, heads, page, dim, tokens, batch, max_len = 9, 2, 5, 12, 7, 3, 11
    store = du.filled_cache(rng, pages, heads, page, dim)
    k, v = du.shares(rng, 1.0, tokens, heads, dim), du.shares(rng, 1.0, tokens, heads, dim)
    q = du.gpu(*du.shares(rng, 1.0, tokens, 4, dim))
    slots, positions, cos, sin = du.gpu(rng.permutation(45)[:tokens].astype(np.int64), rng.integers(0, 20, tokens).astype(np.int32), *du.tables(20, 8, 20))
    kv = du.gpu(*k, *v)
    _, table = du.paged(rng, batch, max_len, page, spare=0)
    heads_q = du.gpu(*du.shares(rng, 0.3, batch, 4, dim))
    where = du.gpu(table, np.array([11, 4, 0], dtype=np.int32))

    def outs(*shape):
        return [torch.full(shape, 3, dtype=torch.int64, device=du.DEV) for _ in range(2)]

    def linear(given, **kw):
        return hb.hb_linear_q4(*lin, *(outs(3, 70) if given else ()), **kw)

    def append(given, **kw):
        keys, values, seeds = du.gpu(*store)
        return (*hb.hb_cache_append(hb.Cache(keys, values, seeds), *kv, slots, positions, cos, sin, 20, SEED, *q, 7, *(outs(tokens, 4, dim) if given else ()), **kw), keys, values)

    def append_plain(given, **kw):
        keys, values, seeds = du.gpu(*store)
        return (*hb.hb_cache_append(hb.Cache(keys, values, seeds), *kv, slots, None, None, None, 20, SEED, **kw), keys, values)

    def attention(given, **kw):
        cache = hb.Cache(*du.gpu(*store))
        room = torch.empty(hb.hb_attention_workspace_bytes(cache, batch, 4, max_len), dtype=torch.uint8, device=du.DEV)
        more = (*outs(batch, 4, dim), room) if given else ()
        return hb.hb_attention(cache, *heads_q, *where, max_len, 12, 20, SEED, *more, **kw)
    return {"linear": linear, "append": append, "append_plain": append_plain, "attention": attention}


@pytest.mark.parametrize("name", ["linear", "append", "append_plain", "attention"])
def test_both_paths(name, monkeypatch):
    call = _calls()[name]
    hb.load()
    served = []
    native = hb._native
    short = name.split("_")[0]

    class Watched:
        def __getattr__(self, attr):
            def run(*args):
                r = getattr(native, attr)(*args)
                if attr == short:
                    served.append(r is not NotImplemented)
                return r
            return run
    monkeypatch.setattr(hb, "_native", Watched())
    results = [call(True)]
    if native.__name__.endswith("_binding"):
        assert served == [True]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    results += [call(True, stream=torch.cuda.current_stream()), call(False), call(False, stream=side), call(False, stream=side.cuda_stream)]
    torch.cuda.synchronize()
    monkeypatch.setattr(hb, "_native", hb._NotThere)
    results.append(call(True))
    for other in results[1:]:
        assert len(other) == len(results[0])
        for a, b in zip(other, results[0]):
            assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b
