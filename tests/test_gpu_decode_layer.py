"""The decoder operators together, as a decoder layer on shares uses them: projections, append with rotation, attention, feed-forward with hb_relu, step after
step on a growing cache; share for share against the oracle, eagerly, on another stream, and in captured graphs that are replayed."""
import numpy as np
import pytest
import torch

import decode_util as du
import oracle
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000051
HIDDEN, HEADS, KV, DIM, WIDE, PAGE, MAX_LEN, BATCH = 64, 4, 2, 16, 160, 4, 18, 3
GROUP, FRAC, K, M = 32, 18, 10, 20


class Layer:
    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.w = {}
        for name, n, k in (("q", HEADS * DIM, HIDDEN), ("k", KV * DIM, HIDDEN), ("v", KV * DIM, HIDDEN), ("o", HIDDEN, HEADS * DIM), ("up", WIDE, HIDDEN), ("down", HIDDEN, WIDE)):
            _, weight, scales = du.layer(rng, 1, k, n, GROUP, FRAC)
            self.w[name] = (weight, scales, *du.gpu(weight, scales))
        self.cos, self.sin = du.tables(MAX_LEN, DIM, FRAC)
        self.turn = du.gpu(self.cos, self.sin)
        self.pages, self.table = du.paged(rng, BATCH, MAX_LEN, PAGE)
        self.page_seeds = du.uniform(rng, self.pages)
        self.keys, self.values = (np.zeros((self.pages, KV, PAGE, DIM), dtype=np.int64) for _ in range(2))
        self.cache = hb.Cache(*du.gpu(self.keys, self.values, self.page_seeds))
        self.d_table = du.gpu(self.table)
        self.q_mul = round((1 << FRAC) / np.sqrt(DIM))

    def slots(self, lens):
        return np.array([self.table[b, n // PAGE] * PAGE + n % PAGE for b, n in enumerate(lens)], dtype=np.int64)

    # one step; x: pair of [batch, hidden]; each call of the protocol has a seed of its own
    def on_gpu(self, x, slots, positions, lens, seed, workspace, stream=None):
        s = [hb.hb_tensor_seed(seed, 100 + i) for i in range(8)]

        def linear(name, x, i):
            return hb.hb_linear_q4(*x, *self.w[name][2:], GROUP, FRAC, s[i], stream=stream)[:2]
        q, k, v = (linear(n, x, i) for i, n in enumerate("qkv"))
        q0, q1, _ = hb.hb_cache_append(self.cache, *(t.view(BATCH, KV, DIM) for t in (*k, *v)), slots, positions, *self.turn, FRAC, s[3],
                                       *(t.view(BATCH, HEADS, DIM) for t in q), self.q_mul, stream=stream)
        a = hb.hb_attention(self.cache, q0, q1, self.d_table, lens, MAX_LEN, K, M, s[4], workspace=workspace, stream=stream)[:2]
        o = linear("o", [t.view(BATCH, HEADS * DIM) for t in a], 5)
        y = [t + u for t, u in zip(x, o)]                          # additions are each party's own
        h = linear("up", y, 6)
        r = hb.hb_relu(*h, K, M, s[7], stream=stream)[:2]
        d = hb.hb_linear_q4(*r, *self.w["down"][2:], GROUP, FRAC, hb.hb_tensor_seed(seed, 200), stream=stream)[:2]
        return [t + u for t, u in zip(y, d)]

    def by_oracle(self, x, slots, positions, lens, seed):
        s = [oracle.tensor_seed(seed, 100 + i) for i in range(8)]

        def linear(name, x, sd):
            return decode.linear(*x, *self.w[name][:2], GROUP, FRAC, sd)
        q, k, v = (linear(n, x, s[i]) for i, n in enumerate("qkv"))
        q_out = [np.empty((BATCH, HEADS, DIM), dtype=np.int64) for _ in range(2)]
        decode.append(self.keys, self.values, self.page_seeds, [t.reshape(BATCH, KV, DIM) for t in k], [t.reshape(BATCH, KV, DIM) for t in v], slots, positions,
                      self.cos, self.sin, DIM, FRAC, s[3], [t.reshape(BATCH, HEADS, DIM) for t in q], self.q_mul, q_out)
        a = decode.attention(self.keys, self.values, self.page_seeds, q_out, self.table, lens, MAX_LEN, K, M, s[4])
        add = lambda a, b: (a.view(np.uint64) + b.view(np.uint64)).view(np.int64)                   # noqa: E731
        y = [add(t, u) for t, u in zip(x, linear("o", [t.reshape(BATCH, HEADS * DIM) for t in a], s[5]))]
        h = linear("up", y, s[6])
        r0, r1, _ = oracle.relu(h[0].ravel(), h[1].ravel(), K, M, s[7])
        return [add(t, u) for t, u in zip(y, linear("down", [r.reshape(BATCH, WIDE) for r in (r0, r1)], oracle.tensor_seed(seed, 200)))]


def _steps(rng, count):
    """Inputs of steps: sequences that start at different lengths; the last one has ended after two steps (its rows are padding)."""
    for step in range(count):
        lens = np.array([step, step + 5, min(step, 2)], dtype=np.int32)
        yield step, du.shares(rng, 1.0, BATCH, HIDDEN), lens


@pytest.mark.parametrize("own_stream", [False, True])
def test_steps(own_stream):
    layer, rng = Layer(1), np.random.default_rng(2)
    need = hb.hb_attention_workspace_bytes(layer.cache, BATCH, HEADS, MAX_LEN)
    stream = torch.cuda.Stream() if own_stream else None
    room = torch.empty(need, dtype=torch.uint8, device=du.DEV)
    torch.cuda.synchronize()
    for step, x, lens in _steps(rng, 7):
        slots = layer.slots(lens)
        if step >= 2:
            slots[2] = -1
        after = np.where(slots >= 0, lens + 1, lens).astype(np.int32)
        inputs = du.gpu(*x, slots, lens, after)
        torch.cuda.synchronize()
        seed = SEED + step
        with torch.cuda.stream(stream if own_stream else torch.cuda.current_stream()):
            out = layer.on_gpu(inputs[:2], *inputs[2:], seed, room, stream if own_stream and step % 2 else None)
        torch.cuda.synchronize()
        want = layer.by_oracle(x, slots, lens, after, seed)
        for p in range(2):
            assert np.array_equal(du.host(out[p])[:2], want[p][:2]), (step, p)             # (a padding row's queries are left as they were)
            assert np.array_equal(du.host((layer.cache.keys, layer.cache.values)[p]), (layer.keys, layer.values)[p]), (step, p)


def test_captured_steps():
    """Two graphs, of the same step with different seeds, that share one workspace; replayed with new inputs, eager work in between."""
    layer, rng = Layer(3), np.random.default_rng(4)
    need = hb.hb_attention_workspace_bytes(layer.cache, BATCH, HEADS, MAX_LEN)
    room = torch.empty(need, dtype=torch.uint8, device=du.DEV)
    held = [torch.zeros((BATCH, HIDDEN), dtype=torch.int64, device=du.DEV) for _ in range(2)]
    slots, positions, lens = (torch.full((BATCH,), -1, dtype=t, device=du.DEV) for t in (torch.int64, torch.int32, torch.int32))
    layer.on_gpu(held, slots, positions, lens, SEED, room)                 # loads the kernels; all rows are padding
    torch.cuda.synchronize()
    side, graphs, outs = torch.cuda.Stream(), [], []
    for g in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            outs.append(layer.on_gpu(held, slots, positions, lens, SEED + g, room))
        graphs.append(graph)
    torch.cuda.synchronize()
    for step, x, at in _steps(rng, 6):
        to = layer.slots(at)
        after = (at + 1).astype(np.int32)
        for t, a in zip((*held, slots, positions, lens), (*x, to, at, after)):
            t.copy_(torch.from_numpy(a))
        room.fill_(0x5A)                                                   # eager work between the replays
        torch.cuda.synchronize()
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        want = layer.by_oracle(x, to, at, after, SEED + step % 2)
        for p in range(2):
            assert np.array_equal(du.host(outs[step % 2][p]), want[p]), (step, p)
            assert np.array_equal(du.host((layer.cache.keys, layer.cache.values)[p]), (layer.keys, layer.values)[p]), (step, p)


def test_calls_at_the_same_time():
    """Two streams with a workspace each, on the same cache and queries."""
    rng = np.random.default_rng(5)
    pages, table = du.paged(rng, 4, 300, 16)
    keys, values, seeds = du.filled_cache(rng, pages, 2, 16, 32)
    q = du.shares(rng, 0.2, 4, 8, 32)
    lens = np.array([300, 17, 0, 130], dtype=np.int32)
    cache = hb.Cache(*du.gpu(keys, values, seeds))
    args = du.gpu(*q, table, lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for turn in range(3):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                outs[i].append(hb.hb_attention(cache, *args, 300, 12, 20, SEED + i)[:2])
    torch.cuda.synchronize()
    for i in range(2):
        want = decode.attention(keys, values, seeds, q, table, lens, 300, 12, 20, SEED + i)
        for got in outs[i]:
            assert all(np.array_equal(du.host(g), w) for g, w in zip(got, want))
