"""hb_attention against the oracle, bit for bit: lengths from none to several splits, pages that end inside every tile, holes, all group sizes."""
import numpy as np
import pytest
import torch

import decode_util as du
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000031


class Case:
    def __init__(self, rng, batch, heads, group, dim, page, max_len, lens=None, k=12, m=20, sigma=1.0, holes=0, extra_width=0):
        self.k, self.m, self.max_len = k, m, max_len
        pages, self.table = du.paged(rng, batch, max_len, page, extra_width=extra_width)
        self.keys, self.values, self.seeds = du.filled_cache(rng, pages, heads, page, dim, sigma)
        self.q = du.shares(rng, None if sigma is None else sigma / np.sqrt(dim), batch, heads * group, dim)
        self.lens = np.array(lens if lens is not None else rng.integers(0, max_len + 1, batch), dtype=np.int32)
        for _ in range(holes):
            self.table[rng.integers(0, batch), rng.integers(0, max(self.table.shape[1], 1))] = rng.choice([-1, pages, 2**31 - 1, -2**31])

    def want(self):
        return decode.attention(self.keys, self.values, self.seeds, self.q, self.table, self.lens, self.max_len, self.k, self.m, SEED)

    def on_gpu(self):
        self.cache = hb.Cache(*du.gpu(self.keys, self.values, self.seeds))
        return (self.cache, *du.gpu(*self.q, self.table, self.lens), self.max_len, self.k, self.m, SEED)

    def check(self):
        o0, o1, bits = hb.hb_attention(*self.on_gpu())
        batch, q_heads, dim = self.q[0].shape
        n = batch * q_heads * self.max_len
        assert bits == 192 * batch * q_heads * dim + 128 * n + hb.hb_opened_bits(1, self.k, self.m, n)
        for got, want in zip((o0, o1), self.want()):
            bad = np.argwhere(du.host(got) != want)
            assert not len(bad), "%d of %d differ, first at %s" % (len(bad), want.size, bad[0])


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 257, 600])
def test_lengths(length):
    rng = np.random.default_rng(length)
    Case(rng, 2, 2, 2, 16, 16, length, [length, max(length - 1, 0)]).check()
    Case(rng, 1, 1, 1, 64, 5, length, [length]).check()


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 16, 17])
def test_query_heads_of_a_key_head(group):
    rng = np.random.default_rng(group)
    Case(rng, 2, 2, group, 20, 7, 90).check()


@pytest.mark.parametrize("dim", [2, 4, 14, 16, 18, 30, 32, 34, 62, 64, 66, 80, 96, 126, 128, 130, 160, 192, 254, 256])
def test_dimensions(dim):
    rng = np.random.default_rng(dim)
    Case(rng, 2, 2, 2, dim, 16, 75).check()
    Case(rng, 1, 1, 8, dim, 6, 40).check()


@pytest.mark.parametrize("page", [1, 2, 3, 8, 12, 16, 20, 64, 100, 1000])
def test_pages(page):
    rng = np.random.default_rng(page)
    Case(rng, 3, 2, 2, 24, page, 150, extra_width=page % 3).check()


@pytest.mark.parametrize("w", list(range(1, 65, 3)) + [64])
def test_slices(w):
    k = 0 if w > 50 else 12 - min(w, 12)
    Case(np.random.default_rng(w), 2, 1, 2, 16, 8, 70, k=k, m=k + w).check()


@pytest.mark.parametrize("lens", [[0, 0, 0], [0, 5, 0], [-1, 40, 2**31 - 1], [-2**31, 41, 1], [40, 40, 40]])
def test_lengths_that_leave_rows_empty(lens):
    Case(np.random.default_rng(5), 3, 2, 3, 16, 8, 40, lens).check()


@pytest.mark.parametrize("seed", range(4))
def test_holes(seed):
    Case(np.random.default_rng(seed), 4, 2, 2, 32, 8, 100, holes=9).check()


@pytest.mark.parametrize("batch,heads,group,dim,page,max_len", [(1, 8, 4, 128, 64, 3000), (7, 4, 2, 64, 16, 700), (33, 1, 1, 64, 16, 130), (2, 3, 8, 256, 12, 500)])
def test_larger(batch, heads, group, dim, page, max_len):
    Case(np.random.default_rng(batch), batch, heads, group, dim, page, max_len).check()


@pytest.mark.parametrize("heads,group,dim,page,max_len,lens", [
    (8, 1, 16, 16, 9000, [5000, 1, 0]), (2, 4, 18, 7, 3001, [0, 0, 3001, 0, 17]), (1, 8, 66, 64, 6000, [130]), (2, 2, 130, 12, 2000, [0, 65, 0, 64, 1999]),
    (1, 1, 4, 9, 700, [i * i % 301 if i % 5 else 0 for i in range(64)]), (1, 3, 4, 9, 300, [i * i % 301 for i in range(65)]),
    (256, 1, 2, 64, 8500, [8500]), (128, 1, 2, 64, 9000, [9000, 7000]), (300, 1, 2, 16, 300, [299, 1])])
def test_sequences_of_any_lengths(heads, group, dim, page, max_len, lens):
    """Lengths far below the greatest, empty sequences between others, as many sequences as are cut together and one more, pieces as long as a sum may be."""
    case = Case(np.random.default_rng(dim), len(lens), heads, group, dim, page, max_len, lens)
    args = case.on_gpu()
    need = hb.hb_attention_workspace_bytes(case.cache, len(lens), heads * group, max_len)
    room = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device=du.DEV)
    want = case.want()
    for _ in range(2):
        got = hb.hb_attention(*args, workspace=room[256: 256 + need])
        for g, w in zip(got, want):
            assert np.array_equal(du.host(g), w)
    assert bool((room[:256] == 0xA5).all()) and bool((room[256 + need:] == 0xA5).all())


@pytest.mark.parametrize("heads,group,dim", [(2, 1, 34), (1, 4, 66), (3, 8, 16)])
def test_replayed_with_other_lengths(heads, group, dim):
    """One captured call on lengths that change in place: the pieces follow them."""
    lens = [[700, 1, 0], [0, 0, 0], [3, 640, 65], [700, 700, 700], [0, 0, 129]]
    case = Case(np.random.default_rng(dim), 3, heads, group, dim, 9, 700, lens[0])
    cache, q0, q1, table, at, max_len, k, m, seed = case.on_gpu()
    outs = [torch.zeros_like(q0) for _ in range(2)]
    room = torch.empty(hb.hb_attention_workspace_bytes(cache, 3, heads * group, 700), dtype=torch.uint8, device=du.DEV)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        hb.hb_attention(cache, q0, q1, table, at, max_len, k, m, seed, outs[0], outs[1], room)
    for now in lens + lens[::-1]:
        case.lens = np.array(now, dtype=np.int32)
        at.copy_(torch.from_numpy(case.lens))
        for t in outs:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, case.want()):
            assert np.array_equal(du.host(got), want), now
        eager = hb.hb_attention(cache, q0, q1, table, at, max_len, k, m, seed)
        assert all(torch.equal(a, b) for a, b in zip(outs, eager[:2]))


@pytest.mark.parametrize("group,dim", [(1, 64), (3, 18), (4, 128), (8, 40)])
def test_any_number_of_the_ring(group, dim):
    """Keys, values and queries over all 64 bits: every carry between digits."""
    Case(np.random.default_rng(dim), 2, 2, group, dim, 5, 100, sigma=None).check()


def test_nothing_to_do():
    rng = np.random.default_rng(1)
    case = Case(rng, 2, 2, 2, 16, 8, 40, [40, 3])
    cache, q0, q1, table, lens, max_len, k, m, seed = case.on_gpu()
    o0, o1, bits = hb.hb_attention(cache, q0[:0], q1[:0], table[:0], lens[:0], max_len, k, m, seed)
    assert o0.shape == (0, 4, 16) and bits == 0
    o0, o1, _ = hb.hb_attention(cache, q0, q1, table, lens, 0, k, m, seed)
    assert not o0.any() and not o1.any()


def test_only_the_outputs_are_written():
    rng = np.random.default_rng(2)
    case = Case(rng, 3, 2, 2, 18, 7, 65)
    keys, values, seeds, q0, q1 = (du.framed(a) for a in (case.keys, case.values, case.seeds, *case.q))
    table, lens = (du.framed(a, before=3, fill=0) for a in (case.table, case.lens))
    outs = [du.framed(np.zeros_like(case.q[0]), before=9) for _ in range(2)]
    cache = hb.Cache(keys[1], values[1], seeds[1])
    need = hb.hb_attention_workspace_bytes(cache, 3, 4, 65)
    room = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device=du.DEV)
    for _ in range(2):                                                   # the second time on what the first left in the workspace
        hb.hb_attention(cache, q0[1], q1[1], table[1], lens[1], 65, case.k, case.m, SEED, outs[0][1], outs[1][1], room[256: 256 + need])
        for (whole, view), want in zip(outs, case.want()):
            assert np.array_equal(du.host(view), want) and du.frame_intact(whole, want.size, 9)
            view.zero_()
    assert bool((room[:256] == 0x5A).all()) and bool((room[256 + need:] == 0x5A).all())
    for (whole, view), a in zip((keys, values, seeds, q0, q1), (case.keys, case.values, case.seeds, *case.q)):
        assert np.array_equal(du.host(view), a) and du.frame_intact(whole, a.size)


def test_refusals():
    rng = np.random.default_rng(3)
    case = Case(rng, 2, 2, 2, 16, 8, 40, [40, 3])
    cache, q0, q1, table, lens, max_len, k, m, seed = case.on_gpu()
    need = hb.hb_attention_workspace_bytes(cache, 2, 4, 40)
    room = torch.zeros(need + 256, dtype=torch.uint8, device=du.DEV)
    outs = [torch.full_like(q0, 5) for _ in range(2)]

    def call(**other):
        a = dict(cache=cache, q0=q0, q1=q1, page_table=table, lens=lens, max_len=40, k=12, m=20, seed=SEED, out0=outs[0], out1=outs[1], workspace=room[:need])
        a.update(other)
        return hb.hb_attention(**a)
    three = torch.zeros((2, 3, 16), dtype=torch.int64, device=du.DEV)
    for other, kind in ((dict(k=20), hb.HbError), (dict(m=65), hb.HbError), (dict(max_len=41), hb.HbError), (dict(max_len=-1), hb.HbError),
                        (dict(workspace=room[: need - 1]), hb.HbError), (dict(workspace=room[8: 8 + need]), hb.HbError), (dict(workspace=room.view(torch.int64)), TypeError),
                        (dict(out0=q0), hb.HbError), (dict(out1=outs[0]), hb.HbError), (dict(out0=room[: q0.numel() * 8].view(torch.int64).view(q0.shape)), hb.HbError),
                        (dict(q0=q0[:1]), ValueError), (dict(q0=q0.to(torch.int32)), TypeError), (dict(lens=lens.long()), TypeError),
                        (dict(lens=lens[:1]), ValueError), (dict(page_table=table.long()), TypeError), (dict(page_table=table[:1]), ValueError),
                        (dict(page_table=table[:, :3].contiguous()), hb.HbError), (dict(q0=three, q1=three, out0=three.clone(), out1=three.clone()), hb.HbError),
                        (dict(cache=None), TypeError), (dict(q0=q0.cpu()), TypeError)):
        with pytest.raises(kind):
            call(**other)
    torch.cuda.synchronize()
    assert all(bool((t == 5).all()) for t in outs)
    assert hb.hb_attention_workspace_bytes(cache, 2, 3, 40) == hb.hb_attention_workspace_bytes(cache, 1 << 16, 4, 40) == 0
    call()
