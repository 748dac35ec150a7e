"""hb_cache_append against the oracle, bit for bit: rotations of a part of the head, odd sizes, padding rows, slots in any order."""
import numpy as np
import pytest
import torch

import decode_util as du
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000021


class Case:
    def __init__(self, rng, tokens, heads, q_heads, dim, rot, page, pages, frac=20, rows=50, sigma=1.0, padding=True):
        self.rot, self.frac = rot, frac
        self.keys, self.values, self.seeds = du.filled_cache(rng, pages, heads, page, dim, None)
        self.k, self.v = du.shares(rng, sigma, tokens, heads, dim), du.shares(rng, sigma, tokens, heads, dim)
        self.q = du.shares(rng, sigma, tokens, q_heads, dim) if q_heads else None
        self.q_out = tuple(du.uniform(rng, tokens, q_heads, dim) for _ in range(2)) if q_heads else None
        self.slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
        self.positions = rng.integers(0, rows, tokens).astype(np.int32)
        if padding and tokens > 3:
            self.slots[1], self.slots[tokens // 2] = -1, pages * page
            self.positions[3] = rows
            self.slots[tokens - 1], self.positions[tokens - 1] = -(1 << 62), -1
        self.cos, self.sin = du.tables(rows, rot, frac)
        self.q_mul = round((1 << frac) / np.sqrt(dim)) if sigma is not None else int(rng.integers(-2**31, 2**31))
        self.bits = 64 * tokens * (heads * (rot + 2 * dim) + q_heads * dim)

    def run(self, in_place=False):
        keys, values, seeds = du.gpu(self.keys, self.values, self.seeds)
        turn = du.gpu(self.positions, self.cos, self.sin) if self.rot else [None, None, None]
        q, out = ([], []) if self.q is None else (du.gpu(*self.q), du.gpu(*self.q_out))
        if in_place:
            out = q
        more = (*q, self.q_mul, *out) if q else ()
        o0, o1, bits = hb.hb_cache_append(hb.Cache(keys, values, seeds), *du.gpu(*self.k, *self.v, self.slots), *turn, self.frac, SEED, *more)
        assert bits == self.bits
        return [keys, values] + ([o0, o1] if q else [])

    def want(self, in_place=False):
        keys, values = self.keys.copy(), self.values.copy()
        out = None if self.q is None else [a.copy() for a in (self.q if in_place else self.q_out)]
        decode.append(keys, values, self.seeds, self.k, self.v, self.slots, self.positions, self.cos, self.sin, self.rot, self.frac, SEED,
                      self.q, self.q_mul, out)
        return [keys, values] + (out or [])

    def check(self, in_place=False):
        for name, got, want in zip(("keys", "values", "q_out0", "q_out1"), self.run(in_place), self.want(in_place)):
            bad = np.argwhere(du.host(got) != want)
            assert not len(bad), "%s: %d of %d differ, first at %s" % (name, len(bad), want.size, bad[0])


@pytest.mark.parametrize("dim", [2, 4, 6, 10, 64, 80, 96, 128, 130, 256])
@pytest.mark.parametrize("part", ["none", "two", "half", "all but two", "all"])
def test_dimensions_and_rotated_parts(dim, part):
    rot = {"none": 0, "two": 2, "half": dim // 2 // 2 * 2, "all but two": dim - 2, "all": dim}[part]
    rng = np.random.default_rng(dim)
    Case(rng, 9, 3, 6, dim, rot, 5, 4).check()


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 31, 64, 100, 257])
@pytest.mark.parametrize("heads,q_heads", [(1, 0), (1, 1), (2, 8), (5, 5)])
def test_tokens_and_heads(tokens, heads, q_heads):
    rng = np.random.default_rng(tokens)
    Case(rng, tokens, heads, q_heads, 32, 32, 7, tokens // 7 + 2).check()


@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (80, 40), (64, 0), (20, 8), (12, 6), (66, 66)])
def test_many_tokens(dim, rot):
    """Launches that fill the chip, whose threads take four numbers each where the parts allow it."""
    rng = np.random.default_rng(dim + rot)
    tokens = 700000 // (16 * dim)
    Case(rng, tokens, 3, 10, dim, rot, 16, tokens // 16 + 3).check()


@pytest.mark.parametrize("page", [1, 3, 16, 64, 100])
def test_pages(page):
    Case(np.random.default_rng(page), 40, 2, 2, 16, 8, page, 80 // page + 2).check()


@pytest.mark.parametrize("frac", [1, 14, 20, 30])
def test_any_number_of_the_ring(frac):
    rng = np.random.default_rng(frac)
    case = Case(rng, 20, 3, 6, 20, 12, 4, 9, frac, sigma=None)
    case.cos, case.sin = (rng.integers(-2**31, 2**31, case.cos.shape).astype(np.int32) for _ in range(2))
    case.check()


@pytest.mark.parametrize("dim,rot", [(64, 64), (10, 4)])
def test_queries_in_place(dim, rot):
    Case(np.random.default_rng(7), 12, 2, 4, dim, rot, 4, 6).check(in_place=True)


def test_only_what_a_row_owns_is_written():
    """Frames around every buffer, rows of padding in the middle."""
    rng = np.random.default_rng(8)
    case = Case(rng, 11, 2, 4, 12, 8, 3, 6)
    frames = [du.framed(a) for a in (case.keys, case.values, *case.q_out)]
    (_, keys), (_, values), (_, o0), (_, o1) = frames
    seeds = du.gpu(case.seeds)
    hb.hb_cache_append(hb.Cache(keys, values, seeds), *(du.framed(a)[1] for a in (*case.k, *case.v, case.slots)), *(du.framed(a, fill=0)[1] for a in
                       (case.positions, case.cos, case.sin)), case.frac, SEED, *(du.framed(a)[1] for a in case.q), case.q_mul, o0, o1)
    for (whole, view), want in zip(frames, case.want()):
        assert np.array_equal(du.host(view), want) and du.frame_intact(whole, want.size)


def test_no_tokens():
    rng = np.random.default_rng(9)
    case = Case(rng, 0, 2, 4, 12, 8, 3, 6)
    case.check()


def test_refusals():
    rng = np.random.default_rng(10)
    case = Case(rng, 4, 2, 4, 12, 8, 3, 6, padding=False)
    keys, values, seeds = du.gpu(case.keys, case.values, case.seeds)
    cache = hb.Cache(keys, values, seeds)
    k0, k1, v0, v1, slots, positions, cos, sin, q0, q1, o0, o1 = du.gpu(*case.k, *case.v, case.slots, case.positions, case.cos, case.sin, *case.q, *case.q_out)

    def call(**other):
        a = dict(cache=cache, k0=k0, k1=k1, v0=v0, v1=v1, slots=slots, positions=positions, cos=cos, sin=sin, frac=20, seed=SEED, q0=q0, q1=q1, q_mul=1,
                 q_out0=o0, q_out1=o1)
        a.update(other)
        return hb.hb_cache_append(**a)
    for other, kind in ((dict(frac=0), hb.HbError), (dict(frac=31), hb.HbError), (dict(k0=k0[:3]), ValueError), (dict(v1=v1.to(torch.int32)), TypeError),
                        (dict(slots=slots.to(torch.int32)), TypeError), (dict(slots=slots[:3]), ValueError), (dict(positions=positions.long()), TypeError),
                        (dict(sin=sin[:-1]), ValueError), (dict(cos=None), TypeError), (dict(q1=None), AttributeError if False else TypeError),
                        (dict(q0=q0[:, :3].contiguous()), ValueError), (dict(k0=k0.cpu()), TypeError), (dict(cache=keys), TypeError),
                        (dict(q_out0=o1), hb.HbError), (dict(q_out0=q1, q_out1=k0.repeat(1, 2, 1)[:, :4].contiguous().copy_(q0)), None),
                        (dict(q_out0=keys.view(-1)[: q0.numel()].view(q0.shape)), hb.HbError), (dict(k0=keys.view(-1)[: k0.numel()].view(k0.shape)), hb.HbError),
                        (dict(cos=torch.zeros((0, 4), dtype=torch.int32, device=du.DEV), sin=torch.zeros((0, 4), dtype=torch.int32, device=du.DEV)), hb.HbError),
                        (dict(cos=torch.zeros((50, 7), dtype=torch.int32, device=du.DEV), sin=torch.zeros((50, 7), dtype=torch.int32, device=du.DEV)), hb.HbError)):
        if kind is None:
            call(**other)
            continue
        with pytest.raises(kind):
            call(**other)
    with pytest.raises(ValueError):
        hb.Cache(keys, values[:5], seeds)
    with pytest.raises(ValueError):
        hb.Cache(keys, values, seeds[:5])
    with pytest.raises(TypeError):
        hb.Cache(keys.cpu(), values, seeds)
    odd = torch.zeros((2, 1, 3, 5), dtype=torch.int64, device=du.DEV)
    wide = torch.zeros((1, 1, 1, 258), dtype=torch.int64, device=du.DEV)
    for store in (odd, wide):
        t = [torch.zeros((1, 1, store.shape[3]), dtype=torch.int64, device=du.DEV) for _ in range(4)]
        with pytest.raises(hb.HbError):
            hb.hb_cache_append(hb.Cache(store, store.clone(), seeds[: store.shape[0]].contiguous()), *t, slots[:1], None, None, None, 20, SEED)
