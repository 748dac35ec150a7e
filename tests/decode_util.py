"""Inputs of the decoder operators' tests: shares, packed weights, caches, page tables."""
import numpy as np
import torch

from oracle import decode

DEV = "cuda"


def uniform(rng, *shape):
    return rng.integers(0, 1 << 64, shape, dtype=np.uint64).view(np.int64)


def shares(rng, sigma, *shape):
    """Shares of Gaussian values at 2^16; sigma None: of any number of the ring."""
    plain = uniform(rng, *shape) if sigma is None else np.rint(rng.normal(0, sigma * 65536.0, shape)).astype(np.int64)
    first = uniform(rng, *shape)
    return first, (plain.view(np.uint64) - first.view(np.uint64)).view(np.int64)


def opened(pair):
    return (np.ascontiguousarray(pair[0]).view(np.uint64) + np.ascontiguousarray(pair[1]).view(np.uint64)).view(np.int64)


def gpu(*arrays):
    out = [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in arrays]
    return out if len(out) > 1 else out[0]


def host(t):
    return t.cpu().numpy()


def framed(array, before=7, after=9, fill=-0x0123456789ABCDEF):
    """A GPU copy inside a larger allocation filled with a sentinel: (whole, view)."""
    array = np.ascontiguousarray(array)
    whole = torch.full((before + array.size + after,), fill, dtype=torch.from_numpy(array).dtype, device=DEV)
    view = whole[before: before + array.size].view(array.shape)
    view.copy_(torch.from_numpy(array))
    return whole, view


def frame_intact(whole, size, before=7, fill=-0x0123456789ABCDEF):
    return bool((whole[:before] == fill).all()) and bool((whole[before + size:] == fill).all())


def layer(rng, rows, inputs, outputs, group, frac, sigma=1.0, big=False):
    """x, packed weights, scales of one linear layer.  big: scales over all of int32."""
    x = shares(rng, sigma, rows, inputs)
    q = rng.integers(-8, 8, (outputs, inputs))
    weight = decode.pack(q)
    if inputs % 2:
        weight[:, -1] |= rng.integers(0, 16, outputs).astype(np.uint8) << 4          # no input has these
    groups = -(-inputs // group)
    if big:
        scales = rng.integers(-2**31, 2**31, (outputs, groups)).astype(np.int32)
    else:
        scales = np.rint(rng.uniform(-1.5, 1.5, (outputs, groups)) * (1 << frac) / (4.6 * np.sqrt(inputs))).astype(np.int32)
    return x, weight, scales


def tables(rows, rot, frac):
    rate = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    angle = np.arange(rows)[:, None] * rate
    return [np.rint(f(angle) * (1 << frac)).astype(np.int32) for f in (np.cos, np.sin)]


def masked(rng, plain, page_seeds, number):
    """What a cache holds of the numbers `plain`, [pages, heads, page, dim]."""
    empty = np.zeros_like(plain)
    return (plain.view(np.uint64) - decode.reveal(empty, page_seeds, number).view(np.uint64)).view(np.int64)


def filled_cache(rng, pages, heads, page, dim, sigma=1.0):
    """keys, values (masked), page_seeds."""
    seeds = uniform(rng, pages)
    shape = (pages, heads, page, dim)
    if sigma is None:
        return uniform(rng, *shape), uniform(rng, *shape), seeds
    return tuple(masked(rng, np.rint(rng.normal(0, sigma * 65536.0, shape)).astype(np.int64), seeds, n) for n in (0, 1)) + (seeds,)


def paged(rng, batch, max_len, page, spare=2, extra_width=0):
    """A page table over a shuffled pool: (pages of the pool, table int32)."""
    each = -(-max_len // page)
    pool = rng.permutation(batch * each + spare)
    return len(pool), np.concatenate([pool[: batch * each].reshape(batch, each), np.full((batch, extra_width), -1)], axis=1).astype(np.int32)
