"""Oracle of the decoder operators (linear layers, paged cache, attention on shares): plain numpy on uint64, one party after the other.

Test infrastructure only, like the rest of this package; it shares no code with the library.  The ReLU inside attention is oracle.relu, which
evaluates the circuit element by element.
"""
import numpy as np

import oracle

M64 = (1 << 64) - 1
U = np.uint64


def words(start, index):
    """Outputs `index` of the SplitMix64 generators started at `start`."""
    with np.errstate(over="ignore"):
        z = np.asarray(start, dtype=U) + (np.asarray(index).astype(U) + U(1)) * U(0x9E3779B97F4A7C15)
        z = (z ^ (z >> U(30))) * U(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> U(27))) * U(0x94D049BB133111EB)
        return z ^ (z >> U(31))


def word(start, index):
    return int(words(np.array([start & M64], dtype=U), np.array([index]))[0])


def u64(x):
    return np.ascontiguousarray(x).view(U) if x.dtype == np.int64 else x


def truncate(y0, y1, f, start, first):
    """Shares of (y0 + y1) / 2^f, words first .. first + 3 of `start`; f: a number.  Truth: floor or floor + 1."""
    with np.errstate(over="ignore"):
        first = np.asarray(first)
        v0, v1, v2, v3 = (words(start, first + j) for j in range(4))
        low = U((1 << 63) - 1)
        r = v0 + v1
        c = (y0 + v0) + (y1 + v1) + U(1 << 62)
        cm, rm = c >> U(63), r >> U(63)
        g = U(1 << (63 - f)) * (U(1) - U(2) * cm)
        t0 = ((c & low) >> U(f)) + cm * U(1 << (63 - f)) - U(1 << (62 - f)) - v2 + g * v3
        t1 = g * (rm - v3) - (((r & low) >> U(f)) - v2)
        return t0, t1


def unpack(weight, inputs):
    """Numbers -8 .. 7 of packed rows: [out, inputs] int64."""
    q = np.stack([weight & 15, weight >> 4], axis=-1).reshape(weight.shape[0], -1)[:, :inputs].astype(np.int64)
    return np.where(q >= 8, q - 16, q)


def pack(q):
    """The layout that hb_linear_q4 reads, of numbers -8 .. 7 [out, inputs]."""
    q = np.concatenate([q, np.zeros((q.shape[0], q.shape[1] % 2), dtype=q.dtype)], axis=1) & 15
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def linear(x0, x1, weight, scales, group, frac, seed):
    """x: [rows, in] int64; returns two [rows, out] int64."""
    rows, inputs = x0.shape
    w = unpack(weight, inputs) * np.repeat(scales.astype(np.int64), group, axis=1)[:, :inputs]
    with np.errstate(over="ignore"):
        y0, y1 = (u64(x) @ w.view(U).T for x in (x0, x1))
    t = truncate(y0, y1, frac, word(seed, 1), 4 * np.arange(y0.size).reshape(y0.shape))
    return tuple(v.view(np.int64) for v in t)


def append(keys, values, page_seeds, k, v, slots, positions, cos, sin, rot, frac, seed, q=None, q_mul=0, q_out=None):
    """Writes into keys, values [pages, heads, page, dim] and q_out (pairs of [tokens, q_heads, dim]); all int64 arrays."""
    pages, heads, page, dim = keys.shape
    start, half = word(seed, 1), rot // 2
    tokens = len(slots)
    with np.errstate(over="ignore"):
        for t in range(tokens):
            slot = int(slots[t])
            if not 0 <= slot < pages * page or (rot and not 0 <= int(positions[t]) < len(cos)):
                continue
            c, s = (tab[positions[t]].astype(np.int64) if rot else np.zeros(0, dtype=np.int64) for tab in (cos, sin))
            at, off = divmod(slot, page)

            def rotated(x, c, s):
                c, s = c.view(U), s.view(U)
                return np.concatenate([x[:, :half] * c - x[:, half:rot] * s, x[:, half:rot] * c + x[:, :half] * s], axis=1)
            for h in range(heads):
                pair = [u64(x[t, h]).copy() for x in k]
                if rot:
                    turned = [rotated(x[None, :], c, s)[0] for x in pair]
                    new = truncate(turned[0], turned[1], frac, start, 4 * ((t * heads + h) * dim + np.arange(rot)))
                    for x, y in zip(pair, new):
                        x[:rot] = y
                for number, cache, shares in ((0, keys, pair), (1, values, [u64(x[t, h]) for x in v])):
                    masks = word(int(page_seeds[at]) & M64, number)
                    e = 2 * ((h * page + off) * dim + np.arange(dim))
                    cache[at, h, off] = ((shares[0] - words(masks, e)) + (shares[1] - words(masks, e + 1))).view(np.int64)
            if q is None:
                continue
            c, s = (((x * q_mul) + (1 << (frac - 1))) >> frac for x in (c, s))
            heads_q = q[0].shape[1]
            for h in range(heads_q):
                turned = []
                for x in q:
                    x = u64(x[t, h])
                    turned.append(np.concatenate([rotated(x[None, :], c, s)[0] if rot else x[:0], x[rot:] * U(q_mul & M64)]))
                i = tokens * heads * dim + (t * heads_q + h) * dim + np.arange(dim)
                for out, y in zip(q_out, truncate(turned[0], turned[1], frac, start, 4 * i)):
                    out[t, h] = y.view(np.int64)


def reveal(cache, page_seeds, number):
    """Keys (number 0) or values (1) in the clear, as int64."""
    pages = cache.shape[0]
    e = 2 * np.arange(cache[0].size).reshape(cache.shape[1:])
    masks = words(u64(page_seeds), np.full(pages, number))[:, None, None, None]
    with np.errstate(over="ignore"):
        return (u64(cache) + words(masks, e) + words(masks, e + 1)).view(np.int64)


def attention(keys, values, page_seeds, q, page_table, lens, max_len, k, m, seed):
    """q: pair of [batch, q_heads, dim] int64; returns two arrays of that shape."""
    pages, heads, page, dim = keys.shape
    batch, heads_q = q[0].shape[:2]
    sub = [word(seed, 2 + j) for j in range(5)]
    scores = [np.zeros((batch, heads_q, max_len), dtype=U) for _ in range(2)]
    out = [np.zeros((batch, heads_q, dim), dtype=U) for _ in range(2)]
    length = np.clip(lens, 0, max_len)

    def masked(b, h, number):
        """Positions that are no holes, their masked numbers and both shares of the masks."""
        t = np.arange(length[b])
        at = page_table[b, t // page].astype(np.int64) if len(t) else t
        t = t[(at >= 0) & (at < pages)]
        at = page_table[b, t // page].astype(np.int64) if len(t) else t
        start = words(u64(page_seeds)[at], np.full(len(t), number))[:, None]
        e = 2 * ((h * page + t % page)[:, None] * dim + np.arange(dim))
        return t, u64((keys, values)[number])[at, h, t % page], words(start, e), words(start, e + 1)
    with np.errstate(over="ignore"):
        for b in range(batch):
            for x in range(heads_q):
                row = b * heads_q + x
                t, delta, b0, b1 = masked(b, x // (heads_q // heads), 0)
                i, j = row * dim + np.arange(dim), row * max_len + t
                a0, a1 = words(sub[0], 2 * i), words(sub[0], 2 * i + 1)
                eps = (u64(q[0][b, x]) - a0) + (u64(q[1][b, x]) - a1)
                c0 = words(sub[1], 5 * j)
                s0 = c0 + delta @ a0 + b0 @ eps + delta @ eps
                s1 = ((b0 + b1) @ (a0 + a1) - c0) + delta @ a1 + b1 @ eps
                scores[0][b, x, t], scores[1][b, x, t] = truncate(s0, s1, 16, sub[1], 5 * j + 1)
        if max_len:
            p0, p1, _ = oracle.relu(scores[0].view(np.int64).ravel(), scores[1].view(np.int64).ravel(), k, m, sub[2])
        for b in range(batch):
            if length[b] == 0:
                continue
            for x in range(heads_q):
                row = b * heads_q + x
                t, delta, b0, b1 = masked(b, x // (heads_q // heads), 1)
                i, j = row * dim + np.arange(dim), row * max_len + t
                a0, a1 = words(sub[3], 2 * j), words(sub[3], 2 * j + 1)
                eps = (u64(p0)[j] - a0) + (u64(p1)[j] - a1)
                c0 = words(sub[4], 9 * i)
                o0 = c0 + a0 @ delta + eps @ b0 + eps @ delta
                o1 = ((a0 + a1) @ (b0 + b1) - c0) + a1 @ delta + eps @ b1
                whole = int(length[b]).bit_length() - 1
                factor = U(((1 << (16 + whole)) + int(length[b]) // 2) // int(length[b]))
                o0, o1 = truncate(o0, o1, 16 + whole, sub[4], 9 * i + 1)
                out[0][b, x], out[1][b, x] = truncate(o0 * factor, o1 * factor, 16, sub[4], 9 * i + 5)
    return tuple(v.view(np.int64) for v in out)
