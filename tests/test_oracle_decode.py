"""The oracle of the decoder operators against what their definitions fix: truncation is floor or one more, linear layers, rotations and
attention agree with the same sums in whole numbers and in 64-bit floats within bounds that follow from the truncations.  No GPU."""
import numpy as np
import pytest

import decode_util as du
from oracle import decode

SEED = 0x2309048750000001


def test_words_are_the_framework_s():
    import oracle
    for t in range(5):
        assert decode.word(SEED, 2 + t) == oracle.tensor_seed(SEED, t)


@pytest.mark.parametrize("f", [1, 2, 7, 16, 20, 31, 40, 46, 61, 62])
def test_truncation_is_floor_or_one_more(f):
    rng = np.random.default_rng(f)
    y = np.concatenate([[0, 1, -1, (1 << 62) - 1, -(1 << 62), (1 << f) - 1, 1 << f, -(1 << f) if f < 62 else -1, -(1 << f) + 1],
                        rng.integers(-(1 << 62), 1 << 62, 4000), rng.integers(-70000, 70000, 1000)]).astype(np.int64)
    y0 = du.uniform(rng, y.size).view(np.uint64)
    y1 = y.view(np.uint64) - y0
    first = 4 * np.arange(y.size)
    t = du.opened(decode.truncate(y0, y1, f, decode.word(SEED, 1), first))
    floor = y >> f
    assert set(np.unique(t - floor)) <= {0, 1}
    exact = (y & ((1 << f) - 1)) == 0
    assert np.array_equal(t[exact], floor[exact])
    # one more exactly where the lower bits of y and of the mask carry
    r = decode.words(decode.word(SEED, 1), first) + decode.words(decode.word(SEED, 1), first + 1)
    low = (1 << f) - 1
    assert np.array_equal(t - floor, (((y & low) + (r.view(np.int64) & low)) >> f))


def test_packing():
    rng = np.random.default_rng(1)
    for inputs in (1, 2, 7, 64):
        q = rng.integers(-8, 8, (5, inputs))
        assert np.array_equal(decode.unpack(decode.pack(q), inputs), q)
    assert decode.pack(np.array([[1, -2, 3]])).tolist() == [[0xE1, 0x03]]


@pytest.mark.parametrize("rows,inputs,outputs,group", [(1, 1, 1, 32), (2, 33, 5, 32), (3, 200, 7, 64)])
def test_linear(rows, inputs, outputs, group):
    rng = np.random.default_rng(inputs)
    x, weight, scales = du.layer(rng, rows, inputs, outputs, group, 18)
    got = du.opened(decode.linear(*x, weight, scales, group, 18, SEED))
    plain = du.opened(x)
    for r in range(rows):
        for n in range(outputs):
            y = sum(int(scales[n, j // group]) * int(decode.unpack(weight, inputs)[n, j]) * int(plain[r, j]) for j in range(inputs))
            assert got[r, n] - (y >> 18) in (0, 1)


@pytest.mark.parametrize("rot", [0, 2, 6, 8])
def test_append_and_reveal(rot):
    rng = np.random.default_rng(rot)
    tokens, heads, q_heads, dim, page, pages, frac = 5, 2, 4, 8, 3, 4, 20
    keys, values, seeds = du.filled_cache(rng, pages, heads, page, dim)
    before = keys.copy(), values.copy()
    k, v, q = (du.shares(rng, 1.0, tokens, h, dim) for h in (heads, heads, q_heads))
    slots = np.array([4, -1, 7, 12, 0])                                 # the second and fourth are padding
    positions = np.array([9, 3, 0, 2, 30], dtype=np.int32)               # as is the last, out of a table of 30 rows
    cos, sin = du.tables(30, rot, frac)
    q_out = du.uniform(rng, tokens, q_heads, dim), du.uniform(rng, tokens, q_heads, dim)
    kept = [a.copy() for a in q_out]
    q_mul = round((1 << frac) / np.sqrt(dim))
    decode.append(keys, values, seeds, k, v, slots, positions, cos, sin, rot, frac, SEED, q, q_mul, q_out)
    live = [0, 2] if rot else [0, 2, 4]
    plain_k, plain_v = decode.reveal(keys, seeds, 0), decode.reveal(values, seeds, 1)
    touched = np.zeros((pages, page), dtype=bool)
    for t in live:
        at, off = divmod(int(slots[t]), page)
        touched[at, off] = True
        assert np.array_equal(plain_v[at, :, off], du.opened(v)[t])
        x, y = du.opened(k)[t].astype(np.float64), du.opened(q)[t].astype(np.float64)
        c, s = (tab[positions[t] if rot else 0] / (1 << frac) for tab in (cos, sin))
        h = rot // 2
        for value, got, factor, slack in ((x, plain_k[at, :, off], 1.0, 1.0), (y, du.opened(q_out)[t], q_mul / (1 << frac), None)):
            want = np.concatenate([value[:, :h] * c - value[:, h:rot] * s, value[:, h:rot] * c + value[:, :h] * s, value[:, rot:]], axis=1) * factor
            # one unit of the truncation; the query's tables are rounded by up to 2^-(frac+1) each besides
            bound = 1.0 + 1e-6 + (0.0 if slack else 2.0 * np.abs(value).max() * 2.0 ** -(frac + 1))
            assert np.abs(got - want).max() <= bound
    assert np.array_equal(keys.transpose(0, 2, 1, 3)[~touched], before[0].transpose(0, 2, 1, 3)[~touched])
    assert np.array_equal(values.transpose(0, 2, 1, 3)[~touched], before[1].transpose(0, 2, 1, 3)[~touched])
    for a, b in zip(q_out, kept):
        dead = [t for t in range(tokens) if t not in live]
        assert np.array_equal(a[dead], b[dead])


def test_attention_against_floats():
    rng = np.random.default_rng(3)
    batch, q_heads, heads, dim, page, max_len = 4, 4, 2, 8, 5, 23
    pages, table = du.paged(rng, batch, max_len, page, extra_width=1)
    keys, values, seeds = du.filled_cache(rng, pages, heads, page, dim)
    q = du.shares(rng, 0.5, batch, q_heads, dim)
    lens = np.array([23, 0, 1, 40], dtype=np.int32)                     # the last counts as max_len
    table[0, 1] = -1                                                     # holes: positions 5 .. 9 of the first sequence
    table[3, 4] = pages
    got = decode.attention(keys, values, seeds, q, table, lens, max_len, 0, 64, SEED)
    assert not got[0][1].any() and not got[1][1].any()
    plain = du.opened(got)
    k, v = decode.reveal(keys, seeds, 0) / 65536.0, decode.reveal(values, seeds, 1) / 65536.0
    x = du.opened(q) / 65536.0
    for b in (0, 2, 3):
        n = min(int(lens[b]), max_len)
        for h in range(q_heads):
            t = np.array([i for i in range(n) if 0 <= table[b, i // page] < pages])
            kk, vv = (c[table[b, t // page], h // 2, t % page] for c in (k, v))
            want = np.maximum(kk @ x[b, h], 0) @ vv / n
            # per weight one unit of 2^-16 times the value; two truncations of the result and the factor's rounding (2^-16 relative)
            bound = (np.abs(vv).sum(0) / n + 2.0 + np.abs(want)) / 65536.0 + np.abs(want) * 2.0 ** -16
            assert (np.abs(plain[b, h] / 65536.0 - want) <= bound).all()
