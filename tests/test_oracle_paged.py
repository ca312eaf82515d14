"""Pins of the plain definitions in oracle/paged.py: closed forms, and the contiguous definitions where both apply."""
import math

import numpy as np
import pytest

from oracle import layer, paged


def test_what_a_row_sees():
    assert paged.sees(4, 0, 0).tolist() == [0, 1, 2, 3, 4]
    assert paged.sees(9, 3, 0).tolist() == [7, 8, 9]
    assert paged.sees(9, 3, 2).tolist() == [0, 1, 7, 8, 9]
    assert paged.sees(2, 3, 2).tolist() == [0, 1, 2]
    assert paged.sees(9, 1, 0).tolist() == [9]
    assert paged.sees(9, 4, 50).tolist() == list(range(10))


def test_attention_is_the_softmax_of_the_gathered_rows():
    rng = np.random.default_rng(0)
    page, h_kv, g, d, n = 4, 2, 3, 8, 3
    K, V = rng.standard_normal((5, page, h_kv, d)), rng.standard_normal((5, page, h_kv, d))
    table, L = [3, 0, 4, -1], 10
    q = rng.standard_normal((n, h_kv * g, d))
    out, mag = paged.attention(q, K, V, table, L, n, 0, 0)
    flat = np.concatenate([K[p] for p in (3, 0, 4)])[:L], np.concatenate([V[p] for p in (3, 0, 4)])[:L]
    for i in range(n):
        for h in range(h_kv * g):
            k, v = (f[:L - n + i + 1, h // g] for f in flat)
            w = np.exp(k @ q[i, h] / math.sqrt(d))
            assert np.allclose(out[i, h], w @ v / w.sum(), atol=1e-12)
            assert np.all(mag[i, h] >= np.abs(out[i, h]) - 1e-12)
    # one key: its value; a missing page is a page of zeros; more rows than tokens: nothing is seen
    one, _ = paged.attention(q[:1], K, V, table, 1, 1, 0, 0)
    assert np.allclose(one[0], np.repeat(V[3, 0], g, axis=0))
    gone, _ = paged.attention(q[:1], K, V, [-1, 0], 4, 1, 0, 0)
    assert not gone.any()
    none, _ = paged.attention(q, K, V, table, 2, 3, 0, 0)
    assert not none[0].any() and none[1].any()


def test_rotary_rules():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 2, 16)), np.array([0, 1, 7, 1000, 65000])
    w = paged.frequencies(1e4, 16)
    assert np.allclose(paged.turn(x, pos, w, False), layer.rope_rotate(x, pos, 1e4), atol=1e-9)
    # interleaved: the half layout of the elements put in order
    order = np.r_[0:16:2, 1:16:2]
    assert np.allclose(paged.turn(x, pos, w, True)[..., order], paged.turn(x[..., order], pos, w, False))
    # part of the head: the rest passes through, and lengths stay
    part = paged.turn(x, pos, paged.frequencies(1e4, 6), False)
    assert np.array_equal(part[..., 6:], x[..., 6:])
    assert np.allclose((part[..., :6] ** 2).sum(-1), (x[..., :6] ** 2).sum(-1))
    assert np.allclose(paged.turn(x, pos, w, False, 1.5), 1.5 * paged.turn(x, pos, w, False))


def test_scaled_frequencies():
    plain = paged.frequencies(1e4, 64)
    assert np.allclose(paged.frequencies(1e4, 64, "linear", 8.0), plain / 8)
    for kind in ("turns", "index"):
        w = paged.frequencies(1e4, 64, kind, 8.0, 8192, 1.0, 32.0)
        assert np.all(np.diff(w) < 0)
        turns = 8192 * plain / (2 * math.pi)
        assert np.allclose(w[turns > 40], plain[turns > 40]) and np.allclose(w[turns < 0.7], plain[turns < 0.7] / 8)
    assert np.allclose(paged.frequencies(1e4, 64, "turns", 1.0, 8192, 1.0, 32.0), plain)


def test_pages_by_hand():
    P = paged.Pages(6, 4, 4, 3)
    assert P.grow([0, 1], [6, 4]) is None
    assert P.table[:2] == [[0, 1, -1], [2, -1, -1]] and P.refs == [1, 1, 1, 0, 0, 0] and P.copies == []
    assert P.fork([0, 0], [2, 3]) is None
    assert P.refs == [3, 3, 1, 0, 0, 0] and P.len == [6, 4, 6, 6] and P.held(3) == [0, 1]
    assert P.grow([3, 1], [1, 1]) is None                 # 3 copies its shared last page, 1 takes a new one
    assert P.copies == [(1, 3, 2)] and P.held(3) == [0, 3] and P.held(1) == [2, 4] and P.refs == [3, 2, 1, 1, 1, 0]
    assert P.grow([0, 2], [3, 3]) == "pages" and P.len[0] == 6
    assert P.grow([0], [7]) == "length" and P.grow([0, 0], [0, 0]) == "index" and P.fork([0], [1]) == "index"
    assert P.free([1, 2]) is None and P.refs == [2, 1, 0, 1, 0, 0] and P.table[1] == [-1, -1, -1]
    P.compact()
    assert P.copies == [(3, 2, 4)] and P.held(3) == [0, 2] and P.refs == [2, 1, 1, 0, 0, 0]


@pytest.mark.parametrize("seed", range(4))
def test_pages_keep_their_books(seed):
    rng = np.random.default_rng(seed)
    P = paged.Pages(40, 4, 8, 10)
    for _ in range(300):
        s = rng.permutation(8)[:rng.integers(1, 5)].tolist()
        [lambda: P.grow(s, rng.integers(0, 9, size=len(s)).tolist()), lambda: P.free(s[:1]), P.compact,
         lambda: P.fork([s[0]] * (len(s) - 1), s[1:])][rng.choice(4, p=[.5, .2, .1, .2])]()
        count = [0] * 40
        for i in range(8):
            for p in P.held(i):
                count[p] += 1
            assert all(p == -1 for p in P.table[i][len(P.held(i)):])
        assert count == P.refs
