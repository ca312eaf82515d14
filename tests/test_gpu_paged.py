"""GPU parity of the paged cache against the plain definitions in oracle/paged.py (fp64).

Bounds, element by element.  Attention: the probabilities are rounded to bf16 (half a step, 2^-8 of each) before they
meet the values, so the sum is off by at most 2^-8 of the same sum over |V| (A below); the scores' fp32 sums, the
exponentials and the sums of up to 2^12 terms stay below 2^-10 A; the result is rounded once, 2^-8 of itself.  Rotary:
one rounding, 2^-8 of the result, and fp32 noise: angle 2^-22, sine and cosine 2^-22, two products and a sum 3 * 2^-24, below
2^-19 (|x| + |y|) mscale together.  Bookkeeping and copies are exact."""
import numpy as np
import pytest
import torch

import paper_2510_10129_amd as cc
from oracle import paged
from paper_2510_10129_amd import _lib

from _gpu_util import DEV, bits_f64, dev_bf16, dev_i32, host_bits

pytestmark = pytest.mark.gpu


def _bf16(rng, shape, std=1.0):
    """Random bf16 values as bits."""
    return host_bits(torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16))


def _ctx(h_q, h_kv, d_h, N=64, M=64, **kw):
    return cc.Context(64, h_q, h_kv, d_h, 64, 1e4, 1e-5, N_cap=N, M_cap=M, T_cap=64, **kw)


class Batch:
    """A pool whose sequences' pages lie anywhere in it, and new rows of some of them."""

    def __init__(self, rng, h_q, h_kv, d_h, page, lens, news, head_major=False, order=None, pad=(0, 0), spare=3, max_pages=None):
        self.dims, self.page, self.lens, self.news = (h_q, h_kv, d_h), page, list(lens), list(news)
        self.seq = list(range(len(lens))) if order is None else list(order)
        used = [-(-n // page) for n in lens]
        n_pages = sum(used) + spare
        cols = max_pages or max(max(used), 1)
        perm = rng.permutation(n_pages)
        self.table = np.full((len(lens), cols), -1, np.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = perm[at:at + u]
            at += u
        self.free = perm[at:]
        shape = (n_pages, h_kv, page, d_h) if head_major else (n_pages, page, h_kv, d_h)
        self.Kb, self.Vb = _bf16(rng, shape, 0.6), _bf16(rng, shape, 0.6)
        self.head_major = head_major
        self.start = np.r_[0, np.cumsum([self.news[b] for b in range(len(self.seq))])] + pad[0]
        self.rows = int(self.start[-1]) + pad[1]
        self.qb = _bf16(rng, (self.rows, h_q * d_h), 2.5)

    def view(self, bits):
        return np.swapaxes(bits, 1, 2) if self.head_major else bits

    def hide(self, value):
        """Every slot that holds no token of a sequence gets `value`."""
        K, V = self.view(self.Kb), self.view(self.Vb)
        keep = np.zeros(K.shape[:2], bool)
        for s, n in enumerate(self.lens):
            for c in range(-(-n // self.page)):
                keep[self.table[s, c], :min(self.page, n - c * self.page)] = True
        K[~keep] = value
        V[~keep] = value

    def device(self):
        self.pool = cc.PagePool(torch.zeros(self.Kb.shape[0], dtype=torch.int32, device=DEV), dev_i32(self.table), dev_i32(self.lens),
                                self.page)
        K, V = dev_bf16(self.Kb), dev_bf16(self.Vb)
        self.kv = cc.PagedKV(K.transpose(1, 2), V.transpose(1, 2)) if self.head_major else cc.PagedKV(K, V)
        self.new = cc.NewRows(dev_i32(self.start), dev_i32(self.seq), self.rows, max(self.news + [0]))
        self.q = dev_bf16(self.qb)
        return self

    def attend(self, ctx, window=0, sinks=0, **kw):
        o = torch.full_like(self.q, 7.0)
        ctx.step_paged_attention(self.q, self.new, self.pool, self.kv, o, window, sinks, **kw)
        return o

    def check(self, o, window=0, sinks=0, sample=None):
        h_q, h_kv, d_h = self.dims
        got = bits_f64(host_bits(o)).reshape(self.rows, h_q, d_h)
        K, V, q = (bits_f64(x) for x in (self.view(self.Kb), self.view(self.Vb), self.qb))
        V = np.where(np.isfinite(V), V, 0.0)               # slots without a token are not looked at
        K = np.where(np.isfinite(K), K, 0.0)
        mine = np.zeros(self.rows, bool)
        for b, s in enumerate(self.seq):
            r0, n = int(self.start[b]), self.news[b]
            mine[r0:r0 + n] = True
            pick = np.arange(n)
            if sample and n > sample:
                pick = np.unique(np.r_[0, n - 1, np.linspace(0, n - 1, sample).astype(int)])
            ref, mag = paged.attention(q[r0:r0 + n].reshape(n, h_q, d_h), K, V, self.table[s], self.lens[s], n, window, sinks, pick)
            err = np.abs(got[r0:r0 + n] - ref)[pick]
            tol = ((2.0 ** -8 + 2.0 ** -10) * (1 + 2.0 ** -8) * mag + 2.0 ** -8 * np.abs(ref))[pick]
            assert np.all(err <= tol + 1e-30), (b, n, self.lens[s], float((err - tol).max()), np.argwhere(err > tol)[:3].tolist())
        assert (got[~mine] == 7.0).all()                   # rows of no sequence stay as they were


HEADS = {"tiny": (4, 2, 64), "d64": (32, 8, 64), "g7": (28, 4, 128), "g4": (32, 8, 128), "g8": (16, 2, 128), "mha": (3, 3, 128),
         "g32": (32, 1, 64), "g5": (5, 1, 128)}


@pytest.mark.parametrize("heads", sorted(HEADS))
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(heads, page):
    """One new token a sequence: lengths of one, at and around page and tile ends, to a few thousand."""
    rng = np.random.default_rng(page)
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 1000, 2500]
    b = Batch(rng, *HEADS[heads], page, lens, [1] * len(lens), head_major=page == 64, order=rng.permutation(len(lens)), pad=(2, 3))
    b.hide(0x7FC0)                                          # NaN behind the last tokens and in free pages
    ctx = _ctx(*HEADS[heads])
    b.device().check(b.attend(ctx))
    ctx.close()


@pytest.mark.parametrize("heads,page,lens,news", [
    ("tiny", 16, [1, 5, 100, 40, 64], [1, 5, 3, 0, 64]),
    ("g4", 16, [300, 17, 2000, 64, 1], [5, 16, 2, 9, 1]),
    ("g7", 32, [500, 700, 33], [33, 2, 10]),
    ("g7", 128, [1500, 129], [300, 129]),
    ("d64", 16, [900, 1024, 70], [130, 257, 70]),
    ("g8", 64, [3000], [64]),
    ("g4", 256, [257, 255, 512], [1, 255, 100]),
    ("g32", 16, [400, 33], [3, 33]),
    ("mha", 16, [333, 70, 300], [333, 1, 65]),
    ("g5", 1024, [2100], [411]),
])
@pytest.mark.parametrize("head_major", [False, True])
def test_chunks(heads, page, lens, news, head_major):
    """Chunks of new tokens, whole prompts among them, sequences without rows, rows of no sequence."""
    rng = np.random.default_rng(len(lens) + page)
    b = Batch(rng, *HEADS[heads], page, lens, news, head_major, pad=(0, 5))
    b.hide(0xFF80)                                          # -inf
    ctx = _ctx(*HEADS[heads])
    b.device().check(b.attend(ctx), sample=40)
    ctx.close()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 0), (64, 4), (100, 65), (1000, 16), (4000, 5), (50, 5000)])
@pytest.mark.parametrize("heads,news", [("g4", [1, 1, 1, 1, 1]), ("g7", [4, 1, 200, 60, 1]), ("d64", [64, 0, 300, 1, 1])])
def test_windows_and_sinks(window, sinks, heads, news):
    """Windows shorter and longer than tiles, chunks and sequences; sinks within, at the ends of and past them."""
    rng = np.random.default_rng(window + sinks)
    lens = [64, 65, 1700, 130, 1]
    b = Batch(rng, *HEADS[heads], 16, lens, news)
    b.hide(0x7F80)
    ctx = _ctx(*HEADS[heads])
    b.device().check(b.attend(ctx, window, sinks), window, sinks, sample=40)
    ctx.close()


@pytest.mark.parametrize("news", [[1, 1], [40, 3], [500, 1]])
def test_pages_that_slid_out_may_be_given_back(news):
    """Entries that no row's window reaches name no page any more; what a window reaches of a page that is none reads as zeros."""
    rng = np.random.default_rng(5)
    window, sinks, page, lens = 100, 20, 16, [1000, 777]
    b = Batch(rng, *HEADS["g4"], page, lens, news)
    for s, n in enumerate(lens):
        low = n - news[s] - window + 1
        for c in range(-(-sinks // page), low // page):
            b.table[s, c] = [-1, b.Kb.shape[0], 2 ** 31 - 1, -2 ** 31][c % 4]
    ctx = _ctx(*HEADS["g4"])
    b.device()
    b.check(b.attend(ctx, window, sinks, flags=_lib.FLAG_CHECK_IDX), window, sinks, sample=30)
    b.table[0, -4], b.table[1, 0] = -7, 1 << 30             # seen, and gone
    b.device()
    b.check(b.attend(ctx, window, sinks), window, sinks, sample=30)
    with pytest.raises(cc.CacheClipError) as e:
        b.attend(ctx, window, sinks, flags=_lib.FLAG_CHECK_IDX)
    assert e.value.status == _lib.CC_ERR_IDX
    ctx.close()


def test_more_rows_than_tokens_and_indexes_that_are_none():
    """Rows in front of a sequence's first token see nothing and get zeros; so do all rows of an index out of range."""
    rng = np.random.default_rng(6)
    b = Batch(rng, *HEADS["g4"], 16, [3, 50, 0], [5, 50, 2])
    ctx = _ctx(*HEADS["g4"])
    b.device()
    o = b.attend(ctx)
    b.check(o)
    assert not host_bits(o)[:2].any() and not host_bits(o)[-2:].any()
    b.new.seq = dev_i32([0, 3, -1])
    o = host_bits(b.attend(ctx))
    assert not o[5:].any() and o[2:5].any()
    for flagged in (b.new, cc.NewRows(dev_i32([0, 5, 60, 60]), None, b.rows, 60)):
        b.new = flagged
        with pytest.raises(cc.CacheClipError) as e:
            b.attend(ctx, flags=_lib.FLAG_CHECK_IDX)
        assert e.value.status == _lib.CC_ERR_IDX
    b.new = cc.NewRows(dev_i32([0]), None, b.rows, 60)      # no sequence at all
    assert (bits_f64(host_bits(b.attend(ctx))) == 7.0).all()
    empty = torch.empty((0, b.q.shape[1]), dtype=torch.bfloat16, device=DEV)
    ctx.step_paged_attention(empty, cc.NewRows(dev_i32([0, 0]), None, 0, 0), b.pool, b.kv, empty)
    ctx.close()


def test_the_bound_on_new_rows_does_not_change_results():
    """max_new only decides launch shapes: too small or too large a bound gives the same rows within the bound of a rounding."""
    rng = np.random.default_rng(7)
    b = Batch(rng, *HEADS["g8"], 32, [700, 300, 90], [100, 1, 17])
    ctx = _ctx(*HEADS["g8"])
    b.device()
    for most in (0, 1, 2, 17, 100, 5000):
        b.new.max_new = most
        b.check(b.attend(ctx), sample=40)
    ctx.close()


def test_same_sequence_twice_and_repeated_calls():
    """Two sets of rows over one sequence; the same call gives the same bits."""
    rng = np.random.default_rng(8)
    b = Batch(rng, *HEADS["g4"], 16, [1500, 900], [3, 3, 3], order=[0, 1, 0])
    ctx = _ctx(*HEADS["g4"])
    b.device()
    first = b.attend(ctx)
    b.check(first)
    for _ in range(3):
        assert torch.equal(b.attend(ctx).view(torch.int16), first.view(torch.int16))
    ctx.close()


@pytest.mark.parametrize("news", [[1] * 300, [1 + (i % 3) for i in range(300)], [40] * 130])
def test_many_sequences(news):
    rng = np.random.default_rng(9)
    lens = [int(v) for v in rng.integers(41, 200, size=len(news))]
    b = Batch(rng, 8, 2, 64, 16, lens, news, order=rng.permutation(len(news)))
    b.news = [news[i] for i in range(len(news))]
    ctx = _ctx(8, 2, 64)
    b.device().check(b.attend(ctx), sample=3)
    ctx.close()


@pytest.mark.parametrize("n_new", [1, 4, 70])
def test_one_long_sequence_is_split(n_new):
    """A sequence of many tiles and few rows, and a short one beside it."""
    rng = np.random.default_rng(10)
    b = Batch(rng, 8, 2, 128, 64, [20000, 40], [n_new, 1])
    ctx = _ctx(8, 2, 128)
    b.device().check(b.attend(ctx), sample=4)
    ctx.close()


@pytest.mark.parametrize("n_new", [1, 90])
def test_pages_behind_32_bit_offsets(n_new):
    """A pool whose pages lie more than 2^32 elements apart."""
    rng = np.random.default_rng(11)
    h_q, h_kv, d_h, page = 8, 2, 128, 16
    b = Batch(rng, h_q, h_kv, d_h, page, [150], [n_new])
    b.device()
    n_pages, gap = b.Kb.shape[0], 7 * 10 ** 8 // 8 * 8
    big = torch.empty(gap * (n_pages - 1) + 2 * page * h_kv * d_h, dtype=torch.bfloat16, device=DEV)
    st = (gap, h_kv * d_h, d_h, 1)
    K = torch.as_strided(big, (n_pages, page, h_kv, d_h), st)
    V = torch.as_strided(big, (n_pages, page, h_kv, d_h), st, page * h_kv * d_h)
    K.copy_(dev_bf16(b.Kb)), V.copy_(dev_bf16(b.Vb))
    b.kv = cc.PagedKV(K, V)
    ctx = _ctx(h_q, h_kv, d_h)
    b.check(b.attend(ctx), sample=20)
    ctx.close()


def test_peaked_and_growing_scores():
    """Queries far along their keys: maxima that jump by hundreds between tiles and probabilities that vanish."""
    rng = np.random.default_rng(12)
    for n_new in (1, 80):
        b = Batch(rng, 8, 2, 128, 16, [700], [n_new])
        b.qb = _bf16(rng, b.qb.shape, 40.0)
        ctx = _ctx(8, 2, 128)
        b.device()
        got = bits_f64(host_bits(b.attend(ctx))).reshape(n_new, 8, 128)
        pick = [0, n_new // 2, n_new - 1]
        ref, mag = paged.attention(bits_f64(b.qb).reshape(n_new, 8, 128), bits_f64(b.Kb), bits_f64(b.Vb), b.table[0], 700, n_new, 0, 0, pick)
        # scores of up to 2^9: their fp32 sums are off by 2^-24 * 130 * 2^9, a probability by 2^-8 of itself
        err, tol = np.abs(got - ref)[pick], ((2.0 ** -8 + 2.0 ** -7) * mag + 2.0 ** -8 * np.abs(ref))[pick]
        assert np.all(err <= tol), float((err - tol).max())
        ctx.close()


@pytest.mark.parametrize("seed", range(30))
def test_batches_at_random(seed):
    """Head layouts, page sizes, batches of 1 to 150 sequences, lengths of 1 to 9000, one to 600 rows, windows: whole blocks, blocks in
    two and in dozens of pieces, ranges with the ends of two blocks; a few rows of each sequence are compared."""
    rng = np.random.default_rng(1000 + seed)
    d_h = int(rng.choice([64, 128]))
    h_kv = int(rng.choice([1, 2, 4, 8]))
    g = int(rng.choice([1, 3, 4, 7, 8]))
    n = int(rng.choice([1, 1, 2, 5, 70, 150]))
    most = int(min(9000, 40000 // n))
    lens = [int(v) for v in np.exp(rng.uniform(0, np.log(most), size=n)).astype(int) + 1]
    cap = int(rng.choice([1, 1, 4, 40, 600]))
    news = [int(min(L, rng.integers(0 if n > 1 else 1, cap + 1))) for L in lens]
    window = int(rng.choice([0, 0, rng.integers(1, 3000)]))
    sinks = int(rng.integers(0, 130)) if window else 0
    b = Batch(rng, h_kv * g, h_kv, d_h, int(rng.choice([16, 32, 64, 256])), lens, news, head_major=bool(rng.integers(2)), pad=(0, 1))
    b.hide(0x7FC0)
    ctx = _ctx(h_kv * g, h_kv, d_h)
    o = b.device().attend(ctx, window, sinks)
    b.check(o, window, sinks, sample=3)
    assert torch.equal(b.attend(ctx, window, sinks).view(torch.int16), o.view(torch.int16))
    ctx.close()


# ---- rotary positions and the append ----

def _rope_case(rng, b, rule, packed, pos=None, in_place=False):
    h_q, h_kv, d_h = b.dims
    ctx = _ctx(h_q, h_kv, d_h)
    kb, vb = _bf16(rng, (b.rows, h_kv * d_h)), _bf16(rng, (b.rows, h_kv * d_h))
    if packed:
        qkv = dev_bf16(np.concatenate([b.qb, kb, vb], axis=1))
        q, k, v = qkv.split((h_q * d_h, h_kv * d_h, h_kv * d_h), dim=1)
    else:
        q, k, v = b.q, dev_bf16(kb), dev_bf16(vb)
    out = q if in_place else torch.full((b.rows, h_q * d_h), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.step_rope_append(q, k, v, b.new, b.pool, b.kv, rule, out, pos=None if pos is None else dev_i32(pos))
    torch.cuda.synchronize()
    freq = paged.frequencies(rule.base, rule.rot, rule.scaling, rule.factor, rule.orig_len, rule.low, rule.high)
    gq = bits_f64(host_bits(out)).reshape(-1, h_q, d_h)
    gK, gV = host_bits(b.kv.K), host_bits(b.kv.V)
    wantV, there, left = b.view(b.Vb).copy(), np.zeros(gK.shape[:2], bool), np.ones(b.rows, bool)

    def close(got, x, at):
        ref = paged.turn(x, at, freq, rule.interleaved, rule.mscale)
        size = np.abs(x).copy()
        half = rule.rot // 2
        p0, p1 = (slice(0, rule.rot, 2), slice(1, rule.rot, 2)) if rule.interleaved else (slice(0, half), slice(half, rule.rot))
        size[..., p0] = size[..., p1] = np.abs(x[..., p0]) + np.abs(x[..., p1])
        tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * size * abs(rule.mscale)
        tol[..., rule.rot:] = 0
        err = np.abs(got - ref)
        assert np.all(err <= tol), (float((err - tol).max()), np.argwhere(err > tol)[:3].tolist())

    for i, s in enumerate(b.seq):
        for t in range(b.news[i]):
            r, p = int(b.start[i]) + t, b.lens[s] - b.news[i] + t
            if p < 0:
                continue
            left[r] = False
            at = np.array([p if pos is None else pos[r]])
            close(gq[r:r + 1], bits_f64(b.qb[r]).reshape(1, h_q, d_h), at)
            page, slot = b.table[s, p // b.page], p % b.page
            if not 0 <= page < gK.shape[0]:
                continue
            there[page, slot] = True
            close(bits_f64(gK[page, slot])[None], bits_f64(kb[r]).reshape(1, h_kv, d_h), at)
            wantV[page, slot] = vb[r].reshape(h_kv, d_h)
    assert np.array_equal(gV, wantV) and np.array_equal(gK[~there], b.view(b.Kb)[~there])
    assert np.array_equal(host_bits(out)[left], b.qb[left]) if in_place else (gq[left] == 7.0).all()
    ctx.close()


RULES = [cc.Rope(1e4, 64), cc.Rope(5e5, 32, True), cc.Rope(1e6, 64, False, "linear", 4.0), cc.Rope(1e4, 20, False, "turns", 8.0, 512, 1.0, 4.0),
         cc.Rope(1e4, 64, True, "index", 16.0, 4096, 1.0, 32.0, 1.277), cc.Rope(1e4, 2), cc.Rope(2.0, 62, True, mscale=-0.5), cc.Rope(1e4, 48)]


@pytest.mark.parametrize("rule", RULES, ids=range(len(RULES)))
@pytest.mark.parametrize("heads", ["tiny", "g7", "mha"])
def test_rope_append(rule, heads):
    rng = np.random.default_rng(20)
    lens, news = [1, 40, 700, 64, 9], [1, 3, 130, 0, 9]
    b = Batch(rng, *HEADS[heads], 16, lens, news, head_major=heads == "mha", order=[4, 0, 2, 1, 3], pad=(1, 2))
    b.news = [9, 1, 130, 3, 0]
    b.start = np.r_[0, np.cumsum(b.news)] + 1
    _rope_case(rng, b.device(), rule, packed=heads == "g7")


@pytest.mark.parametrize("rot", [128, 64, 96, 70])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_append_wide_heads_in_place_and_far(rot, interleaved):
    """Head dim 128, queries turned where they lie, positions of their own up to 2^31 - 1."""
    rng = np.random.default_rng(rot)
    b = Batch(rng, 8, 2, 128, 32, [100, 5], [60, 5])
    pos = rng.integers(0, 2 ** 31, size=b.rows).astype(np.int32)
    pos[:4] = [0, 1, 2 ** 31 - 1, 65536]
    _rope_case(rng, b.device(), cc.Rope(5e5, rot, interleaved), False, pos, in_place=True)


def test_rope_append_skips_what_has_no_place():
    """Rows in front of the first token, sequences that are none and pages that are none."""
    rng = np.random.default_rng(21)
    b = Batch(rng, *HEADS["tiny"], 16, [2, 40, 30], [4, 40, 1])
    b.table[1, 1], b.table[2, 1] = -1, b.Kb.shape[0]
    _rope_case(rng, b.device(), cc.Rope(1e4, 64), True)
    ctx = _ctx(*HEADS["tiny"])
    k = torch.zeros((b.rows, 128), dtype=torch.bfloat16, device=DEV)
    for new in (b.new, cc.NewRows(dev_i32([0, 1]), dev_i32([7]), b.rows, 1), cc.NewRows(dev_i32([0, 1, 0]), None, b.rows, 1)):
        with pytest.raises(cc.CacheClipError) as e:
            ctx.step_rope_append(b.q, k, k, new, b.pool, b.kv, cc.Rope(1e4, 64), torch.empty_like(b.q), flags=_lib.FLAG_CHECK_IDX)
        assert e.value.status == _lib.CC_ERR_IDX
    ctx.close()


# ---- pages ----

def _compare(pool, P, kvs, mirror):
    assert pool.refs.tolist() == P.refs and pool.len.tolist() == P.len
    for s in range(len(P.len)):
        n = len(P.held(s))
        assert pool.table[s, :n].tolist() == P.table[s][:n], s
    for (K, V), kv in zip(mirror, kvs):
        assert np.array_equal(host_bits(kv.K), K) and np.array_equal(host_bits(kv.V), V)


def _apply(P, mirror):
    for K, V in mirror:
        for old, new, n in P.copies:
            K[new, :n], V[new, :n] = K[old, :n], V[old, :n]


STATUS = {None: 0, "index": _lib.CC_ERR_IDX, "length": _lib.CC_ERR_SHAPE, "pages": _lib.CC_ERR_WORKSPACE}


@pytest.mark.parametrize("seed,n_pages,page,n_seqs,max_pages,layers,d_h,head_major", [
    (0, 60, 16, 12, 8, 2, 64, False), (1, 300, 32, 40, 12, 1, 128, True), (2, 9, 16, 5, 9, 3, 64, True), (3, 20000, 16, 1500, 30, 1, 64, False)])
def test_random_histories(seed, n_pages, page, n_seqs, max_pages, layers, d_h, head_major):
    """Calls of all four kinds, refused ones among them, against the books kept one page at a time."""
    rng = np.random.default_rng(seed)
    h_kv = 1 + seed % 3
    ctx = _ctx(2 * h_kv, h_kv, d_h)
    pool = cc.PagePool.empty(n_pages, page, n_seqs, max_pages, device=DEV)
    P = paged.Pages(n_pages, page, n_seqs, max_pages)
    mirror, kvs = [], []
    for _ in range(layers):
        shape = (n_pages, h_kv, page, d_h) if head_major else (n_pages, page, h_kv, d_h)
        pair = [_bf16(rng, shape) for _ in range(2)]
        dev = [dev_bf16(x) for x in pair]
        mirror.append([np.swapaxes(x, 1, 2) if head_major else x for x in pair])
        kvs.append(cc.PagedKV(*[x.transpose(1, 2) if head_major else x for x in dev]))
    seen = set()
    for step in range(40):
        kind = rng.choice(["grow", "free", "fork", "compact"], p=[.5, .15, .25, .1])
        n = int(rng.integers(0, n_seqs + 1))
        some = rng.permutation(n_seqs)[:n].tolist()
        P.copies = []
        try:
            if kind == "grow":
                more = rng.integers(0, 2 * page + 1, size=n).tolist()
                if rng.random() < 0.1 and n:
                    some[0] = [n_seqs, -1, some[-1]][rng.integers(3)]
                if rng.random() < 0.1 and n:
                    more[-1] = int(rng.choice([-1, max_pages * page + 1, 2 ** 31 - 1]))
                want = P.grow(some, more)
                ctx.grow_pages(pool, kvs, dev_i32(some), dev_i32(more))
            elif kind == "free":
                some = some[:max(1, n // 3)]
                want = P.free(some)
                ctx.free_pages(pool, dev_i32(some))
            elif kind == "fork":
                dst = [s for s in some if P.len[s] == 0 or rng.random() < 0.01]
                src = rng.integers(0, n_seqs, size=len(dst)).tolist()
                want = P.fork(src, dst)
                ctx.fork_pages(pool, dev_i32(src), dev_i32(dst))
            else:
                want = P.compact()
                ctx.compact_pages(pool, kvs)
            got = 0
        except cc.CacheClipError as e:
            got = e.status
        if want is not None:
            P.copies = []
        assert got == STATUS[want] == pool.status.item(), (step, kind, want, got)
        seen.add((kind, want))
        _apply(P, mirror)
        _compare(pool, P, kvs, mirror)
    assert {"grow", "free", "fork", "compact"} <= {k for k, w in seen if w is None}
    ctx.close()


def test_lists_longer_than_a_workgroup():
    """More entries than threads, more pages than are found in one step, entries of none to many pages, copies in every part."""
    rng = np.random.default_rng(31)
    n_seqs, n_pages, page, max_pages = 5000, 40001, 16, 64
    ctx = _ctx(1, 1, 64)
    pool, P = cc.PagePool.empty(n_pages, page, n_seqs, max_pages, device=DEV), paged.Pages(n_pages, page, n_seqs, max_pages)
    mirror = [[_bf16(rng, (n_pages, page, 1, 64)) for _ in range(2)]]
    kvs = [cc.PagedKV(dev_bf16(K), dev_bf16(V)) for K, V in mirror]
    order = rng.permutation(n_seqs).tolist()
    first, rest = order[:2300], order[2300:]
    more = [int(x) for x in rng.choice([0, 1, 15, 16, 17, 33, 81, 97, 640], size=2300, p=[.1, .2, .1, .1, .1, .2, .1, .05, .05])]
    src = rng.choice(first, size=2500).tolist()
    fine = rng.permutation(first + rest[:2500]).tolist()
    steps = [("grow", first, more), ("fork", src, rest[:2500]), ("grow", fine, rng.integers(0, 40, size=4800).tolist()),
             ("grow", fine + [fine[4000]], [1] * 4801), ("free", fine[::3], None), ("grow", fine[1::3], [300] * 1600),
             ("grow", fine[1:3900:3], [300] * 1300)]
    for kind, a, b in steps:
        P.copies, got = [], 0
        call = dict(grow=lambda: ctx.grow_pages(pool, kvs, dev_i32(a), dev_i32(b)), fork=lambda: ctx.fork_pages(pool, dev_i32(a), dev_i32(b)),
                    free=lambda: ctx.free_pages(pool, dev_i32(a)))[kind]
        want = P.free(a) if kind == "free" else getattr(P, kind)(a, b)
        try:
            call()
        except cc.CacheClipError as e:
            got = e.status
        assert got == STATUS[want], (kind, want, got)
        if want is None:
            _apply(P, mirror)
        _compare(pool, P, kvs, mirror)
    ctx.close()


def test_many_layers_take_several_launches():
    """More layers than one copy launch takes; a cow copy of 1 and of 15 tokens and a compaction."""
    rng = np.random.default_rng(30)
    ctx = _ctx(1, 1, 64)
    pool, P = cc.PagePool.empty(12, 16, 4, 4, device=DEV), paged.Pages(12, 16, 4, 4)
    mirror = [[_bf16(rng, (12, 16, 1, 64)) for _ in range(2)] for _ in range(131)]
    kvs = [cc.PagedKV(dev_bf16(K), dev_bf16(V)) for K, V in mirror]
    for kind, a, b in (("grow", [0, 1], [17, 31]), ("fork", [0, 1], [2, 3]), ("grow", [3, 0], [1, 40]), ("free", [1, 0], None), ("compact",) * 3):
        if kind == "compact":
            P.compact(), ctx.compact_pages(pool, kvs)
        elif kind == "free":
            P.free(a), ctx.free_pages(pool, dev_i32(a))
        elif kind == "fork":
            P.fork(a, b), ctx.fork_pages(pool, dev_i32(a), dev_i32(b))
        else:
            P.grow(a, b), ctx.grow_pages(pool, kvs, dev_i32(a), dev_i32(b))
        _apply(P, mirror)
        P.copies = []
        _compare(pool, P, kvs, mirror)
    ctx.close()


def test_refusals_leave_no_trace():
    ctx = _ctx(4, 2, 64)
    pool = cc.PagePool.empty(8, 16, 3, 4, device=DEV)
    K = torch.zeros((8, 16, 2, 64), dtype=torch.bfloat16, device=DEV)
    kv = cc.PagedKV(K, K.clone())
    for call in (lambda: ctx.grow_pages(pool, [kv], dev_i32([0, 1, 2, 2]), dev_i32([1, 1, 1, 1])),
                 lambda: ctx.free_pages(pool, dev_i32([0, 1, 2, 0])),
                 lambda: ctx.step_paged_attention(torch.zeros((1, 256), dtype=torch.bfloat16, device=DEV), cc.NewRows(dev_i32([0, 1]), None, 1, 1),
                                                  pool, kv, torch.zeros((1, 256), dtype=torch.bfloat16, device=DEV), window=-1),
                 lambda: ctx.compact_pages(cc.PagePool(pool.refs, pool.table, pool.len, 24), [])):
        with pytest.raises(cc.CacheClipError) as e:
            call()
        assert e.value.status == _lib.CC_ERR_SHAPE
    buf, new = torch.zeros(4096, dtype=torch.bfloat16, device=DEV), cc.NewRows(dev_i32([0, 2]), None, 2, 2)
    q, qkv = buf[:512].view(2, 256), buf.view(2, 2048)[:, :512]
    for call in (lambda: ctx.step_paged_attention(q, new, pool, kv, q), lambda: ctx.step_paged_attention(q, new, pool, kv, buf[504:1016].view(2, 256)),
                 lambda: ctx.step_rope_append(qkv[:, :256], qkv[:, 256:384], qkv[:, 384:], new, pool, kv, cc.Rope(1e4, 64), buf[248:760].view(2, 256)),
                 lambda: ctx.step_rope_append(q, qkv[:, 256:384], buf[512:].view(2, 1792)[:, :128], new, pool, kv, cc.Rope(1e4, 64), q),
                 lambda: ctx.step_rope_append(q, buf[1024:].view(2, 1536)[:, :128], qkv[:, 384:], new, pool, kv, cc.Rope(1e4, 64), q)):
        with pytest.raises(cc.CacheClipError) as e:          # results over what is still read
            call()
        assert e.value.status == _lib.CC_ERR_SHAPE and "overlap" in str(e.value)
    small = cc.PagePool(pool.refs, pool.table, pool.len, 16, work=torch.zeros(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(cc.CacheClipError) as e:
        ctx.free_pages(small, dev_i32([0]))
    assert e.value.status == _lib.CC_ERR_WORKSPACE
    host, x = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 256), dtype=torch.bfloat16, device=DEV)
    for call in (lambda: ctx.free_pages(pool, host), lambda: ctx.fork_pages(pool, dev_i32([0]), host),
                 lambda: cc.PagePool(pool.refs, pool.table, pool.len.cpu(), 16),
                 lambda: ctx.compact_pages(pool, [cc.PagedKV(K.cpu(), K.cpu())]),
                 lambda: ctx.step_paged_attention(x, cc.NewRows(torch.tensor([0, 1], dtype=torch.int32), None, 1, 1), pool, kv, x.clone()),
                 lambda: ctx.step_paged_attention(x.cpu(), cc.NewRows(dev_i32([0, 1]), None, 1, 1), pool, kv, x),
                 lambda: ctx.step_rope_append(x, x[:, :128], x[:, :128], cc.NewRows(dev_i32([0, 1]), None, 1, 1), pool, kv, cc.Rope(1e4, 64), x,
                                              pos=host)):
        with pytest.raises(ValueError):                      # host memory does not reach the device
            call()
    assert not pool.refs.any() and not pool.len.any()
    ctx.grow_pages(pool, [], dev_i32([]), dev_i32([]))       # nothing to do
    ctx.fork_pages(pool, dev_i32([]), dev_i32([]))
    ctx.compact_pages(pool, [kv])
    assert pool.status.item() == 0
    ctx.close()


# ---- together ----

def test_answers_from_a_recomputed_cache():
    """A contiguous cache becomes pages as it lies; attention over it is the contiguous attention; then answers fork from it,
    grow, are turned and attend layer by layer, and the freed pool is empty again."""
    rng = np.random.default_rng(40)
    h_q, h_kv, d_h, page, N, layers = 8, 2, 128, 16, 203, 2
    ctx = _ctx(h_q, h_kv, d_h, N=512, M=64)
    n_pages = 40
    Kb, Vb = ([_bf16(rng, (n_pages * page, h_kv, d_h), 0.6) for _ in range(layers)] for _ in range(2))
    K, V = [dev_bf16(x) for x in Kb], [dev_bf16(x) for x in Vb]
    kvs = [cc.PagedKV(k.view(n_pages, page, h_kv, d_h), v.view(n_pages, page, h_kv, d_h)) for k, v in zip(K, V)]
    pool, P = cc.PagePool.empty(n_pages, page, 6, 20, device=DEV), paged.Pages(n_pages, page, 6, 20)
    P.grow([0], [N]), ctx.grow_pages(pool, kvs, dev_i32([0]), dev_i32([N]))      # the lowest pages: the cache itself
    qb = _bf16(rng, (40, h_q * d_h), 2.5)
    q, one, two = dev_bf16(qb), torch.empty((40, h_q * d_h), dtype=torch.bfloat16, device=DEV), torch.empty((40, h_q * d_h), dtype=torch.bfloat16, device=DEV)
    ctx.step_sparse_attention(q, 40, dev_i32(np.arange(N - 40, N)), cc.KVLayer(K[0][:N], V[0][:N]), one)
    ctx.step_paged_attention(q, cc.NewRows(dev_i32([0, 40]), None, 40, 40), pool, kvs[0], two)
    ref, mag = paged.attention(bits_f64(qb).reshape(40, h_q, d_h), bits_f64(Kb[0]).reshape(n_pages, page, h_kv, d_h),
                               bits_f64(Vb[0]).reshape(n_pages, page, h_kv, d_h), P.table[0], N, 40, 0, 0)
    for got in (one, two):
        assert np.all(np.abs(bits_f64(host_bits(got)).reshape(ref.shape) - ref) <= 1.3 * 2.0 ** -8 * mag + 2.0 ** -8 * np.abs(ref))

    mirror = [[k.reshape(n_pages, page, h_kv, d_h), v.reshape(n_pages, page, h_kv, d_h)] for k, v in zip(Kb, Vb)]
    rule = cc.Rope(5e5, 64, True, "index", 4.0, 128, 1.0, 8.0, 1.1)
    freq = paged.frequencies(rule.base, rule.rot, rule.scaling, rule.factor, rule.orig_len, rule.low, rule.high)
    P.fork([0, 0, 0], [3, 1, 5]), ctx.fork_pages(pool, dev_i32([0, 0, 0]), dev_i32([3, 1, 5]), sync=False)
    for step, (seqs, more) in enumerate((([3, 1, 5], [1, 1, 1]), ([5, 3], [6, 30]), ([1, 3, 5, 0], [1, 1, 1, 9]))):
        P.grow(seqs, more), ctx.grow_pages(pool, kvs, dev_i32(seqs), dev_i32(more), sync=False)
        _apply(P, mirror)
        start, rows = np.r_[0, np.cumsum(more)], sum(more)
        new = cc.NewRows(dev_i32(start), dev_i32(seqs), rows, max(more))
        for l in range(layers):
            qkv = _bf16(rng, (rows, (h_q + 2 * h_kv) * d_h))
            qd, kd, vd = dev_bf16(qkv).split((h_q * d_h, h_kv * d_h, h_kv * d_h), dim=1)
            turned, o = torch.empty((rows, h_q * d_h), dtype=torch.bfloat16, device=DEV), torch.empty((rows, h_q * d_h), dtype=torch.bfloat16, device=DEV)
            ctx.step_rope_append(qd, kd, vd, new, pool, kvs[l], rule, turned, flags=_lib.FLAG_CHECK_IDX)
            ctx.step_paged_attention(turned, new, pool, kvs[l], o, window=100, sinks=4, flags=_lib.FLAG_CHECK_IDX)
            gK, gV = host_bits(kvs[l].K), host_bits(kvs[l].V)
            for i, s in enumerate(seqs):
                pos = np.arange(P.len[s] - more[i], P.len[s])
                pages = np.array(P.table[s])[pos // page]
                x = bits_f64(qkv[start[i]:start[i + 1]]).reshape(more[i], -1, d_h)
                k = paged.turn(x[:, h_q:h_q + h_kv], pos, freq, True, rule.mscale)
                assert np.allclose(bits_f64(gK[pages, pos % page]), k, rtol=2.0 ** -8, atol=1e-5)
                mirror[l][0][pages, pos % page] = gK[pages, pos % page]        # rounded as the device rounds
                mirror[l][1][pages, pos % page] = qkv[start[i]:start[i + 1]].reshape(more[i], -1, d_h)[:, h_q + h_kv:]
                tq = bits_f64(host_bits(turned[start[i]:start[i + 1]])).reshape(more[i], h_q, d_h)
                assert np.allclose(tq, paged.turn(x[:, :h_q], pos, freq, True, rule.mscale), rtol=2.0 ** -8, atol=1e-5)
                ref, mag = paged.attention(tq, bits_f64(mirror[l][0]), bits_f64(mirror[l][1]), P.table[s], P.len[s], more[i], 100, 4)
                got = bits_f64(host_bits(o[start[i]:start[i + 1]])).reshape(ref.shape)
                assert np.all(np.abs(got - ref) <= 1.3 * 2.0 ** -8 * mag + 2.0 ** -8 * np.abs(ref)), (step, l, s)
        _compare(pool, P, kvs, mirror)
    P.free([0]), ctx.free_pages(pool, dev_i32([0]))
    P.compact(), ctx.compact_pages(pool, kvs)
    _apply(P, mirror)
    _compare(pool, P, kvs, mirror)
    ctx.free_pages(pool, dev_i32([1, 5, 3]))
    assert not pool.refs.any() and not pool.len.any()
    ctx.close()


def test_a_captured_decode_loop_replays():
    """Grow by one, turn, append and attend, recorded once and replayed, between eager work; every replay against the same
    calls made eagerly on a pool of their own."""
    rng = np.random.default_rng(41)
    h_q, h_kv, d_h, page = 8, 2, 64, 16
    b, lens = 3, [30, 47, 1]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    shape = (32, page, h_kv, d_h)
    Kb, Vb, qkv = _bf16(rng, shape, 0.6), _bf16(rng, shape, 0.6), _bf16(rng, (b, (h_q + 2 * h_kv) * d_h))

    def make():
        pool = cc.PagePool.empty(32, page, b, 10, device=DEV)
        kv = cc.PagedKV(dev_bf16(Kb), dev_bf16(Vb))
        s = dict(pool=pool, kv=kv, x=dev_bf16(qkv), seq=dev_i32(range(b)), more=dev_i32([1] * b), q=torch.zeros((b, h_q * d_h), dtype=torch.bfloat16, device=DEV),
                 o=torch.zeros((b, h_q * d_h), dtype=torch.bfloat16, device=DEV), new=cc.NewRows(dev_i32(range(b + 1)), None, b, 1))
        s["parts"] = s["x"].split((h_q * d_h, h_kv * d_h, h_kv * d_h), dim=1)
        return s

    def step(ctx, s):
        ctx.grow_pages(s["pool"], [s["kv"]], s["seq"], s["more"], sync=False)
        ctx.step_rope_append(*s["parts"], s["new"], s["pool"], s["kv"], cc.Rope(1e4, 64), s["q"])
        ctx.step_paged_attention(s["q"], s["new"], s["pool"], s["kv"], s["o"], window=40, sinks=2)

    eager, graphed = make(), make()
    ctx, ctx2 = _ctx(h_q, h_kv, d_h), _ctx(h_q, h_kv, d_h, stream=side.cuda_stream)
    for c, s in ((ctx, eager), (ctx2, graphed)):
        torch.cuda.synchronize()
        c.grow_pages(s["pool"], [s["kv"]], s["seq"], dev_i32(lens))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(ctx2, graphed)
    for i in range(25):
        x = dev_bf16(_bf16(rng, qkv.shape))
        eager["x"].copy_(x), graphed["x"].copy_(x)
        step(ctx, eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for key in ("o", "q"):
            assert torch.equal(eager[key].view(torch.int16), graphed[key].view(torch.int16)), (i, key)
        assert torch.equal(eager["pool"].table, graphed["pool"].table) and torch.equal(eager["pool"].len, graphed["pool"].len)
        assert torch.equal(eager["kv"].K.view(torch.int16), graphed["kv"].K.view(torch.int16)) and graphed["pool"].status.item() == 0
        (x.float() @ x.float().t()).sum().item()             # the program's own work between replays
    ctx.close(), ctx2.close()


def test_every_kernel_is_timed():
    ctx = _ctx(4, 2, 64)
    pool = cc.PagePool.empty(8, 16, 2, 4, device=DEV)
    K = torch.zeros((8, 16, 2, 64), dtype=torch.bfloat16, device=DEV)
    kv, x = cc.PagedKV(K, K.clone()), torch.zeros((1, 256), dtype=torch.bfloat16, device=DEV)
    ctx.profile_enable(True)
    ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([1]))
    new = cc.NewRows(dev_i32([0, 1]), None, 1, 1)
    ctx.step_rope_append(x, x[:, :128], x[:, :128], new, pool, kv, cc.Rope(1e4, 64), torch.empty_like(x))
    ctx.step_paged_attention(x, new, pool, kv, torch.empty_like(x))
    prof = ctx.profile_read()
    assert {k for k, (_, n) in prof.items() if n} == {"pages", "page_copy", "rope_append", "paged_attn"}
    ctx.close()
