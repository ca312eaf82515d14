"""Paged attention of few rows holds its probabilities in two bf16 parts: what it loses is the rounding of its result and the noise
of sums in 32 bits, not a rounding of the probabilities.

Bound per element: the result is rounded once, 2^-8 of itself.  A probability keeps 2^-16 of itself (what the first part leaves is 2^-8
of it at most and is rounded to 2^-8 of that).  Scores: 128 products of a sum of magnitudes below 16 (in base 2) in 32 bits, 128 * 2^-24 * 16 =
2^-13, as relative errors of the probabilities twice (numerator and denominator); sums of up to 2500 terms 2500 * 2^-24 < 2^-12.7,
twice.  Together below 2^-11 of the same sum over |V|."""
import numpy as np
import pytest

from oracle import paged

from _gpu_util import bits_f64, host_bits
from test_gpu_paged import HEADS, Batch, _ctx

pytestmark = pytest.mark.gpu


def _check(b, o, window=0, sinks=0):
    h_q, _, d_h = b.dims
    got = bits_f64(host_bits(o)).reshape(b.rows, h_q, d_h)
    K, V, q = (bits_f64(x) for x in (b.view(b.Kb), b.view(b.Vb), b.qb))
    for i, s in enumerate(b.seq):
        r0, n = int(b.start[i]), b.news[i]
        ref, mag = paged.attention(q[r0:r0 + n].reshape(n, h_q, d_h), K, V, b.table[s], b.lens[s], n, window, sinks)
        err, tol = np.abs(got[r0:r0 + n] - ref), 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * mag
        assert np.all(err <= tol), (i, n, b.lens[s], float((err / tol).max()), int((err > tol).sum()), err.size)


@pytest.mark.parametrize("heads", ["tiny", "d64", "g4", "g7", "g8", "mha", "g5"])
def test_single_tokens(heads):
    rng = np.random.default_rng(50)
    lens = [1, 2, 3, 9, 16, 17, 33, 64, 65, 129, 700, 2500]
    b = Batch(rng, *HEADS[heads], 16, lens, [1] * len(lens))
    ctx = _ctx(*HEADS[heads])
    o = b.device().attend(ctx)
    _check(b, o)
    ctx.close()


@pytest.mark.parametrize("heads,most", [("d64", 8), ("tiny", 16), ("g4", 4), ("g7", 2), ("g8", 2), ("mha", 16), ("g5", 3)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_drafted_tokens(heads, most, page, window, sinks):
    """Up to 16 (row, query head) columns a kv head, 32 at head dim 64, whole blocks and blocks in pieces."""
    rng = np.random.default_rng(51)
    lens = [most, most + 1, 40, 65, 300, 2500]
    b = Batch(rng, *HEADS[heads], page, lens, [most, 1, most, most, 2, most], head_major=page == 64)
    ctx = _ctx(*HEADS[heads])
    o = b.device().attend(ctx, window, sinks)
    _check(b, o, window, sinks)
    ctx.close()
