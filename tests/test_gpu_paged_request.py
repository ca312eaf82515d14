"""A request from its selection to its answers: the cache that a recomputed layer leaves becomes pages as it lies, answers fork from it
and grow; rows of the answers against the plain definitions (fp64).

Bounds: the rotation rounds once, 2^-8 of the result, and 2^-19 of the pair in 32 bits; attention rounds its result, 2^-8 of itself, and
probabilities lose 2^-8 of themselves at most, with 2^-10 for the sums in 32 bits."""
import numpy as np
import pytest
import torch

import paper_2510_10129_amd as cc
from oracle import fixture, paged
from oracle import select as osel
from paper_2510_10129_amd import _lib
from workloads import CONFIGS, gen

from _gpu_util import DEV, bits_f64, dev_bf16, dev_i32, dev_weights, host_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 64])
def test_answers_from_the_cache_of_a_recomputed_layer(page):
    wl = CONFIGS["C1"]
    m = wl.model
    w = gen.layer_weights(m, 0, wl.seed)
    xl, xg = gen.hidden_pair(wl)
    Ks, Vs = fixture.stale_cache_one_layer(xl, w, m)
    Ks[wl.P + wl.T:], Vs[wl.P + wl.T:] = 0, 0
    N, used = wl.N, -(-wl.N // page)
    n_pages = used + 12

    # the prompt: selection and one layer over a cache with room for pages behind it
    K, V = (torch.zeros((n_pages * page, m.H_kv, m.d_h), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    K[:N], V[:N] = dev_bf16(Ks), dev_bf16(Vs)
    ctx = cc.Context.for_model(m, N_cap=N, M_cap=N, T_cap=wl.T)
    A = gen.aux_attention(wl)
    idx, M = ctx.select(torch.from_numpy(A).to(DEV), wl.recomp_bp[0], wl.window, wl.tau, 0, wl.P, wl.Q)
    assert np.array_equal(idx[:M].cpu().numpy(), osel.select(A, wl.recomp_bp[0], wl.window, wl.tau, True, wl.P, wl.Q))
    out = torch.empty((M, m.d), dtype=torch.bfloat16, device=DEV)
    ctx.recompute_layer(dev_bf16(xg), idx, cc.KVLayer(K[:N], V[:N]), idx, M, dev_weights(w), out, _lib.FLAG_CHECK_IDX)

    # its pages are the lowest of a new pool; three answers share them and copy the last one where it is not full
    kv = cc.PagedKV(K.view(n_pages, page, m.H_kv, m.d_h), V.view(n_pages, page, m.H_kv, m.d_h))
    pool, P = cc.PagePool.empty(n_pages, page, 4, used + 3, device=DEV), paged.Pages(n_pages, page, 4, used + 3)
    P.grow([0], [N]), ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([N]))
    assert pool.table[0, :used].tolist() == list(range(used))
    prompt = [host_bits(K[:N]), host_bits(V[:N])]
    assert not np.array_equal(prompt[0], Ks)
    P.fork([0, 0, 0], [1, 2, 3]), ctx.fork_pages(pool, dev_i32([0, 0, 0]), dev_i32([1, 2, 3]))

    rng = np.random.default_rng(70)
    rule, freq = cc.Rope(m.rope_base, m.d_h), paged.frequencies(m.rope_base, m.d_h)
    nq, heads = m.H_q * m.d_h, m.H_q + 2 * m.H_kv
    want = [bits_f64(host_bits(kv.K)), bits_f64(host_bits(kv.V))]
    for seqs, more in (([1, 2, 3], [1, 1, 1]), ([3, 1], [30, 4]), ([2, 1, 3], [1, 1, 1])):
        P.grow(seqs, more), ctx.grow_pages(pool, [kv], dev_i32(seqs), dev_i32(more), sync=False)
        for old, new_page, n in P.copies:
            for x in want:
                x[new_page, :n] = x[old, :n]
        start, rows = np.r_[0, np.cumsum(more)], sum(more)
        x = rng.standard_normal((rows, m.d)).astype(np.float32)
        qkv = gen.f32_to_bf16_bits((x @ bits_f64(w["w_qkv"]).T).astype(np.float32))         # the caller's product
        q, k, v = dev_bf16(qkv).split((nq, m.H_kv * m.d_h, m.H_kv * m.d_h), dim=1)
        new, turned, o = cc.NewRows(dev_i32(start), dev_i32(seqs), rows, max(more)), *(torch.empty((rows, nq), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ctx.step_rope_append(q, k, v, new, pool, kv, rule, turned, flags=_lib.FLAG_CHECK_IDX)
        ctx.step_paged_attention(turned, new, pool, kv, o, flags=_lib.FLAG_CHECK_IDX)
        assert pool.status.item() == 0 and not pool.refused.any()
        gK, gV = bits_f64(host_bits(kv.K)), bits_f64(host_bits(kv.V))
        for i, s in enumerate(seqs):
            pos = np.arange(P.len[s] - more[i], P.len[s])
            at = np.array(P.table[s])[pos // page], pos % page
            rest = bits_f64(qkv[start[i]:start[i + 1]]).reshape(more[i], heads, m.d_h)
            kt = paged.turn(rest[:, m.H_q:m.H_q + m.H_kv], pos, freq, False)
            pair = np.abs(rest[:, m.H_q:m.H_q + m.H_kv])
            pair = np.tile(pair[..., :m.d_h // 2] + pair[..., m.d_h // 2:], 2)
            assert np.all(np.abs(gK[at] - kt) <= 2.0 ** -8 * np.abs(kt) + 2.0 ** -19 * pair)
            assert np.array_equal(gV[at], rest[:, m.H_q + m.H_kv:])
            want[0][at], want[1][at] = gK[at], gV[at]
            tq = bits_f64(host_bits(turned[start[i]:start[i + 1]])).reshape(more[i], m.H_q, m.d_h)
            ref, mag = paged.attention(tq, want[0], want[1], P.table[s], P.len[s], more[i], 0, 0)
            got = bits_f64(host_bits(o[start[i]:start[i + 1]])).reshape(ref.shape)
            tol = (2.0 ** -8 + 2.0 ** -10) * (1 + 2.0 ** -8) * mag + 2.0 ** -8 * np.abs(ref)
            assert np.all(np.abs(got - ref) <= tol), (seqs, s, float((np.abs(got - ref) / tol).max()))
        assert np.array_equal(gK, want[0]) and np.array_equal(gV, want[1])                  # nothing else was written
    assert np.array_equal(host_bits(K[:N]), prompt[0]) and np.array_equal(host_bits(V[:N]), prompt[1])
    ctx.free_pages(pool, dev_i32([3, 1, 2]))
    P.free([3, 1, 2])
    assert pool.refs.tolist() == P.refs and pool.len.tolist() == [N, 0, 0, 0]
    ctx.close()
