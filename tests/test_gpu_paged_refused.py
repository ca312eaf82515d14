"""A grow that is refused and not waited for: the append behind it must not take the last places of the unchanged length, which hold
other tokens, of a page that other answers may hold too."""
import numpy as np
import pytest
import torch

import paper_2510_10129_amd as cc
from paper_2510_10129_amd import _lib

from _gpu_util import DEV, dev_bf16, dev_i32, host_bits
from test_gpu_paged import _bf16, _ctx

pytestmark = pytest.mark.gpu
H_Q, H_KV, D_H, PAGE = 8, 2, 64, 16


def _make(rng, n_pages, n_seqs, max_pages=8):
    pool = cc.PagePool.empty(n_pages, PAGE, n_seqs, max_pages, device=DEV)
    shape = (n_pages, PAGE, H_KV, D_H)
    return pool, cc.PagedKV(dev_bf16(_bf16(rng, shape)), dev_bf16(_bf16(rng, shape)))


def _rows(rng, seqs, more):
    start = np.r_[0, np.cumsum(more)]
    x = dev_bf16(_bf16(rng, (int(start[-1]), (H_Q + 2 * H_KV) * D_H)))
    parts = x.split((H_Q * D_H, H_KV * D_H, H_KV * D_H), dim=1)
    return cc.NewRows(dev_i32(start), dev_i32(seqs), int(start[-1]), max(more)), parts


def _bits(pool, kv):
    return [host_bits(kv.K), host_bits(kv.V), pool.refs.tolist(), pool.table.tolist(), pool.len.tolist()]


def _same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


RULE = cc.Rope(1e4, 64)


@pytest.mark.parametrize("seqs,more,status", [([1, 2, 3], [1, 1, 1], _lib.CC_ERR_WORKSPACE), ([1, 2], [5, 200], _lib.CC_ERR_SHAPE),
                                              ([1, 2, 1], [1, 2, 1], _lib.CC_ERR_IDX), ([2, 9], [1, 1], _lib.CC_ERR_IDX)])
def test_a_refused_grow_costs_no_tokens(seqs, more, status):
    """Answers of one context whose last page they share; too few pages, too long, a repeated index, an index that is none."""
    rng = np.random.default_rng(60)
    pool, kv = _make(rng, 4, 4)
    ctx = _ctx(H_Q, H_KV, D_H)
    ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([PAGE + 5]))            # two pages, two are left
    ctx.fork_pages(pool, dev_i32([0, 0, 0]), dev_i32([1, 2, 3]))
    before = _bits(pool, kv)
    ctx.grow_pages(pool, [kv], dev_i32(seqs), dev_i32(more), sync=False)
    assert pool.status.item() == status
    mine = [(s, n) for s, n in dict(zip(seqs, more)).items() if s < 4]
    new, parts = _rows(rng, [s for s, _ in mine], [min(n, 20) for _, n in mine])
    out = torch.full((new.rows, H_Q * D_H), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.step_rope_append(*parts, new, pool, kv, RULE, out)
    assert _same(_bits(pool, kv), before) and bool((out == 7.0).all())
    with pytest.raises(cc.CacheClipError) as e:
        ctx.step_rope_append(*parts, new, pool, kv, RULE, out, flags=_lib.FLAG_CHECK_IDX)
    assert e.value.status == _lib.CC_ERR_IDX
    # the refusal outlives other calls; sequences that were not asked about are as before
    ctx.compact_pages(pool, [kv]), ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([0]))
    assert pool.status.item() == 0
    assert pool.refused.tolist() == [status if s in [m[0] for m in mine] else 0 for s in range(4)]
    ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([1]))
    other, parts0 = _rows(rng, [0], [1])
    got = torch.full((1, H_Q * D_H), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.step_rope_append(*parts0, other, pool, kv, RULE, got, flags=_lib.FLAG_CHECK_IDX)
    page = pool.table[0, 1].item()
    assert np.array_equal(host_bits(kv.V[page, 5]), host_bits(parts0[2]).reshape(H_KV, D_H)) and not bool((got == 7.0).all())
    # a grow that is made, or freeing, ends it
    ctx.free_pages(pool, dev_i32([3]))
    ctx.grow_pages(pool, [kv], dev_i32([1]), dev_i32([1]))
    assert pool.refused.tolist() == [0, 0, status if any(m[0] == 2 for m in mine) else 0, 0]
    one, parts1 = _rows(rng, [1], [1])
    ctx.step_rope_append(*parts1, one, pool, kv, RULE, got, flags=_lib.FLAG_CHECK_IDX)
    page = pool.table[1, 1].item()
    assert np.array_equal(host_bits(kv.V[page, 5]), host_bits(parts1[2]).reshape(H_KV, D_H))
    pool.refused.zero_()                                                     # so does the caller
    ctx.step_rope_append(*_rows(rng, [2], [1])[1], _rows(rng, [2], [1])[0], pool, kv, RULE, got, flags=_lib.FLAG_CHECK_IDX)
    ctx.close()


def test_an_entry_without_tokens_asks_for_nothing():
    """Of a refused list, an entry of no tokens is not refused anything, and a made grow of none clears nothing."""
    rng = np.random.default_rng(61)
    pool, kv = _make(rng, 2, 3)
    ctx = _ctx(H_Q, H_KV, D_H)
    ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([3]))
    ctx.grow_pages(pool, [kv], dev_i32([0, 1, 2]), dev_i32([0, 50, -1]), sync=False)
    assert pool.refused.tolist() == [0, _lib.CC_ERR_IDX, _lib.CC_ERR_IDX]
    ctx.grow_pages(pool, [kv], dev_i32([1, 0]), dev_i32([0, 1]), sync=False)
    assert pool.status.item() == 0 and pool.refused.tolist() == [0, _lib.CC_ERR_IDX, _lib.CC_ERR_IDX]
    with pytest.raises(cc.CacheClipError):
        ctx.grow_pages(pool, [kv], dev_i32([0]), dev_i32([200]))             # also where it is waited for
    assert pool.refused.tolist() == [_lib.CC_ERR_SHAPE, _lib.CC_ERR_IDX, _lib.CC_ERR_IDX]
    ctx.free_pages(pool, dev_i32([2, 0, 1]))
    assert not pool.refused.any()
    ctx.close()


def test_a_captured_loop_that_runs_out_of_pages():
    """Eight answers of one context, each a token a replay, recorded once: the steps that there are pages for are made, the others
    leave every key and value as it is, and after answers were freed the loop goes on."""
    rng = np.random.default_rng(62)
    n, first = 8, 2 * PAGE + 3
    pool, kv = _make(rng, 14, n + 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx = _ctx(H_Q, H_KV, D_H, stream=side.cuda_stream)
    ctx.grow_pages(pool, [kv], dev_i32([n]), dev_i32([first]))
    ctx.fork_pages(pool, dev_i32([n] * n), dev_i32(range(n)))                # 3 pages shared, 11 free: a copy each, and 3 over
    new, parts = _rows(rng, range(n), [1] * n)
    more, seq, q = dev_i32([1] * n), dev_i32(range(n)), torch.zeros((n, H_Q * D_H), dtype=torch.bfloat16, device=DEV)
    o = torch.zeros_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.grow_pages(pool, [kv], seq, more, sync=False)
        ctx.step_rope_append(*parts, new, pool, kv, RULE, q)
        ctx.step_paged_attention(q, new, pool, kv, o)
    room = PAGE - 3                                                          # tokens until every answer needs a page more
    for i in range(room + 4):
        before = _bits(pool, kv)
        g.replay()
        torch.cuda.synchronize()
        if i < room:
            assert pool.len[:n].tolist() == [first + i + 1] * n and not pool.refused.any()
            for s in range(n):
                p = first + i
                assert np.array_equal(host_bits(kv.V[pool.table[s, p // PAGE].item(), p % PAGE]), host_bits(parts[2][s]).reshape(H_KV, D_H))
        else:
            assert _same(_bits(pool, kv), before)
            ctx.free_pages(pool, dev_i32([]))                                # a later call's status is its own
            torch.cuda.synchronize()
            assert pool.status.item() == 0 and pool.refused.tolist() == [_lib.CC_ERR_WORKSPACE] * n + [0]
        (o.float() @ o.float().t()).sum().item()                             # the program's own work between replays
    torch.cuda.synchronize()
    kept = _bits(pool, kv)[4]
    ctx.free_pages(pool, dev_i32([3, 4, 5, 6, 7]))
    torch.cuda.synchronize()
    rest, parts = _rows(rng, range(3), [1] * 3)
    ctx.grow_pages(pool, [kv], dev_i32(range(3)), dev_i32([1] * 3), sync=False)
    ctx.step_rope_append(*parts, rest, pool, kv, RULE, q[:3])
    torch.cuda.synchronize()
    assert not pool.refused.any() and pool.len[:3].tolist() == [x + 1 for x in kept[:3]]
    for s in range(3):
        assert np.array_equal(host_bits(kv.V[pool.table[s, kept[s] // PAGE].item(), kept[s] % PAGE]), host_bits(parts[2][s]).reshape(H_KV, D_H))
    ctx.close()


def test_a_sequence_with_two_sets_of_rows_is_reported():
    """Its last places would be written by both: the index check of the append refuses it; a second entry without rows is none."""
    rng = np.random.default_rng(63)
    pool, kv = _make(rng, 80, 70)
    ctx = _ctx(H_Q, H_KV, D_H)
    ctx.grow_pages(pool, [kv], dev_i32(range(70)), dev_i32([9] * 70))
    before = _bits(pool, kv)
    for seqs, more, ok in (([4, 5, 4], [1, 1, 1], False), ([4, 5, 4], [1, 1, 0], True), ([4, 5, 4], [0, 1, 2], True),
                           (list(range(70)) + [0], [1] * 71, False), (list(range(69)) + [68], [1] * 70, False), (list(range(70)), [1] * 70, True)):
        new, parts = _rows(rng, seqs, more)
        out = torch.full((new.rows, H_Q * D_H), 7.0, dtype=torch.bfloat16, device=DEV)
        if ok:
            ctx.step_rope_append(*parts, new, pool, kv, RULE, out, flags=_lib.FLAG_CHECK_IDX)
            before = _bits(pool, kv)
            continue
        with pytest.raises(cc.CacheClipError) as e:
            ctx.step_rope_append(*parts, new, pool, kv, RULE, out, flags=_lib.FLAG_CHECK_IDX)
        assert e.value.status == _lib.CC_ERR_IDX and _same(_bits(pool, kv), before) and bool((out == 7.0).all())
        ctx.step_paged_attention(out, new, pool, kv, torch.empty_like(out), flags=_lib.FLAG_CHECK_IDX)      # may look twice
    ctx.close()


def test_a_new_pool_is_ready_for_every_stream():
    """The words of a new pool lie in memory that held other numbers, and torch's stream is busy: a context on a stream of its own does
    not wait for it."""
    rng = np.random.default_rng(64)
    made, kv = _make(rng, 8, 3)
    side = torch.cuda.Stream()
    ctx = _ctx(H_Q, H_KV, D_H, stream=side.cuda_stream)
    new, parts = _rows(rng, [0, 1, 2], [4, 1, 20])
    q = torch.zeros((25, H_Q * D_H), dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    ctx.grow_pages(made, [kv], dev_i32([0, 1, 2]), dev_i32([4, 1, 20]))
    x = torch.randn((4096, 4096), device=DEV)
    old = [torch.full((3,), -4, dtype=torch.int32, device=DEV) for _ in range(200)]
    torch.cuda.synchronize()
    del old
    for _ in range(20):
        y = x @ x                                           # some milliseconds
    pool = cc.PagePool(made.refs, made.table, made.len, PAGE, status=made.status, work=made.work)
    ctx.step_rope_append(*parts, new, pool, kv, RULE, q)
    torch.cuda.synchronize()
    del y
    assert pool.status.item() == 0 and not pool.refused.any() and bool(q.any(dim=1).all())
    for s, (r0, n) in enumerate(((0, 4), (4, 1), (5, 20))):
        pages, pos = pool.table[s].cpu().numpy(), np.arange(n)
        assert np.array_equal(host_bits(kv.V)[pages[pos // PAGE], pos % PAGE], host_bits(parts[2][r0:r0 + n]).reshape(n, H_KV, D_H))
    ctx.close()
