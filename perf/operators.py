"""The operators of the paged cache: plain form, calls and sizes that are measured.

After a request's cache has been recomputed a server answers from it: sequences grow by single
tokens or by chunks (a follow-up question), several answers fork from one context, finished ones
are freed, and the pool is compacted.  A case is one of these calls at one size: `attend` (new rows
over a paged cache, optionally a sliding window with sinks), `rope` (rotary positions of new rows
and their keys and values into pages), `fork` (answers forked from contexts, each grown by a few tokens) and
`compact`.  Head layouts are those of the layers in `cases.py`.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"

#        H_q, H_kv, d_h, rope_base
HEADS = {
    "d256": (4, 2, 64, 1.0e4),
    "d2048": (32, 8, 64, 5.0e5),
    "d3584": (28, 4, 128, 1.0e6),
    "d4096": (32, 8, 128, 5.0e5),
    "d8192": (64, 8, 128, 5.0e5),
}


def listed():
    return [
        # the smallest model's first answer token after a 1k request: latency is all there is
        dict(name="decode_1k", kind="attend", heads="d256", page=16, batch=1, ctx=1073, new=1, ragged=False, window=0,
             sinks=0, head_major=False),
        # a server's decode step: one token each of 32 sequences of ragged lengths
        dict(name="decode_16k_batch", kind="attend", heads="d4096", page=16, batch=32, ctx=16577, new=1, ragged=True,
             window=0, sinks=0, head_major=False),
        # few long contexts: the keys of one sequence spread over the chip
        dict(name="decode_64k", kind="attend", heads="d8192", page=64, batch=4, ctx=65857, new=1, ragged=False, window=0,
             sinks=0, head_major=True),
        # decode under a sliding window with sinks, groups of seven query heads
        dict(name="decode_window_29k", kind="attend", heads="d3584", page=32, batch=64, ctx=28865, new=1, ragged=True,
             window=4096, sinks=4, head_major=False),
        # a few drafted tokens a sequence, verified in one pass
        dict(name="verify_16k", kind="attend", heads="d4096", page=16, batch=16, ctx=16581, new=5, ragged=True, window=0,
             sinks=0, head_major=False),
        # a batch of ragged follow-up chunks at short context, head dim 64
        dict(name="chunk_4k", kind="attend", heads="d2048", page=16, batch=6, ctx=4224, new=512, ragged=True, window=0,
             sinks=0, head_major=False),
        # two chunks under a window with sinks
        dict(name="chunk_window_29k", kind="attend", heads="d3584", page=32, batch=2, ctx=28865, new=1024, ragged=False,
             window=4096, sinks=64, head_major=True),
        # one chunk over a 64k context: the largest call
        dict(name="chunk_64k", kind="attend", heads="d8192", page=64, batch=1, ctx=66560, new=1024, ragged=False, window=0,
             sinks=0, head_major=False),
        # the rotary step of a decode batch
        dict(name="rope_decode", kind="rope", heads="d4096", page=16, batch=32, ctx=16577, new=1, ragged=True, rot=128,
             interleaved=False, scaling="plain", packed=True),
        # the rotary step of one long chunk: interleaved pairs, half of the head, a context stretched eightfold
        dict(name="rope_chunk", kind="rope", heads="d8192", page=64, batch=1, ctx=66560, new=4096, ragged=False, rot=64,
             interleaved=True, scaling="index", packed=True),
        # eight answers from each of four contexts, every one grown by three tokens: 28 layers
        dict(name="fork_8_of_4", kind="fork", heads="d3584", page=16, layers=28, contexts=4, answers=8, ctx=6553, grow=3),
        # a pool of 32 layers, two fifths of its pages freed here and there
        dict(name="compact_16k", kind="compact", heads="d4096", page=16, layers=32, seqs=12, ctx=1400, free=40),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """A call of the same kinds: contexts of one to 66k tokens, batches up to 64, one to 2048 new rows."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        kind = rng.choices(("attend", "rope", "fork", "compact"), (6, 2, 1, 1))[0]
        c = dict(kind=kind, heads=rng.choice(sorted(HEADS)), page=rng.choice((16, 32, 64, 128)))
        if kind in ("attend", "rope"):
            ctx = _log_int(rng, 1, 66560)
            new = rng.choice((1, 1, rng.randint(1, 8), _log_int(rng, 1, 2048)))
            c.update(batch=_log_int(rng, 1, 64), ctx=max(ctx, new), new=new, ragged=rng.random() < 0.6)
        if kind == "attend":
            window = rng.choice((0, 0, _log_int(rng, 1, 8192)))
            c.update(window=window, sinks=rng.choice((0, rng.randint(1, 80))) if window else 0, head_major=rng.random() < 0.4)
        elif kind == "rope":
            d_h = HEADS[c["heads"]][2]
            c.update(rot=rng.choice((d_h, d_h, d_h // 2, 2 * rng.randint(1, d_h // 2))), interleaved=rng.random() < 0.5,
                     scaling=rng.choice(("plain", "linear", "turns", "index")), packed=rng.random() < 0.5)
        elif kind == "fork":
            c.update(layers=rng.randint(1, 32), contexts=rng.randint(1, 8), answers=rng.randint(1, 8),
                     ctx=_log_int(rng, 1, 8192), grow=_log_int(rng, 1, 200))
        else:
            c.update(layers=rng.randint(1, 32), seqs=rng.randint(1, 24), ctx=_log_int(rng, 16, 4096), free=rng.randint(5, 80))
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and _pool_bytes(c) < 4e9:
            return c


# ---- sizes ----

def _lens(c):
    """Tokens and new rows of every sequence of a batch."""
    n, L, new = c["batch"], c["ctx"], c["new"]
    if not c["ragged"]:
        return [L] * n, [new] * n
    r = random.Random(n * 100003 + L)
    news = [new if i == 0 else r.randint(max(1, new // 2), new) for i in range(n)]
    return [max(k, r.randint(max(1, L // 3), L)) for k in news], news


def _holds(c):
    """Tokens of every sequence that the pool holds pages for."""
    if c["kind"] in ("attend", "rope"):
        return _lens(c)[0]
    if c["kind"] == "fork":
        r = random.Random(c["contexts"] * 100003 + c["ctx"])
        return [r.randint(max(1, c["ctx"] // 2), c["ctx"]) for _ in range(c["contexts"])]
    r = random.Random(c["seqs"] * 100003 + c["ctx"])
    return [r.randint(max(1, c["ctx"] // 2), c["ctx"]) for _ in range(c["seqs"])]


def _pages(c, tokens):
    return -(-tokens // c["page"])


def _n_pages(c):
    held = sum(_pages(c, t) for t in _holds(c))
    if c["kind"] == "fork":
        return held + c["contexts"] * (c["answers"] + 1) * (_pages(c, c["grow"]) + 2)
    if c["kind"] == "compact":
        return held * 100 // (100 - c["free"]) + 1
    return held + held // 8 + 1


def _row_bytes(c):
    _, h_kv, d_h, _ = HEADS[c["heads"]]
    return h_kv * d_h * 2


def _pool_bytes(c):
    return 2 * c.get("layers", 1) * _n_pages(c) * c["page"] * _row_bytes(c)


def _seen(p, window, sinks):
    """Keys that a row at position p sees."""
    if window == 0 or p < window:
        return p + 1
    return window + min(sinks, p - window + 1)


def _moves(c):
    """Pages that a compaction moves: the live ones behind the first `live` pages."""
    held = sum(_pages(c, t) for t in _holds(c))
    order = _page_order(c)[:held]
    return sum(1 for p in order if p >= held)


def _page_order(c):
    """The pages in the order in which the pool's sequences took them: a pool that has served for a while."""
    order = list(range(_n_pages(c)))
    random.Random(c["page"] * 7919 + len(order)).shuffle(order)
    return order


def work(case):
    c = case
    h_q, h_kv, d_h, _ = HEADS[c["heads"]]
    row = _row_bytes(c)
    if c["kind"] == "attend":
        keys, flops, q_rows = 0, 0, 0
        for L, n in zip(*_lens(c)):
            first = L - n
            low = max(0, first - c["window"] + 1) if c["window"] else 0
            keys += L - low + min(low, c["sinks"])
            q_rows += n
            flops += sum(_seen(p, c["window"], c["sinks"]) for p in range(first, L))
        return {"bytes": 2 * row * keys + 2 * 2 * h_q * d_h * q_rows, "flops": 4 * d_h * h_q * flops}
    if c["kind"] == "rope":
        q_rows = sum(_lens(c)[1])
        return {"bytes": 2 * q_rows * (2 * row + 2 * h_q * d_h), "flops": 3 * q_rows * (h_q + h_kv) * c["rot"]}
    held = _holds(c)
    if c["kind"] == "fork":
        part = sum(t % c["page"] for t in held) * (c["answers"] + 1)
        entries = sum(_pages(c, t) for t in held) * (c["answers"] + 1)
        return {"bytes": 2 * 2 * c["layers"] * row * part + 8 * entries + 4 * _n_pages(c), "flops": entries}
    return {"bytes": 2 * 2 * c["layers"] * c["page"] * row * _moves(c) + 8 * _n_pages(c), "flops": _n_pages(c)}


# ---- inputs ----

class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=self.g)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c, r = dict(case), _Draw(seed)
    h_q, h_kv, d_h, base = HEADS[c["heads"]]
    page, n_pages, held = c["page"], _n_pages(c), _holds(c)
    s = {"c": c}

    # the pool: every sequence's pages lie where earlier ones left room
    order = _page_order(c)
    if c["kind"] in ("attend", "rope", "fork"):
        random.Random(seed).shuffle(order)
    children = c["contexts"] * c["answers"] if c["kind"] == "fork" else 0
    most = max(_pages(c, t + c.get("grow", 0)) for t in held)
    refs, table, at = [0] * n_pages, [], 0
    for t in held + [0] * children:
        mine = order[at:at + _pages(c, t)]
        at += len(mine)
        for p in mine:
            refs[p] += 1
        table.append(mine + [-1] * (most - len(mine)))
    s["refs"], s["table"], s["len"] = _i32(refs), _i32(table), _i32(held + [0] * children)
    s["status"] = _i32([0])

    # keys and values of all layers; tokens or heads outermost in a page
    shape = (c.get("layers", 1), n_pages) + ((h_kv, page, d_h) if c.get("head_major") else (page, h_kv, d_h))
    s["K"], s["V"] = r.normal(shape, 0.6), r.normal(shape, 0.6)
    kvs = s["kvs"] = [(K.transpose(1, 2), V.transpose(1, 2)) if c.get("head_major") else (K, V) for K, V in zip(s["K"], s["V"])]

    if c["kind"] in ("attend", "rope"):
        news = _lens(c)[1]
        start = [0]
        for n in news:
            start.append(start[-1] + n)
        s["start"], s["rows"] = _i32(start), start[-1]
        s["host_start"], s["host_len"] = start, held
    if c["kind"] == "attend":
        s["q"] = r.normal((s["rows"], h_q * d_h), 2.5)
        s["o"] = torch.zeros_like(s["q"])
    elif c["kind"] == "rope":
        qkv = r.normal((s["rows"], (h_q + 2 * h_kv) * d_h))
        parts = qkv.split((h_q * d_h, h_kv * d_h, h_kv * d_h), dim=1)
        s["q"], s["k"], s["v"] = parts if c["packed"] else [p.contiguous() for p in parts]
        s["q_out"] = torch.zeros((s["rows"], h_q * d_h), dtype=torch.bfloat16, device=DEV)
        s["rope"] = dict(base=base, rot=c["rot"], interleaved=c["interleaved"], scaling=c["scaling"],
                         factor=1.0 if c["scaling"] == "plain" else 8.0, orig_len=8192, low=1.0, high=32.0,
                         mscale=0.1 * math.log(8.0) + 1.0 if c["scaling"] == "index" else 1.0)
    elif c["kind"] == "fork":
        n, a = c["contexts"], c["answers"]
        s["src"], s["dst"] = _i32([i for i in range(n) for _ in range(a)]), _i32(list(range(n, n + n * a)))
        s["all"] = _i32(list(range(n + n * a)))
        s["more"] = torch.full((n + n * a,), c["grow"], dtype=torch.int32, device=DEV)
        s["refs0"], s["table0"], s["len0"] = s["refs"].clone(), s["table"].clone(), s["len"].clone()
    else:
        s["refs0"], s["table0"] = s["refs"].clone(), s["table"].clone()

    if own:
        import paper_2510_10129_amd as cc
        s["ctx"] = cc.Context(64, h_q, h_kv, d_h, 64, base, 1e-5, N_cap=64, M_cap=64, T_cap=64)
        s["pool"] = cc.PagePool(s["refs"], s["table"], s["len"], page, status=s["status"])
        s["paged"] = [cc.PagedKV(K, V) for K, V in kvs]
        if "start" in s:
            s["new"] = cc.NewRows(s["start"], None, s["rows"], max(news))
        if "rope" in s:
            s["rule"] = cc.Rope(**s["rope"])
    return s


# ---- plain form ----

def _plain_attend(s):
    c = s["c"]
    h_q, h_kv, d_h, _ = HEADS[c["heads"]]
    g, page, (K, V) = h_q // h_kv, c["page"], s["kvs"][0]
    for b, L in enumerate(s["host_len"]):
        r0, r1 = s["host_start"][b], s["host_start"][b + 1]
        first = L - (r1 - r0)
        low = max(0, first - c["window"] + 1) if c["window"] else 0
        j = torch.arange(L, device=DEV)
        j = j[(j >= low) | (j < c["sinks"])]
        at = s["table"][b].long()[j // page], j % page
        k = K[at].float().permute(1, 2, 0).contiguous()                         # [H_kv, d_h, keys]
        v = V[at].float().permute(1, 0, 2).contiguous()                         # [H_kv, keys, d_h]
        step = max(1, int(2.5e8 // (h_q * j.numel())))
        for i0 in range(r0, r1, step):
            i1 = min(r1, i0 + step)
            p = first + torch.arange(i0 - r0, i1 - r0, device=DEV)
            hide = j[None, :] > p[:, None]
            if c["window"]:
                hide = hide | ((j[None, :] <= p[:, None] - c["window"]) & (j[None, :] >= c["sinks"]))
            q = s["q"][i0:i1].float().view(i1 - i0, h_kv, g, d_h).permute(1, 0, 2, 3).reshape(h_kv, -1, d_h)
            z = (torch.matmul(q, k) / math.sqrt(d_h)).view(h_kv, i1 - i0, g, -1)
            z = z.masked_fill(hide[None, :, None, :], float("-inf"))
            e = torch.exp(z - z.amax(dim=-1, keepdim=True))
            w = (e / e.sum(dim=-1, keepdim=True)).view(h_kv, (i1 - i0) * g, -1)
            o = torch.matmul(w, v).view(h_kv, i1 - i0, g, d_h).permute(1, 0, 2, 3)
            s["o"][i0:i1] = o.reshape(i1 - i0, h_q * d_h).to(torch.bfloat16)
    return s["o"]


def _plain_angles(rule, pos):
    """cos and sin [rows, rot / 2] in 32 bits, from angles in 64."""
    j = torch.arange(rule["rot"] // 2, device=DEV, dtype=torch.float64)
    inv = rule["base"] ** (-2.0 * j / rule["rot"])
    f, kind = rule["factor"], rule["scaling"]
    if kind == "linear":
        inv = inv / f
    elif kind == "turns":
        keep = ((rule["orig_len"] * inv / (2 * math.pi) - rule["low"]) / (rule["high"] - rule["low"])).clamp(0, 1)
        inv = inv * ((1 - keep) / f + keep)
    elif kind == "index":
        def index_of(turns):
            return rule["rot"] * math.log(rule["orig_len"] / (turns * 2 * math.pi)) / (2 * math.log(rule["base"]))
        lo, hi = max(math.floor(index_of(rule["high"])), 0), min(math.ceil(index_of(rule["low"])), rule["rot"] - 1)
        keep = 1 - ((j - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        inv = inv * ((1 - keep) / f + keep)
    a = pos.double()[:, None] * inv
    return (torch.cos(a) * rule["mscale"]).float(), (torch.sin(a) * rule["mscale"]).float()


def _plain_turn(x, cos, sin, rot, interleaved):
    """x [rows, heads, d_h] in 32 bits."""
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    c, s = cos[:, None, :], sin[:, None, :]
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    return y


def _plain_rope(s):
    c = s["c"]
    h_q, h_kv, d_h, _ = HEADS[c["heads"]]
    n, rows = s["start"].numel() - 1, torch.arange(s["rows"], device=DEV)
    b = torch.searchsorted(s["start"].long(), rows, right=True) - 1
    count = (s["start"][1:] - s["start"][:n]).long()
    pos = s["len"].long()[b] - count[b] + rows - s["start"].long()[b]
    cos, sin = _plain_angles(s["rope"], pos)
    turn = lambda x, h: _plain_turn(x.float().view(-1, h, d_h), cos, sin, c["rot"], c["interleaved"]).to(torch.bfloat16)
    s["q_out"].copy_(turn(s["q"], h_q).view(s["rows"], -1))
    K, V = s["kvs"][0]
    at = s["table"].long()[b, pos // c["page"]], pos % c["page"]
    K[at] = turn(s["k"], h_kv)
    V[at] = s["v"].view(-1, h_kv, d_h)
    return s["q_out"], K, V


def _plain_count(refs, pages, by):
    refs.index_add_(0, pages.long(), torch.full_like(pages, by))


def _plain_free(s, seqs):
    rows = s["table"][seqs.long()]
    _plain_count(s["refs"], rows[rows >= 0], -1)
    s["table"][seqs.long()] = -1
    s["len"][seqs.long()] = 0


def _plain_fork(s):
    c, page = s["c"], s["c"]["page"]
    _plain_free(s, s["dst"])
    rows = s["table"][s["src"].long()]
    s["table"][s["dst"].long()] = rows
    s["len"][s["dst"].long()] = s["len"][s["src"].long()]
    _plain_count(s["refs"], rows[rows >= 0], 1)
    # grow: the lowest free pages in the list's order, a shared last page is copied first
    seqs, more = s["all"].long(), s["more"].long()
    n = s["len"].long()[seqs]
    have, need = (n + page - 1) // page, (n + more + page - 1) // page
    tail = s["table"][seqs, (have - 1).clamp(min=0)].long()
    copies = (more > 0) & (n % page != 0) & (s["refs"][tail.clamp(min=0)] > 1)
    take = need - have + copies
    first = torch.cumsum(take, 0) - take
    free = torch.nonzero(s["refs"] == 0)[:, 0]
    if int(take.sum()) > free.numel():
        s["status"].fill_(-4)
        return
    new = free[first.clamp(max=max(free.numel() - 1, 0))]
    for i in torch.nonzero(copies)[:, 0].tolist():
        k = int(n[i]) % page
        for K, V in s["kvs"]:
            K[new[i], :k], V[new[i], :k] = K[tail[i], :k], V[tail[i], :k]
    _plain_count(s["refs"], tail[copies].int(), -1)
    s["table"][seqs[copies], have[copies] - 1] = new[copies].int()
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    fresh = (col >= have[:, None]) & (col < need[:, None])
    at = (first + copies)[:, None] + col - have[:, None]
    rows = s["table"][seqs]
    s["table"][seqs] = torch.where(fresh, free[at.clamp(0, free.numel() - 1)].int(), rows)
    _plain_count(s["refs"], s["table"][seqs][fresh], 1)
    _plain_count(s["refs"], new[copies].int(), 1)
    s["len"][seqs] = (n + more).int()
    s["status"].zero_()


def _plain_compact(s):
    live = s["refs"] > 0
    n = int(live.sum())
    to, frm = torch.nonzero(~live[:n])[:, 0], torch.nonzero(live[n:])[:, 0] + n
    moved = torch.arange(live.numel(), device=DEV)
    moved[frm] = to
    for K, V in s["kvs"]:
        K[to], V[to] = K[frm], V[frm]
    s["refs"][to] = s["refs"][frm]
    s["refs"][frm] = 0
    held = s["table"] >= 0
    s["table"][held] = moved[s["table"][held].long()].int()
    s["status"].zero_()


# ---- one pass ----

def _pool_out(s):
    return s["status"], s["refs"], s["table"], s["len"], s["K"], s["V"]


def run(s):
    c = s["c"]
    if c["kind"] == "attend":
        if not own:
            return _plain_attend(s)
        s["ctx"].step_paged_attention(s["q"], s["new"], s["pool"], s["paged"][0], s["o"], window=c["window"], sinks=c["sinks"])
        return s["o"]
    if c["kind"] == "rope":
        if not own:
            return _plain_rope(s)
        s["ctx"].step_rope_append(s["q"], s["k"], s["v"], s["new"], s["pool"], s["paged"][0], s["rule"], s["q_out"])
        return s["q_out"], *s["kvs"][0]
    if c["kind"] == "fork":
        # the contexts as they were before the last answers
        s["refs"].copy_(s["refs0"]), s["table"].copy_(s["table0"]), s["len"].copy_(s["len0"])
        if own:
            s["ctx"].free_pages(s["pool"], s["dst"], sync=False)
            s["ctx"].fork_pages(s["pool"], s["src"], s["dst"], sync=False)
            s["ctx"].grow_pages(s["pool"], s["paged"], s["all"], s["more"], sync=False)
        else:
            _plain_fork(s)
        return _pool_out(s)
    # the scattered pool again: a compaction reads pages that it does not write
    s["refs"].copy_(s["refs0"]), s["table"].copy_(s["table0"])
    if own:
        s["ctx"].compact_pages(s["pool"], s["paged"], sync=False)
    else:
        _plain_compact(s)
    return _pool_out(s)


# ---- from the definitions, in 64 bits ----

def _exact_attend(s):
    c = s["c"]
    h_q, h_kv, d_h, _ = HEADS[c["heads"]]
    K, V = s["kvs"][0]
    out = torch.empty((s["rows"], h_q, d_h), dtype=torch.float64, device=DEV)
    q = s["q"].double().view(s["rows"], h_q, d_h)
    for b, L in enumerate(s["host_len"]):
        pages = [int(p) for p in s["table"][b, :_pages(c, L)].cpu()]
        r0, r1 = s["host_start"][b], s["host_start"][b + 1]
        for h in range(h_kv):
            keys = torch.cat([K[pages[i:i + 64], :, h].reshape(-1, d_h) for i in range(0, len(pages), 64)])[:L].double()
            vals = torch.cat([V[pages[i:i + 64], :, h].reshape(-1, d_h) for i in range(0, len(pages), 64)])[:L].double()
            for hq in range(h * h_q // h_kv, (h + 1) * h_q // h_kv):
                for i0 in range(r0, r1, 512):
                    i1 = min(r1, i0 + 512)
                    here = torch.arange(L - (r1 - i0), L - (r1 - i1), device=DEV).unsqueeze(1)
                    key = torch.arange(L, device=DEV).unsqueeze(0)
                    sees = key <= here
                    if c["window"] > 0:
                        sees &= (here - key < c["window"]) | (key < c["sinks"])
                    z = torch.mm(q[i0:i1, hq].contiguous(), keys.t().contiguous()).div_(d_h ** 0.5)
                    z[~sees] = -math.inf
                    out[i0:i1, hq] = torch.mm(torch.softmax(z, dim=1), vals)
    return out.view(s["rows"], -1)


def _exact_rope(s):
    c, rule = s["c"], s["rope"]
    h_q, h_kv, d_h, _ = HEADS[c["heads"]]
    rot, base, f = rule["rot"], rule["base"], rule["factor"]
    freq = []
    for j in range(rot // 2):
        w = base ** (-2.0 * j / rot)
        if rule["scaling"] == "linear":
            w /= f
        elif rule["scaling"] == "turns":
            turns = rule["orig_len"] * w / (2 * math.pi)
            part = min(1.0, max(0.0, (turns - rule["low"]) / (rule["high"] - rule["low"])))
            w = (1.0 - part) * w / f + part * w
        elif rule["scaling"] == "index":
            ends = [rot / 2 * math.log(rule["orig_len"] / (2 * math.pi * t), base) for t in (rule["high"], rule["low"])]
            lo, hi = max(0, math.floor(ends[0])), min(rot - 1, math.ceil(ends[1]))
            part = min(1.0, max(0.0, (j - lo) / max(hi - lo, 0.001)))
            w = part * w / f + (1.0 - part) * w
        freq.append(w)
    freq = torch.tensor(freq, dtype=torch.float64, device=DEV)
    at, slot = [], []
    for b, L in enumerate(s["host_len"]):
        n = s["host_start"][b + 1] - s["host_start"][b]
        mine = s["table"][b].cpu().tolist()
        for p in range(L - n, L):
            at.append(p)
            slot.append(mine[p // c["page"]] * c["page"] + p % c["page"])
    wave = torch.polar(torch.full((1, 1), rule["mscale"], dtype=torch.float64, device=DEV),
                       torch.tensor(at, dtype=torch.float64, device=DEV)[:, None] * freq[None, :])[:, None, :]

    def turned(x, h):
        x = x.double().view(-1, h, d_h).clone()
        low = x[..., :rot]
        pair = (low.unflatten(-1, (rot // 2, 2)) if c["interleaved"] else low.unflatten(-1, (2, rot // 2)).transpose(-1, -2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * wave)
        x[..., :rot] = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return x

    K, V = (t.double().flatten(0, 1) for t in s["kvs"][0])
    slot = torch.tensor(slot, device=DEV)
    K[slot], V[slot] = turned(s["k"], h_kv), s["v"].double().view(-1, h_kv, d_h)
    shape = s["kvs"][0][0].shape
    return turned(s["q"], h_q).view(s["rows"], -1), K.view(shape), V.view(shape)


def _exact_fork(s):
    c, page = s["c"], s["c"]["page"]
    refs, table, length = s["refs"].tolist(), s["table"].tolist(), s["len"].tolist()
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        table[b], length[b] = list(table[a]), length[a]
        for p in table[a]:
            if p >= 0:
                refs[p] += 1
    before, copies = list(refs), []
    free = iter([p for p, k in enumerate(before) if k == 0])
    for b, more in zip(s["all"].tolist(), s["more"].tolist()):
        used, part = -(-length[b] // page), length[b] % page
        if more and part and before[table[b][used - 1]] > 1:
            p, old = next(free), table[b][used - 1]
            copies.append((old, p, part))
            refs[old], refs[p], table[b][used - 1] = refs[old] - 1, 1, p
        length[b] += more
        for i in range(used, -(-length[b] // page)):
            table[b][i] = next(free)
            refs[table[b][i]] = 1
    return refs, table, length, copies


def _exact_compact(s):
    refs, table, page = s["refs"].tolist(), s["table"].tolist(), s["c"]["page"]
    n = sum(1 for k in refs if k)
    to = dict(zip([p for p, k in enumerate(refs) if k and p >= n], [p for p, k in enumerate(refs) if not k and p < n]))
    for p, t in to.items():
        refs[t], refs[p] = refs[p], 0
    return refs, [[to.get(p, p) for p in row] for row in table], s["len"].tolist(), [(p, t, page) for p, t in to.items()]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attend":
        if work(case)["flops"] > 6e13:
            return None
        return _exact_attend(s)
    if case["kind"] == "rope":
        return _exact_rope(s)
    refs, table, length, copies = (_exact_fork if case["kind"] == "fork" else _exact_compact)(s)
    if copies:
        frm, to, _ = (torch.tensor(x, device=DEV) for x in zip(*copies))
        rows = torch.arange(case["page"], device=DEV)[None, :] < torch.tensor([k for _, _, k in copies], device=DEV)[:, None]
        for t in (t for kv in s["kvs"] for t in kv):
            t[to] = torch.where(rows[:, :, None, None], t[frm], t[to])
    return _i32([0]), _i32(refs), _i32(table), _i32(length), s["K"], s["V"]
