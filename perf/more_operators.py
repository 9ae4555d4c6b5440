"""The operators of beam and tree decoding over a paged cache that follow a step's logits, as they are timed.

A batch of users decodes with beams, or over drafted trees, whose keys and values live in pages that rows of a block table
share.  When a step's logits are there, four operators make the next step's state on the GPU:

  select   the best continuations of every user's beams over the whole vocabulary: log-softmax of each beam's logits (over the
           tokens that its grammar state allows, or over all), added to the beam's score, the best `width` of all
  fork     the chosen beams' block tables from their parents': full pages are shared, a partial last page goes to one child and
           fresh pages to the others, pages that nobody holds any more are free again
  copy     the filled part of those partial pages into the fresh ones, keys and values of all layers
  compact  after a tree's verification: keys and values of the accepted path move to the places behind the cached ones, all layers

Sizes are those of the benchmark's workloads (beams K = 10 .. 20, drafts N = 40 .. 80, 12 heads of 64 in 4 layers, 32 heads of 128 in
32 layers, 1 to 16 users, trees of 240 nodes in three levels, vocabulary 33024) and generic ones: grouped key heads, odd vocabularies,
hundreds of requests, tables of some thousand pages.
"""
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
NEG = float("-inf")
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f16": (torch.float16, torch.float16),
         "mixed": (torch.bfloat16, torch.float16)}   # of k and of v; mixed: the library's own cache layout


def listed():
    return [
        # one user's ten beams: latency, the smallest selection
        dict(name="select_k10", kind="select", n=1, w_lo=10, w_hi=10, V=33024, width=10, inp="f32", states=0, norm="masked",
             ends=0.0, shape=1),
        # the first step of 16 users, one row each, forty drafts wanted, only some tokens may begin an item
        dict(name="select_first_b16", kind="select", n=16, w_lo=1, w_hi=1, V=33024, width=40, inp="f32", states=4, norm="full",
             ends=0.0, shape=2),
        # 16 users' twenty beams, each in a state of its own among the valid continuations
        dict(name="select_b16_k20", kind="select", n=16, w_lo=20, w_hi=20, V=33024, width=20, inp="f32", states=64, norm="masked",
             ends=0.0, shape=3),
        # conversations with up to 16 beams each, some of them at their end, 16-bit logits of an odd vocabulary, two candidates a beam
        dict(name="select_b61_ends", kind="select", n=61, w_lo=8, w_hi=16, V=100003, width=32, inp="bf16", states=0, norm="masked",
             ends=0.2, shape=4),
        # eighty drafts from eighty for 48 users: 507 MB of logits, memory traffic
        dict(name="select_b48_k80", kind="select", n=48, w_lo=80, w_hi=80, V=33024, width=80, inp="f32", states=0, norm="masked",
             ends=0.0, shape=5),
        # one user's ten beams over one history: latency
        dict(name="fork_k10", kind="fork", n=1, w=10, q_lo=1, q_hi=1, ctx_lo=522, ctx_hi=522, page=64, spare=1.0, shape=6),
        # 16 users' twenty beams in small pages
        dict(name="fork_b16_k20", kind="fork", n=16, w=20, q_lo=1, q_hi=1, ctx_lo=256, ctx_hi=1024, page=16, spare=1.0, shape=7),
        # a large batch after its trees were verified: every row keeps some of its new tokens, the rest's pages come back
        dict(name="fork_trim_b1021", kind="fork", n=1021, w=1, q_lo=1, q_hi=61, ctx_lo=30, ctx_hi=32000, page=16, spare=1.0,
             shape=8),
        # the draft model's caches of one user's ten beams: latency
        dict(name="copy_k10", kind="copy", n=1, w=10, ctx_lo=522, ctx_hi=522, page=64, layers=4, Hkv=12, hd=64, types="mixed",
             layout="token", shape=9),
        # the 7B-shape caches of 16 users' ten beams: memory traffic
        dict(name="copy_b16_k10", kind="copy", n=16, w=10, ctx_lo=256, ctx_hi=1024, page=16, layers=32, Hkv=32, hd=128,
             types="mixed", layout="token", shape=10),
        # the accepted path of one tree in the draft model's caches: latency
        dict(name="compact_b1", kind="compact", n=1, q_lo=120, q_hi=120, levels=3, page=64, layers=4, Hkv=12, hd=64, types="mixed",
             layout="token", shape=11),
        # 16 users' trees in the 7B-shape caches
        dict(name="compact_b16", kind="compact", n=16, q_lo=240, q_hi=240, levels=3, page=64, layers=32, Hkv=32, hd=128,
             types="mixed", layout="token", shape=12),
    ]


def _log(rng, lo, hi):
    """An integer, uniform over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["select", "select", "select", "fork", "fork", "copy", "copy", "compact", "compact"])
    shape = rng.randrange(1 << 30)
    while True:
        n, page = _log(rng, 1, 1021), rng.choice([16, 32, 64, 128, 256])
        w = _log(rng, 1, 100)
        ctx_hi = _log(rng, 1, 32000)
        ctx_lo = max(1, ctx_hi // rng.choice([1, 2, 8, 32]) - rng.choice([0, 1]))
        store = dict(layers=rng.choice([1, 2, 4, 12, 28, 32]), hd=rng.choice([32, 64, 64, 128, 128]), Hkv=rng.choice([1, 2, 4, 8, 12, 32]),
                     types=rng.choice(["bf16", "f16", "mixed"]), layout=rng.choice(["token", "token", "head"]))
        token = 4.0 * store["layers"] * store["hd"] * store["Hkv"]
        if kind == "select":
            c = dict(kind=kind, n=n, w_lo=max(1, w // rng.choice([1, 1, 2, 7])), w_hi=w, V=_log(rng, 300, 130000),
                     width=_log(rng, 1, 128), inp=rng.choice(["f32", "bf16", "f16"]), states=rng.choice([0, 0, 1, 16, 64]),
                     norm=rng.choice(["masked", "full"]), ends=rng.choice([0.0, 0.0, 0.2]), shape=shape)
            if n * w * c["V"] <= 120e6 and n * w <= 8192:
                return c
        elif kind == "fork":
            q_hi = 1 if rng.random() < 0.6 else _log(rng, 2, 240)
            c = dict(kind=kind, n=n, w=w if q_hi == 1 else 1, q_lo=1, q_hi=q_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page,
                     spare=rng.choice([0.5, 1.0, 1.0, 1.5]), shape=shape)
            if n * c["w"] <= 4096 and n * c["w"] * (ctx_hi / page + 2) <= 2.2e6:
                return c
        elif kind == "copy":
            c = dict(kind=kind, n=n, w=max(2, w), ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page, shape=shape, **store)
            if n * c["w"] * page * token <= 0.6e9:
                return c
        else:
            levels = rng.choice([1, 2, 3, 4, 7])
            q_hi = _log(rng, 2 * levels, 512)
            c = dict(kind=kind, n=n, q_lo=max(levels, q_hi // rng.choice([1, 2])), q_hi=q_hi, levels=levels, page=page, shape=shape, **store)
            if n * (q_hi + 2 * page) * token <= 2.6e9:
                return c


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    return t.mul_(std) if std != 1.0 else t


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _up(a, page):
    return -(-a // page)


def _spread(rng, lo, hi, n):
    """n lengths, uniform over the logarithm of [lo, hi]."""
    return np.clip(np.rint(lo * (hi / lo) ** rng.random(n)), lo, hi).astype(np.int64)


def _offsets(q):
    return np.concatenate([[0], np.cumsum(q)])


# Sizes, parents and accepted paths belong to the case, so that its work is known; values and the pages' order are the seed's.
def _beams(c):
    return np.random.default_rng([c["shape"], 3]).integers(c["w_lo"], c["w_hi"] + 1, size=c["n"])


def _prepare_select(c, seed):
    rng, g, w, V = np.random.default_rng([seed, 13]), _gen(seed), _beams(c), c["V"]
    R = int(w.sum())
    s = SimpleNamespace(c=c, R=R, w=w, cu=_i32(_offsets(w)), logits=_normal(g, (R, V), 3.0, FLOAT[c["inp"]]), final=None, grammar=None,
                        state=None)
    # a user's beams, best first
    score = np.concatenate([-np.cumsum(rng.exponential(0.4, size=k)) for k in w]) - 5.0
    s.score = torch.from_numpy(score.astype(np.float32)).to(DEV)
    if c["ends"]:
        s.final = _i32(np.where(rng.random(R) < c["ends"], V - 1, -1))
    if c["states"]:
        # half of the states allow a few tokens (the continuations of a list of items), half forbid a few
        bits = np.zeros((c["states"], _up(V, 32) * 32), np.uint8)
        for i in range(c["states"]):
            few = rng.choice(V, size=min(V, 256), replace=False)
            bits[i, :V] = i & 1
            bits[i, few] = 1 - (i & 1)
        s.grammar = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)
        s.state = _i32(rng.integers(-1, c["states"], size=R))
    return s


def _fork_sizes(c):
    """Of every row: cached and new tokens, its parent and what it keeps (beams: all; trees: a part of the new ones)."""
    rng, n, w = np.random.default_rng([c["shape"], 5]), c["n"], c["w"]
    kv = np.repeat(_spread(rng, c["ctx_lo"], c["ctx_hi"], n), w)
    q = rng.integers(c["q_lo"], c["q_hi"] + 1, size=n * w)
    if w == 1:
        return kv, q, None, kv + 1 + np.minimum(q - 1, rng.integers(0, 5, size=n))
    # a few good beams have most of the children
    up = np.minimum(rng.geometric(2.0 / w if w > 2 else 0.7, size=(n, w)) - 1, w - 1) + w * np.arange(n)[:, None]
    return kv, q, np.sort(up, axis=1).reshape(-1), None


def _fork_copies(c):
    kv, q, up, _ = _fork_sizes(c)
    if up is None:
        return 0
    again = np.concatenate([[False], up[1:] == up[:-1]])
    return int((again & ((kv + q)[up] % c["page"] != 0)).sum())


def _prepare_fork(c, seed):
    page, (kv, q, up, keep) = c["page"], _fork_sizes(c)
    rows, rng = len(kv), np.random.default_rng([seed, 11])
    # a user's rows share the full pages of the history; each has its own last one, and those of its new tokens that the plan
    # has just taken from the front of the free list
    full, have, need = kv // page, _up(kv, page), _up(kv + q, page)
    first = np.arange(0, rows, c["w"])
    fresh, copies = need - have, _fork_copies(c)
    left = int(np.ceil(c["spare"] * copies)) + 7
    n_pages = int(full[first].sum() + (have - full).sum() + fresh.sum()) + left
    order, width = rng.permutation(n_pages).astype(np.int32), int(need.max()) + 2
    table, ref, i = np.full((rows, width), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for b in range(rows):
        if b % c["w"]:
            table[b, :full[b]] = table[b - b % c["w"], :full[b]]
        else:
            table[b, :full[b]] = order[i:i + full[b]]
            ref[order[i:i + full[b]]] = c["w"]
            i += int(full[b])
        if have[b] > full[b]:
            table[b, full[b]] = order[i]
            ref[order[i]] = 1
            i += 1
    free, at = order[i:], _offsets(fresh)
    for b in np.nonzero(fresh)[0]:
        table[b, have[b]:need[b]] = free[at[b]:at[b + 1]]
    return SimpleNamespace(c=c, table=_i32(table), kv=_i32(kv), q=_i32(q), state=_i32(np.zeros(rows)), ref=_i32(ref), free=_i32(free),
                           n_free=_i32([free.size]), used=_i32([at[-1]]), parent=None if up is None else _i32(up),
                           length=None if keep is None else _i32(keep))


def _caches(c, g, pages):
    """K and V as [layers][pages][page][heads][hd], in memory token by token or head by head."""
    kt, vt = TYPES[c["types"]]
    head = c["layout"] == "head"
    shape = (c["layers"], pages, c["Hkv"] if head else c["page"], c["page"] if head else c["Hkv"], c["hd"])
    k, v = _normal(g, shape, dtype=kt), _normal(g, shape, dtype=vt)
    return (k.transpose(2, 3), v.transpose(2, 3)) if head else (k, v)


def _copy_sizes(c):
    """Sequence lengths, and which of every user's beams need a copy of their parent's last page."""
    rng, n, w = np.random.default_rng([c["shape"], 7]), c["n"], c["w"]
    length = np.repeat(_spread(rng, c["ctx_lo"], c["ctx_hi"], n), w)
    up = np.sort(np.minimum(rng.geometric(2.0 / w if w > 2 else 0.7, size=(n, w)) - 1, w - 1), axis=1)
    again = np.concatenate([np.zeros((n, 1), bool), up[:, 1:] == up[:, :-1]], axis=1).reshape(-1)
    return length, (up + w * np.arange(n)[:, None]).reshape(-1), again & (length % c["page"] != 0)


def _prepare_copy(c, seed):
    length, up, need = _copy_sizes(c)
    rows, copies = len(length), int(need.sum())
    order = np.random.default_rng([seed, 17]).permutation(rows + copies + 3).astype(np.int32)
    src, dst = np.full(rows, -1), np.full(rows, -1)
    src[need], dst[need] = order[up[need]], order[rows:rows + copies]
    k, v = _caches(c, _gen(seed), rows + copies + 3)
    s = SimpleNamespace(c=c, k=k, v=v, src=_i32(src), dst=_i32(dst), length=_i32(length))
    s.layers = _own_layers(k, v) if own else None
    return s


def _compact_sizes(c):
    """Trees, where the accepted path's nodes are (one a level, from the first on), and how many of them there are."""
    rng, n, L = np.random.default_rng([c["shape"], 9]), c["n"], c["levels"]
    q, kv = rng.integers(c["q_lo"], c["q_hi"] + 1, size=n), rng.integers(1, 3000, size=n)
    keep, count = np.zeros((n, L), np.int64), rng.integers(0, L + 1, size=n)
    for b in range(n):
        per = max(1, int(q[b]) // L)
        for i in range(L):
            at = i * per + rng.integers(0, per)
            # (the places that a pass writes are not read by the next one, which has to find what the first one found: a node is
            # where it stays, or behind the path's end)
            keep[b, i] = at if at >= L else i
    return q, kv, keep, count


def _prepare_compact(c, seed):
    q, kv, keep, count = _compact_sizes(c)
    page, rng = c["page"], np.random.default_rng([seed, 19])
    have = _up(kv % page + q, page)
    order, at = rng.permutation(int(have.sum()) + 3).astype(np.int64), _offsets(have)
    slot = []
    for b in range(c["n"]):
        p = kv[b] % page + np.arange(q[b])
        slot.append(order[at[b] + p // page] * page + p % page)
    k, v = _caches(c, _gen(seed), order.size)
    s = SimpleNamespace(c=c, k=k, v=v, slot=torch.from_numpy(np.concatenate(slot)).to(DEV), cu=_i32(_offsets(q)), kv=_i32(kv),
                        keep=_i32(keep), count=_i32(count))
    s.layers = _own_layers(k, v) if own else None
    return s


def _own_layers(k, v):
    """The description of all layers' caches, which a program makes once."""
    import paper_2410_05165_gb300 as ats
    return ats.CacheLayers(list(zip(k.unbind(0), v.unbind(0))))


def prepare(case, seed):
    return {"select": _prepare_select, "fork": _prepare_fork, "copy": _prepare_copy, "compact": _prepare_compact}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------
def _unpack(words, n):
    """Bits of 32-bit words [rows][w] as truth values [rows][n]."""
    b = (words[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
    return b.reshape(words.shape[0], -1)[:, :n] != 0


def _plain_select(s):
    """Request after request, in 64 bits: the places of two beams' candidates may lie closer than 32 bits tell."""
    c, V, W, off = s.c, s.c["V"], s.c["width"], _offsets(s.w)
    token = torch.full((c["n"], W), -1, dtype=torch.int32, device=DEV)
    parent, best = torch.full_like(token, -1), torch.full((c["n"], W), NEG, dtype=torch.float32, device=DEV)
    table = None
    if s.grammar is not None:
        table = torch.cat([_unpack(s.grammar, V), torch.ones(1, V, dtype=torch.bool, device=DEV)])   # (-1: the last row)
    for b in range(c["n"]):
        rows = slice(int(off[b]), int(off[b + 1]))
        x = s.logits[rows].double()
        x = torch.where(x != x, NEG, x).clamp_max_(torch.finfo(s.logits.dtype).max)
        ok = None if table is None else table[s.state[rows].long()]
        if ok is not None and c["norm"] == "masked":
            x = torch.where(ok, x, NEG)
        m = x.amax(1, keepdim=True).clamp_min_(-1e300)
        x = x - m
        x = s.score[rows].double()[:, None] + (x - x.exp().sum(1, keepdim=True).log_())
        if ok is not None and c["norm"] == "full":
            x = torch.where(ok, x, NEG)
        if s.final is not None:   # a beam at its end goes on as it is, as one candidate
            f = s.final[rows].long()
            one = torch.arange(V, device=DEV)[None, :] == f[:, None]
            x = torch.where((f >= 0)[:, None], torch.where(one, s.score[rows].double()[:, None], NEG), x)
        x = torch.where(x != x, NEG, x).reshape(-1)
        k = min(W, x.numel())
        at = torch.nonzero((x >= torch.topk(x, k).values[-1]) & (x > NEG)).reshape(-1)   # (ties: the lowest first)
        at = at[torch.sort(x[at], descending=True, stable=True).indices[:k]]
        token[b, :at.numel()], parent[b, :at.numel()] = (at % V).int(), (at // V + rows.start).int()
        best[b, :at.numel()] = x[at].float()
    return {"token": token, "parent": parent, "score": best}


def _plain_fork(s):
    page, n_pages, width = s.c["page"], s.ref.numel(), s.table.shape[1]
    held = (s.kv + torch.where(s.state == 0, s.q, 0)).long()
    rows, table = held.numel(), s.table.long()
    up = torch.arange(rows, device=DEV) if s.parent is None else s.parent.long()
    m = up.numel()
    length = held[up] if s.length is None else s.length.long()
    pages, j, col = (length + page - 1) // page, torch.arange(m, device=DEV), torch.arange(width, device=DEV)[None, :]
    # the child with the most tokens, the first of them, may go on in its parent's last page
    most = torch.zeros(rows, dtype=torch.long, device=DEV).scatter_reduce_(0, up, length, "amax")
    heir = torch.full((rows,), m, device=DEV).scatter_reduce_(0, up, torch.where(length == most[up], j, m), "amin")
    last = table[up, (pages - 1).clamp_min(0)]
    copies = (length % page != 0) & ~((heir[up] == j) & (s.ref[last] <= 1))
    nth = torch.cumsum(copies, 0) - copies.long() + s.used.long()
    ok = ~copies | (nth < s.n_free.long())
    copies = copies & ok
    fresh = s.free[nth.clamp(0, s.free.numel() - 1)].long()
    new = torch.where(ok[:, None] & (col < pages[:, None]), table[up], -1)
    new = torch.where(copies[:, None] & (col == pages[:, None] - 1), fresh[:, None], new)
    ref = s.ref.long()
    out = torch.arange(s.free.numel(), device=DEV) < s.used.long()
    ref = ref.index_add(0, s.free.long(), out.long())
    old = table[col < ((held + page - 1) // page)[:, None]]
    ref = ref.index_add(0, old, torch.full_like(old, -1))
    now = new[new >= 0]
    ref = ref.index_add(0, now, torch.ones_like(now))
    left = torch.cumsum(ref <= 0, 0)
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    free[torch.where(ref <= 0, left - 1, n_pages - 1)] = torch.where(ref <= 0, torch.arange(n_pages, device=DEV), -1).int()
    free = torch.where(torch.arange(n_pages, device=DEV) < left[-1], free, -1)
    return {"table": new.int(), "kv_len": torch.where(ok, length, -1).int(), "state": torch.where(ok, 0, 1).int(),
            "src": torch.where(copies, last, -1).int(), "dst": torch.where(copies, fresh, -1).int(), "ref": ref.int(),
            "free": free, "n_free": left[-1:].int()}


def _plain_copy(s):
    page = s.c["page"]
    rows = torch.where(s.src >= 0, (s.length - 1) % page + 1, 0)
    j, r = torch.nonzero(torch.arange(page, device=DEV)[None, :] < rows[:, None], as_tuple=True)
    a, b = s.src.long()[j], s.dst.long()[j]
    for t in (s.k, s.v):
        t[:, b, r] = t[:, a, r]
    return {"k": s.k, "v": s.v}


def _plain_compact(s):
    page, L = s.c["page"], s.keep.shape[1]
    b, i = torch.nonzero(torch.arange(L, device=DEV)[None, :] < s.count[:, None], as_tuple=True)
    a = s.slot[s.cu.long()[b] + s.keep.long()[b, i]]
    to = s.slot[s.cu.long()[b] + i]
    for t in (s.k, s.v):
        t[:, to // page, to % page] = t[:, a // page, a % page]
    return {"k": s.k, "v": s.v, "kv_len": s.kv + s.count}


def _run_own(s):
    import paper_2410_05165_gb300 as ats
    kind = s.c["kind"]
    if kind == "select":
        r = ats.op_beam_select(s.logits, s.cu, s.c["width"], score=s.score, final=s.final, grammar=s.grammar, state=s.state,
                               norm=ats.NORM_MASKED if s.c["norm"] == "masked" else ats.NORM_FULL)
        return {"token": r.token, "parent": r.parent, "score": r.score}
    if kind == "fork":
        r = ats.op_fork_pages(s.table, s.kv, s.ref, s.free, s.n_free, s.c["page"], q_len=s.q, state=s.state, used=s.used,
                              parent=s.parent, length=s.length)
        return {"table": r.table, "kv_len": r.kv_len, "state": r.state, "src": r.src, "dst": r.dst, "ref": r.ref, "free": r.free,
                "n_free": r.n_free}
    if kind == "copy":
        ats.op_copy_pages(s.layers, s.src, s.dst, length=s.length)
        return {"k": s.k, "v": s.v}
    kv_len = ats.op_compact_tokens(s.layers, s.slot, s.cu, s.kv, s.keep, s.count)
    return {"k": s.k, "v": s.v, "kv_len": kv_len}


def run(s):
    if own:
        return _run_own(s)
    return {"select": _plain_select, "fork": _plain_fork, "copy": _plain_copy, "compact": _plain_compact}[s.c["kind"]](s)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "select":
        R = float(_beams(c).sum())
        logits = R * c["V"]
        return {"bytes": logits * (4.0 if c["inp"] == "f32" else 2.0) + c["states"] * c["V"] / 8.0 + 12.0 * R + 12.0 * c["n"] * c["width"],
                "flops": 4.0 * logits}
    if c["kind"] == "fork":
        kv, q, up, keep = _fork_sizes(c)
        need = _up(kv + q, c["page"])
        kept = need[up] if up is not None else _up(keep, c["page"])
        rows, width = float(len(kv)), float(need.max()) + 2.0
        # parents' entries in, the new table out; counts in and out, the free list out (its size: about the pages that rows hold alone)
        pool = float((kv // c["page"])[::c["w"]].sum() + (need - kv // c["page"]).sum()) + c["spare"] * _fork_copies(c) + 7.0
        return {"bytes": 4.0 * float(kept.sum()) + 4.0 * rows * width + 12.0 * pool + 36.0 * rows, "flops": rows * width}
    store = 4.0 * c["layers"] * c["Hkv"] * c["hd"]
    if c["kind"] == "copy":
        length, _, need = _copy_sizes(c)
        moved = float(((length - 1) % c["page"] + 1)[need].sum())
        return {"bytes": 2.0 * moved * store + 12.0 * len(length), "flops": moved}
    q, _, keep, count = _compact_sizes(c)
    moved = float(sum((keep[b, :count[b]] != np.arange(count[b])).sum() for b in range(c["n"])))
    return {"bytes": 2.0 * moved * store + 16.0 * c["n"] + 12.0 * float(count.sum()), "flops": moved + c["n"]}


# ---------------------------------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The selection's scores and their places; the other operators move values and count, which 64 bits do not do otherwise."""
    c = case
    if c["kind"] != "select" or int(_beams(c).sum()) > 20000:   # (a row at a time)
        return None
    s = _prepare_select(c, seed)
    off, W, V = _offsets(s.w), c["width"], c["V"]
    token, parent = np.full((c["n"], W), -1, np.int32), np.full((c["n"], W), -1, np.int32)
    best = np.full((c["n"], W), NEG)
    score, final = s.score.cpu().numpy().astype(np.float64), None if s.final is None else s.final.cpu().numpy()
    state = None if s.state is None else s.state.cpu().numpy()
    for b in range(c["n"]):
        got = []
        for r in range(int(off[b]), int(off[b + 1])):
            if final is not None and final[r] >= 0:
                got.append((torch.tensor([score[r]], dtype=torch.float64, device=DEV), torch.tensor([int(final[r])], device=DEV), r))
                continue
            x = s.logits[r].double()
            at = torch.arange(V, device=DEV)
            if state is not None and state[r] >= 0:
                bits = np.unpackbits(s.grammar[state[r]].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                at = torch.from_numpy(np.nonzero(bits)[0]).to(DEV)
            lse = torch.logsumexp(x if c["norm"] == "full" else x[at], 0)
            y = x[at]
            y, order = torch.sort(y, descending=True, stable=True)
            got.append((score[r] + (y[:W] - lse), at[order[:W]], r))
        y = torch.cat([g[0] for g in got])
        t = torch.cat([g[1] for g in got])
        p = torch.cat([torch.full_like(g[1], g[2]) for g in got])
        y, order = torch.sort(y, descending=True, stable=True)
        k = min(W, y.numel())
        best[b, :k], token[b, :k], parent[b, :k] = y[:k].cpu().numpy(), t[order[:k]].cpu().numpy(), p[order[:k]].cpu().numpy()
    return {"token": torch.from_numpy(token), "parent": torch.from_numpy(parent), "score": torch.from_numpy(best)}
