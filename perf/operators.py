"""The operators of one serving step over drafted trees of a batch of requests, as they are timed.

A batch of requests, each with cached keys and values in pages and with a few new tokens (one token, a drafted
tree, or a piece of a prompt), takes four operators a step:

  plan    block tables and slot maps on the GPU from the requests' lengths: pages taken from a free list, the
          cache slot, position and request of every new token, and every tree node's ancestors as bits
  append  the new tokens' q rotated, their k rotated and v stored into the cache by slot
  attn    attention of the new tokens over their request's cached keys and their own ancestors
  logits  penalties for repeated tokens, biases, grammar masks and temperature on the logits of every token

Sizes are those of the benchmark's workloads (12 heads of 64, 32 heads of 64 or 128, trees of K = 10 .. 20, N = 40 .. 80
over three levels, 1 to 16 users, 512-token histories, vocabulary 33024) and generic ones: grouped key heads,
caches of some ten thousand tokens, hundreds of requests, vocabularies that are no power of two.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
NEG = float("-inf")
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f16": (torch.float16, torch.float16),
         "mixed": (torch.bfloat16, torch.float16)}   # of q / k and of v; mixed: the library's own cache layout


def listed():
    return [
        # 16 users' drafted trees (K = 20, N = 80, three levels) over their histories
        dict(name="plan_trees_b16", kind="plan", n=16, q_lo=240, q_hi=240, ctx_lo=256, ctx_hi=1024, page=64, levels=3,
             spare=1.0, shape=1),
        # one token each for a large batch of conversations, an odd number of them, more pages wanted than free
        dict(name="plan_decode_b1021", kind="plan", n=1021, q_lo=1, q_hi=1, ctx_lo=30, ctx_hi=32000, page=16, levels=0,
             spare=0.7, shape=2),
        # ten beams through the draft model: latency
        dict(name="append_t10", kind="append", n=1, q_lo=10, q_hi=10, ctx_lo=512, ctx_hi=512, H=12, Hkv=12, hd=64, page=64,
             types="mixed", src="f32", layout="token", shape=3),
        # 16 users' trees through the 7B-shape model, from the 32-bit sums of the QKV projection
        dict(name="append_t3840", kind="append", n=16, q_lo=240, q_hi=240, ctx_lo=256, ctx_hi=1024, H=32, Hkv=32, hd=128,
             page=64, types="mixed", src="f32", layout="token", shape=4),
        # one beam of the draft model over one history: latency, the smallest call
        dict(name="attn_decode_b1", kind="attn", n=1, q_lo=1, q_hi=1, ctx_lo=512, ctx_hi=512, H=12, Hkv=12, hd=64, page=64,
             types="mixed", layout="token", levels=0, shape=5),
        # one token each for 61 conversations of very different lengths, grouped heads: memory traffic
        dict(name="attn_decode_b61", kind="attn", n=61, q_lo=1, q_hi=1, ctx_lo=500, ctx_hi=16000, H=32, Hkv=8, hd=128, page=64,
             types="bf16", layout="token", levels=0, shape=6),
        # 16 users' drafted trees over their histories, 7B-shape heads, the library's cache layout
        dict(name="attn_trees_b16", kind="attn", n=16, q_lo=240, q_hi=240, ctx_lo=256, ctx_hi=1024, H=32, Hkv=32, hd=128,
             page=64, types="mixed", layout="token", levels=3, shape=7),
        # a tree of 61 tokens over three very long contexts in small pages, grouped heads
        dict(name="attn_tree_long", kind="attn", n=3, q_lo=61, q_hi=61, ctx_lo=20000, ctx_hi=65000, H=32, Hkv=8, hd=128, page=16,
             types="bf16", layout="token", levels=4, shape=8),
        # pieces of two prompts, causal, over what is cached already; pages laid out head by head: tensor work
        dict(name="attn_prompt_4001", kind="attn", n=2, q_lo=4001, q_hi=4001, ctx_lo=1500, ctx_hi=3001, H=32, Hkv=8, hd=64,
             page=128, types="f16", layout="head", levels=0, shape=9),
        # the logits of one token of one user: latency
        dict(name="logits_r1", kind="logits", n=1, q_lo=1, q_hi=1, V=33024, hist_lo=512, hist_hi=512, bias=20, states=1,
             inp="f32", out="f32", levels=0, shape=10),
        # the logits of 16 users' trees, every node with the tokens of its own path
        dict(name="logits_trees_b16", kind="logits", n=16, q_lo=240, q_hi=240, V=33024, hist_lo=256, hist_hi=1024, bias=300,
             states=64, inp="f32", out="f32", levels=3, shape=11),
        # one token each for a large batch, long histories, 16-bit logits of an odd vocabulary
        dict(name="logits_decode_b509", kind="logits", n=509, q_lo=1, q_hi=1, V=100003, hist_lo=50, hist_hi=8000, bias=100,
             states=32, inp="bf16", out="bf16", levels=0, shape=12),
    ]


def _log(rng, lo, hi):
    """An integer, uniform over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attn", "attn", "attn", "attn", "logits", "logits"])
    shape = rng.randrange(1 << 30)
    while True:
        n = _log(rng, 1, 1021)
        if rng.random() < 0.5:
            q_lo = q_hi = 1
        else:
            q_lo = _log(rng, 1, 4001)
            q_hi = min(4001, q_lo + _log(rng, 1, 100))
        levels = 0 if q_hi == 1 or q_hi > 1024 or rng.random() < 0.3 else rng.choice([1, 2, 3, 4, 7])
        ctx_hi = _log(rng, 1, 65000)
        ctx_lo = max(0, ctx_hi // rng.choice([1, 2, 8, 32]) - rng.choice([0, 1]))
        page = rng.choice([16, 32, 64, 128, 256])
        H, Hkv, hd = rng.choice([(12, 12, 64), (32, 32, 64), (32, 32, 128), (32, 8, 128), (32, 8, 64), (28, 4, 128), (12, 4, 64),
                                 (8, 1, 128), (4, 4, 32), (6, 2, 32)])
        types, layout = rng.choice(["bf16", "f16", "mixed"]), rng.choice(["token", "token", "head"])
        if kind == "plan":
            c = dict(kind=kind, n=n, q_lo=q_lo, q_hi=q_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page, levels=levels,
                     spare=rng.choice([0.5, 1.0, 1.0, 1.5]), shape=shape)
            if n * q_hi <= 16384:
                return c
        elif kind == "append":
            c = dict(kind=kind, n=n, q_lo=q_lo, q_hi=q_hi, ctx_lo=ctx_lo // 16, ctx_hi=max(1, ctx_hi // 16), H=H, Hkv=Hkv, hd=hd,
                     page=page, types=types, src=rng.choice(["f32", "same"]), layout=layout, shape=shape)
            if n * q_hi <= 4096 and n * (c["ctx_hi"] + q_hi + page) <= 65536:
                return c
        elif kind == "attn":
            c = dict(kind=kind, n=n, q_lo=q_lo, q_hi=q_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, H=H, Hkv=Hkv, hd=hd, page=page, types=types,
                     layout=layout, levels=levels, shape=shape)
            if (4.0 * n * q_hi * (ctx_hi + q_hi) * H * hd < 2.5e11 and 4.0 * n * (ctx_hi + q_hi) * Hkv * hd < 1.1e9
                    and n * Hkv <= 4096):
                return c
        else:
            V = _log(rng, 500, 130000)
            c = dict(kind=kind, n=n, q_lo=q_lo, q_hi=q_hi, V=V, hist_lo=rng.choice([0, 1, 50]), hist_hi=_log(rng, 60, 8000),
                     bias=rng.choice([0, 1, 30, 300]), states=rng.choice([0, 1, 16, 64]), inp=rng.choice(["f32", "bf16", "f16"]),
                     out="f32", levels=levels, shape=shape)
            if rng.random() < 0.6:
                c["out"] = c["inp"]
            if n * q_hi * V <= 120e6:
                return c


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    return t.mul_(std) if std != 1.0 else t


def _spread(rng, lo, hi, n):
    """n lengths, uniform over the logarithm of [lo, hi]."""
    x = (lo + 1.0) * ((hi + 1.0) / (lo + 1.0)) ** rng.random(n) - 1.0
    return np.clip(np.rint(x), lo, hi).astype(np.int64)


def _lengths(c):
    """New tokens and cached tokens of each request; they belong to the case, so that its work is known."""
    rng = np.random.default_rng([c["shape"], 3])
    q = rng.integers(c["q_lo"], c["q_hi"] + 1, size=c["n"])
    return q, (_spread(rng, c["ctx_lo"], c["ctx_hi"], c["n"]) if "ctx_hi" in c else None)


def _parents(c, q):
    """Drafted trees, level after level, the parent of a node drawn from the level before (-1: none), and every
    request's ancestor bits [q][q] (a node among them)."""
    rng = np.random.default_rng([c["shape"], 5])
    par, bits = [], []
    for m in q:
        per = -(-int(m) // c["levels"])
        p = np.full(m, -1, np.int32)
        for i in range(per, m, per):
            k = min(per, m - i)
            p[i:i + k] = rng.integers(i - per, i, size=k)
        b = np.eye(m, dtype=bool)
        for i in range(m):
            if p[i] >= 0:
                b[i] |= b[p[i]]
        par.append(p)
        bits.append(b)
    return par, bits


def _words(bits, words):
    """Rows of bits as 32-bit words, the lowest bit first."""
    out = np.zeros((sum(len(b) for b in bits), words * 32), np.uint8)
    i = 0
    for b in bits:
        out[i:i + len(b), :b.shape[1]] = b
        i += len(b)
    return torch.from_numpy(np.packbits(out, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _offsets(q):
    return np.concatenate([[0], np.cumsum(q)])


def _pages(c, q, ctx, seed, spare=0.0):
    """A pool in random order, the requests' block tables (entries not yet taken are -1) and the pages left."""
    rng = np.random.default_rng([seed, 11])
    have = -(-(ctx + (0 if spare else q)) // c["page"])
    want = int((-(-(ctx + q) // c["page"]) - -(-ctx // c["page"])).sum())
    left = int(math.ceil(spare * want)) if spare else 3
    width = int((-(-(ctx + q) // c["page"])).max()) + 2
    order = rng.permutation(int(have.sum()) + left).astype(np.int32)
    table = np.full((c["n"], width), -1, np.int32)
    i = 0
    for b in range(c["n"]):
        table[b, :have[b]] = order[i:i + have[b]]
        i += int(have[b])
    return table, order[i:], order.size


def _cache(c, g, pages):
    """K and V as [pages][page][heads][hd], in memory token by token or head by head."""
    kt, vt = TYPES[c["types"]]
    shape = (pages, c["page"], c["Hkv"], c["hd"])
    if c["layout"] == "head":
        shape = (pages, c["Hkv"], c["page"], c["hd"])
    k, v = _normal(g, shape, dtype=kt), _normal(g, shape, dtype=torch.bfloat16 if c["types"] == "mixed" else vt).to(vt)
    return (k.transpose(1, 2), v.transpose(1, 2)) if c["layout"] == "head" else (k, v)


def _slots(c, table, q, ctx):
    s = [table[b, (ctx[b] + np.arange(q[b])) // c["page"]].astype(np.int64) * c["page"] + (ctx[b] + np.arange(q[b])) % c["page"]
         for b in range(c["n"])]
    return np.concatenate(s)


def _prepare_plan(c, seed):
    q, ctx = _lengths(c)
    table, free, _ = _pages(c, q, ctx, seed, c["spare"])
    s = SimpleNamespace(c=c, T=int(q.sum()), q_len=_i32(q), kv_len=_i32(ctx), table=_i32(table), n_free=_i32([free.size]),
                        free=_i32(free if free.size else [0]), parent=None, words=0)
    if c["levels"]:
        s.parent = _i32(np.concatenate(_parents(c, q)[0]))
        s.words = -(-int(q.max()) // 32)
    return s


def _prepare_append(c, seed):
    q, ctx = _lengths(c)
    table, _, pages = _pages(c, q, ctx, seed)
    g = _gen(seed)
    k, v = _cache(c, g, pages)
    T, rows = int(q.sum()), (c["H"] + 2 * c["Hkv"]) * c["hd"]
    pos = np.concatenate([ctx[b] + np.minimum(np.arange(q[b]), 4) for b in range(c["n"])])   # nodes of a level share one
    return SimpleNamespace(c=c, T=T, k=k, v=v, qkv=_normal(g, (T, rows), dtype=torch.float32 if c["src"] == "f32" else k.dtype),
                           slot=torch.from_numpy(_slots(c, table, q, ctx)).to(DEV), pos=_i32(pos))


def _prepare_attn(c, seed):
    q, ctx = _lengths(c)
    table, _, pages = _pages(c, q, ctx, seed)
    g = _gen(seed)
    k, v = _cache(c, g, pages)
    s = SimpleNamespace(c=c, q_host=q, ctx_host=ctx, k=k, v=v, q=_normal(g, (int(q.sum()), c["H"], c["hd"]), dtype=k.dtype),
                        table=_i32(table), cu_q=_i32(_offsets(q)), ctx=_i32(ctx), mask=None)
    if c["levels"]:
        s.mask = _words(_parents(c, q)[1], -(-int(q.max()) // 32))
    return s


def _hist_lens(c):
    return _spread(np.random.default_rng([c["shape"], 7]), c["hist_lo"], c["hist_hi"], c["n"])


def _prepare_logits(c, seed):
    q, _ = _lengths(c)
    g, rng, n, V, R = _gen(seed), np.random.default_rng([seed, 13]), c["n"], c["V"], int(q.sum())
    hist = _hist_lens(c)
    # tokens recur, as words do: ranks of a Zipf law through a permutation
    perm = rng.permutation(V)

    def words(k):
        return perm[np.minimum((V ** rng.random(k)).astype(np.int64) - 1, V - 1)]

    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    s = SimpleNamespace(c=c, R=R, q_host=q, logits=_normal(g, (R, V), 3.0, dt[c["inp"]]), out_type=dt[c["out"]],
                        req=_i32(np.repeat(np.arange(n), q)), hist=_i32(words(max(1, int(hist.sum())))),
                        hist_off=_i32(_offsets(hist)), prompt_len=_i32(hist * rng.integers(2, 9, size=n) // 10),
                        mask=None, tree_tok=None, cu_q=None, bias_off=None, bias_tok=None, bias_val=None, grammar=None,
                        state=None)

    def per_request(lo, hi, neutral):
        x = rng.uniform(lo, hi, size=n)
        x[rng.random(n) < 0.2] = neutral
        return torch.from_numpy(x.astype(np.float32)).to(DEV)

    s.repetition, s.frequency = per_request(1.0, 1.5, 1.0), per_request(-0.2, 1.0, 0.0)
    s.presence, s.temperature = per_request(-0.2, 1.0, 0.0), per_request(0.5, 1.5, 1.0)
    if c["bias"]:
        nb = np.minimum(rng.integers(0, c["bias"] + 1, size=n), V)
        s.bias_off = _i32(_offsets(nb))
        s.bias_tok = _i32(np.concatenate([rng.choice(V, size=k, replace=False) for k in nb] + [np.zeros(1, np.int64)]))
        s.bias_val = _normal(g, (s.bias_tok.numel(),), 4.0, torch.float32)
    if c["states"]:
        # half of the states allow a few tokens (a closed list), half forbid a few
        w = np.zeros((c["states"], -(-V // 32) * 32), np.uint8)
        for i in range(c["states"]):
            few = rng.choice(V, size=min(V, 256), replace=False)
            w[i, :V] = i & 1
            w[i, few] = 1 - (i & 1)
        s.grammar = torch.from_numpy(np.packbits(w, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)
        s.state = _i32(rng.integers(-1, c["states"], size=R))
    if c["levels"]:
        s.mask = _words(_parents(c, q)[1], -(-int(q.max()) // 32))
        s.tree_tok, s.cu_q = _i32(words(R)), _i32(_offsets(q))
    return s


def prepare(case, seed):
    return {"plan": _prepare_plan, "append": _prepare_append, "attn": _prepare_attn, "logits": _prepare_logits}[case["kind"]](
        case, seed)


# ---------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------
def _unpack(words, n):
    """Bits of 32-bit words [rows][w] as truth values [rows][n]."""
    b = (words[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
    return b.reshape(words.shape[0], -1)[:, :n] != 0


def _plain_plan(s):
    c, page, T, n = s.c, s.c["page"], s.T, s.c["n"]
    q, kv = s.q_len.long(), s.kv_len.long()
    end = torch.cumsum(q, 0)
    start = end - q
    have, need = (kv + page - 1) // page, (kv + q + page - 1) // page
    new = need - have
    upto = torch.cumsum(new, 0)
    ok = (new == 0) | (upto <= s.n_free.long())
    taken = torch.where(ok, upto, torch.zeros_like(upto)).max()
    col = torch.arange(s.table.shape[1], device=DEV)[None, :]
    fresh = ok[:, None] & (col >= have[:, None]) & (col < need[:, None])
    src = (upto - new)[:, None] + col - have[:, None]
    table = torch.where(fresh, s.free.long()[src.clamp(0, s.free.numel() - 1)], s.table.long())
    t = torch.arange(T, device=DEV)
    req = torch.searchsorted(end, t, right=True)
    i = t - start[req]
    at = kv[req] + i
    slot = torch.where(ok[req], table[req, at // page] * page + at % page, torch.full_like(at, -1))
    mask, depth = None, i
    if s.parent is not None:
        # a node's ancestors: the walk up from every node at once, one level a turn
        node, live = i.clone(), torch.ones_like(i, dtype=torch.bool)
        bits = torch.zeros(T, s.words * 32, dtype=torch.bool, device=DEV)
        depth = torch.full_like(i, -1)
        for _ in range(c["levels"]):
            bits[t, node] = bits[t, node] | live
            depth = depth + live
            up = s.parent.long()[start[req] + node]
            live = live & (up >= 0)
            node = torch.where(live, up, node)
        w = bits.reshape(T, s.words, 32).long() << torch.arange(32, device=DEV)
        mask = w.sum(2)
        mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask).int()
    return {"table": table.int(), "cu_q": torch.cat([start[:1] * 0, end]).int(), "ctx_len": torch.where(ok, kv, -1).int(),
            "req": req.int(), "pos": (kv[req] + depth).int(), "slot": slot, "mask": mask, "taken": taken.int()}


def _rope(x, pos, half, dtype):
    """Each head's first half against its second, turned by position x 10000^(-i / half)."""
    freq = 10000.0 ** (-torch.arange(half, device=DEV, dtype=dtype) / half)
    ang = pos.to(dtype)[:, None] * freq
    cos, sin = ang.cos()[:, None, :], ang.sin()[:, None, :]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], 2)


def _append_parts(s, dtype):
    c = s.c
    q, k, v = s.qkv.to(dtype).split([c["H"] * c["hd"], c["Hkv"] * c["hd"], c["Hkv"] * c["hd"]], 1)
    q, k, v = q.reshape(s.T, -1, c["hd"]), k.reshape(s.T, -1, c["hd"]), v.reshape(s.T, -1, c["hd"])
    return _rope(q, s.pos, c["hd"] // 2, dtype), _rope(k, s.pos, c["hd"] // 2, dtype), v


def _plain_append(s):
    page = s.c["page"]
    q, k, v = _append_parts(s, torch.float32)
    s.k[s.slot // page, s.slot % page] = k.to(s.k.dtype)
    s.v[s.slot // page, s.slot % page] = v.to(s.v.dtype)
    return {"q": q.to(s.k.dtype), "k": s.k, "v": s.v}


def _attend(s, dtype):
    """Request after request: scores, masked softmax, weighted values (rows that see nothing: zero)."""
    c, off = s.c, _offsets(s.q_host)
    G, out = c["H"] // c["Hkv"], torch.empty(s.q.shape, device=DEV, dtype=dtype)
    for b in range(c["n"]):
        L, ctx = int(s.q_host[b]), int(s.ctx_host[b])
        S = ctx + L
        rows = s.table[b, :-(-S // c["page"])].long()
        see = torch.ones(L, S, dtype=torch.bool, device=DEV)
        sl = slice(int(off[b]), int(off[b]) + L)
        see[:, ctx:] = _unpack(s.mask[sl], L) if s.mask is not None else torch.ones(L, L, dtype=torch.bool, device=DEV).tril()
        for h in range(c["Hkv"]):
            k = s.k[rows, :, h].reshape(-1, c["hd"])[:S].to(dtype)
            v = s.v[rows, :, h].reshape(-1, c["hd"])[:S].to(dtype)
            q = s.q[sl, h * G:(h + 1) * G].to(dtype).transpose(0, 1)
            w = torch.matmul(q, k.T).mul_(c["hd"] ** -0.5).masked_fill_(~see, NEG)
            w = torch.exp(w - w.amax(2, keepdim=True).clamp_min(-3e38)).masked_fill_(~see, 0.0)
            w = w / w.sum(2, keepdim=True).clamp_min(1e-30)
            out[sl, h * G:(h + 1) * G] = torch.matmul(w, v).transpose(0, 1)
    return out


def _adjust(s, dtype):
    c, n, V, R = s.c, s.c["n"], s.c["V"], s.R
    req = s.req.long()
    hist = (s.hist_off[1:] - s.hist_off[:-1]).long()
    own_req = torch.repeat_interleave(torch.arange(n, device=DEV), hist)
    tok = s.hist[:own_req.numel()].long()
    prompt = torch.arange(own_req.numel(), device=DEV) - s.hist_off[:-1].long()[own_req] < s.prompt_len.long()[own_req]
    seen, count = torch.zeros(n * V, device=DEV), torch.zeros(n * V, device=DEV)
    seen.index_fill_(0, own_req * V + tok, 1.0)
    count.index_add_(0, own_req * V + tok, (~prompt).float())
    seen, count = seen.reshape(n, V)[req], count.reshape(n, V)[req]
    if s.mask is not None:
        row, j = torch.nonzero(_unpack(s.mask, int(s.q_host.max())), as_tuple=True)
        at = row * V + s.tree_tok.long()[s.cu_q.long()[req[row]] + j]
        count.view(-1).index_add_(0, at, torch.ones(at.numel(), device=DEV))
        seen.view(-1).index_fill_(0, at, 1.0)
    x = s.logits.to(dtype)
    r = s.repetition.to(dtype)[req][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
    del seen
    x = x - s.frequency.to(dtype)[req][:, None] * count - s.presence.to(dtype)[req][:, None] * (count > 0)
    del count
    if s.bias_off is not None:
        nb = (s.bias_off[1:] - s.bias_off[:-1]).long()
        b = torch.repeat_interleave(torch.arange(n, device=DEV), nb)
        add = torch.zeros(n * V, device=DEV, dtype=dtype)
        add.index_add_(0, b * V + s.bias_tok[:b.numel()].long(), s.bias_val[:b.numel()].to(dtype))
        x = x + add.reshape(n, V)[req]
    if s.grammar is not None:
        ok = torch.cat([_unpack(s.grammar, V), torch.ones(1, V, dtype=torch.bool, device=DEV)])   # (-1: the last row)
        x = torch.where(ok[s.state.long()], x, NEG)
    return x / s.temperature.to(dtype)[req][:, None]


def _own_rules(s):
    import paper_2410_05165_gb300 as ats
    return ats.LogitRules(hist=s.hist, hist_off=s.hist_off, prompt_len=s.prompt_len, repetition=s.repetition,
                          frequency=s.frequency, presence=s.presence, temperature=s.temperature, bias_off=s.bias_off,
                          bias_tok=s.bias_tok, bias_val=s.bias_val, grammar=s.grammar, tree_tok=s.tree_tok, cu_q=s.cu_q)


def _run_own(s):
    import paper_2410_05165_gb300 as ats
    c = s.c
    if c["kind"] == "plan":
        p = ats.op_batch_plan(s.q_len, s.kv_len, s.table, s.free, s.n_free, c["page"], s.T, parent=s.parent, mask_words=s.words)
        return {"table": s.table, "cu_q": p.cu_q, "ctx_len": p.ctx_len, "req": p.req, "pos": p.pos, "slot": p.slot,
                "mask": p.mask, "taken": p.taken}
    if c["kind"] == "append":
        q = ats.op_rope_append(s.qkv, c["H"], s.k, s.v, s.slot, pos=s.pos, theta=10000.0)
        return {"q": q, "k": s.k, "v": s.v}
    if c["kind"] == "attn":
        return ats.op_tree_attention(s.q, s.k, s.v, s.cu_q, s.ctx, s.table, mask=s.mask)
    return ats.op_adjust_logits(s.logits, s.req, _own_rules(s), mask=s.mask, state=s.state, out_dtype=s.out_type)


def run(s):
    if own:
        return _run_own(s)
    c = s.c
    if c["kind"] == "plan":
        return _plain_plan(s)
    if c["kind"] == "append":
        return _plain_append(s)
    if c["kind"] == "attn":
        return _attend(s, torch.float32).to(s.q.dtype)
    return _adjust(s, torch.float32).to(s.out_type)


# ---------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------
def work(case):
    c = case
    q, ctx = _lengths(c)
    T = float(q.sum())
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}
    if c["kind"] == "plan":
        # lengths, the table entries of the new tokens' pages (read or written), four numbers a token and its bits
        entries = float((-(-(ctx + q) // c["page"]) - ctx // c["page"]).sum())
        bits = T * (4.0 + 4.0 * -(-int(q.max()) // 32)) if c["levels"] else 0.0
        return {"bytes": 20.0 * c["n"] + 4.0 * entries + 20.0 * T + bits, "flops": 10.0 * T}
    if c["kind"] == "append":
        d, dk = c["H"] * c["hd"], c["Hkv"] * c["hd"]
        src = 4.0 if c["src"] == "f32" else 2.0
        return {"bytes": T * ((d + 2 * dk) * (src + 2.0) + 12.0), "flops": 3.0 * T * (d + dk)}
    if c["kind"] == "attn":
        if c["levels"]:
            tree = float(sum(b.sum() for b in _parents(c, q)[1]))
        else:
            tree = float((q * (q + 1.0) / 2).sum())
        pairs = float((q * 1.0 * ctx).sum()) + tree
        return {"bytes": 4.0 * float((ctx + q).sum()) * c["Hkv"] * c["hd"] + 4.0 * T * c["H"] * c["hd"],
                "flops": 4.0 * pairs * c["H"] * c["hd"]}
    by = T * c["V"] * (size[c["inp"]] + size[c["out"]]) + 4.0 * float(_hist_lens(c).sum()) + 4.0 * c["n"] * c["bias"]
    return {"bytes": by + c["states"] * c["V"] / 8.0, "flops": 6.0 * T * c["V"]}


# ---------------------------------------------------------------------------------------------------
# the same in 64 bits, on the host where the work is small in number and on the GPU where it is large
# ---------------------------------------------------------------------------------------------------
def _exact_append(c, seed):
    s = _prepare_append(c, seed)
    half, page = c["hd"] // 2, c["page"]
    ang = s.pos.double()[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV),
                                              -torch.arange(half, device=DEV, dtype=torch.float64) / half)
    turn = torch.polar(torch.ones_like(ang), ang)[:, None, :]
    x = s.qkv.double().reshape(s.T, -1, c["hd"])
    nr = c["H"] + c["Hkv"]
    z = torch.complex(x[:, :nr, :half].contiguous(), x[:, :nr, half:].contiguous()) * turn
    y = torch.cat([z.real, z.imag], 2)
    k, v = s.k.double(), s.v.double()
    k[s.slot // page, s.slot % page] = y[:, c["H"]:]
    v[s.slot // page, s.slot % page] = x[:, nr:]
    return {"q": y[:, :c["H"]], "k": k, "v": v}


def _exact_attn(c, seed):
    s = _prepare_attn(c, seed)
    out, off, G = torch.empty(s.q.shape, dtype=torch.float64, device=DEV), _offsets(s.q_host), c["H"] // c["Hkv"]
    bits = _parents(c, s.q_host)[1] if c["levels"] else None
    table = s.table.cpu().numpy()
    for b in range(c["n"]):
        L, ctx = int(s.q_host[b]), int(s.ctx_host[b])
        at = np.arange(ctx + L)
        page, row = torch.from_numpy(table[b, at // c["page"]].astype(np.int64)).to(DEV), torch.from_numpy(at % c["page"]).to(DEV)
        hide = torch.zeros(L, ctx + L, dtype=torch.float64, device=DEV)
        own_bits = torch.from_numpy(bits[b]).to(DEV) if bits else torch.ones(L, L, device=DEV).tril() > 0
        hide[:, ctx:].masked_fill_(~own_bits, NEG)
        for h in range(c["H"]):
            k, v = s.k[page, row, h // G].double(), s.v[page, row, h // G].double()
            score = s.q[off[b]:off[b + 1], h].double() @ k.T / math.sqrt(c["hd"]) + hide
            out[off[b]:off[b + 1], h] = torch.softmax(score, 1) @ v
    return out


def _exact_logits(c, seed):
    s = _prepare_logits(c, seed)
    host = {k: v.cpu().numpy() for k, v in vars(s).items() if torch.is_tensor(v) and k != "logits"}
    out = torch.empty(s.R, c["V"], dtype=torch.float64, device=DEV)
    bits = _parents(c, s.q_host)[1] if c["levels"] else None
    row = 0
    for b in range(c["n"]):
        h = host["hist"][host["hist_off"][b]:host["hist_off"][b + 1]]
        p = int(host["prompt_len"][b])
        base_seen, base = np.zeros(c["V"], bool), np.zeros(c["V"])
        base_seen[h] = True
        np.add.at(base, h[p:], 1.0)
        bias = np.zeros(c["V"])
        if "bias_off" in host:
            sl = slice(host["bias_off"][b], host["bias_off"][b + 1])
            bias[host["bias_tok"][sl]] = host["bias_val"][sl]
        bias, base, base_seen = torch.from_numpy(bias).to(DEV), torch.from_numpy(base).to(DEV), torch.from_numpy(base_seen).to(DEV)
        for i in range(int(s.q_host[b])):
            seen, count = base_seen, base
            if bits:
                path = s.tree_tok[int(host["cu_q"][b]) + torch.from_numpy(np.nonzero(bits[b][i])[0]).to(DEV)].long()
                seen, count = seen.clone(), count.clone()
                seen[path] = True
                count.index_put_((path,), torch.ones(path.numel(), dtype=torch.float64, device=DEV), accumulate=True)
            x = s.logits[row].double()
            rp = float(host["repetition"][b])
            x = torch.where(seen, torch.where(x > 0, x / rp, x * rp), x)
            x = x - float(host["frequency"][b]) * count - float(host["presence"][b]) * (count > 0).double() + bias
            if "state" in host and host["state"][row] >= 0:
                words = host["grammar"][host["state"][row]].view(np.uint8)
                allowed = torch.from_numpy(np.unpackbits(words, bitorder="little")[:c["V"]].astype(bool)).to(DEV)
                x = x.masked_fill(~allowed, NEG)
            out[row] = x / float(host["temperature"][b])
            row += 1
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None
    if c["kind"] == "append":
        return _exact_append(c, seed)
    if c["kind"] == "attn":
        # (many small products: one for each request and head)
        return _exact_attn(c, seed) if work(c)["flops"] < 2e12 and c["n"] * c["H"] < 20000 else None
    return _exact_logits(c, seed)
