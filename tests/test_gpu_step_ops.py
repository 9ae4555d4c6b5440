"""The batched serving step's operators (plan, cache append, tree attention, logit rules) against plain
implementations in 64 bits or whole numbers, through the C ABI."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
NEG = float("-inf")


@pytest.fixture(scope="module")
def ats():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2410_05165_gb300 as m
    return m


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def _np64(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------------------------------
# plan
# ---------------------------------------------------------------------------------------------------
def _plan_reference(q, kv, table, free, n_free, page, T, parent, words):
    n, width = table.shape
    table = table.copy()
    cu, ctx, state = [0], [], []
    req, pos, slot = np.full(T, -1), np.zeros(T, np.int64), np.full(T, -1, np.int64)
    mask = np.zeros((T, words * 32), np.uint8)
    upto = used = taken = first = 0
    for b in range(n):
        L = max(0, q[b])
        need, have = -(-(kv[b] + L) // page), -(-kv[b] // page)
        limit = q[b] < 0 or kv[b] < 0 or need > width or first + L > T or (parent is not None and L > 32 * words)
        new = 0 if limit else need - have
        ok = not limit and (new == 0 or upto + new <= n_free)
        if ok and new:
            table[b, have:need] = free[upto:upto + new]
            used = upto + new
        upto += new
        if ok:
            taken = upto
        state.append(2 if limit else 0 if ok else 1)
        ctx.append(kv[b] if ok else -1)
        for i in range(L):
            t = first + i
            if t >= T:
                break
            req[t] = b
            depth = i
            if parent is not None:
                seen, node = [], i
                end = min(min(T, first + L) - min(T, first), 32 * words)
                while 0 <= node < end and len(seen) < end:
                    seen.append(node)
                    mask[t, node] = 1
                    node = parent[first + node]
                depth = max(0, len(seen) - 1)
            pos[t] = kv[b] + depth
            if ok:
                slot[t] = int(table[b, (kv[b] + i) // page]) * page + (kv[b] + i) % page
        first += L
        cu.append(min(T, first))
    bits = np.packbits(mask, axis=1, bitorder="little").view(np.int32) if words else None
    return dict(table=table, cu_q=cu, ctx_len=ctx, state=state, req=req, pos=pos, slot=slot, mask=bits, used=used, taken=taken)


def _check_plan(ats, q, kv, page, width, n_free, T, parent=None, words=0, seed=0):
    rng = np.random.default_rng(seed)
    n = len(q)
    order = rng.permutation(n * width + n_free + 1).astype(np.int32)
    table = np.full((n, width), -7, np.int32)
    for b in range(n):
        have = min(width, max(0, -(-kv[b] // page)))
        table[b, :have] = order[-1 - b * width - np.arange(have)]
    free = order[:max(1, n_free)]
    ref = _plan_reference(q, kv, table, free, n_free, page, T, parent, words)
    tb = _dev(table)
    p = ats.op_batch_plan(_dev(q), _dev(kv), tb, _dev(free), _dev([n_free]), page, T,
                          parent=None if parent is None else _dev(parent), mask_words=words)
    for k in ("cu_q", "ctx_len", "state", "req", "pos", "slot", "used", "taken"):
        np.testing.assert_array_equal(getattr(p, k).cpu().numpy(), ref[k], err_msg=k)
    np.testing.assert_array_equal(tb.cpu().numpy(), ref["table"])
    if words:
        np.testing.assert_array_equal(p.mask.cpu().numpy(), ref["mask"])
    # (a second call finds the table extended and writes the same)
    p2 = ats.op_batch_plan(_dev(q), _dev(kv), tb, _dev(free), _dev([n_free]), page, T,
                           parent=None if parent is None else _dev(parent), mask_words=words)
    np.testing.assert_array_equal(p2.slot.cpu().numpy(), ref["slot"])


def _tree(rng, m, p_root=0.1):
    return np.array([-1 if i == 0 or rng.random() < p_root else rng.integers(0, i) for i in range(m)], np.int32)


@pytest.mark.parametrize("n,page,spare", [(1, 16, 4), (7, 64, 100), (300, 16, 40), (1021, 32, 5000), (5000, 16, 9000)])
def test_plan_chains(ats, n, page, spare):
    rng = np.random.default_rng(n)
    q, kv = rng.integers(0, 40, size=n), rng.integers(0, 300, size=n)
    kv[rng.random(n) < 0.3] //= page
    kv[rng.random(n) < 0.3] *= 0
    width = int((-(-(kv + q) // page)).max()) + 1
    _check_plan(ats, q, kv, page, width, spare, int(max(1, q.sum())) + 5, seed=n)


@pytest.mark.parametrize("sizes,words", [([1], 1), ([240, 0, 31, 32, 33], 8), ([100] * 40, 4), ([1500, 3, 4096], 128)])
def test_plan_trees(ats, sizes, words):
    rng = np.random.default_rng(len(sizes) + words)
    parent = np.concatenate([_tree(rng, m) for m in sizes])
    kv = rng.integers(0, 1000, size=len(sizes))
    _check_plan(ats, np.array(sizes), kv, 64, 90, 400, sum(sizes), parent, words)


def test_plan_deep_chain_and_odd_parents(ats):
    """A chain of 200 nodes, parents out of range (roots), parents that come later, and a cycle (it ends)."""
    chain = np.arange(-1, 199)
    odd = np.array([5, -9, 77, 2, 3, 1])
    cycle = np.array([1, 2, 0])
    _check_plan(ats, np.array([200, 6, 3]), np.array([10, 0, 64]), 16, 40, 100, 209, np.concatenate([chain, odd, cycle]), 7)


def test_plan_limits(ats):
    """Negative lengths, too narrow a table, tokens past the rows given or past the mask, no free page at all."""
    _check_plan(ats, np.array([3, -1, 5, 100, 2, 0]), np.array([4, 9, -2, 30, 16, 7]), 16, 3, 50, 200)
    _check_plan(ats, np.array([10, 10, 10, 0]), np.array([0, 5, 5, 5]), 16, 3, 50, 17)
    _check_plan(ats, np.array([33, 32]), np.array([0, 5]), 16, 9, 50, 65, np.full(65, -1), 1)
    _check_plan(ats, np.array([1, 1, 1]), np.array([16, 15, 32]), 16, 9, 0, 3)


# ---------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f16": (torch.float16, torch.float16),
         "mixed": (torch.bfloat16, torch.float16)}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # unit roundoff: 8 and 11 significant bits


def _cache(types, pages, page, heads, hd, layout="token", seed=0, fill=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for t in TYPES[types]:
        shape = (pages, heads, page, hd) if layout == "head" else (pages, page, heads, hd)
        x = torch.randn(shape, generator=g, device="cuda").to(t) if fill is None else torch.full(shape, fill, device="cuda",
                                                                                               dtype=t)
        out.append(x.transpose(1, 2) if layout == "head" else x)
    return out


@pytest.mark.parametrize("T,H,Hkv,hd,page,types,src,layout,theta", [
    (1, 4, 4, 32, 16, "bf16", "f32", "token", 10000.0), (10, 12, 12, 64, 64, "mixed", "f32", "token", 10000.0),
    (37, 32, 8, 128, 16, "f16", "same", "head", 500000.0), (200, 0, 1, 128, 64, "bf16", "same", "token", 10000.0),
    (5, 3, 1, 48, 8, "bf16", "f32", "head", 2.0), (5, 2, 2, 256, 32, "mixed", "same", "token", 0.5)])
def test_rope_append(ats, T, H, Hkv, hd, page, types, src, layout, theta):
    rng = np.random.default_rng(T + hd)
    pages = T // page + 3
    kc, vc = _cache(types, pages, page, Hkv, hd, layout, seed=T)
    slot = rng.permutation(pages * page)[:T].astype(np.int64)
    slot[::7] = -1
    slot[3::11] = pages * page + 5
    pos = rng.integers(0, 1 << 20, size=T).astype(np.int32)
    pos[0] = 0
    wide = torch.randn(T, (H + 2 * Hkv) * hd + 16, device="cuda").to(torch.float32 if src == "f32" else kc.dtype)
    qkv = wide[:, 8:8 + (H + 2 * Hkv) * hd]   # rows that are not contiguous
    k_ref, v_ref = _np64(kc), _np64(vc)
    for rotate in (True, False):
        q = ats.op_rope_append(qkv, H, kc, vc, _dev(slot, torch.int64), pos=_dev(pos) if rotate else None, theta=theta)
        x = _np64(qkv).reshape(T, -1, hd)
        half = hd // 2
        ang = (pos[:, None] * float(np.float32(theta)) ** (-np.arange(half) / half))[:, None, :] * rotate
        y = np.concatenate([x[..., :half] * np.cos(ang) - x[..., half:] * np.sin(ang),
                            x[..., half:] * np.cos(ang) + x[..., :half] * np.sin(ang)], 2)
        y[:, H + Hkv:] = x[:, H + Hkv:]
        mag = np.concatenate([np.abs(x[..., :half]) + np.abs(x[..., half:])] * 2, 2)
        for t in range(T):
            if 0 <= slot[t] < pages * page:
                k_ref[slot[t] // page, slot[t] % page], v_ref[slot[t] // page, slot[t] % page] = y[t, H:H + Hkv], y[t, H + Hkv:]
        # one rounding (its unit, and half the least subnormal of fp16), and the angle: 2^-25 half turns from its 32 bits,
        # a few 2^-24 of the values
        bound = np.zeros(k_ref.shape)
        for t in range(T):
            if 0 <= slot[t] < pages * page:
                bound[slot[t] // page, slot[t] % page] = mag[t, H:H + Hkv]
        assert np.all(np.abs(_np64(q) - y[:, :H]) <= UNIT[kc.dtype] * np.abs(y[:, :H]) + 1e-6 * mag[:, :H] + 3e-8)
        assert np.all(np.abs(_np64(kc) - k_ref) <= UNIT[kc.dtype] * np.abs(k_ref) + 1e-6 * bound + 3e-8)
        assert np.all(np.abs(_np64(vc) - v_ref) <= UNIT[vc.dtype] * np.abs(v_ref) + 3e-8)
        k_ref, v_ref = _np64(kc), _np64(vc)


# ---------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------
def _attention_reference(q, k, v, see, scale):
    """q [L][H][hd], k / v [S][Hkv][hd], see [L][S] in 64 bits -> out, sum of weight x |v|, log-sum-exp."""
    L, H, hd = q.shape
    G = H // k.shape[1]
    out, mag, lse = np.zeros(q.shape), np.zeros(q.shape), np.full((L, H), NEG)
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        s = q[:, h] @ np.where(see.any(0)[:, None], kk, 0.0).T * scale
        for i in range(L):
            on = see[i]
            if not on.any():
                continue
            si = s[i, on]
            w = np.exp(si - si.max())
            lse[i, h] = si.max() + np.log(w.sum())
            w /= w.sum()
            out[i, h], mag[i, h] = w @ vv[on], w @ np.abs(vv[on])
    return out, mag, lse


def _attention_case(ats, q_len, ctx, H, Hkv, hd, page, types="bf16", layout="token", tree=None, scale=None, poison=True, seed=0,
                    q_std=1.0, stream=None):
    """Random pages in random order; every cache row that no token of its request may see holds a NaN or an infinity
    (poison), the rows of the step's own tokens too where the mask hides them from all."""
    rng = np.random.default_rng(seed)
    n, T = len(q_len), int(np.sum(q_len))
    need = [-(-(max(0, c) + m) // page) for c, m in zip(ctx, q_len)]
    pages = sum(need) + 3
    order = rng.permutation(pages)
    table = np.full((n, max(need) + 1), -1, np.int32)
    at = 0
    for b in range(n):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    kc, vc = _cache(types, pages, page, Hkv, hd, layout, seed=seed)
    seen_rows = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    cu = np.concatenate([[0], np.cumsum(q_len)])
    sees, mask = [], None
    words = max(1, -(-int(max(q_len)) // 32))
    bits = np.zeros((T, words * 32), np.uint8)
    for b in range(n):
        L, c = q_len[b], max(0, ctx[b])
        see = np.zeros((L, c + L), bool)
        if ctx[b] >= 0:
            see[:, :c] = True
            see[:, c:] = np.tril(np.ones((L, L), bool)) if tree is None else tree(rng, L)
        bits[cu[b]:cu[b + 1], :L] = see[:, c:]
        sees.append(see)
        for p in np.nonzero(see.any(0))[0]:
            seen_rows[table[b, p // page], p % page] = True
    if poison:
        for x in (kc, vc):
            x[~seen_rows] = float("nan")
            idx = torch.nonzero(~seen_rows)[::2]
            x[idx[:, 0], idx[:, 1]] = float("inf")
    if tree is not None:
        mask = _dev(np.packbits(bits, axis=1, bitorder="little").view(np.int32))
    q = (torch.randn(T, H, hd, device="cuda") * q_std).to(kc.dtype)
    lse = torch.full((T, H), 7.0, device="cuda")
    args = (q, kc, vc, _dev(cu), _dev(ctx), _dev(table))
    torch.cuda.synchronize()
    out = ats.op_tree_attention(*args, mask=mask, scale=scale, lse=lse, stream=stream)
    torch.cuda.synchronize()
    assert ats.op_status(noalloc=True) == 0
    again = ats.op_tree_attention(*args, mask=mask, scale=scale, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))   # the same call, the same bits
    K, V, Q, O, S = _np64(kc), _np64(vc), _np64(q), _np64(out), lse.cpu().numpy()
    for b in range(n):
        L, c = q_len[b], max(0, ctx[b])
        rows = np.arange(c + L)
        k, v = K[table[b, rows // page], rows % page], V[table[b, rows // page], rows % page]
        sl = slice(cu[b], cu[b + 1])
        ref, mag, ls = _attention_reference(Q[sl], k, v, sees[b], hd ** -0.5 if scale is None else scale)
        # weights rounded to V's type, the result to q's, scores from sums of hd products and exponentials in 32 bits
        tol = UNIT[kc.dtype] * np.abs(ref) + (UNIT[vc.dtype] + 1e-4) * mag + 1e-6
        err = np.abs(O[sl] - ref)
        assert np.all(err <= tol), (b, L, c, np.nanmax(err - tol), np.isnan(err).sum())
        hidden = np.isinf(ls)
        assert np.all(S[sl][hidden] == NEG) and np.all(O[sl][hidden] == 0)
        assert np.all(np.abs(S[sl][~hidden] - ls[~hidden]) <= 1e-4 * (1 + np.abs(ls[~hidden])))


def _drafted(rng, L):
    see = np.eye(L, dtype=bool)
    for i, p in enumerate(_tree(rng, L)):
        if p >= 0:
            see[i] |= see[p]
    return see


def _any_bits(rng, L):
    """Bits of no tree: later tokens, rows without a single one."""
    see = rng.random((L, L)) < 0.3
    see[rng.random(L) < 0.3] = False
    return see


@pytest.mark.parametrize("H,Hkv,hd,page,types,layout", [
    (4, 4, 32, 16, "bf16", "token"), (12, 12, 64, 64, "mixed", "token"), (8, 2, 128, 16, "f16", "head"),
    (8, 1, 128, 256, "bf16", "token"), (6, 2, 64, 128, "f16", "token"), (7, 1, 32, 32, "mixed", "head"),
    (32, 32, 128, 64, "mixed", "token")])
@pytest.mark.parametrize("tree", [None, _drafted, _any_bits])
def test_tree_attention_batch(ats, H, Hkv, hd, page, types, layout, tree):
    """Ragged batches: no cached token, one, ends inside and at the end of pages and key tiles; no new token, one, many;
    a request that was not served; small and large groups."""
    _attention_case(ats, [1, 5, 0, 33, 2, 1, 70], [0, 1, 17, 300, -1, 127, 128], H, Hkv, hd, page, types, layout, tree, seed=hd + H)


@pytest.mark.parametrize("q_len,ctx", [([1], [0]), ([1], [1000]), ([1] * 40, list(range(0, 400, 10))), ([130], [0]), ([129, 1], [64, 2000]),
                                       ([257], [31]), ([128], [128]), ([1, 300], [5000, 0]), ([600], [700])])
@pytest.mark.parametrize("tree", [None, _drafted])
def test_tree_attention_lengths(ats, q_len, ctx, tree):
    _attention_case(ats, q_len, ctx, 4, 2, 64, 16, "bf16", "token", tree, seed=len(q_len) + q_len[0])


@pytest.mark.parametrize("q_len,ctx,H,hd,page", [([1] * 12, [11000 + 37 * i for i in range(12)], 4, 128, 64),
                                                  ([1] * 19, [9000 - 100 * i for i in range(19)], 8, 64, 16),
                                                  ([150] * 12, [4000 + 64 * i for i in range(12)], 4, 128, 32)])
def test_tree_attention_long_ranges(ats, q_len, ctx, H, hd, page):
    """Some ten key tiles in a row for every CTA, under the memory traffic of all of them: the copies' ring goes round many
    times, on few rows (alternate tiles to two streams) and on many (every tile to both)."""
    _attention_case(ats, q_len, ctx, H, H, hd, page, "bf16", tree=_drafted, poison=False, seed=hd + page)


@pytest.mark.parametrize("q_len,ctx,H,hd,tree", [([65] * 45, [500 + 23 * i for i in range(45)], 8, 64, _drafted),
                                                  ([130, 3] * 20, [40 * i for i in range(40)], 8, 128, _drafted),
                                                  ([1] * 300, [10 * i for i in range(300)], 8, 32, None),
                                                  ([700, 900], [100, 0], 24, 64, None)])
def test_tree_attention_many_blocks(ats, q_len, ctx, H, hd, tree):
    """Several blocks a CTA, of one kind or mixed, so that ranges end at blocks' borders or next to them as well as inside; a
    causal prompt, whose blocks see their own tokens' keys in part."""
    _attention_case(ats, q_len, ctx, H, H // 4, hd, 16, "bf16", tree=tree, seed=len(q_len) + H)
    _attention_case(ats, q_len, ctx, H, H, hd, 64, "f16", tree=tree, seed=len(q_len) + hd)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 16, 127, 128])
def test_tree_attention_groups(ats, G):
    _attention_case(ats, [3, 1, 9], [200, 77, 513], 2 * G if G < 100 else G, 2 if G < 100 else 1, 32, 16, "f16", tree=_drafted, seed=G)


def test_tree_attention_large_scores(ats):
    """Scores of some hundreds: the running maximum moves far, weights vanish (q.k of 8 N(0,1) heads of 64)."""
    _attention_case(ats, [4, 40], [3000, 100], 8, 2, 64, 64, "bf16", tree=_drafted, q_std=30.0, seed=5)
    _attention_case(ats, [4, 40], [3000, 100], 8, 2, 128, 64, "f16", scale=2.0, seed=6)


def test_tree_attention_only_masked_context(ats):
    """No cached token and a mask that hides everything: zeros, and no NaN from rows never written."""
    _attention_case(ats, [5, 200], [0, 0], 4, 1, 128, 16, "bf16", tree=lambda rng, L: np.zeros((L, L), bool), seed=8)


def test_tree_attention_attended_infinity_and_nan(ats):
    """A NaN or infinity in V reaches the tokens that attend to it, and no other."""
    H, hd, page, ctx, L = 4, 64, 16, 50, 20
    rng = np.random.default_rng(4)
    kc, vc = _cache("bf16", 8, page, 2, hd, seed=9)
    table = np.arange(8, dtype=np.int32)[None]
    see = _drafted(rng, L)
    bad = {3: float("nan"), 7: float("inf"), 11: NEG}
    clean = vc.clone()
    for a, x in bad.items():
        vc[(ctx + a) // page, (ctx + a) % page, 1, 5] = x
    words = np.packbits(np.pad(see, ((0, 0), (0, 12))), axis=1, bitorder="little").view(np.int32)
    q = torch.randn(L, H, hd, device="cuda").to(torch.bfloat16)
    args = (_dev([0, L]), _dev([ctx]), _dev(table))
    got = ats.op_tree_attention(q, kc, vc, *args, mask=_dev(words))
    ref = ats.op_tree_attention(q, kc, clean, *args, mask=_dev(words))
    for i in range(L):
        hit = [x for a, x in bad.items() if see[i, a]]
        want = sum(hit) if hit else None
        for h in (2, 3):   # the heads of key head 1
            x = float(got[i, h, 5])
            if want is None:
                assert x == float(ref[i, h, 5])
            else:
                assert (np.isnan(want) and np.isnan(x)) or x == want, (i, h, x, want)
    keep = torch.ones(H, hd, dtype=torch.bool, device="cuda")
    keep[2:, 5] = False
    assert torch.equal(got[:, keep], ref[:, keep])


@pytest.mark.parametrize("G,hd", [(2, 64), (8, 128), (1, 32)])
def test_causal_attention_of_infinity_and_nan(ats, G, hd):
    """The same in a causal call of several blocks: from the token on whose value it is, and not before."""
    H, page, ctx, L = 2 * G, 16, 70, 300
    kc, vc = _cache("bf16", 24, page, 2, hd, seed=12)
    clean = vc.clone()
    bad = {0: (0, float("inf")), 3: (1, float("nan")), 127: (2, NEG), 128: (3, float("nan")), 150: (4, float("inf")),
           299: (5, float("nan"))}
    for a, (c, x) in bad.items():
        vc[(ctx + a) // page, (ctx + a) % page, 1, c] = x
    q = torch.randn(L, H, hd, device="cuda").to(torch.bfloat16)
    args = (_dev([0, L]), _dev([ctx]), _dev(np.arange(24, dtype=np.int32)[None]))
    got = ats.op_tree_attention(q, kc, vc, *args)
    ref = ats.op_tree_attention(q, kc, clean, *args)
    for a, (c, x) in bad.items():
        assert torch.equal(got[:a, G:, c], ref[:a, G:, c])
        after = got[a:, G:, c].float()
        assert bool(torch.isnan(after).all()) if np.isnan(x) else bool((after == x).all())
    assert torch.equal(got[:, :G], ref[:, :G]) and torch.equal(got[:, G:, 6:], ref[:, G:, 6:])


def test_tree_attention_strides_streams_and_shared_pages(ats):
    """q and out as slices of wider rows, two requests over the same prefix pages, a stream of the caller's."""
    H, Hkv, hd, page = 8, 2, 64, 32
    kc, vc = _cache("mixed", 20, page, Hkv, hd, seed=3)
    table = np.array([[0, 1, 2, 3, 4, 5], [0, 1, 2, 9, 8, 7]], np.int32)
    ctx, q_len = [100, 130], [9, 17]
    wide = torch.randn(26, 2 * H * hd + 24, device="cuda").to(torch.bfloat16)
    q = wide[:, 16:16 + H * hd].unflatten(1, (H, hd))
    out = wide[:, 24 + H * hd:].unflatten(1, (H, hd))
    before = wide[:, :24 + H * hd].clone()
    s = torch.cuda.Stream()
    args = (_dev([0, 9, 26]), _dev(ctx), _dev(table))
    torch.cuda.synchronize()
    ats.op_tree_attention(q, kc, vc, *args, out=out, stream=s)
    s.synchronize()
    assert torch.equal(before, wide[:, :24 + H * hd])
    K, V, Q, O = _np64(kc), _np64(vc), _np64(q), _np64(out)
    for b, sl in enumerate((slice(0, 9), slice(9, 26))):
        rows = np.arange(ctx[b] + q_len[b])
        k, v = K[table[b, rows // page], rows % page], V[table[b, rows // page], rows % page]
        see = np.concatenate([np.ones((q_len[b], ctx[b]), bool), np.tril(np.ones((q_len[b],) * 2, bool))], 1)
        ref, mag, _ = _attention_reference(Q[sl], k, v, see, hd ** -0.5)
        assert np.all(np.abs(O[sl] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 1e-4) * mag + 1e-6)


def test_tree_attention_offsets_past_32_bits(ats):
    """Pages that start past 2^32 elements of a cache of 8.6 GB per tensor."""
    heads, hd, page = 8, 128, 64
    pages = (1 << 32) // (page * heads * hd) + 40
    kc = torch.empty(pages, page, heads, hd, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    use = np.array([pages - 1, 5, pages - 20, 33000], np.int64)
    for p in use:
        kc[p], vc[p] = torch.randn(2, page, heads, hd, device="cuda").to(torch.bfloat16)
    q = torch.randn(3, heads, hd, device="cuda").to(torch.bfloat16)
    out = ats.op_tree_attention(q, kc, vc, _dev([0, 3]), _dev([200]), _dev(use[None]))
    ix = torch.from_numpy(use).cuda()
    k, v = _np64(kc[ix]).reshape(-1, heads, hd)[:203], _np64(vc[ix]).reshape(-1, heads, hd)[:203]
    see = np.concatenate([np.ones((3, 200), bool), np.tril(np.ones((3, 3), bool))], 1)
    ref, mag, _ = _attention_reference(_np64(q), k, v, see, hd ** -0.5)
    assert np.all(np.abs(_np64(out) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-4) * mag + 1e-6)
    slot = torch.tensor([(pages - 3) * page + 7], dtype=torch.int64, device="cuda")
    qkv = torch.randn(1, 3 * heads * hd, device="cuda")
    ats.op_rope_append(qkv, heads, kc, vc, slot)
    assert torch.equal(kc[pages - 3, 7].flatten(), qkv[0, heads * hd:2 * heads * hd].to(torch.bfloat16))
    assert torch.equal(vc[pages - 3, 7].flatten(), qkv[0, 2 * heads * hd:].to(torch.bfloat16))


def test_tree_attention_in_a_graph(ats):
    """Captured once, replayed over other lengths, tables and values."""
    H, Hkv, hd, page = 8, 2, 64, 16
    kc, vc = _cache("bf16", 300, page, Hkv, hd, seed=12)
    table = _dev(np.random.default_rng(0).permutation(300).reshape(3, 100))
    cu, ctx = _dev([0, 1, 2, 3]), _dev([10, 20, 30])
    q = torch.randn(3, H, hd, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ats.op_tree_attention(q, kc, vc, cu, ctx, table, out=out)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ats.op_tree_attention(q, kc, vc, cu, ctx, table, out=out)
    for lens in ([1500, 3, 0], [7, 700, 1598]):
        ctx.copy_(_dev(lens))
        q.copy_(torch.randn(3, H, hd, device="cuda"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = ats.op_tree_attention(q, kc, vc, cu, ctx, table)
        assert torch.equal(out, want)


def test_tree_attention_in_a_graph_of_another_stream(ats):
    """Captured on a stream that the attention was never called on, and replayed on the caller's, twice."""
    kc, vc = _cache("bf16", 40, 16, 2, 64, seed=31)
    q = torch.randn(9, 4, 64, device="cuda").to(torch.bfloat16)
    args = (_dev([0, 1, 9]), _dev([300, 100]), _dev(np.arange(40).reshape(2, 20)))
    want = ats.op_tree_attention(q, kc, vc, *args)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        for _ in range(3):
            ats.op_tree_attention(q, kc, vc, *args, out=out)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert ats.op_status(noalloc=True) == 0


def test_a_timeout_once_read_clears_the_workspaces(ats, monkeypatch):
    """(The status is a fake's: nothing waits in vain here.)  Counters that a call left behind are cleared, on every stream."""
    from paper_2410_05165_gb300 import binding
    streams = [torch.cuda.current_stream(), torch.cuda.Stream()]
    spaces = [binding.op_tree_attention_workspace(torch.device("cuda", 0), s.cuda_stream) for s in streams]
    torch.cuda.synchronize()
    for w in spaces:
        w[:64] = 1
    torch.cuda.synchronize()

    class Failed:
        @staticmethod
        def atspeed_op_status(stream, ws):
            return binding.E_TIMEOUT

    with monkeypatch.context() as m:
        m.setattr(binding, "load", lambda: Failed)
        assert binding.op_status(noalloc=True) == binding.E_TIMEOUT
    torch.cuda.synchronize()
    assert all(int(w[:binding.TREE_ATTENTION_COUNTER_BYTES].sum()) == 0 for w in spaces)


def test_step_ops_refuse_wrong_tensors(ats):
    kc, vc = _cache("bf16", 4, 16, 2, 64)
    q = torch.zeros(3, 4, 64, device="cuda", dtype=torch.bfloat16)
    cu, ctx, table = _dev([0, 3]), _dev([5]), _dev([[0, 1]])
    ok = ats.op_tree_attention(q, kc, vc, cu, ctx, table)
    assert ok.shape == q.shape
    for bad in ((q.half(), kc, vc, cu, ctx, table), (q[:, :3], kc, vc, cu, ctx, table), (q, kc, vc[:3], cu, ctx, table),
                (q, kc, vc, cu[:1], ctx, table), (q, kc, vc, cu.long(), ctx, table), (q, kc, vc, cu, ctx, table[0]),
                (q.cpu(), kc, vc, cu, ctx, table), (q, kc[..., ::2], vc[..., ::2], cu, ctx, table)):
        with pytest.raises(ats.AtSpeedError) as e:
            ats.op_tree_attention(*bad)
        assert e.value.status in (ats.E_ARG, ats.E_SHAPE)
    with pytest.raises(ats.AtSpeedError):
        ats.op_tree_attention(q, kc, vc, cu, ctx, table, mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ats.AtSpeedError):
        ats.op_rope_append(torch.zeros(3, 7 * 64, device="cuda"), 4, kc, vc, torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ats.AtSpeedError):
        ats.op_batch_plan(_dev([1, 1]), _dev([1]), table, _dev([0]), _dev([1]), 16, 2)
    with pytest.raises(ats.AtSpeedError):
        ats.op_adjust_logits(torch.zeros(3, 10, device="cuda"), _dev([0]), ats.LogitRules(n_req=1))
    with pytest.raises(ats.AtSpeedError):
        ats.LogitRules(n_req=2, repetition=torch.ones(1, device="cuda"))


# ---------------------------------------------------------------------------------------------------
# logits
# ---------------------------------------------------------------------------------------------------
def _logits_reference(x, req, d, mask, state):
    out = x.astype(np.float64)
    R, V = x.shape
    n = d["n_req"]
    for r in range(R):
        b, y = req[r], out[r]
        if 0 <= b < n:
            count, seen = np.zeros(V), np.zeros(V, bool)
            toks = []
            if "hist" in d:
                h = d["hist"][d["hist_off"][b]:d["hist_off"][b + 1]]
                p = d["prompt_len"][b] if "prompt_len" in d else 0
                toks = list(h[p:])
                for v in h[:p]:
                    if 0 <= v < V:
                        seen[v] = True
            if mask is not None:
                t0, t1 = d["cu_q"][b], d["cu_q"][b + 1]
                toks += [d["tree_tok"][t0 + a] for a in range(min(t1 - t0, mask.shape[1])) if mask[r, a]]
            for v in toks:
                if 0 <= v < V:
                    count[v] += 1
                    seen[v] = True
            if "repetition" in d:
                rp = float(d["repetition"][b])
                with np.errstate(all="ignore"):
                    y = np.where(seen, np.where(y > 0, y / rp, y * rp), y)
            y = y - float(d["frequency"][b] if "frequency" in d else 0) * count
            y = y - float(d["presence"][b] if "presence" in d else 0) * (count > 0)
            if "bias_off" in d:
                last = {}
                for k in range(d["bias_off"][b], d["bias_off"][b + 1]):
                    last[d["bias_tok"][k]] = d["bias_val"][k]
                for v, w in last.items():
                    if 0 <= v < V:
                        y[v] += w
        if state is not None and state[r] >= 0:
            w = np.unpackbits(d["grammar"][state[r]].view(np.uint8), bitorder="little")[:V]
            y = np.where(w > 0, y, NEG)
        if 0 <= b < n and "temperature" in d and d["temperature"][b] > 0:
            y = y / float(d["temperature"][b])
        out[r] = y
    return out


def _logits_case(ats, V, q_len, hist_max, inp, out_dtype, seed, leave=(), tree=True, stride=0, inplace=False):
    rng = np.random.default_rng(seed)
    n, R = len(q_len), int(np.sum(q_len))
    hist_len = rng.integers(0, hist_max + 1, size=n)
    d = dict(n_req=n, hist_off=np.concatenate([[0], np.cumsum(hist_len)]).astype(np.int32),
             hist=rng.integers(-2, (V if hist_max > 4000 else min(V, 60)) + 2, size=max(1, hist_len.sum())).astype(np.int32),
             prompt_len=(hist_len * rng.random(n)).astype(np.int32), repetition=rng.uniform(0.8, 1.6, n).astype(np.float32),
             frequency=rng.uniform(-0.5, 1.0, n).astype(np.float32), presence=rng.uniform(-0.5, 1.0, n).astype(np.float32),
             temperature=np.where(rng.random(n) < 0.3, 0.0, rng.uniform(0.5, 2.0, n)).astype(np.float32))
    nb = rng.integers(0, 30, size=n)
    d.update(bias_off=np.concatenate([[0], np.cumsum(nb)]).astype(np.int32),
             bias_tok=rng.integers(-1, V + 1, size=max(1, nb.sum())).astype(np.int32),
             bias_val=rng.normal(0, 4, size=max(1, nb.sum())).astype(np.float32))
    words = -(-V // 32)
    grammar = (rng.random((3, words * 32)) < 0.5).astype(np.uint8)
    grammar[1] = 0
    d["grammar"] = np.packbits(grammar, axis=1, bitorder="little").view(np.int32)
    state = rng.integers(-1, 3, size=R)
    req = np.repeat(np.arange(n), q_len)
    req[rng.random(R) < 0.1] = -1
    mask = None
    if tree:
        d["cu_q"] = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
        d["tree_tok"] = rng.integers(0, min(V, 60), size=R).astype(np.int32)
        mask = rng.random((R, 32 * max(1, -(-max(q_len) // 32)))) < 0.2
    for k in leave:
        d.pop(k, None)
    if "grammar" in leave:
        state = None
    x = torch.randn(R, V + stride, device="cuda").mul_(3).to(inp)[:, :V]
    x[0, 0], x[0, V - 1] = NEG, float("inf")
    given = {k: _dev(v, torch.float32 if v.dtype == np.float32 else torch.int32) for k, v in d.items() if k != "n_req"}
    rules = ats.LogitRules(n_req=n, **given)
    before = x.clone()
    got = ats.op_adjust_logits(x, _dev(req), rules,
                               mask=None if mask is None else _dev(np.packbits(mask, axis=1, bitorder="little").view(np.int32)),
                               state=None if state is None else _dev(state), out=x if inplace else None,
                               out_dtype=None if inplace else out_dtype)
    ref = _logits_reference(_np64(before), req, d, mask, state)
    g = _np64(got)
    if not inplace:
        assert torch.equal(before, x)
    fin = np.isfinite(ref)
    np.testing.assert_array_equal(g[~fin], ref[~fin])
    # five operations in 32 bits on terms of up to |x| + 40 (counts x frequency, biases), then one rounding to 16 bits
    unit = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[got.dtype]
    scale = np.abs(ref) + np.abs(np.where(np.isfinite(_np64(before)), _np64(before), 0)) + 40.0
    assert np.all(np.abs(g[fin] - ref[fin]) <= unit * np.abs(ref[fin]) + 2.0 ** -20 * scale[fin])


@pytest.mark.parametrize("V,q_len,hist", [(100, [1], 10), (33024, [1, 30, 7], 700), (8191, [3, 3], 100), (8193, [40], 50),
                                          (1, [2], 3), (20011, [5, 1, 64, 33], 3000)])
@pytest.mark.parametrize("inp,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                     (torch.float16, torch.float16), (torch.float16, torch.float32)])
def test_adjust_logits(ats, V, q_len, hist, inp, out):
    _logits_case(ats, V, q_len, hist, inp, out, seed=V + len(q_len))


@pytest.mark.parametrize("leave", [("hist", "hist_off", "prompt_len"), ("bias_off", "bias_tok", "bias_val"), ("grammar",), ("repetition",),
                                   ("frequency", "presence"), ("temperature",), ("prompt_len",)])
def test_adjust_logits_rules_left_out(ats, leave):
    _logits_case(ats, 9001, [4, 9], 300, torch.float32, torch.float32, 17, leave=leave)


@pytest.mark.parametrize("stride,inplace", [(1, False), (7, True), (8, True), (0, True)])
def test_adjust_logits_strides_and_in_place(ats, stride, inplace):
    _logits_case(ats, 9000, [4, 9], 300, torch.bfloat16, torch.bfloat16, 18, stride=stride, inplace=inplace)
    _logits_case(ats, 9001, [4, 9], 300, torch.float32, torch.float32, 19, stride=stride, inplace=inplace, tree=False)


@pytest.mark.parametrize("inplace", [False, True])
def test_adjust_logits_long_lists_and_paths(ats, inplace):
    """Histories that touch most of the vocabulary (lists longer than a CTA), paths of hundreds of tokens, rows of one
    request and of others in turn."""
    _logits_case(ats, 5003, [300, 1, 17], 9000, torch.float32, torch.float32, 23, inplace=inplace)
    _logits_case(ats, 60, [520, 2], 100, torch.float16, torch.float16, 24, inplace=inplace)


def test_adjust_logits_forbids_nan_and_keeps_the_rest(ats):
    """A forbidden token is -infinity whatever its logit was; a row whose state allows nothing is -infinity throughout."""
    x = torch.full((2, 70), float("nan"), device="cuda")
    grammar = np.zeros((2, 3), np.int32)
    grammar[0, 0] = 6
    got = ats.op_adjust_logits(x, _dev([0, 0]), ats.LogitRules(n_req=1, grammar=_dev(grammar)), state=_dev([0, 1])).cpu()
    assert torch.isnan(got[0, 1:3]).all() and (got[0, 3:] == NEG).all() and got[0, 0] == NEG and (got[1] == NEG).all()
