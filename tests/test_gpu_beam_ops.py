"""Beam selection, fork of block tables, page copies and token compaction against plain implementations in 64 bits or whole
numbers, through the binding."""
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


# ---------------------------------------------------------------------------------------------------
# selection
# ---------------------------------------------------------------------------------------------------
def _log_probs(x, dtype, allowed, full):
    """[R][V] float64 logits -> log-probabilities of the allowed ones (others -inf)."""
    x = np.minimum(np.where(np.isnan(x), NEG, x), float(torch.finfo(dtype).max))
    over = x if full else np.where(allowed, x, NEG)
    m = np.maximum(over.max(axis=1, keepdims=True), -1e300)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        y = (x - m) - np.log(np.exp(over - m).sum(axis=1, keepdims=True))
    return np.where(allowed, y, NEG), x


def _select_reference(x, dtype, cu, width, score, final, allowed, full):
    lp, x = _log_probs(x, dtype, allowed, full)
    out = []
    for b in range(len(cu) - 1):
        got = []
        for r in range(cu[b], cu[b + 1]):
            if final is not None and final[r] >= 0:
                got.append(np.array([[score[r]], [r], [0.0], [final[r]]]))
                continue
            v = np.arange(x.shape[1])
            got.append(np.stack([score[r] + lp[r], np.full(v.size, r), x[r], v]))
        c = np.concatenate(got, axis=1) if got else np.zeros((4, 0))
        with np.errstate(over="ignore"):
            c = c[:, c[0].astype(np.float32) > NEG]   # (NaN is not)
        if c.shape[1] > 4 * width:   # (what is well below the last one chosen is not sorted)
            c = c[:, c[0] >= np.partition(c[0], -width)[-width] - 1e-3]
        order = np.lexsort((c[3], -c[2], c[1], -c[0]))
        out.append(c[:, order])
    return out


def _rows(logits):
    return logits.double().cpu().numpy()


def _bits(table):
    """[states][V] truth values as 32-bit words."""
    s, v = table.shape
    w = np.zeros((s, -(-v // 32) * 32), np.uint8)
    w[:, :v] = table
    return _dev(np.packbits(w, axis=1, bitorder="little").view(np.int32))


def _tolerance(V):
    """Of a score, absolute, without its own rounding.  A term e^d of a row's sum is off by 2.3 |d| 2^-24 (a difference, a product, the
    constant) and an exponential's 2 units in the last place, 2^-22; sum |d| e^d / sum e^d is at most log V; a thread's sum
    has at most V / 256 + 16 terms and the threads' sums 13 more additions of half a step, 2^-24, and a rescaling."""
    return ((V / 256 + 16) + 13 + 2.3 * np.log(V) + 4 + 2 + 4) * 2.0 ** -24


def _check_select(ats, logits, counts, width, score=None, final=None, table=None, state=None, norm="masked", exact=False, first=0):
    """exact: the places of all candidates are far enough apart, or equal, to be told by 32 bits."""
    R, V = logits.shape
    cu = first + np.concatenate([[0], np.cumsum(counts)])
    allowed = np.ones((R, V), bool)
    if table is not None:
        for r in range(R):
            if state[r] >= 0:
                allowed[r] = table[state[r]] if state[r] < len(table) else False
    sc = np.zeros(R) if score is None else np.asarray(score, np.float32).astype(np.float64)
    ref = _select_reference(_rows(logits), logits.dtype, cu, width, sc, final, allowed, norm == "full")
    kw = dict(score=None if score is None else _dev(np.asarray(score, np.float32), torch.float32),
              final=None if final is None else _dev(final), norm=ats.NORM_FULL if norm == "full" else ats.NORM_MASKED)
    if table is not None:
        kw.update(grammar=_bits(table), state=_dev(state))
    got = ats.op_beam_select(logits, _dev(cu), width, **kw)
    tok, par, out = got.token.cpu().numpy(), got.parent.cpu().numpy(), got.score.double().cpu().numpy()
    tol = _tolerance(V)
    for b, c in enumerate(ref):
        k = min(width, c.shape[1])
        assert (tok[b, k:] == -1).all() and (par[b, k:] == -1).all() and (out[b, k:] == NEG).all()
        if exact:
            np.testing.assert_array_equal(par[b, :k], c[1, :k].astype(int))
            np.testing.assert_array_equal(tok[b, :k], c[3, :k].astype(int))
        place = {(int(r), int(v)): s for s, r, _, v in c.T}
        mine = np.array([place[p, t] for p, t in zip(par[b, :k], tok[b, :k])])   # (none that may not be chosen)
        assert len(set(zip(par[b, :k], tok[b, :k]))) == k
        finite = np.isfinite(mine)
        np.testing.assert_array_equal(out[b, :k][~finite], mine[~finite])
        assert (np.abs(out[b, :k] - mine)[finite] <= tol + np.abs(mine[finite]) * 2.0 ** -24).all()
        with np.errstate(invalid="ignore"):
            assert not (np.abs(mine - c[0, :k])[finite] > 2 * tol).any()   # (places may be changed by two rows' errors alone)
    again = ats.op_beam_select(logits, _dev(cu), width, **kw)
    assert torch.equal(again.token, got.token) and torch.equal(again.parent, got.parent) and torch.equal(again.score, got.score)
    return got


def _logits(seed, R, V, dtype, std=3.0, pitch=0, lead=0):
    """Rows of V logits, V + pitch elements apart, the first `lead` elements into its memory."""
    g = torch.Generator("cuda").manual_seed(seed)
    t = torch.randn(lead + R * (V + pitch), generator=g, device="cuda") * std
    return t.to(dtype)[lead:].view(R, V + pitch)[:, :V]


TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,width", [(1, 1), (2, 3), (31, 40), (300, 10), (4095, 64), (4096, 65), (4097, 256), (8200, 100), (33024, 20)])
def test_select_sizes(ats, dtype, V, width):
    counts = [3, 0, 1, 7]
    rng = np.random.default_rng(V)
    _check_select(ats, _logits(V, 11, V, dtype), counts, width, score=-rng.exponential(2.0, 11))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pitch,lead", [(1, 0), (3, 1), (7, 5), (8, 8), (100, 2)])
def test_select_strides(ats, dtype, pitch, lead):
    V = 5003
    _check_select(ats, _logits(7, 9, V, dtype, pitch=pitch, lead=lead), [4, 5], 33, score=np.linspace(-1, -3, 9))


@pytest.mark.parametrize("R,V,width", [(1, 33024, 40), (1, 200003, 256), (1, 300007, 30), (101, 40000, 12), (150, 40001, 12), (700, 5000, 17), (2600, 700, 8)])
def test_select_one_piece_and_many(ats, R, V, width):
    counts = [R] if R == 1 else [R // 4, 1, R - R // 4 - 1]
    _check_select(ats, _logits(R, R, V, torch.float32), counts, width, score=-np.random.default_rng(R).exponential(2.0, R))


@pytest.mark.parametrize("width", [10, 70])
def test_select_one_request_of_many_beams_among_small_ones(ats, width):
    counts = [1] * 99 + [3000] + [0, 2]
    _check_select(ats, _logits(6, 3101, 300, torch.float32), counts, width, score=-np.random.default_rng(6).exponential(2.0, 3101),
                  final=np.where(np.arange(3101) % 7 == 3, 5, -1))


@pytest.mark.parametrize("norm", ["masked", "full"])
@pytest.mark.parametrize("dtype", TYPES)
def test_select_grammar(ats, norm, dtype):
    V, R = 9001, 12
    rng = np.random.default_rng(3)
    table = np.zeros((5, V), bool)
    table[0, rng.choice(V, 30, replace=False)] = True
    table[1] = ~table[0]
    table[2] = True
    table[4, [0, V - 1]] = True   # (3: nothing)
    state = np.array([-1, 0, 1, 2, 3, 4, 5, 99, 0, 4, 3, 3])
    _check_select(ats, _logits(5, R, V, dtype), [5, 5, 2], 25, score=-rng.exponential(1.0, R), table=table, state=state, norm=norm)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,V", [(761, 12289), (1500, 8193), (900, 16385), (2000, 12290)])
def test_select_more_rows_than_run_at_once(ats, dtype, R, V):
    """Rows of four tiles and more that CTAs take one after the other: ended beams, states of every kind and rows of no request among
    them, at the beginning too."""
    rng = np.random.default_rng(R)
    logits = _logits(R, R, V, dtype, pitch=R % 3)
    final = np.where(rng.random(R) < 0.3, rng.integers(0, V, size=R), -1)
    final[:5] = 3
    table = rng.random((4, V)) < np.array([0.5, 0.001, 0.0, 1.0])[:, None]
    state = rng.integers(-1, 6, size=R)
    first, last = 7, 11
    counts = [R // 3, 0, 1, R - first - last - R // 3 - 1]
    logits[:first] = float("nan")
    logits[R - last:] = float("nan")
    for kw in (dict(), dict(final=final), dict(final=final, table=table, state=state, norm="full"), dict(table=table, state=state)):
        _check_select(ats, logits, counts, 15, score=-rng.exponential(2.0, R), first=first, **kw)
    _check_select(ats, logits, counts, 15, score=-rng.exponential(2.0, R), first=first, final=np.zeros(R, int))   # (every one of them)


def test_select_ended_beams(ats):
    V, R = 5000, 8
    final = np.array([-1, 7, -1, 3, 4999, -5, 0, 1])
    score = np.array([-1.0, -2.0, -30.0, -0.5, -1.0, -1.5, -2.5, NEG], np.float32)
    logits = _logits(9, R, V, torch.float32)
    logits[1] = float("nan")   # an ended beam's logits do not count
    _check_select(ats, logits, [4, 2, 2], 12, score=score, final=final)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 31, 64, 65, 256])
def test_select_ties(ats, dtype, width):
    """Few different logits, the same in every row: equal scores, by row and token."""
    V, R = 9001, 6
    rng = np.random.default_rng(width)
    row = rng.integers(0, 3, size=V).astype(np.float32) * 4
    logits = torch.from_numpy(np.tile(row, (R, 1))).to("cuda", dtype)
    _check_select(ats, logits, [6], width, score=np.zeros(R), exact=True)
    _check_select(ats, logits, [2, 4], width, exact=True)
    const = torch.zeros(R, V, dtype=dtype, device="cuda")
    _check_select(ats, const, [6], width, exact=True)
    # (rows that begin at other places of a 16-byte word have the same sums)
    wide = torch.empty(R, V + 3, dtype=dtype, device="cuda")
    view = wide[:, 1:1 + V]
    view.copy_(logits)
    _check_select(ats, view, [6], width, exact=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fill", [NEG, "lowest"])
@pytest.mark.parametrize("few", [0, 1, 5, 400])
def test_select_masked_values(ats, dtype, fill, few):
    """Logits that a mask filled with -infinity or the type's lowest value, but for a few."""
    V, R, width = 12500, 4, 40
    rng = np.random.default_rng(few)
    low = NEG if fill == NEG else float(torch.finfo(dtype).min)
    x = np.full((R, V), low)
    for r in range(R):
        x[r, rng.choice(V, few, replace=False)] = rng.permutation(few) * 0.5   # (far apart in every type)
    logits = torch.from_numpy(x).to("cuda", dtype)
    # (scores of rows 40 apart: no two rows' candidates are near each other)
    _check_select(ats, logits, [1, 3], width, score=np.arange(R) * -401.0, exact=True)


def test_select_values_that_are_not_finite(ats):
    V = 6000
    logits = _logits(2, 5, V, torch.float32)
    logits[0, 100:200] = float("nan")
    logits[1, 17] = float("inf")
    logits[2, 5000] = logits[2, 30] = float("inf")
    logits[3] = float("nan")
    logits[4] = NEG
    logits[4, 77] = 1.0
    _check_select(ats, logits, [1, 1, 1, 1, 1], 9)
    _check_select(ats, logits, [5], 9, score=[-1, -2, -3, -4, -5])
    for dtype in (torch.bfloat16, torch.float16):
        _check_select(ats, logits.to(dtype), [5], 300 - 44, score=[-1, -2, -3, -4, -5])


@pytest.mark.parametrize("at", [1000.0, 2.0 ** 20, -2.0 ** 20, 3e6, -1e9, 1e30, -3e38])
def test_select_logits_far_out(ats, at):
    """Maxima on both sides of where sums change their units; a row's parts on both sides."""
    V = 9000
    g = torch.Generator("cuda").manual_seed(1)
    logits = (torch.randn(4, V, generator=g, device="cuda") * 3 + at).contiguous()
    logits[1, ::3] = -5.0
    logits[2, 4096:] -= 1e7 if abs(at) < 1e8 else 0.0
    for dtype in (torch.float32, torch.bfloat16):
        for r in range(4):
            x = logits[r:r + 1].to(dtype)
            lp, _ = _log_probs(_rows(x), dtype, np.ones((1, V), bool), False)
            got = ats.op_beam_select(x, _dev([0, 1]), 20)
            best = np.sort(lp[0])[::-1][:20]
            out = got.score[0].double().cpu().numpy()
            # (where only the differences of far out logits count: a difference, a product, the constant of a term's exponent, 2.3 steps of
            # differences of up to 100 that count)
            assert (np.abs(out - best) <= _tolerance(V) + 230 * 2.0 ** -24 + np.abs(best) * 2.0 ** -24).all(), (dtype, r)


def test_select_scores_far_out(ats):
    """Beams marked as empty by a score far down or -infinity, and scores of any size."""
    logits = _logits(4, 6, 5000, torch.float32)
    _check_select(ats, logits, [6], 50, score=[0.0, -1e9, -1e9, NEG, -1e20, 3e38], exact=False)
    got = _check_select(ats, logits, [6], 5, score=[NEG] * 6)
    assert (got.token == -1).all()
    got = _check_select(ats, logits, [6], 5, score=[float("nan")] * 6)
    assert (got.token == -1).all()
    # (a row of score +infinity comes first, by its logits)
    got = ats.op_beam_select(logits, _dev([0, 6]), 5, score=_dev(np.array([0, 1, np.inf, 0, 0, 0], np.float32), torch.float32))
    assert got.parent[0].tolist() == [2] * 5 and got.score[0].tolist() == [float("inf")] * 5
    assert got.token[0].tolist() == torch.sort(logits[2], descending=True).indices[:5].tolist()
    # (a row whose score swallows its logits' differences: by the logits)
    got = ats.op_beam_select(logits, _dev([0, 1]), 5, score=_dev(np.full(6, -1e20, np.float32), torch.float32))
    assert got.token[0].tolist() == torch.sort(logits[0], descending=True).indices[:5].tolist()


@pytest.mark.parametrize("order", ["up", "down", "lane", "tile", "few", "row"])
@pytest.mark.parametrize("width", [10, 80, 256])
def test_select_orders_that_meet_one_group(ats, order, width):
    """The best tokens in one thread's places, in one tile, or every one better than those before it."""
    V, R = 41000, 2
    base = np.linspace(-8, 8, V)
    if order == "up":
        x = base
    elif order == "down":
        x = base[::-1]
    else:
        x = np.random.default_rng(0).permutation(base[:V - 2000] - 8)
        i = np.arange(2000)
        hot = {"lane": i * 16 % V, "tile": 20000 + i, "few": i // 100 + i % 20 * 2048 + i % 100 // 20 * 300,   # a hundred places of each 2048
               "row": i // 20 + i % 20 * 2048}[order]
        assert len(set(hot.tolist())) == 2000
        x = np.concatenate([x, np.zeros(2000)])
        x[hot] = np.linspace(0, 8, 2000)
    logits = torch.from_numpy(np.tile(x, (R, 1)).astype(np.float32)).to("cuda")
    _check_select(ats, logits, [1, 1], width, exact=True)


@pytest.mark.parametrize("width", [8, 20, 64, 256])
def test_select_many_equal_beams(ats, width):
    """More candidates of one score than the ranking holds at a time."""
    logits = torch.zeros(90, 700, device="cuda")
    _check_select(ats, logits, [90], width, exact=True)
    logits = _logits(1, 1, 700, torch.float32).expand(90, 700).contiguous()
    _check_select(ats, logits, [90], width, exact=True)
    # (better and better beams)
    _check_select(ats, logits, [90], width, score=np.linspace(-90, 0, 90), exact=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [20, 80, 256])
@pytest.mark.parametrize("rules", [False, True])
def test_select_whole_numbers(ats, dtype, width, rules):
    """A few different logits, each of them many times, in beams that come in turn from the worst to the best."""
    V, R, tokens = 12500, 90, 9000
    rng = np.random.default_rng(width)
    x = np.round(rng.normal(0, 1.2, V))
    x[rng.permutation(V)[:30]] = np.arange(30) // 6 + 5
    logits = torch.from_numpy(np.tile(x, (R, 1)).astype(np.float32)).to("cuda", dtype)
    score = np.arange(R) // 3 % 4 * 0.25 - 1   # (a sum of whole and quarter steps tells which it is of)
    kw = {}
    if rules:
        kw = dict(table=np.arange(V)[None, :] % 25 < 18, state=np.zeros(R, int))
        assert kw["table"].sum() == tokens
    _check_select(ats, logits, [R], width, score=score, exact=True, **kw)
    _check_select(ats, logits, [1, R - 1], width, score=score, exact=True, **kw)


def test_select_leaves_other_rows(ats):
    logits = _logits(8, 10, 3000, torch.float32)
    logits[:2] = float("nan")
    logits[8:] = float("nan")
    _check_select(ats, logits, [3, 3], 7, first=2)


def test_select_past_2_31_logits(ats):
    """66 000 rows of 33 001: two requests of 33 000 beams, whose best continuations lie in the last rows."""
    R, V = 66000, 33001
    logits = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    assert logits.numel() > 2 ** 31
    score = np.full(R, -100.0, np.float32)
    want = [[], []]
    for b, (first, step) in enumerate(((32990, 1), (65999, -1))):
        for i in range(10):
            r, v = first + i * step, V - 1 - 7 * i
            logits[r, v] = 8.0
            score[r] = -1.0 - i
            # (the rows' log-sums are the same; a row's other tokens, the first ten of them, have equal scores)
            want[b] += [(-1.0 - i + 8.0, r, v, 8.0)] + [(-1.0 - i, r, t, 0.0) for t in range(10)]
    got = ats.op_beam_select(logits, _dev([0, 33000, 66000]), 10, score=_dev(score, torch.float32))
    lse = np.log(V - 1 + np.exp(8.0))
    for b in range(2):
        best = sorted(want[b], key=lambda c: (-c[0], c[1], -c[3], c[2]))[:10]
        assert list(zip(got.parent[b].tolist(), got.token[b].tolist())) == [c[1:3] for c in best]
        assert np.abs(got.score[b].double().cpu().numpy() - [c[0] - lse for c in best]).max() <= _tolerance(V) + 16 * 2.0 ** -24


def test_select_on_streams_and_in_graphs(ats):
    a, b = _logits(1, 20, 33024, torch.float32), _logits(2, 20, 33024, torch.float32)
    cu = _dev([0, 10, 20])
    want = [ats.op_beam_select(x, cu, 10) for x in (a, b)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        got = [ats.op_beam_select(a, cu, 10, stream=s1), ats.op_beam_select(b, cu, 10, stream=s2)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.token, w.token) and torch.equal(g.score, w.score) and torch.equal(g.parent, w.parent)
    x = a.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ats.op_beam_select(x, cu, 10)
    for src, w in ((a, want[0]), (b, want[1]), (a, want[0])):
        x.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.token, w.token) and torch.equal(got.score, w.score)


def test_select_workspaces_are_given_back(ats):
    """A call's workspace is free after it, on every stream and after a refusal; calls that are captured have their graph's memory."""
    cu, logits = _dev([0, 10, 20]), _logits(1, 20, 33024, torch.float32)
    side = torch.cuda.Stream()
    for stream in (None, side):
        ats.op_beam_select(logits, cu, 10, stream=stream)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        for _ in range(50):
            ats.op_beam_select(logits, cu, 10, stream=stream)
        with pytest.raises(ats.AtSpeedError):
            ats.op_beam_select(logits, cu, 257, stream=stream)
        torch.cuda.synchronize()
        assert torch.cuda.memory_allocated() == before
    # (two graphs of calls one after the other, replayed beside each other and beside calls of their own)
    want = ats.op_beam_select(logits, cu, 10)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = [ats.op_beam_select(logits, cu, 10) for _ in range(5)]
        graphs.append((g, got, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        own = ats.op_beam_select(logits, cu, 10)
        torch.cuda.synchronize()
        for r in [own] + [r for _, got, _ in graphs for r in got]:
            assert torch.equal(r.token, want.token) and torch.equal(r.parent, want.parent) and torch.equal(r.score, want.score)


# ---------------------------------------------------------------------------------------------------
# fork
# ---------------------------------------------------------------------------------------------------
def _fork_reference(table, held, ref, free, n_free, used, parent, length, page):
    n, width = table.shape
    n_pages, m = len(ref), len(parent)
    pool = lambda e: 0 <= e < n_pages  # noqa: E731
    up = lambda x: -(-int(x) // page)  # noqa: E731
    new = np.full((m, width), -1, np.int32)
    out_len, state, src, dst = np.zeros(m, int), np.zeros(m, int), np.full(m, -1), np.full(m, -1)
    lens = {}
    for j in range(m):
        p = parent[j]
        if p < 0:
            continue
        h = held[p] if p < n else -1
        x = h if length is None else length[j]
        if x < 0 or x > h or up(x) > width:
            state[j], out_len[j] = 2, -1
        else:
            lens[j] = int(x)
    heir = {}
    for j, x in lens.items():
        p = parent[j]
        if p not in heir or x > lens[heir[p]]:
            heir[p] = j
    nth, served = 0, []
    for j, x in lens.items():
        p, k = parent[j], up(x)
        row = list(table[p, :k])
        if x % page and pool(row[-1]) and not (heir[p] == j and ref[row[-1]] <= 1):
            if used + nth >= n_free:
                state[j], out_len[j] = 1, -1
                nth += 1
                continue
            src[j], dst[j] = row[-1], free[used + nth]
            row[-1] = dst[j]
            nth += 1
        out_len[j] = x
        new[j, :k] = row
        served.append(j)
    count = ref.astype(np.int64).copy()
    for i in range(used):
        count[free[i]] += 1
    for p in range(n):
        for e in table[p, :min(width, up(held[p]))]:
            if pool(e):
                count[e] -= 1
    for j in served:
        for e in new[j, :up(out_len[j])]:
            if pool(e):
                count[e] += 1
    now_free = np.nonzero(count <= 0)[0]
    return dict(table=new, kv_len=out_len, state=state, src=src, dst=dst, ref=count, free=now_free, n_free=[len(now_free)])


def _check_fork(ats, table, kv, ref, free, n_free, page, q=None, old_state=None, used=None, parent=None, length=None):
    n = len(kv)
    held = np.maximum(kv, 0) + (np.where(np.zeros(n, int) == (0 if old_state is None else old_state), np.maximum(q, 0), 0) if q is not None else 0)
    want = _fork_reference(table, held, ref, free, n_free, used or 0, np.arange(n) if parent is None else parent, length, page)
    opt = lambda a: None if a is None else _dev(a)  # noqa: E731
    args = (_dev(table), _dev(kv), _dev(ref), _dev(free), _dev([n_free]), page)
    kw = dict(q_len=opt(q), state=opt(old_state), used=None if used is None else _dev([used, 99]), parent=opt(parent), length=opt(length))
    before = [t.clone() for t in args[:5]]
    got = ats.op_fork_pages(*args, **kw)
    for k in ("table", "kv_len", "state", "src", "dst", "ref", "n_free"):
        np.testing.assert_array_equal(getattr(got, k).cpu().numpy(), want[k], err_msg=k)
    f = got.free.cpu().numpy()
    np.testing.assert_array_equal(f[:len(want["free"])], want["free"])
    assert (f[len(want["free"]):] == -1).all()
    for t, old in zip(args[:5], before):
        assert torch.equal(t, old)
    return got


def _pool(rng, n, width, page, n_pages, q_hi=1, shared=0.5):
    """Rows of a table that share their first pages, whose counts are right; the rows' tokens; the pages left."""
    order = list(rng.permutation(n_pages))
    table, ref = np.full((n, width), -9, np.int32), np.zeros(n_pages, np.int32)
    kv = np.zeros(n, int)
    for b in range(n):
        kv[b] = rng.integers(0, (width - 1) * page)
        k = -(-kv[b] // page)
        start = 0
        if b and rng.random() < shared:
            other = rng.integers(0, b)
            start = min(kv[b] // page, kv[other] // page)
            table[b, :start] = table[other, :start]
        for i in range(start, k):
            table[b, i] = order.pop()
        for e in table[b, :k]:
            ref[e] += 1
    return table, kv, ref, np.array(order, np.int32)


@pytest.mark.parametrize("n,m,width,page", [(1, 1, 3, 16), (1, 10, 9, 64), (10, 10, 9, 64), (7, 33, 21, 5), (160, 300, 40, 16), (40, 3, 33, 1)])
@pytest.mark.parametrize("seed", [0, 1])
def test_fork_beams(ats, n, m, width, page, seed):
    rng = np.random.default_rng([n, m, seed])
    table, kv, ref, free = _pool(rng, n, width, page, n * width + 3 * m + 11)
    parent = rng.integers(-1, n, size=m)
    for n_free in (0, min(len(free), m // 2), len(free)):
        _check_fork(ats, table, kv, ref, free, n_free, page, parent=parent)
    # lengths: anything that the parent holds, and some that it does not
    length = np.where(parent >= 0, rng.integers(-1, kv.max() + 2, size=m), 0)
    _check_fork(ats, table, kv, ref, free, len(free), page, parent=parent, length=length)
    length = (kv[np.maximum(parent, 0)] * rng.random(m)).astype(int)
    _check_fork(ats, table, kv, ref, free, len(free), page, parent=parent, length=length)
    _check_fork(ats, table, kv, ref, free, len(free), page, parent=np.where(rng.random(m) < 0.3, n + 2, parent))


def test_fork_shared_last_pages_and_foreign_entries(ats):
    """A partial last page that something else holds is copied by every child; entries outside the pool are handed on."""
    page = 4
    table = np.array([[5, 6, 7], [5, 6, 8], [5, 6, 7], [1, 99, -3]], np.int32)
    ref = np.array([0, 1, 0, 0, 0, 3, 4, 2, 1, 0], np.int32)   # (6: once more by someone else)
    kv = np.array([10, 9, 10, 10])
    free = np.array([0, 2, 3, 4, 9], np.int32)
    _check_fork(ats, table, kv, ref, free, 5, page)
    _check_fork(ats, table, kv, ref, free, 5, page, parent=np.array([0, 0, 2, 3, 3]))
    _check_fork(ats, table, kv, ref, free, 1, page, parent=np.array([0, 1, 1, 2, -1]))
    _check_fork(ats, table, kv, ref, free, 5, page, parent=np.array([1, 1, 1]), length=np.array([6, 8, 5]))
    _check_fork(ats, table, kv, ref, free, 5, page, parent=np.array([-1, -1]))


@pytest.mark.parametrize("n", [1, 61, 1021, 16384])
def test_fork_gives_back_what_was_not_kept(ats, n):
    rng = np.random.default_rng(n)
    page, width = 16, 12
    kv, q = rng.integers(0, 100, size=n), rng.integers(0, 60, size=n)
    state = (rng.random(n) < 0.1).astype(int)
    n_pages = n * width + 5
    order = rng.permutation(n_pages).astype(np.int32)
    have, need = -(-kv // page), -(-(kv + np.where(state == 0, q, 0)) // page)
    table, ref, i = np.full((n, width), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for b in range(n):
        table[b, :have[b]] = order[i:i + have[b]]
        i += have[b]
    ref[order[:i]] = 1
    free, used = order[i:], 0
    for b in range(n):
        k = max(0, need[b] - have[b])
        table[b, have[b]:have[b] + k] = free[used:used + k]
        used += k
    length = kv + np.where(state == 0, (q * rng.random(n)).astype(int), 0)
    _check_fork(ats, table, kv, ref, free, len(free), page, q=q, old_state=state, used=used, length=length)
    _check_fork(ats, table, kv, ref, free, len(free), page, q=q, old_state=state, used=used)
    _check_fork(ats, table, kv, ref, free, len(free), page, q=q, old_state=state, used=used, parent=rng.integers(-1, n, size=n))


@pytest.mark.parametrize("n_pages", [1, 7, 1024, 8191, 8193, 100003, 1000000])
def test_fork_free_list_of_any_pool(ats, n_pages):
    rng = np.random.default_rng(n_pages)
    ref = (rng.random(n_pages) < 0.5).astype(np.int32)
    free = np.nonzero(ref == 0)[0].astype(np.int32)
    _check_fork(ats, np.array([[-1]], np.int32), np.array([0]), ref, free, len(free), 16)


def test_fork_of_more_pages_handed_out_than_there_are(ats):
    """A count of pages taken that is past the free list's end or below 0."""
    table, ref, free = _dev([[0, 1]]), _dev([1, 1, 0, 0, 0]), _dev([2, 3, 4])
    for used, left in ((-7, [2, 3, 4]), (99, [])):
        f = ats.op_fork_pages(table, _dev([20]), ref, free, _dev([3]), 16, used=_dev([used]))
        assert f.ref.tolist() == [1, 1] + [0 if left else 1] * 3 and f.free.tolist()[:int(f.n_free)] == left


def test_fork_without_a_free_page(ats):
    table, ref = np.array([[0, 1]], np.int32), np.array([1, 1], np.int32)
    _check_fork(ats, table, np.array([20]), ref, np.zeros(0, np.int32), 0, 16, parent=np.array([0, 0]))


def test_fork_writes_into_given_outputs_and_in_graphs(ats):
    rng = np.random.default_rng(5)
    table, kv, ref, free = _pool(rng, 20, 9, 16, 400)
    a = (_dev(table), _dev(kv), _dev(ref), _dev(free), _dev([len(free)]), 16)
    parents = [_dev(rng.integers(0, 20, size=20)) for _ in range(3)]
    want = [ats.op_fork_pages(*a, parent=p) for p in parents]
    out = ats.op_fork_pages(*a)
    p = parents[0].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ats.op_fork_pages(*a, parent=p, out=out)
    for src, w in zip(parents, want):
        p.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        for k in ats.PageFork.__slots__:
            assert torch.equal(getattr(out, k), getattr(w, k)), k


@pytest.mark.parametrize("page", [16, 3])
def test_plan_and_fork_keep_the_pages(ats, page):
    """Beams of several users, step after step on the GPU alone: every row finds its own tokens, counts and free list are
    those of the rows, and a page that two rows hold is never written to."""
    rng = np.random.default_rng(page)
    users, w, n_pages, width = 3, 6, 400, 30
    n = users * w
    ref, table = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.arange(n_pages, dtype=torch.int32, device="cuda"), _dev([n_pages])
    kv = torch.zeros(n, dtype=torch.int32, device="cuda")
    cache = torch.full((n_pages * page,), -1, dtype=torch.int64, device="cuda")   # a token's number in its cache row
    said = [[] for _ in range(n)]
    number = 0
    for step in range(25):
        q = rng.integers(5, 20, size=n) if step == 0 else rng.integers(0, 3, size=n)
        if step == 0:
            q[np.arange(n) % w > 0] = 0   # (a user's first row alone has a prompt)
        T = max(1, int(q.sum()))
        plan = ats.op_batch_plan(_dev(q), kv, table, free, n_free, page, T)
        assert (plan.state == ats.PLAN_OK).all()
        slot = plan.slot.cpu().numpy()
        t = 0
        for b in range(n):
            for _ in range(q[b]):
                assert slot[t] >= 0
                cache[slot[t]] = number
                said[b].append(number)
                number += 1
                t += 1
        parent = np.concatenate([u * w + (rng.integers(0, w, size=w) if step else np.zeros(w, int)) for u in range(users)])
        if step % 5 == 4:
            parent[rng.integers(0, n)] = -1
        fork = ats.op_fork_pages(table, kv, ref, free, n_free, page, q_len=_dev(q), state=plan.state, used=plan.pages, parent=_dev(parent))
        assert (fork.state == ats.PLAN_OK).all()
        kv, table, ref, free, n_free = fork.kv_len, fork.table, fork.ref, fork.free, fork.n_free
        # the copies, here by torch
        for a, b, length in zip(fork.src.tolist(), fork.dst.tolist(), kv.tolist()):
            if a >= 0:
                rows = (length - 1) % page + 1
                cache[b * page:b * page + rows] = cache[a * page:a * page + rows]
        said = [list(said[p]) if p >= 0 else [] for p in parent]
        assert kv.tolist() == [len(s) for s in said]
        tab, holds = table.cpu().numpy(), np.zeros(n_pages, int)
        for b in range(n):
            k = -(-len(said[b]) // page)
            rows = (tab[b, :k, None].astype(np.int64) * page + np.arange(page)).reshape(-1)[:len(said[b])]
            assert cache[torch.from_numpy(rows).cuda()].tolist() == said[b]
            assert (tab[b, k:] == -1).all()
            np.add.at(holds, tab[b, :k], 1)
        np.testing.assert_array_equal(ref.cpu().numpy(), holds)
        assert int(n_free) == (holds == 0).sum()
        np.testing.assert_array_equal(free.cpu().numpy()[:int(n_free)], np.nonzero(holds == 0)[0])


# ---------------------------------------------------------------------------------------------------
# copies and compaction
# ---------------------------------------------------------------------------------------------------
def _layers(seed, layers, pages, page, heads, hd, types, layout):
    g = torch.Generator("cuda").manual_seed(seed)
    out = []
    for _ in range(layers):
        pair = []
        for t in types:
            if layout == "head":
                x = torch.randn(pages, heads, page, hd, generator=g, device="cuda").to(t).transpose(1, 2)
            elif layout == "wide":   # rows and heads apart from each other
                x = torch.randn(pages, page + 1, heads + 1, hd + 8, generator=g, device="cuda").to(t)[:, :page, :heads, :hd]
            else:
                x = torch.randn(pages, page, heads, hd, generator=g, device="cuda").to(t)
            pair.append(x)
        out.append(tuple(pair))
    return out


def _whole(t):
    """The memory under a view, its gaps too."""
    n = t.untyped_storage().nbytes() // t.element_size()
    return torch.as_strided(t, (n,), (1,), 0)


MIXED, F16 = (torch.bfloat16, torch.float16), (torch.float16, torch.float16)


def _copied(caches, src, dst, rows, pages):
    for pair in caches:
        for t in pair:
            for a, b, r in zip(src, dst, rows):
                if 0 <= a < pages and 0 <= b < pages and a != b and r > 0:
                    t[b, :r] = t[a, :r].clone()


@pytest.mark.parametrize("layout", ["token", "head", "wide"])
@pytest.mark.parametrize("layers,page,heads,hd,types", [(1, 16, 1, 8, MIXED), (4, 64, 12, 64, MIXED), (3, 5, 3, 24, F16),
                                                          (130, 16, 2, 32, F16), (2, 256, 32, 128, MIXED), (2, 1, 1, 264, MIXED)])
def test_copy_pages(ats, layout, layers, page, heads, hd, types):
    pages, n = 23, 14
    rng = np.random.default_rng(page)
    order = rng.permutation(pages)
    src, dst = order[rng.integers(0, 6, size=n)], order[6:6 + n].copy()
    src[3], dst[5], src[7], dst[8], dst[9] = -1, -1, pages, pages + 5, src[9]
    for length in (None, rng.integers(-1, 5 * page, size=n)):
        mine = _layers(1, layers, pages, page, heads, hd, types, layout)
        want = [tuple(t.clone() if layout == "token" else _whole(t).clone().as_strided(t.shape, t.stride(), t.storage_offset()) for t in p)
                for p in mine]
        rows = np.full(n, page) if length is None else np.where(length > 0, (length - 1) % page + 1, 0)
        _copied(want, src, dst, rows, pages)
        ats.op_copy_pages(ats.CacheLayers(mine), _dev(src), _dev(dst), length=None if length is None else _dev(length))
        for p, q in zip(mine, want):
            for x, y in zip(p, q):
                assert torch.equal(_whole(x).view(torch.int16), _whole(y).view(torch.int16))


@pytest.mark.parametrize("n", [255, 257, 1024, 1025, 2500])
def test_copy_many_pages(ats, n):
    """More pairs than a CTA lists at a time, most of them none."""
    rng = np.random.default_rng(n)
    order = rng.permutation(2 * n)
    src, dst = order[:n].copy(), order[n:].copy()
    src[rng.random(n) < 0.6] = -1
    length = rng.integers(0, 50, size=n)
    mine = _layers(4, 2, 2 * n, 7, 2, 16, MIXED, "token")
    want = [tuple(t.clone() for t in p) for p in mine]
    _copied(want, src, dst, np.where(length > 0, (length - 1) % 7 + 1, 0), 2 * n)
    ats.op_copy_pages(ats.CacheLayers(mine), _dev(src), _dev(dst), length=_dev(length))
    for p, q in zip(mine, want):
        for x, y in zip(p, q):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def _compacted(caches, slot, cu, keep, n_keep, ok, page, rows):
    moved = []
    for b in range(len(cu) - 1):
        q, last, count = cu[b + 1] - cu[b], -1, 0
        while ok[b] and count < min(n_keep[b], keep.shape[1]) and last < keep[b, count] < q:
            last = keep[b, count]
            count += 1
        moved.append(count)
        for pair in caches:
            for t in pair:
                old = {}
                for i in range(count):
                    a = slot[cu[b] + keep[b, i]]
                    old[i] = t[a // page, a % page].clone() if 0 <= a < rows else None
                for i in range(count):
                    a, to = slot[cu[b] + keep[b, i]], slot[cu[b] + i]
                    if a != to and old[i] is not None and 0 <= to < rows:
                        t[to // page, to % page] = old[i]
    return np.array(moved)


@pytest.mark.parametrize("layout", ["token", "head", "wide"])
@pytest.mark.parametrize("layers,page,heads,hd,types,q_hi", [(1, 16, 1, 8, MIXED, 5), (4, 64, 12, 64, MIXED, 120), (130, 5, 2, 24, F16, 9),
                                                               (2, 16, 32, 128, MIXED, 240)])
def test_compact_tokens(ats, layout, layers, page, heads, hd, types, q_hi):
    rng = np.random.default_rng(q_hi)
    n, width = 6, 12
    q = rng.integers(1, q_hi + 1, size=n)
    q[2] = 0
    cu = np.concatenate([[0], np.cumsum(q)])
    kv = rng.integers(0, 50, size=n)
    need = -(-(kv % page + q) // page)
    pages = int(need.sum()) + 2
    order, at = rng.permutation(pages), np.concatenate([[0], np.cumsum(need)])
    slot = np.concatenate([order[at[b] + (kv[b] % page + np.arange(q[b])) // page] * page + (kv[b] % page + np.arange(q[b])) % page for b in range(n)])
    keep, n_keep = np.full((n, width), -1), np.zeros(n, int)
    for b in range(n):
        k = min(width, q[b], rng.integers(0, width + 1))
        keep[b, :k] = np.sort(rng.choice(q[b], size=k, replace=False)) if k else []
        n_keep[b] = k
    keep[0, :min(4, q[0])] = np.arange(1, 1 + min(4, q[0]))   # every move lands where the one before it came from (the last: out)
    n_keep[0] = min(4, q[0])
    n_keep[1] = 99
    state = np.array([0, 0, 0, 1, 0, 0])
    for st in (None, state):
        mine = _layers(3, layers, pages, page, heads, hd, types, layout)
        want = [tuple(_whole(t).clone().as_strided(t.shape, t.stride(), t.storage_offset()) for t in p) for p in mine]
        count = _compacted(want, slot, cu, keep, n_keep, np.ones(n, bool) if st is None else st == 0, page, pages * page)
        got = ats.op_compact_tokens(ats.CacheLayers(mine), _dev(slot, torch.int64), _dev(cu), _dev(kv), _dev(keep), _dev(n_keep),
                                    state=None if st is None else _dev(st))
        np.testing.assert_array_equal(got.cpu().numpy(), kv + count)
        for p, r in zip(mine, want):
            for x, y in zip(p, r):
                assert torch.equal(_whole(x).view(torch.int16), _whole(y).view(torch.int16))


def test_compact_long_chains_and_odd_lists(ats):
    """Hundreds of kept tokens, each in the place of the next; lists that are not ascending; slots outside the cache."""
    page, pages, q = 16, 80, 1200
    mine = _layers(5, 2, pages, page, 4, 64, MIXED, "token")
    slot = np.random.default_rng(1).permutation(pages * page)[:q].astype(np.int64)
    slot[700], slot[3] = -1, pages * page
    keep = np.stack([np.arange(1, 1100), np.concatenate([[5, 9, 9], np.arange(3, 1099)])])
    cu, kv, n_keep = np.array([0, 1150, 1200]), np.array([3, 4]), np.array([1099, 1000])
    want = [tuple(t.clone() for t in p) for p in mine]
    count = _compacted(want, slot, cu, keep, n_keep, np.ones(2, bool), page, pages * page)
    got = ats.op_compact_tokens(ats.CacheLayers(mine), _dev(slot, torch.int64), _dev(cu), _dev(kv), _dev(keep), _dev(n_keep))
    assert got.tolist() == [3 + 1099, 4 + 2] and count.tolist() == [1099, 2]
    for p, r in zip(mine, want):
        for x, y in zip(p, r):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_rows_past_2_31_elements(ats):
    """A layer of 5 GB a cache: rows behind element 2^31."""
    pages, page, heads, hd = 5000, 64, 64, 128
    k, v = (torch.zeros(pages, page, heads, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 31
    for t in (k, v):
        t[pages - 2] = torch.randn(page, heads, hd, device="cuda")
    layers = ats.CacheLayers([(k, v)])
    ats.op_copy_pages(layers, _dev([pages - 2, -1]), _dev([pages - 1, 3]), length=_dev([40, 1]))
    for t in (k, v):
        assert torch.equal(t[pages - 1, :40], t[pages - 2, :40]) and not t[pages - 1, 40:].any() and not t[3].any()
    slot = torch.arange(pages * page - 2 * page, pages * page, dtype=torch.int64, device="cuda")   # the last two pages
    want = [t[pages - 2, 33].clone() for t in (k, v)]
    got = ats.op_compact_tokens(layers, slot, _dev([0, 2 * page]), _dev([7]), _dev([[0, 33]]), _dev([2]))
    assert got.tolist() == [9]
    for t, w in zip((k, v), want):
        assert torch.equal(t[pages - 2, 1], w)


def test_moves_on_streams_and_in_graphs(ats):
    mine = _layers(2, 3, 40, 16, 4, 64, MIXED, "token")
    layers = ats.CacheLayers(mine)
    src, dst, length = _dev([0, 1, 2]), _dev([10, 11, 12]), _dev([16, 3, 40])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ats.op_copy_pages(layers, src, dst, length=length, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(mine[2][1][10], mine[2][1][0]) and torch.equal(mine[1][0][11, :3], mine[1][0][1, :3])
    slot, cu, kv = torch.arange(64, device="cuda"), _dev([0, 64]), _dev([0])
    keep, n_keep = _dev([[2, 20]]), _dev([1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ats.op_compact_tokens(layers, slot, cu, kv, keep, n_keep)
        ats.op_copy_pages(layers, src, dst)
    keep.copy_(_dev([[4, 21]]))
    n_keep.fill_(2)
    want = [[t[0, 4].clone(), t[1, 5].clone()] for p in mine for t in p]
    graph.replay()
    torch.cuda.synchronize()
    assert out.tolist() == [2]
    for w, t in zip(want, [t for p in mine for t in p]):
        assert torch.equal(t[0, 0], w[0]) and torch.equal(t[0, 1], w[1]) and torch.equal(t[10], t[0])
