"""Beam selection, page fork and moves at the edges of what they allow: lists that fill to their last place, scores near a type's largest
number, and forks, copies and moves whose counts, lists and buffers are at their limits."""
import numpy as np
import pytest
import torch

from test_gpu_beam_ops import NEG, TYPES, _bits, _check_select, _dev, _logits, ats  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------
# selection: a ranking in several rounds whose list fills up
# ---------------------------------------------------------------------------------------------------
def _equal_logits(V, hot, dtype, alone):
    """A row with `hot` equal best logits, the others 25 and more below them (alone: -infinity), and where those are."""
    rng = np.random.default_rng(hot)
    row = np.full(V, NEG) if alone else np.floor(rng.uniform(-30, -20, size=V))
    at = np.sort(rng.choice(V, size=hot, replace=False))
    row[at] = 5.0
    return torch.from_numpy(row.astype(np.float32)).to("cuda", dtype), at


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("better", [False, True])
@pytest.mark.parametrize("over", [-2, -1, 0, 1, 2])
# width, threads that rank, rows whose candidates are looked at in a round, more rows, other requests
@pytest.mark.parametrize("width,threads,round_rows,more,others", [
    (16, 1024, 512, 8, []), (16, 1024, 512, 600, []), (64, 256, 32, 8, [2]), (64, 256, 32, 90, [1, 1, 0, 3]), (30, 256, 64, 80, [3, 1, 2]),
    (10, 256, 128, 72, [1, 2, 1]), (80, 1024, 128, 12, []), (80, 1024, 128, 300, []), (120, 1024, 64, 20, []), (256, 1024, 32, 8, [])])
def test_select_fills_the_list_and_goes_on(ats, width, threads, round_rows, more, others, over, better, dtype):  # noqa: F811
    """Equal scores whose first round fills the list of 2 * threads places, but for a quarter of the threads or one, just so, or one or many too
    far, before more of them come.  Rows are the same, so that their sums are; what a state allows (of a sum over all) says how many are equal."""
    V, hot = 1000, 100
    total = 2 * threads + {-2: -threads // 4, -1: -1, 0: 0, 1: 1, 2: threads // 4 + 3}[over]
    allow = np.full(round_rows, total // round_rows)
    allow[:total % round_rows] += 1
    assert allow.max() <= hot and allow.sum() == total
    beams = round_rows + more
    state = np.concatenate([allow, np.full(more + sum(others), total // round_rows)])
    # (a bound at the equal ones needs `width` threads that meet one: an eighth of them do at least; without others there is no other bound)
    row, at = _equal_logits(V, hot, dtype, alone=width > threads // 8)
    table = np.ones((hot + 1, V), bool)
    for s in range(hot + 1):
        table[s, at[s:]] = False
    score = np.zeros(state.size)
    if better:   # (fewer than `width` of them: the bound stays)
        score[[round_rows // 2, beams - 1]] = 1.0
        state[[round_rows // 2, beams - 1]] = 3
    logits = row.expand(state.size, V).contiguous()
    _check_select(ats, logits, [beams] + others, width, score=score, table=table, state=state, norm="full", exact=True)


@pytest.mark.parametrize("width,beams,tied,others", [(80, 140, [*range(24), *range(128, 140)], []),
                                                     (10, 200, [*range(51), *range(128, 200)], [1] * 9)])
def test_select_equal_beams_among_far_ones(ats, width, beams, tied, others):  # noqa: F811
    """Rows of equal logits, some of them beams of one score, the others far below: nearly a full list, then more."""
    score = np.full(beams + sum(others), -50.0)
    score[tied] = 0.0
    _check_select(ats, torch.zeros(score.size, 700, device="cuda"), [beams] + others, width, score=score, exact=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 3, 9, 513, 2049, 4095, 4101, 8193])
def test_select_rows_that_end_early_in_a_tile(ats, dtype, V):  # noqa: F811
    """Rows that begin at every place of a 16-byte word and leave most of their last tile's lanes nothing to read."""
    _check_select(ats, _logits(V, 9, V, dtype, pitch=(1 - V) % 16), [4, 5], 12, score=np.linspace(-1, -2, 9))
    _check_select(ats, _logits(V, 1, V, dtype, lead=1), [1], 12)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("down", [float(np.finfo(np.float32).min), -1e38])
@pytest.mark.parametrize("V", [3, 5000])
def test_select_scores_and_logits_near_the_largest_number(ats, dtype, down, V):  # noqa: F811
    """Beams marked as empty by a score far down, whose logits have an infinity or a number near the largest: the one continuation whose
    score is finite fills a place that nothing better takes."""
    logits = torch.full((4, V), -1e6, device="cuda")
    logits[0, :2] = torch.tensor([0.5, -3.0])
    logits[1, 1] = float("inf")
    logits[2, 2] = 3e38
    logits[3, 0] = -2.0
    logits = logits.to(dtype)
    got = _check_select(ats, logits, [4], 9, score=[0.0, down, down, NEG])
    pairs = list(zip(got.parent[0].tolist(), got.token[0].tolist()))
    assert pairs[:2] == [(0, 0), (0, 1)] and (V > 3 or pairs[3:] == [(1, 1), (2, 2)] + [(-1, -1)] * 4)
    got = _check_select(ats, logits, [1, 2, 1], 3, score=[0.0, down, down, NEG])
    assert list(zip(got.parent[1].tolist(), got.token[1].tolist())) == [(1, 1), (2, 2), (-1, -1)]


def test_select_with_a_tensor_as_workspace(ats, monkeypatch):  # noqa: F811
    """As in a torch without raw allocations: the same results, on another stream and in a graph too."""
    from paper_2410_05165_gb300 import binding
    logits, cu = _logits(1, 20, 33024, torch.float32), _dev([0, 10, 20])
    want = ats.op_beam_select(logits, cu, 10)
    monkeypatch.setattr(binding, "_raw_alloc", None)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = ats.op_beam_select(logits, cu, 10)
    for _ in range(20):
        graph.replay()
        calls = [captured, ats.op_beam_select(logits, cu, 10), ats.op_beam_select(logits, cu, 10, stream=side)]
        torch.cuda.synchronize()
        for got in calls:
            assert torch.equal(got.token, want.token) and torch.equal(got.parent, want.parent) and torch.equal(got.score, want.score)


# ---------------------------------------------------------------------------------------------------
# selection: what scores are worth
# ---------------------------------------------------------------------------------------------------
# Of a logarithm in two 32-bit parts: 2^-29 (the rest of its series is below 2^-7 and rounded in 32 bits, some operations of 2^-31 each).
# Twice that for the sums with it, which are exact but for their lower parts' roundings.
LOG = 2.0 ** -28


def _counted(V, counts):
    """Rows of n zeros among -infinities: their sums are n, without a rounding."""
    logits = torch.full((len(counts), V), NEG, device="cuda")
    for r, n in enumerate(counts):
        logits[r, torch.randperm(V, generator=torch.Generator().manual_seed(r))[:n].cuda()] = 0.0
    return logits


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 100, 33024, 100003])   # one piece a row, many
@pytest.mark.parametrize("cum", [0.0, -3.7, 11.0, -1e4])
def test_select_scores_of_sums_without_a_rounding(ats, dtype, V, cum):  # noqa: F811
    """cum - log n, off by its own rounding and what the logarithm is off."""
    counts = [n for n in (1, 2, 3, 5, 7, 100, 1023, 4097, 16384, 33023, 65521, 99991) if n <= V]
    cum = float(np.float32(cum))
    got = ats.op_beam_select(_counted(V, counts).to(dtype), _dev(range(len(counts) + 1)), 1, score=_dev(np.full(len(counts), cum), torch.float32))
    want = cum - np.log(np.array(counts, np.float64))
    assert (np.abs(got.score[:, 0].double().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -24 + LOG).all()


@pytest.mark.parametrize("beams", [17, 64])   # as many in a request
def test_select_tells_scores_apart_that_32_bits_do_not(ats, beams):  # noqa: F811
    """Beams whose scores take back all of their sums' logarithms but what 32 bits leave of those, some 2^-22: the order and what is left."""
    V, R = 20011, 3 * beams
    rng = np.random.default_rng(beams)
    counts = rng.choice(np.arange(2000, V), size=R, replace=False)
    logits, table = _counted(V, counts), np.zeros((R, V), bool)
    table[np.arange(R), torch.argmax(logits, dim=1).cpu().numpy()] = True   # (one of its tokens may follow a beam)
    score = np.log(counts.astype(np.float64)).astype(np.float32)
    exact = score.astype(np.float64) - np.log(counts.astype(np.float64))
    assert np.abs(exact).max() > 2.0 ** -24
    got = ats.op_beam_select(logits, _dev([0, beams, 2 * beams, R]), beams, score=_dev(score, torch.float32), grammar=_bits(table),
                             state=_dev(np.arange(R)), norm=ats.NORM_FULL)
    for b in range(3):
        rows = got.parent[b].cpu().numpy()
        assert sorted(rows) == list(range(b * beams, (b + 1) * beams))
        assert (np.abs(got.score[b].double().cpu().numpy() - exact[rows]) <= np.abs(exact[rows]) * 2.0 ** -24 + LOG).all()
        assert (np.diff(exact[rows]) <= 2 * LOG).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,V,std", [(10, 33024, 3.0), (320, 33024, 0.5), (200, 100003, 3.0), (300, 33024, 1.5)])
def test_select_scores_of_random_rows(ats, dtype, R, V, std):  # noqa: F811
    """In steps of 2^-24 a sum is off by 4 for the exponential (2^-22 at most, of one sign at the worst) and by what roundings of either sign leave:
    2.3 |d| for a term e^d, |d| 9 on average of a sum that a few terms make (9 / sqrt 3 / 2: 2.7), some 50 additions of a thread's (sqrt 50 / sqrt 3
    / 2: 2) and ten of the threads' sums (1.8): 3.8 in the mean square, seven times that for the worst row.  32 together."""
    logits = _logits(R, R, V, dtype, std=std)
    score = (-np.random.default_rng(V).exponential(2.0, R)).astype(np.float32)
    got = ats.op_beam_select(logits, _dev(range(R + 1)), 8, score=_dev(score, torch.float32))
    lp = torch.log_softmax(logits.double(), dim=1) + _dev(score, torch.float64)[:, None]
    want, token = torch.sort(lp, dim=1, descending=True, stable=True)
    assert torch.equal(got.token, token[:, :8].int())   # (within a row the order is the logits')
    off = (got.score.double() - want[:, :8]).abs()
    assert bool((off <= want[:, :8].abs() * 2.0 ** -24 + 32 * 2.0 ** -24).all()), float(off.max())


# ---------------------------------------------------------------------------------------------------
# fork
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_pages", [8, 20000])   # counts by one CTA, by several
@pytest.mark.parametrize("entries", [0, 1, 3])
@pytest.mark.parametrize("used", [None, 1, 6])
def test_fork_with_a_count_past_the_free_lists_end(ats, n_pages, entries, used):  # noqa: F811
    """Five children of one partial page, four of which want a copy; n_free says 7, the list has fewer entries."""
    memory = _dev([2, 3, 4, 5, 6, 7, 5, 5])   # (what lies behind the list is not its)
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ref[:2] = 1
    f = ats.op_fork_pages(_dev([[0, 1, -1]]), _dev([20]), ref, memory[:entries], _dev([7]), 16, parent=_dev([0] * 5),
                          used=None if used is None else _dev([used]))
    taken = min(entries, used or 0)
    copies = min(4, entries - taken)
    fresh = memory.tolist()[taken:taken + copies]
    assert f.state.tolist() == [0] * (1 + copies) + [1] * (4 - copies)
    assert f.dst.tolist() == [-1] + fresh + [-1] * (4 - copies) and f.src.tolist() == [-1] + [1] * copies + [-1] * (4 - copies)
    assert f.table.tolist() == [[0, 1, -1]] + [[0, e, -1] for e in fresh] + [[-1] * 3] * (4 - copies)
    held = [1 + copies, 1] + [0] * (n_pages - 2)
    for e in memory.tolist()[:taken] + fresh:
        held[e] = 1
    free = [e for e, h in enumerate(held) if h == 0]
    assert f.ref.tolist() == held and int(f.n_free) == len(free) and f.free.tolist() == free + [-1] * (n_pages - len(free))


def test_fork_writes_side_by_side_but_not_over(ats):  # noqa: F811
    """Inputs and outputs in one buffer, each next to the other: right.  With an output one entry into its neighbour: refused."""
    n, m, width, pages = 2, 3, 3, 8
    given = dict(table=[0, 1, -1, 2, -1, -1], kv_len=[20, 3], ref=[1, 1, 1, 0, 0, 0, 0, 0], free=[3, 4, 5, 6, 7], n_free=[5], parent=[0, 0, 1])
    sizes = dict(table=m * width, kv_len=m, state=m, src=m, dst=m, ref=pages, free=pages, n_free=1)
    for shifted in (None, *sizes):
        buffer = torch.full((200,), -7, dtype=torch.int32, device="cuda")
        at, ins, outs = 50, {}, {}
        for k, v in given.items():
            ins[k] = buffer[at:at + len(v)]
            ins[k].copy_(_dev(v))
            at += len(v)
        for k, size in sizes.items():
            outs[k] = buffer[at - (k == shifted):at - (k == shifted) + size]
            at += size
        outs["table"] = outs["table"].view(m, width)
        ins["table"] = ins["table"].view(n, width)
        before = buffer.clone()
        call = lambda: ats.op_fork_pages(**ins, page_size=16, out=ats.PageFork(**outs))  # noqa: E731
        if shifted:
            with pytest.raises(ats.AtSpeedError):
                call()
            assert torch.equal(buffer, before)
            continue
        f, want = call(), ats.op_fork_pages(**ins, page_size=16)
        for k in sizes:
            assert torch.equal(getattr(f, k), getattr(want, k)), k
        assert f.table.tolist() == [[0, 1, -1], [0, 3, -1], [2, -1, -1]] and f.free.tolist() == [4, 5, 6, 7, -1, -1, -1, -1]
        assert (buffer[:50] == -7).all() and (buffer[at:] == -7).all() and torch.equal(buffer[50:50 + 25], before[50:50 + 25])
