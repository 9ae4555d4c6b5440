"""The batched serving step's operators where lengths, weights, states and streams are unusual."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
NEG = float("-inf")
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # unit roundoff
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f16": (torch.float16, torch.float16), "mixed": (torch.bfloat16, torch.float16)}


@pytest.fixture(scope="module")
def ats():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2410_05165_gb300 as m
    return m


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


# ---------------------------------------------------------------------------------------------------
# small weights beside a large one
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("types", ["f16", "mixed", "bf16"])
@pytest.mark.parametrize("L,heads", [(1, 320), (200, 160)])   # one row a block, and blocks of more than 128; whole blocks a CTA
@pytest.mark.parametrize("score", [15.5, 17.0, 17.375, 20.0])
def test_small_weights_add_up(ats, types, L, heads, score):
    """One key with a value of 0 that is `score` nats above 20 000 others with a value of 1: the others' sum is the result."""
    kt, vt = TYPES[types]
    hd, page, ctx = 32, 256, 20000
    pages = -(-(ctx + L) // page)
    kc = torch.zeros(pages, page, heads, hd, dtype=kt, device="cuda")
    vc = torch.ones(pages, page, heads, hd, dtype=vt, device="cuda")
    kc[0, 0, :, 3], vc[0, 0] = score, 0
    q = torch.zeros(L, heads, hd, dtype=kt, device="cuda")
    q[:, :, 3] = 1
    lse = torch.zeros(L, heads, device="cuda")
    out = ats.op_tree_attention(q, kc, vc, _dev([0, L]), _dev([ctx]), _dev(np.arange(pages)[None]), scale=1.0, lse=lse)
    assert ats.op_status(noalloc=True) == 0
    n = (ctx + np.arange(L))[:, None, None].astype(np.float64)   # keys with a score of 0
    ref, log_sum = n / (n + np.exp(score)), np.log(n + np.exp(score))
    # weights rounded to V's type: UNIT of each, and in fp16 at least the 2^-32 of the largest below which a weight has no
    # bits; exponentials and sums in 32 bits; the result rounded to q's type
    tol = UNIT[kt] * ref + (UNIT[vt] + 1e-4) * ref + n * 2.0 ** -32
    err = np.abs(out.double().cpu().numpy() - ref)
    assert np.all(err <= tol), (err.max(), ref.max(), tol.min())
    assert np.all(np.abs(lse.double().cpu().numpy() - log_sum[..., 0]) <= 1e-4 * (1 + log_sum[..., 0]))


# ---------------------------------------------------------------------------------------------------
# requests that change from row to row, each with a list and a path
# ---------------------------------------------------------------------------------------------------
def test_lists_of_requests_in_turn(ats):
    """A few rows a request, so that a CTA's rows are of several: the path of a request's first row joins the list that was
    made just before, and leaves it whole to the next row."""
    rng = np.random.default_rng(41)
    n, V = 300, 700
    q_len = rng.integers(1, 6, size=n)
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    R = int(cu[-1])
    hist = rng.integers(0, 40, size=(n, 12)).astype(np.int32) + (np.arange(n)[:, None] % 600)
    tok = rng.integers(0, V, size=R).astype(np.int32)
    req = np.repeat(np.arange(n), q_len).astype(np.int32)
    at = np.arange(R) - cu[req]
    mask = np.array([(2 << i) - 1 for i in at], np.int32)[:, None]   # a chain: a token and all before it
    x = torch.randn(R, V, device="cuda")
    want = x.double().cpu().numpy()
    for r in range(R):
        b = req[r]
        count, seen = np.zeros(V), np.zeros(V, bool)
        path = tok[cu[b]:cu[b] + at[r] + 1]
        np.add.at(count, np.concatenate([hist[b, 5:], path]), 1)
        seen[hist[b, :5]] = True
        y = want[r]
        y = np.where(seen | (count > 0), np.where(y > 0, y / 1.25, y * 1.25), y)
        want[r] = y - 0.5 * count - 3.0 * (count > 0)
    full = lambda v: torch.full((n,), v, device="cuda")   # noqa: E731
    rules = ats.LogitRules(hist=_dev(hist.ravel()), hist_off=_dev(12 * np.arange(n + 1)), prompt_len=_dev(np.full(n, 5)),
                           repetition=full(1.25), frequency=full(0.5), presence=full(3.0), tree_tok=_dev(tok), cu_q=_dev(cu))
    first = None
    for _ in range(20):
        got = ats.op_adjust_logits(x, _dev(req), rules, mask=_dev(mask))
        first = got if first is None else first
        assert torch.equal(got, first)
    # four operations in 32 bits on terms of up to |x| + 12
    assert np.all(np.abs(first.double().cpu().numpy() - want) <= 2.0 ** -21 * (np.abs(want) + 20))


# ---------------------------------------------------------------------------------------------------
# grammar states past the table
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("inp", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [70, 9001])
def test_a_grammar_state_past_the_table_allows_nothing(ats, V, inp):
    x = torch.randn(5, V, device="cuda").to(inp)
    words = -(-V // 32)
    rules = ats.LogitRules(n_req=1, grammar=torch.full((2, words), -1, dtype=torch.int32, device="cuda"),
                           bias_off=_dev([0, 1]), bias_tok=_dev([5]), bias_val=torch.full((1,), 3.0, device="cuda"))
    got = ats.op_adjust_logits(x, _dev([0, 0, 0, -1, 0]), rules, state=_dev([1, 2, 2 ** 31 - 1, 5, -1]))
    assert bool((got[1:4] == NEG).all())
    want = x.float()
    want[:, 5] += 3
    assert torch.equal(got[[0, 4]], want.to(inp)[[0, 4]])


# ---------------------------------------------------------------------------------------------------
# a wait that gives up
# ---------------------------------------------------------------------------------------------------
def test_a_wait_that_gives_up_is_reported(ats):
    """Counters of partial results that start far below zero: the CTAs that wait for them give up after the kernel's own limit
    and return, the status says so once, and with the counters zeroed the same call is right."""
    from paper_2410_05165_gb300 import binding
    kc, vc = (torch.randn(300, 16, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16)
    args = (q, kc, vc, _dev([0, 1]), _dev([4700]), _dev(np.arange(300)[None]))
    want = ats.op_tree_attention(*args)   # (one block of 37 tiles: cut for many CTAs)
    assert ats.op_status(noalloc=True) == ats.OK
    w = binding.op_tree_attention_workspace(q.device, torch.cuda.current_stream().cuda_stream)
    counters = w[:binding.TREE_ATTENTION_COUNTER_BYTES].view(torch.int32)
    counters[:torch.cuda.get_device_properties(0).multi_processor_count] = -100000   # (the arrivals come first)
    ats.op_tree_attention(*args)
    assert ats.op_status(noalloc=True) == ats.E_TIMEOUT
    assert ats.op_status(noalloc=True) == ats.OK
    assert int(counters.abs().max()) == 0
    assert torch.equal(ats.op_tree_attention(*args), want)
    assert ats.op_status(noalloc=True) == ats.OK


# ---------------------------------------------------------------------------------------------------
# streams
# ---------------------------------------------------------------------------------------------------
def _calls(ats):
    """Each operator's call on a stream: the output that is looked at, as a function of the stream."""
    kc, vc = (torch.randn(60, 16, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(9, 4, 64, device="cuda").to(torch.bfloat16)
    cu, ctx, table = _dev([0, 1, 9]), _dev([300, 100]), _dev(np.arange(60).reshape(2, 30))
    qkv, slot = torch.randn(9, 8 * 64, device="cuda"), torch.arange(900, 909, device="cuda")
    x, req = torch.randn(9, 1003, device="cuda"), _dev([0] + [1] * 8)
    rules = ats.LogitRules(n_req=2, temperature=torch.full((2,), 0.5, device="cuda"))
    q_len, kv_len, n_free = _dev([1, 8]), _dev([300, 100]), _dev([5])
    return {"plan": lambda s: ats.op_batch_plan(q_len, kv_len, table, table.flatten(), n_free, 16, 9, stream=s).slot,
            "append": lambda s: ats.op_rope_append(qkv, 4, kc, vc, slot, stream=s),
            "attention": lambda s: ats.op_tree_attention(q, kc, vc, cu, ctx, table, stream=s),
            "logits": lambda s: ats.op_adjust_logits(x, req, rules, stream=s)}


@pytest.mark.parametrize("op", ["plan", "append", "attention", "logits"])
def test_outputs_on_a_stream_take_no_memory_that_the_current_one_reads(ats, op):
    """Memory given back on the current stream, with a read of it still to come there, is not what a call on another stream
    writes its output into."""
    call, s = _calls(ats)[op], torch.cuda.Stream()
    want = call(None).clone()
    torch.cuda.synchronize()
    old = torch.full_like(want, 5)
    kept, at = torch.empty_like(old), old.data_ptr()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)   # (some 50 ms)
    kept.copy_(old)
    del old
    out = call(s)
    assert out.data_ptr() != at
    torch.cuda.synchronize()
    assert bool((kept == 5).all()) and torch.equal(out, want)


@pytest.mark.parametrize("op", ["plan", "append", "attention", "logits"])
def test_outputs_on_a_stream_stay_until_the_current_one_has_read_them(ats, op):
    """Given back with a read of it still to come on the current stream, an output is not the next tensor of its own stream."""
    call, s = _calls(ats)[op], torch.cuda.Stream()
    want = call(None).clone()
    torch.cuda.synchronize()
    out = call(s)
    s.synchronize()
    kept, at = torch.empty_like(out), out.data_ptr()
    torch.cuda._sleep(100_000_000)
    kept.copy_(out)
    del out
    with torch.cuda.stream(s):
        other = torch.full_like(want, 5)
    assert other.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(kept, want)


def test_attention_on_a_stream_that_a_capture_forks_to(ats):
    """The workspace of a captured call is of the stream that the call is on, not of the one that was current: its counters are
    zeroed before the call, and its memory is not given to the capturing stream's next tensors."""
    kc, vc = (torch.randn(60, 16, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(9, 4, 64, device="cuda").to(torch.bfloat16)
    args = (_dev([0, 1, 9]), _dev([300, 100]), _dev(np.arange(60).reshape(2, 30)))
    want = ats.op_tree_attention(q, kc, vc, *args)
    out = torch.zeros(3, *q.shape, dtype=q.dtype, device="cuda")
    main, side, g = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=main):
        side.wait_stream(main)
        others = []
        for i in range(3):
            ats.op_tree_attention(q, kc, vc, *args, out=out[i], stream=side)
            others.append(torch.full((50_000_000,), 255, dtype=torch.uint8, device="cuda"))   # (more than a workspace)
        main.wait_stream(side)
    for _ in range(5):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in out) and all(bool((x == 255).all()) for x in others)
    assert ats.op_status(noalloc=True) == ats.OK


def test_captured_attention_shares_no_workspace(ats, monkeypatch):
    """Two graphs captured on a stream that had a workspace: each has its own, one for all its calls, and replays beside each
    other and beside calls on that stream are right."""
    from paper_2410_05165_gb300 import binding
    kc, vc = (torch.randn(300, 16, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    qs = torch.randn(3, 4, 8, 64, device="cuda").to(torch.bfloat16)
    args = (_dev([0, 4]), _dev([4700]), _dev(np.arange(300)[None]))   # (one block, cut for many CTAs)
    want = torch.stack([ats.op_tree_attention(q, kc, vc, *args) for q in qs])
    got = torch.zeros_like(want)
    torch.cuda.synchronize()
    lib, used = binding.load(), []

    class Watched:
        def __getattr__(self, name):
            f = getattr(lib, name)
            if name != "atspeed_op_tree_attention":
                return f
            return lambda *a: used.append(a[-1]) or f(*a)

    warm = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with monkeypatch.context() as m:
        m.setattr(binding, "load", Watched)
        with torch.cuda.stream(warm):
            ats.op_tree_attention(qs[2], kc, vc, *args, out=got[2])
        warm.synchronize()
        for i, g in enumerate(graphs):
            with torch.cuda.graph(g, stream=warm):
                for _ in range(4):
                    ats.op_tree_attention(qs[i], kc, vc, *args, out=got[i])
    assert len(used) == 9 and len({used[0], used[1], used[5]}) == 3
    assert len(set(used[1:5])) == 1 and len(set(used[5:])) == 1   # (one a graph, zeroed once)
    assert not {used[1], used[5]} & {w.data_ptr() for w in binding._tree_ws.values()}
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        got.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            with torch.cuda.stream(warm):
                ats.op_tree_attention(qs[2], kc, vc, *args, out=got[2])
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    assert ats.op_status(noalloc=True) == ats.OK


def test_attention_on_two_streams_at_once(ats):
    kc, vc = (torch.randn(300, 16, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    qs = torch.randn(2, 4, 8, 64, device="cuda").to(torch.bfloat16)
    args = (_dev([0, 4]), _dev([4700]), _dev(np.arange(300)[None]))
    want = torch.stack([ats.op_tree_attention(q, kc, vc, *args) for q in qs])
    got = torch.zeros_like(want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            ats.op_tree_attention(qs[i], kc, vc, *args, out=got[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and ats.op_status(noalloc=True) == ats.OK


def test_a_timeout_once_read_asks_nothing_of_a_stream_that_is_gone(ats, monkeypatch):
    """(The status is a fake's.)  The workspace of a stream that its owner has destroyed is cleared with the others."""
    import ctypes

    from paper_2410_05165_gb300 import binding
    rt, handle = torch.cuda.cudart(), ctypes.c_size_t()
    assert int(rt.cudaStreamCreate(ctypes.addressof(handle))) == 0
    w = binding.op_tree_attention_workspace(torch.device("cuda", 0), handle.value)
    torch.cuda.synchronize()
    assert int(rt.cudaStreamDestroy(handle.value)) == 0
    w[:64] = 1

    class Failed:
        @staticmethod
        def atspeed_op_status(stream, ws):
            return binding.E_TIMEOUT

    with monkeypatch.context() as m:
        m.setattr(binding, "load", lambda: Failed)
        assert binding.op_status(noalloc=True) == binding.E_TIMEOUT
    assert int(w[:binding.TREE_ATTENTION_COUNTER_BYTES].sum()) == 0
    binding._tree_ws.pop((0, handle.value))


# ---------------------------------------------------------------------------------------------------
# nothing to take, nothing listed, one row
# ---------------------------------------------------------------------------------------------------
def test_plan_with_no_free_page(ats):
    """An empty free list: requests that need no page are served, the others are not."""
    table = _dev([[4, 0], [7, 0]])
    p = ats.op_batch_plan(_dev([1, 1]), _dev([15, 16]), table, _dev(np.zeros(0, np.int32)), _dev([0]), 16, 2)
    assert p.state.tolist() == [ats.PLAN_OK, ats.PLAN_NO_PAGES] and p.slot.tolist() == [4 * 16 + 15, -1]
    assert int(p.used) == 0 and table.tolist() == [[4, 0], [7, 0]]


def test_no_bias_listed(ats):
    """Lists of biases that hold none in this step."""
    x = torch.randn(3, 100, device="cuda")
    none = _dev(np.zeros(0, np.int32))
    rules = ats.LogitRules(n_req=2, bias_off=_dev([0, 0, 0]), bias_tok=none, bias_val=none.float(),
                           temperature=torch.full((2,), 2.0, device="cuda"))
    assert torch.equal(ats.op_adjust_logits(x, _dev([0, 1, 1]), rules), x / 2)


def test_one_row_of_any_stride(ats):
    """The distance between rows means nothing where there is one: logits and projections as columns that were transposed."""
    col = torch.randn(1003, 1, device="cuda")
    rules = ats.LogitRules(n_req=1, temperature=torch.full((1,), 2.0, device="cuda"))
    out = torch.empty(1003, 1, device="cuda").t()
    assert torch.equal(ats.op_adjust_logits(col.t(), _dev([0]), rules), col.t() / 2)
    assert torch.equal(ats.op_adjust_logits(col.t(), _dev([0]), rules, out=out), col.t() / 2)
    kc, vc = (torch.randn(4, 16, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    qkv = torch.randn(8 * 64, 1, device="cuda")
    slot = torch.tensor([35], device="cuda")
    q = ats.op_rope_append(qkv.t(), 4, kc, vc, slot)
    assert torch.equal(q.flatten(), qkv[:256, 0].to(torch.bfloat16))
    assert torch.equal(kc[2, 3].flatten(), qkv[256:384, 0].to(torch.bfloat16))
    args = (kc, vc, _dev([0, 1]), _dev([35]), _dev([[0, 1, 2]]))
    odd = torch.as_strided(q.clone(), (1, 4, 64), (1, 64, 1))
    assert torch.equal(ats.op_tree_attention(odd, *args), ats.op_tree_attention(q, *args))
    into = torch.empty_like(q)
    ats.op_tree_attention(q, *args, out=torch.as_strided(into, (1, 4, 64), (1, 64, 1)))
    assert torch.equal(into, ats.op_tree_attention(q, *args))


def test_one_head_of_any_stride(ats):
    kc, vc = (torch.randn(4, 16, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(3, 1, 64, device="cuda").to(torch.bfloat16)
    args = (kc, vc, _dev([0, 3]), _dev([40]), _dev([[0, 1, 2]]))
    other = q.reshape(1, 3, 64).transpose(0, 1)   # (the heads' stride is that of all tokens)
    assert other.stride(1) != 64
    out = torch.empty(1, 3, 64, dtype=q.dtype, device="cuda").transpose(0, 1)
    want = ats.op_tree_attention(q, *args)
    assert torch.equal(ats.op_tree_attention(other, *args), want)
    assert torch.equal(ats.op_tree_attention(q, *args, out=out), want)


def test_lists_that_end_near_31_bits(ats):
    """Entries at the end of lists of 2^31 - 1: the places past them do not come round to negative ones."""
    end, V = (1 << 31) - 1, 100
    hist, bias_tok = (torch.empty(end, dtype=torch.int32, device="cuda") for _ in range(2))
    bias_val = torch.empty(end, device="cuda")
    hist[-3:] = _dev([7, 9, 9])
    bias_tok[-2:], bias_val[-2:] = _dev([7, 50]), torch.tensor([2.0, -1.0], device="cuda")
    rules = ats.LogitRules(hist=hist, hist_off=_dev([end - 3, end]), frequency=torch.full((1,), 0.5, device="cuda"),
                           bias_off=_dev([end - 2, end]), bias_tok=bias_tok, bias_val=bias_val)
    x = torch.zeros(2, V, device="cuda")
    want = x.clone()
    want[:, 7], want[:, 9], want[:, 50] = 1.5, -1.0, -1.0
    assert torch.equal(ats.op_adjust_logits(x, _dev([0, 0]), rules), want)


def test_plan_of_positions_near_31_bits(ats):
    """Pages of 2^30 tokens and a request whose last position is 2^31 - 2; the next one would need a position past that."""
    page, kv = 1 << 30, (1 << 31) - 9
    table = _dev([[5, 6, -7], [8, 9, -7], [-7, -7, -7]])
    p = ats.op_batch_plan(_dev([8, 9, 2]), _dev([kv, kv, 0]), table, _dev([3]), _dev([1]), page, 20)
    assert p.state.tolist() == [ats.PLAN_OK, ats.PLAN_LIMIT, ats.PLAN_OK] and p.ctx_len.tolist() == [kv, -1, 0]
    assert table.tolist() == [[5, 6, -7], [8, 9, -7], [3, -7, -7]]
    assert p.pos.tolist()[:8] == [kv + i for i in range(8)] and p.pos.tolist()[17:] == [0, 1, 0]
    assert p.slot.tolist() == [6 * page + kv - page + i for i in range(8)] + [-1] * 9 + [3 * page, 3 * page + 1, -1]


# ---------------------------------------------------------------------------------------------------
# rows of no request
# ---------------------------------------------------------------------------------------------------
def test_rows_of_no_request_are_left_as_they_are(ats):
    """So that a step can be divided among calls over neighbouring requests, each with its own kind of mask."""
    kc, vc = (torch.randn(12, 16, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(40, 4, 64, device="cuda").to(torch.bfloat16)
    cu, ctx, table = _dev([0, 5, 6, 30]), _dev([20, 33, 10]), _dev([[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]])
    lse = torch.full((40, 4), 7.0, device="cuda")
    out = torch.full_like(q, 3.0)
    ats.op_tree_attention(q, kc, vc, cu, ctx, table, out=out, lse=lse)
    assert bool((out[30:] == 3).all()) and bool((lse[30:] == 7).all())
    parts = torch.full_like(q, 3.0)
    ats.op_tree_attention(q, kc, vc, cu[2:], ctx[2:], table[2:], out=parts)
    assert bool((parts[:6] == 3).all())
    ats.op_tree_attention(q, kc, vc, cu[:3], ctx[:2], table[:2], out=parts)
    tol = 2.0 ** -8 * out.float().abs() + 2.0 ** -7 * vc.float().abs().max()   # (each call divides its key ranges its own way)
    assert bool(((parts.float() - out.float()).abs() <= tol).all())
