"""Beam selection, page fork, page copies and token compaction together, as examples/beam_decode.py runs them: the beams' scores and
what is cached for them against the model in 64 bits, shared pages, and trees whose accepted paths stay in the cache."""
import importlib.util
import os
import sys
from types import SimpleNamespace

import pytest
import torch

from test_gpu_tree_decode import _exact_logits

pytestmark = pytest.mark.gpu
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
# one logit's error against 64 bits, as test_gpu_tree_decode derives it: 5 * 4 * 2^-8 / sqrt 3
LOGIT = 0.045
SAY = 12


@pytest.fixture(scope="module")
def ex():
    import __graft_entry__
    __graft_entry__.build()
    sys.path.insert(0, EXAMPLES)
    spec = importlib.util.spec_from_file_location("beam_decode", os.path.join(EXAMPLES, "beam_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def prompts(ex):
    g = torch.Generator().manual_seed(5)
    return [torch.randint(0, ex.td.VOCAB, (n,), generator=g).tolist() for n in (1, 33, 130, 16)]


@pytest.fixture(scope="module")
def beams(ex, prompts):
    b = ex.Beams(ex.td.Model(3), prompts, width=5, say=SAY)
    b.run()
    return b


NO_RULES = SimpleNamespace(repetition=[1.0] * 2, frequency=[0.0] * 2, temperature=[1.0] * 2, prompt_len=[1, 1])


def _log_probs(ex, model, text):
    """Of the token after each of a text's places, in 64 bits, over the allowed ones (row 1 of _exact_logits: no rule but the grammar)."""
    x = _exact_logits(ex.td, model, NO_RULES, 1, text)
    return torch.log_softmax(x, dim=1)


def test_scores_are_the_models(ex, prompts, beams):
    """A step's log-probability is off by a logit's error and the log-sum's, which is at most a logit's."""
    for u, p in enumerate(prompts):
        scores = beams.score.view(-1, beams.width)[u].tolist()
        assert scores == sorted(scores, reverse=True)
        lists = beams.lists()[u]
        assert len(set(map(tuple, lists))) == beams.width
        for said, score in zip(lists, scores):
            lp = _log_probs(ex, beams.model, (p + said)[:-1])[len(p) - 1:]
            want = float(lp.gather(1, torch.tensor(said, device="cuda")[:, None]).sum())
            assert abs(score - want) <= 2 * LOGIT * SAY, (u, score, want)


def test_beams_are_the_best(ex, prompts, beams):
    """No continuation that was left out is better than the worst beam by more than both scores may be off, seen from the beams' last step."""
    for u, p in enumerate(prompts):
        lists, worst = beams.lists()[u], float(beams.score.view(-1, beams.width)[u, -1])
        parents = {tuple(s[:-1]) for s in lists}
        for said in parents:
            lp = _log_probs(ex, beams.model, p + list(said))[len(p) - 1:]
            at = sum(float(lp[i, t]) for i, t in enumerate(said))
            for v in torch.topk(lp[-1], beams.width).indices.tolist():
                if list(said) + [v] not in lists:
                    assert at + float(lp[-1, v]) <= worst + 4 * LOGIT * SAY


def _first_keys(ex, model, tokens):
    """The first layer's keys [T][heads][HD] in 64 bits: of the token and its position alone."""
    td = ex.td
    h = model.embed[torch.tensor(tokens, device="cuda")].double()
    x = h / (h.square().mean(1, keepdim=True) + td.EPS).sqrt()
    k = (x @ model.layers[0]["qkv"].double().T).view(len(tokens), -1, td.HD)[:, td.HEADS:td.HEADS + td.KV_HEADS]
    half = td.HD // 2
    ang = torch.arange(len(tokens), device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(half, device="cuda", dtype=torch.float64) / half)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    return torch.cat([k[..., :half] * cos - k[..., half:] * sin, k[..., half:] * cos + k[..., :half] * sin], -1)


def _check_keys(ex, model, cache, row, tokens):
    """Cached keys of a row of a block table.  The norm's rows are rounded to 16 bits (2^-8 of each of 256 terms of a sum of unit size,
    in the root mean square 2^-8 / sqrt 3, five times that for the worst), a key once more (2^-8 of up to 5)."""
    td = ex.td
    k = cache[torch.tensor(row, device="cuda").long()].reshape(-1, td.KV_HEADS, td.HD)[:len(tokens)].double()
    assert float((k - _first_keys(ex, model, tokens)).abs().max()) <= 5 * 2 ** -8 / 3 ** 0.5 + 5 * 2 ** -8


def test_every_beam_finds_its_own_tokens(ex, prompts, beams):
    for u, p in enumerate(prompts):
        for i, said in enumerate(beams.lists()[u]):
            r = u * beams.width + i
            tokens = p + said[:-1]
            assert int(beams.kv_len[r]) == len(tokens)
            _check_keys(ex, beams.model, beams.caches[0][0], beams.table[r, :-(-len(tokens) // ex.td.PAGE)].tolist(), tokens)


def test_pages_are_shared_and_given_back(ex, prompts, beams):
    pages = beams.ref.numel()
    holds = [0] * pages
    for row, k in zip(beams.table.tolist(), beams.kv_len.tolist()):
        used = -(-k // ex.td.PAGE)
        assert all(e == -1 for e in row[used:])
        for e in row[:used]:
            holds[e] += 1
    assert beams.ref.tolist() == holds
    assert beams.free.tolist()[:int(beams.n_free)] == [i for i, h in enumerate(holds) if h == 0]
    # full pages of the prompts are in one place, partial last ones in a place of their own for every beam
    for u, p in enumerate(prompts):
        rows = beams.table[u * beams.width:(u + 1) * beams.width].tolist()
        for c in range((len(p) - 1) // ex.td.PAGE):
            assert len({row[c] for row in rows}) == 1
        k = len(p) + SAY - 1
        if k % ex.td.PAGE:
            assert len({row[k // ex.td.PAGE] for row in rows}) == beams.width
    assert beams.close() == pages


def test_replayed_steps_are_those_of_single_calls(ex, prompts, beams):
    again = ex.Beams(beams.model, prompts, width=5, say=SAY)
    while int(again.steps) < SAY:
        again.step()
    for name in ("said", "score", "table", "kv_len", "ref", "free", "n_free"):
        assert torch.equal(getattr(again, name), getattr(beams, name)), name


def test_ended_beams_stay_as_they_are(ex, prompts, beams):
    """With the most frequent token of the sequences as the end: a beam that said it keeps its score and says it again."""
    said = [t for user in beams.lists() for s in user for t in s[:SAY // 2]]
    end = max(set(said), key=said.count)
    b = ex.Beams(beams.model, prompts, width=5, say=SAY, end=end)
    scores = []
    while int(b.steps) < SAY:
        b.step()
        scores.append((b.said[:, :int(b.steps)].tolist(), b.score.tolist()))
    seen = 0
    for (before, s0), (after, s1) in zip(scores, scores[1:]):
        ended = {tuple(x): s for x, s in zip(before, s0) if x[-1] == end}
        for x, s in zip(after, s1):
            if tuple(x[:-1]) in ended:
                seen += 1
                assert x[-1] == end and s == ended[tuple(x[:-1])]
    assert seen


def test_accepted_paths_are_kept(ex, prompts):
    td = ex.td
    model = td.Model(3)
    plain = td.Decoder(model, prompts)
    plain.run(24, td.no_draft)
    known = [t[:] for t in plain.text]

    def knows(b, text):   # a wrong draft before each right one, below each other
        rest = known[b][len(text):len(text) + 2]
        tokens = [x for t in rest for x in ((t + 1) % td.VOCAB, t)]
        return tokens, [2 * (j // 2) - 1 for j in range(len(tokens))]

    d = ex.Keeper(model, prompts)
    d.run(24, knows)
    assert d.moved > 0
    for b, text in enumerate(d.text):
        assert d.kv_len[b] == len(text) - 1   # all but the last one, which was chosen from them
        _check_keys(ex, model, d.caches[0][0], d.table[b, :-(-d.kv_len[b] // td.PAGE)].tolist(), text[:-1])
        x = _exact_logits(td, model, d, b, text[:-1])[d.prompt_len[b] - 1:]
        chosen = x.gather(1, torch.tensor(text[d.prompt_len[b]:], device="cuda")[:, None])[:, 0]
        assert bool((chosen >= x.max(1).values - 0.113).all())   # (test_gpu_tree_decode's bound)
    held = sorted(e for row, k in zip(d.table.tolist(), d.kv_len) for e in row[:-(-k // td.PAGE)])
    assert held == [i for i, r in enumerate(d.ref.tolist()) if r] and max(d.ref.tolist()) == 1
    assert d.pages.tolist()[:int(d.n_free)] == [i for i, r in enumerate(d.ref.tolist()) if r == 0]


def _small_pool(ex, pages):
    """One user's 17 prompt tokens, five beams: one full page that all share, a second one of each, and up to four copies a step."""
    g = torch.Generator().manual_seed(7)
    prompt = torch.randint(0, ex.td.VOCAB, (ex.td.PAGE + 1,), generator=g).tolist()
    return prompt, ex.Beams(ex.td.Model(3), [prompt], width=5, say=SAY, pages=pages)


def test_a_pool_that_is_just_large_enough(ex):
    (_, a), (_, b) = _small_pool(ex, 10), _small_pool(ex, 256)
    a.run()
    b.run()
    assert torch.equal(a.said, b.said) and torch.equal(a.score, b.score)


def test_beams_that_get_no_page_are_dropped(ex):
    """With six pages nothing is left for a beam that goes on twice: an error at the end, and what has a score then is the model's."""
    prompt, b = _small_pool(ex, 6)
    with pytest.raises(RuntimeError, match="not all beams"):
        b.run()
    assert int(b.steps) == SAY
    left = [r for r, s in enumerate(b.score.tolist()) if s > float("-inf")]
    assert 0 < len(left) < 5
    for r in left:
        said = b.said[r].tolist()
        tokens = prompt + said[:-1]
        assert int(b.kv_len[r]) == len(tokens)
        _check_keys(ex, b.model, b.caches[0][0], b.table[r, :-(-len(tokens) // ex.td.PAGE)].tolist(), tokens)
        lp = _log_probs(ex, b.model, tokens)[len(prompt) - 1:]
        want = float(lp.gather(1, torch.tensor(said, device="cuda")[:, None]).sum())
        assert abs(float(b.score[r]) - want) <= 2 * LOGIT * SAY


def test_a_prompt_that_gets_no_page(ex):
    with pytest.raises(RuntimeError, match="not all beams"):
        _small_pool(ex, 1)
