"""The serving step's operators together, as examples/tree_decode.py runs them: what a batch of users is told by tree
decoding, against one token a step and against the model in 64 bits over the whole texts."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    import __graft_entry__
    __graft_entry__.build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tree_decode.py")
    spec = importlib.util.spec_from_file_location("tree_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


SAY = 24


@pytest.fixture(scope="module")
def told(ex):
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, ex.VOCAB, (n,), generator=g).tolist() for n in (1, 33, 130)]
    model = ex.Model(3)
    plain = ex.Decoder(model, prompts)
    plain.run(SAY, ex.no_draft)
    known = [t[:] for t in plain.text]

    def knows(b, text):   # two right drafts, below each other, a wrong one beside each
        rest = known[b][len(text):len(text) + 2]
        tokens = [x for t in rest for x in ((t + 1) % ex.VOCAB, t)]
        return tokens, [2 * (j // 2) - 1 for j in range(len(tokens))]

    tree = ex.Decoder(model, prompts)
    tree.run(SAY, knows)
    return model, prompts, plain, tree


def _exact_logits(ex, model, d, b, text):
    """Adjusted logits of the token after each of a text's places, in 64 bits."""
    T, f64 = len(text), torch.float64
    tok = torch.tensor(text, device="cuda")
    h = model.embed[tok].double()
    half = ex.HD // 2
    ang = torch.arange(T, device="cuda", dtype=f64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=f64) / half)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]

    def norm(x):
        return x / (x.square().mean(1, keepdim=True) + ex.EPS).sqrt()

    def rope(x):
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

    for w in model.layers:
        qkv = (norm(h) @ w["qkv"].double().T).view(T, -1, ex.HD)
        q, k, v = rope(qkv[:, :ex.HEADS]), rope(qkv[:, ex.HEADS:ex.HEADS + ex.KV_HEADS]), qkv[:, ex.HEADS + ex.KV_HEADS:]
        k, v = (x.repeat_interleave(ex.HEADS // ex.KV_HEADS, 1) for x in (k, v))
        s = torch.einsum("ihc,jhc->hij", q, k) * ex.HD ** -0.5
        s = s.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        h = h + torch.einsum("hij,jhc->ihc", s.softmax(-1), v).reshape(T, -1) @ w["o"].double().T
        up = norm(h) @ w["up"].double().T
        h = h + (torch.nn.functional.silu(up[:, :ex.FF]) * up[:, ex.FF:]) @ w["down"].double().T
    x = norm(h) @ model.head.double().T
    rep, freq, temp = (float(t[b]) for t in (d.repetition, d.frequency, d.temperature))
    for i in range(d.prompt_len[b] - 1, T):
        seen = torch.bincount(tok[:i + 1], minlength=ex.VOCAB)
        count = torch.bincount(tok[d.prompt_len[b]:i + 1], minlength=ex.VOCAB)
        y = torch.where(seen > 0, torch.where(x[i] > 0, x[i] / rep, x[i] * rep), x[i]) - freq * count
        if b == 0:
            y[7] = float("-inf")
            y[11] += 1.0
        if i % 2 == 1:
            y[1::2] = float("-inf")
        x[i] = y / temp
    return x


def test_what_is_told_is_the_models_choice(ex, told):
    """Each told token is the best of the exact logits, but for the roundings to 16 bits on the way.  Those: about 16 places
    (q, k, v, weights, attention, SwiGLU, norms of two layers), each a relative error of up to 2^-8, 2^-8 / sqrt 3 in the
    root mean square, of a stream that the head turns into logits of unit size: 4 * 2^-8 / sqrt 3 = 0.009 together, five
    times that for the worst of the choices, for both of the logits compared, divided by the temperature 0.8: 0.113."""
    model, prompts, plain, tree = told
    for d in (plain, tree):
        for b, text in enumerate(d.text):
            x = _exact_logits(ex, model, d, b, text[:-1])[d.prompt_len[b] - 1:]
            chosen = x.gather(1, torch.tensor(text[d.prompt_len[b]:], device="cuda")[:, None])[:, 0]
            assert bool((chosen >= x.max(1).values - 0.113).all())


def test_tree_tells_what_one_token_a_step_does(told):
    """In a third of the steps (two drafts and the token after them).  A result's last bits may differ with the step it is
    computed in, a choice with them where two logits are next to each other: the first difference of a user ends the comparison,
    and the exact logits (above) have the last word on both."""
    model, prompts, plain, tree = told
    same = 0
    for t, u, p in zip(tree.text, plain.text, prompts):
        n = min(len(t), len(u))
        same += next((i for i in range(n) if t[i] != u[i]), n) - len(p)
    assert same >= 2 * SAY * len(prompts) // 3
    if all(t[:len(p) + SAY] == u[:len(p) + SAY] for t, u, p in zip(tree.text, plain.text, prompts)):
        assert tree.steps == SAY // 3 and plain.steps == SAY


def test_rules_hold(ex, told):
    _, prompts, plain, tree = told
    for d in (plain, tree):
        for b, (t, p) in enumerate(zip(d.text, prompts)):
            assert all(x % 2 == 0 for i, x in enumerate(t[len(p):], len(p)) if (i - 1) % 2 == 1)
            assert b != 0 or 7 not in t[len(p):]


def test_pages_are_kept_once(ex, told):
    _, _, plain, tree = told
    for d in (plain, tree):
        held = [x for row, k in zip(d.table.tolist(), d.kv_len) for x in row[:-(-k // ex.PAGE)]]
        assert sorted(held + d.free) == list(range(d.caches[0][0].shape[0]))
        assert all(k < len(t) for k, t in zip(d.kv_len, d.text))


def test_a_step_that_does_not_fit_is_told(ex, told):
    model, prompts, _, _ = told
    d = ex.Decoder(model, prompts, pages=13)
    with pytest.raises(RuntimeError):
        d.run(300, ex.no_draft)
