"""Tree decoding for a batch of users with the stateless operators: a small decoder with grouped heads, random weights.

    python examples/tree_decode.py            # drafts from what followed a token before; compared with one token a step

Every step is plan -> (rope_append -> tree_attention, once per layer) -> adjust_logits.  A step's tokens of a user are the
accepted ones that are not in the cache yet, as a chain, and below the last of them a tree of drafts.  Where the chosen
next token is one of the drafts, it and the walk below it are accepted.  The chain's keys and values stay in the cache, the
drafts' are written over by the next step.  A page that only drafts had reached goes back to the free list.
"""
import os
import sys
from typing import Callable, List, Sequence, Tuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_05165_gb300 as ats  # noqa: E402

LAYERS, D, HEADS, KV_HEADS, HD, FF, VOCAB, PAGE = 2, 256, 8, 2, 32, 512, 1003, 16
MAX_TOKENS = 256      # of a step, all users' together (the matrix products' rows)
MASK_WORDS = 4        # up to 128 tokens a user and step
EPS = 1e-5

Draft = Tuple[List[int], List[int]]   # tokens, and each one's parent among them (-1: the last accepted token)


class Model:
    def __init__(self, seed: int = 0):
        g = torch.Generator("cuda").manual_seed(seed)

        def weight(rows, cols):
            return torch.randn(rows, cols, generator=g, device="cuda").mul_(cols ** -0.5).to(torch.bfloat16)

        self.embed = torch.randn(VOCAB, D, generator=g, device="cuda")
        self.layers = [dict(qkv=weight((HEADS + 2 * KV_HEADS) * HD, D), o=weight(D, HEADS * HD), up=weight(2 * FF, D),
                            down=weight(D, FF)) for _ in range(LAYERS)]
        self.head = weight(VOCAB, D)
        self.norm = torch.ones(D, dtype=torch.bfloat16, device="cuda")

    def logits(self, tokens: torch.Tensor, plan: "ats.BatchPlan", table: torch.Tensor, caches) -> torch.Tensor:
        """Logits of a step's MAX_TOKENS rows (those past its tokens mean nothing)."""
        T = MAX_TOKENS
        h = self.embed[tokens.clamp(min=0)]
        for w, (k, v) in zip(self.layers, caches):
            qkv = ats.op_gemm(w["qkv"], ats.op_rmsnorm(h, self.norm, EPS), T)
            q = ats.op_rope_append(qkv, HEADS, k, v, plan.slot, pos=plan.pos)
            out = torch.zeros_like(q)   # (rows of no request are not written)
            ats.op_tree_attention(q, k, v, plan.cu_q, plan.ctx_len, table, mask=plan.mask, out=out)
            ats.op_gemm(w["o"], out.view(T, HEADS * HD), T, Y=h, accumulate=True)
            ats.op_gemm(w["down"], ats.op_gemm_swiglu(w["up"], ats.op_rmsnorm(h, self.norm, EPS), T), T, Y=h, accumulate=True)
        return ats.op_gemm(self.head, ats.op_rmsnorm(h, self.norm, EPS), T)


def _i32(x) -> torch.Tensor:
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Decoder:
    """Users' texts, their caches and the rules of what may be said."""

    def __init__(self, model: Model, prompts: Sequence[Sequence[int]], pages: int = 256, width: int = 32):
        self.model, n = model, len(prompts)
        self.text = [list(p) for p in prompts]
        self.prompt_len = [len(p) for p in prompts]
        self.kv_len = [0] * n
        # BF16 keys, FP16 values: the layout of the library's own caches
        self.caches = [(torch.zeros(pages, PAGE, KV_HEADS, HD, dtype=torch.bfloat16, device="cuda"),
                        torch.zeros(pages, PAGE, KV_HEADS, HD, dtype=torch.float16, device="cuda")) for _ in range(LAYERS)]
        self.table = torch.zeros(n, width, dtype=torch.int32, device="cuda")
        self.free = list(range(pages))
        self.steps = 0
        # penalties by user; user 0 is not to say token 7 and likes token 11; at odd positions only every other token is allowed
        self.repetition = torch.linspace(1.0, 1.3, n, device="cuda")
        self.frequency = torch.linspace(0.0, 0.4, n, device="cuda")
        self.temperature = torch.full((n,), 0.8, device="cuda")
        self.bias = dict(bias_off=_i32([0] + [2] * n), bias_tok=_i32([7, 11]),
                         bias_val=torch.tensor([float("-inf"), 1.0], device="cuda"))
        words = -(-VOCAB // 32)
        self.grammar = torch.stack([torch.full((words,), -1, dtype=torch.int32), torch.full((words,), 0x55555555, dtype=torch.int32)])
        self.grammar = self.grammar.to("cuda")
        self._prefill()

    def _plan(self, q_len: Sequence[int], parent=None) -> "ats.BatchPlan":
        plan = ats.op_batch_plan(_i32(q_len), _i32(self.kv_len), self.table, _i32(self.free), _i32([len(self.free)]), PAGE, MAX_TOKENS,
                                 parent=parent, mask_words=MASK_WORDS if parent is not None else 0)
        if int(plan.state.max()) != ats.PLAN_OK:
            raise RuntimeError(f"not all users can be served: {plan.state.tolist()}")
        self.free = self.free[int(plan.used):]
        return plan

    def _commit(self, kept: Sequence[int], q_len: Sequence[int]) -> None:
        """The first kept[b] of a step's q_len[b] tokens stay in the cache; pages past them are free again."""
        for b, row in enumerate(self.table.tolist()):
            have = -(-(self.kv_len[b] + q_len[b]) // PAGE)
            self.kv_len[b] += kept[b]
            self.free += row[-(-self.kv_len[b] // PAGE):have]

    def _step_tokens(self, parts: Sequence[Sequence[int]]) -> torch.Tensor:
        flat = [t for p in parts for t in p]
        if len(flat) > MAX_TOKENS:
            raise ValueError(f"{len(flat)} tokens in a step of {MAX_TOKENS}")
        return _i32(flat + [-1] * (MAX_TOKENS - len(flat)))

    def _prefill(self) -> None:
        """All but the prompts' last tokens, in pieces; causal within a piece (no parents, no mask)."""
        piece = MAX_TOKENS // len(self.text)
        while any(k < len(t) - 1 for k, t in zip(self.kv_len, self.text)):
            parts = [t[k:min(k + piece, len(t) - 1)] for k, t in zip(self.kv_len, self.text)]
            q_len = [len(p) for p in parts]
            plan = self._plan(q_len)
            self.model.logits(self._step_tokens(parts), plan, self.table, self.caches)
            self._commit(q_len, q_len)

    def step(self, drafts: Sequence[Draft]) -> torch.Tensor:
        """One step; appends what is accepted to each user's text.  Returns the adjusted logits [MAX_TOKENS][VOCAB]."""
        n = len(self.text)
        chains = [t[k:] for k, t in zip(self.kv_len, self.text)]
        parts = [c + d[0] for c, d in zip(chains, drafts)]
        parents = [list(range(-1, len(c) - 1)) + [len(c) + (p if p >= 0 else -1) for p in d[1]] for c, d in zip(chains, drafts)]
        q_len = [len(p) for p in parts]
        tokens = self._step_tokens(parts)
        plan = self._plan(q_len, parent=self._step_tokens(parents))
        logits = self.model.logits(tokens, plan, self.table, self.caches)
        # the texts are the history; of a path only the drafts come on top of it
        text = [t for u in self.text for t in u]
        off = [0]
        for u in self.text:
            off.append(off[-1] + len(u))
        rules = ats.LogitRules(hist=_i32(text), hist_off=_i32(off), prompt_len=_i32(self.prompt_len), repetition=self.repetition,
                               frequency=self.frequency, temperature=self.temperature, grammar=self.grammar,
                               tree_tok=self._step_tokens([[-1] * len(c) + d[0] for c, d in zip(chains, drafts)]),
                               cu_q=plan.cu_q, **self.bias)
        state = torch.where(plan.req < 0, -1, plan.pos & 1).to(torch.int32)
        ats.op_adjust_logits(logits, plan.req, rules, mask=plan.mask, state=state, out=logits)
        best, first = logits.argmax(dim=1).tolist(), 0
        self.path = []   # each user's tokens of this step that are accepted
        for b in range(n):
            at = len(chains[b]) - 1   # the last accepted token; then down the tree as long as a draft is what was chosen
            self.path.append(list(range(at)))
            while at is not None:
                self.path[b].append(at)
                self.text[b].append(best[first + at])
                at = next((j for j in range(len(chains[b]), q_len[b])
                           if parents[b][j] == at and parts[b][j] == self.text[b][-1]), None)
            first += q_len[b]
        self._commit([len(c) for c in chains], q_len)
        self.steps += 1
        return logits

    def run(self, tokens: int, draft: Callable[[int, List[int]], Draft]) -> None:
        """Until every user has said `tokens` tokens or more."""
        while any(len(t) - p < tokens for t, p in zip(self.text, self.prompt_len)):
            self.step([draft(b, t) for b, t in enumerate(self.text)])


def no_draft(_: int, text: List[int]) -> Draft:
    return [], []


def seen_before(_: int, text: List[int], depth: int = 4) -> Draft:
    """A chain of what followed the last token when it was last said, and beside its start what followed the time before."""
    places = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:2]
    tokens, parents = [], []
    for i in places:
        for j, t in enumerate(text[i + 1:i + 1 + depth]):
            tokens.append(t)
            parents.append(len(tokens) - 2 if j else -1)
    return tokens, parents


def main() -> None:
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (40, 200, 7, 93)]
    model, say = Model(), 48
    plain = Decoder(model, prompts)
    plain.run(say, no_draft)
    tree = Decoder(model, prompts)
    tree.run(say, seen_before)
    # the best case: drafts that know what will be said, and a wrong one beside each
    known = [t[:] for t in plain.text]

    def knows(b: int, text: List[int]) -> Draft:
        rest = known[b][len(text):len(text) + 4]
        tokens = [x for t in rest for x in ((t + 1) % VOCAB, t)]
        return tokens, [2 * (j // 2) - 1 for j in range(len(tokens))]

    best = Decoder(model, prompts)
    best.run(say, knows)
    for name, d in (("one token a step", plain), ("drafts from the text", tree), ("drafts that know", best)):
        same = sum(a == b for t, u in zip(d.text, plain.text) for a, b in zip(t, u))
        total = sum(min(len(t), len(u)) for t, u in zip(d.text, plain.text))
        print(f"{name}: {d.steps} steps, {same} of {total} tokens as with one token a step")
    if ats.op_status(noalloc=True) != 0 or ats.op_status() != 0:
        raise RuntimeError("a device-side wait gave up")


if __name__ == "__main__":
    main()
