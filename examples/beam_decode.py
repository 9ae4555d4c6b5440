"""Beam search for a batch of users over a paged cache whose pages the beams share, and tree decoding that keeps an accepted
path's keys and values, with the stateless operators: the small decoder of tree_decode.py, random weights.

    python examples/beam_decode.py

A beam step is plan -> (rope_append -> tree_attention, once per layer) -> beam_select -> fork_pages -> copy_pages.  Nothing of it
comes to the host, so that one captured graph is replayed step after step.  All of a user's beams share the pages of its prompt; a
beam that goes on twice shares its full pages with both and has its last one copied; the pages of beams that nothing goes on from
are free again.

A tree step is that of tree_decode.py; then compact_tokens moves the accepted path behind what is cached and fork_pages gives
the rest of the step's pages back, so that no accepted token is computed twice.
"""
import os
import sys
from typing import List, Sequence

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import tree_decode as td  # noqa: E402
from tree_decode import ats  # noqa: E402


def _i32(x) -> torch.Tensor:
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Beams:
    """`width` beams of every user; tokens at odd positions are even ones (the grammar of tree_decode.py)."""

    def __init__(self, model: td.Model, prompts: Sequence[Sequence[int]], width: int = 4, say: int = 16, end: int = -1, pages: int = 256,
                 columns: int = 32):
        self.model, self.width, self.users, self.say, self.end = model, width, len(prompts), say, end
        self.prompts = [list(p) for p in prompts]
        n = self.n = width * len(prompts)
        if n > td.MAX_TOKENS:
            raise ValueError(f"{n} beams in a step of {td.MAX_TOKENS} tokens")
        shape = (pages, td.PAGE, td.KV_HEADS, td.HD)
        self.caches = [(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.float16, device="cuda"))
                       for _ in range(td.LAYERS)]
        self.layers = ats.CacheLayers(self.caches)
        words = -(-td.VOCAB // 32)
        self.grammar = torch.stack([torch.full((words,), -1, dtype=torch.int32), torch.full((words,), 0x55555555, dtype=torch.int32)]).cuda()
        # what a step reads and the next one's takes the place of
        self.table = torch.full((n, columns), -1, dtype=torch.int32, device="cuda")
        self.kv_len, self.ref = _i32([0] * n), _i32([0] * pages)
        self.free, self.n_free = _i32(range(pages)), _i32([pages])
        self.token, self.final = _i32([-1] * td.MAX_TOKENS), _i32([-1] * n)
        self.score, self.lost = torch.zeros(n, device="cuda"), torch.zeros((), dtype=torch.bool, device="cuda")
        self.said, self.steps = _i32([[-1] * say] * n), torch.zeros((), dtype=torch.int64, device="cuda")
        self.one, self.every, self.graph = _i32([1] * n), _i32(range(0, n + 1, width)), None
        self._prefill()

    def _forward(self, q_len: torch.Tensor):
        plan = ats.op_batch_plan(q_len, self.kv_len, self.table, self.free, self.n_free, td.PAGE, td.MAX_TOKENS)
        self._drop(plan.state)
        return plan, self.model.logits(self.token, plan, self.table, self.caches)

    def _drop(self, state: torch.Tensor) -> None:
        """A row for which there were no pages has no history: it is not chosen again, and run() says so."""
        out = state != ats.PLAN_OK
        self.lost.logical_or_((out & (self.score > -torch.inf)).any())
        self.score.masked_fill_(out, -torch.inf)

    def _check(self) -> None:
        if bool(self.lost):
            raise RuntimeError("not all beams could go on: too few pages, or rows of the table that are too short")

    def _fork(self, plan, q_len, parent=None) -> None:
        """The rows' pages after a step, and from their parents."""
        f = ats.op_fork_pages(self.table, self.kv_len, self.ref, self.free, self.n_free, td.PAGE, q_len=q_len, state=plan.state, used=plan.pages,
                              parent=parent)
        ats.op_copy_pages(self.layers, f.src, f.dst, length=f.kv_len)
        for name in ("table", "kv_len", "ref", "free", "n_free"):
            getattr(self, name).copy_(getattr(f, name))
        self._drop(f.state)

    def _prefill(self) -> None:
        """The prompts, but for their last tokens, in each user's first row; then all of its rows share their pages."""
        done, piece = [0] * self.users, td.MAX_TOKENS // self.users
        while any(k < len(p) - 1 for k, p in zip(done, self.prompts)):
            parts = [p[k:min(k + piece, len(p) - 1)] for k, p in zip(done, self.prompts)]
            q_len = _i32([x for part in parts for x in [len(part)] + [0] * (self.width - 1)])
            flat = [t for part in parts for t in part]
            self.token.copy_(_i32(flat + [-1] * (td.MAX_TOKENS - len(flat))))
            plan, _ = self._forward(q_len)
            self._fork(plan, q_len)
            done = [k + len(part) for k, part in zip(done, parts)]
        # The first step: the last prompt token in the first rows, whose best continuations begin the beams.
        first = self.every[:-1]
        q_len = torch.zeros_like(self.one).index_fill_(0, first.long(), 1)
        self.token.fill_(-1)
        self.token[:self.users] = _i32([p[-1] for p in self.prompts])
        plan, logits = self._forward(q_len)
        best = ats.op_beam_select(logits[:self.users], _i32(range(self.users + 1)), self.width, grammar=self.grammar,
                                  state=plan.pos[:self.users] & 1)
        # (a row of the logits is a user here, a beam's parent the user's first row)
        self._choose(best, (best.parent * self.width).view(-1))
        self._fork(plan, q_len, best.parent.view(-1) * self.width)
        self._check()

    def _choose(self, best, parent: torch.Tensor) -> None:
        token, rows = best.token.view(-1), parent.long()
        self.said.copy_(self.said[rows].index_copy(1, self.steps.view(1), token[:, None]))
        self.steps += 1
        self.token[:self.n] = token
        self.score.copy_(best.score.view(-1))
        if self.end >= 0:
            self.final.copy_(torch.where(token == self.end, token, -1))

    def step(self) -> None:
        plan, logits = self._forward(self.one)
        best = ats.op_beam_select(logits[:self.n], self.every, self.width, score=self.score, final=self.final, grammar=self.grammar,
                                  state=plan.pos[:self.n] & 1)
        parent = best.parent.view(-1)
        self._choose(best, parent)
        self._fork(plan, self.one, parent)

    def run(self) -> None:
        """Until `say` tokens are said: one step as it is, the others as replays of a graph of one.  An error if pages ran out; the
        beams that are left (those with a score) are right all the same."""
        left = self.say - int(self.steps)
        if left > 0:
            self.step()
        if left > 1 and self.graph is None:
            torch.cuda.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.step()
        for _ in range(left - 1):
            self.graph.replay()
        self._check()

    def lists(self) -> List[List[List[int]]]:
        """Every user's sequences, best first."""
        said = self.said[:, :int(self.steps)].tolist()
        return [said[u * self.width:(u + 1) * self.width] for u in range(self.users)]

    def close(self) -> int:
        """Ends all beams; the free pages."""
        f = ats.op_fork_pages(self.table, self.kv_len, self.ref, self.free, self.n_free, td.PAGE, parent=torch.full_like(self.one, -1))
        return int(f.n_free)


class Keeper(td.Decoder):
    """Tree decoding whose accepted paths stay in the cache.  The page counts and the free list are on the GPU."""

    def __init__(self, model: td.Model, prompts: Sequence[Sequence[int]], pages: int = 256, width: int = 32):
        self.ref, self.pages, self.n_free = _i32([0] * pages), _i32(range(pages)), _i32([pages])
        self.moved = 0
        self.path = None
        super().__init__(model, prompts, pages, width)

    def _plan(self, q_len, parent=None):
        self.q_len, self.kv = _i32(q_len), _i32(self.kv_len)
        self.plan = ats.op_batch_plan(self.q_len, self.kv, self.table, self.pages, self.n_free, td.PAGE, td.MAX_TOKENS, parent=parent,
                                      mask_words=td.MASK_WORDS if parent is not None else 0)
        if int(self.plan.state.max()) != ats.PLAN_OK:
            raise RuntimeError(f"not all users can be served: {self.plan.state.tolist()}")
        return self.plan

    def _commit(self, kept, q_len) -> None:
        path, self.path = self.path or [list(range(k)) for k in kept], None
        most = max(1, max(len(p) for p in path))
        keep, count = _i32([p + [-1] * (most - len(p)) for p in path]), _i32([len(p) for p in path])
        if not hasattr(self, "layers"):
            self.layers = ats.CacheLayers(self.caches)
        length = ats.op_compact_tokens(self.layers, self.plan.slot, self.plan.cu_q, self.kv, keep, count, state=self.plan.state)
        f = ats.op_fork_pages(self.table, self.kv, self.ref, self.pages, self.n_free, td.PAGE, q_len=self.q_len, state=self.plan.state,
                              used=self.plan.pages, length=length)
        self.table, self.ref, self.pages, self.n_free = f.table, f.ref, f.free, f.n_free
        self.kv_len = length.tolist()
        self.moved += sum(i != k for p in path for i, k in enumerate(p))


def main() -> None:
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, td.VOCAB, (n,), generator=g).tolist() for n in (40, 200, 7, 93)]
    model = td.Model()
    beams = Beams(model, prompts, width=6, say=16)
    beams.run()
    for u, (lists, score) in enumerate(zip(beams.lists(), beams.score.view(-1, 6).tolist())):
        print(f"user {u}: {score[0]:.2f} {lists[0]}")
    used = beams.caches[0][0].shape[0] - int(beams.n_free)
    alone = sum(6 * -(-(len(p) + 15) // td.PAGE) for p in prompts)
    print(f"{used} pages for 24 beams, {alone} if none were shared; {beams.close()} free after their end")
    plain = td.Decoder(model, prompts)
    plain.run(48, td.no_draft)
    known = [t[:] for t in plain.text]

    def knows(b: int, text: List[int]) -> td.Draft:   # the best case: two right drafts, a wrong one before each
        rest = known[b][len(text):len(text) + 2]
        tokens = [x for t in rest for x in ((t + 1) % td.VOCAB, t)]
        return tokens, [2 * (j // 2) - 1 for j in range(len(tokens))]

    kept = Keeper(model, prompts)
    kept.run(48, knows)
    same = sum(a == b for t, u in zip(kept.text, plain.text) for a, b in zip(t, u))
    total = sum(min(len(t), len(u)) for t, u in zip(kept.text, plain.text))
    print(f"trees: {kept.steps} steps, {kept.moved} accepted tokens moved, {same} of {total} tokens as in {plain.steps} steps of one token")
    if ats.op_status(noalloc=True) != 0 or ats.op_status() != 0:
        raise RuntimeError("a device-side wait gave up")


if __name__ == "__main__":
    main()
