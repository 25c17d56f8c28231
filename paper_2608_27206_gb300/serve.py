"""The attention of one decoder layer while a pruned prompt is answered.

ServeLayer owns a layer's paged 8-bit cache, its block table, lengths and scratch, and issues the
calls of a serving loop:

    prompt  append the prompt's kept rows (as pace_prune_index lists them) and attend, every token
    step    append one token per sequence and attend: a decode step
    draft   append a tree of drafted tokens per sequence and attend from each of its nodes;
    accept  then keeps the path that agrees with the tokens picked after the nodes
    prune   keeps some of the cached tokens (a prompt's, once a later layer has scored them)
    fork    copies a sequence's tokens to others, for several answers to one prompt

Everything is allocated once, and what a step needs is on the device, lengths included, so a step
can be captured in a CUDA graph and replayed while the sequences grow.  The host counts along: a call
or a replay that would take a sequence past max_len raises before it issues anything, and one that
raises for another reason takes its tokens back.  What the kernels report (numbers out of range,
values that are not finite) shows in check().

    python -m paper_2608_27206_gb300.serve

prunes the visual tokens of a 4K image (10549 of them) to 40 %, fills the cache with what is left
and times decode steps, and steps of drafted trees where --nodes is given.
"""
from __future__ import annotations

import argparse
import contextlib
import time
from typing import Optional, Sequence

import torch

from . import pace as P
from . import synth


class CapturedStep(torch.cuda.CUDAGraph):
    """A captured step of a ServeLayer, whose replays count like its steps."""

    layer: "ServeLayer"

    def replay(self) -> None:
        self.layer._require_one()
        super().replay()
        self.layer._steps += 1


class ServeLayer:
    """max_len bounds a sequence's slots; sections are the pairs that each row of position ids turns.

    lens, on the device, are the sequences' lengths: the methods, replays and reset change them, nobody else may.  How many drafted
    tokens were accepted only the device knows: the host counts all of them, and reads the lengths when that would be too many."""

    def __init__(self, max_seqs: int, max_len: int, page_size: int = 64, n_q_heads: int = synth.LLM_QHEADS,
                 n_kv_heads: int = synth.LLM_KVHEADS, head_dim: int = synth.LLM_DIM, sections: Optional[Sequence[int]] = None,
                 rope_base: float = 1e6, max_positions: Optional[int] = None, window: int = 0, sinks: int = 0, device="cuda"):
        self.B, self.max_len, self.window, self.sinks = max_seqs, max_len, window, sinks
        self.n_q_heads = n_q_heads
        self.sections = list(sections) if sections is not None else [head_dim // 8, head_dim * 3 // 16, head_dim * 3 // 16]
        pages = -(-max_len // page_size)
        self.cache = P.KvCache.empty(max_seqs * pages, page_size, n_kv_heads, head_dim, device)
        # each sequence has the pages of max_len slots for itself (a program short of memory hands them out as sequences grow)
        self.table = torch.arange(max_seqs * pages, dtype=torch.int32, device=device).view(max_seqs, pages)
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self._of_prompts, self._steps = [0] * max_seqs, 0      # the same on the host: tokens of prompts, and of steps
        self._tree, self._loose = None, False                  # a tree not yet accepted; whether there may be fewer tokens than counted
        self.rope = P.pace_rope_table(max_positions or max_len, head_dim, rope_base, device=device)
        self.one = list(range(max_seqs + 1))
        self.q = torch.empty((max_seqs, n_q_heads, head_dim), dtype=torch.bfloat16, device=device)
        self.out = torch.empty_like(self.q)
        n = P.pace_kv_attention_workspace_size(self.cache, self.one, n_q_heads, max_len)
        self.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)

    def _lengths(self) -> list:
        """The sequences' lengths, read from the device where the host does not know them."""
        if self._loose:
            self._of_prompts, self._loose = [n - self._steps for n in self.lens.tolist()], False
        return [n + self._steps for n in self._of_prompts]

    def _require(self, new: Sequence[int], what: str) -> None:
        """Raises unless new[b] more tokens fit each sequence b."""
        if self._tree is not None:
            raise ValueError(f"{what} before the drafted tokens have been accepted")
        if max(a + b for a, b in zip(self._of_prompts, new)) + self._steps > self.max_len and \
                (not self._loose or max(a + b for a, b in zip(self._lengths(), new)) > self.max_len):
            raise ValueError(f"{what} past max_len ({self.max_len})")

    @contextlib.contextmanager
    def _taking(self, cu_new: Sequence[int], what: str):
        """Counts new tokens (a prefix over the sequences) for the calls inside: raises if they do not fit, and counts them no more if a call
        raises (what it may have stored lies behind the sequences' ends then)."""
        new = [int(b) - int(a) for a, b in zip(cu_new, cu_new[1:])]
        if len(new) != self.B or min(new) < 0:
            raise ValueError(f"cu_new: expected a prefix of {self.B} numbers of tokens")
        self._require(new, what)
        more = torch.tensor(new, dtype=torch.int32, device=self.lens.device)
        self.lens += more
        try:
            yield
        except BaseException:
            self.lens -= more
            raise
        self._of_prompts = [a + b for a, b in zip(self._of_prompts, new)]

    def _require_one(self) -> None:
        self._require([1] * self.B, "a step")

    def _require_heads(self, Q: torch.Tensor) -> None:
        """Raises unless the attention takes as many heads as Q has: before the keys beside it are stored."""
        heads, of = self.cache.n_kv_heads, Q.shape[1] if Q.dim() == 3 else 0
        if of < 1 or of % heads or of // heads > 64:
            raise ValueError(f"Q: expected [rows, heads, D], heads a multiple of {heads}")

    def reset(self) -> None:
        """Empties the sequences."""
        self.lens.zero_()
        self._of_prompts, self._steps = [0] * self.B, 0
        self._tree, self._loose = None, False

    def check(self) -> None:
        """Waits for the device and raises if a call since the last check has reported an error."""
        code, where = P.pace_device_status(clear=True)
        if code != P.PACE_OK:
            raise RuntimeError(f"{P.status_string(code)} (device status {code} from kernel {where})")

    def prompt(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, cu_new: Sequence[int], positions: torch.Tensor,
               rows: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Appends cu_new[b + 1] - cu_new[b] tokens to every sequence b (0: none) and attends from each of them: a whole prompt, a
        chunk of one or a chat's next turn.  rows picks the tokens out of K, V, Q and positions.  bf16 [cu_new[-1], heads, D]."""
        self._require_heads(Q)
        with self._taking(cu_new, "a prompt"):
            q = P.pace_kv_append(self.cache, K, V, cu_new, self.lens, self.table, rows=rows, rope=self.rope, positions=positions,
                                 sections=self.sections, q=Q)
            return P.pace_kv_attention(self.cache, q, cu_new, self.lens, self.table, self.max_len, window=self.window, sinks=self.sinks)

    def step(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """One token for every sequence: row b of K, V, Q and of the position ids.  The result is overwritten by the next step."""
        self._require_one()
        out = self._step(K, V, Q, positions)
        self._steps += 1
        return out

    def _step(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        if Q.dim() != 3 or Q.shape[1] != self.n_q_heads:      # (self.q has room for fewer)
            raise ValueError(f"Q: expected [{self.B}, {self.n_q_heads}, D]")
        self.lens += 1
        try:
            P.pace_kv_append(self.cache, K, V, self.one, self.lens, self.table, rope=self.rope, positions=positions,
                             sections=self.sections, q=Q, q_out=self.q)
            return P.pace_kv_attention(self.cache, self.q, self.one, self.lens, self.table, self.max_len, window=self.window,
                                       sinks=self.sinks, out=self.out, ws=self.ws)
        except BaseException:
            self.lens -= 1
            raise

    def draft(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, parents: torch.Tensor, cu_nodes: Sequence[int],
              positions: torch.Tensor) -> torch.Tensor:
        """Appends cu_nodes[b + 1] - cu_nodes[b] drafted tokens to every sequence b, the nodes of a tree (parents, device int32: the
        number of each one's parent in its tree, before it, or -1; node 0 is the token that the model picked last), and attends from each:
        bf16 [nodes, heads, D].  positions are the ids of the sequence's end and the nodes' depths.  accept() is to follow, and
        reads parents again."""
        if max(int(b) - int(a) for a, b in zip(cu_nodes, cu_nodes[1:])) > P.TREE_MAX:
            raise ValueError(f"a tree of more than {P.TREE_MAX} nodes")
        self._require_heads(Q)
        P._int32(parents, int(cu_nodes[-1]), "parents")      # (raises before anything is stored)
        with self._taking(cu_nodes, "a tree"):
            q = P.pace_kv_append(self.cache, K, V, cu_nodes, self.lens, self.table, rope=self.rope, positions=positions,
                                 sections=self.sections, q=Q)
            out = P.pace_kv_tree_attention(self.cache, q, cu_nodes, parents, self.lens, self.table, self.max_len, window=self.window,
                                           sinks=self.sinks)
        self._tree = list(cu_nodes), parents
        return out

    def accept(self, tokens: torch.Tensor, picked: torch.Tensor):
        """Of the drafted tokens (device int32, as are those picked after each node) keeps the path that the picked ones agree with.
        Returns its rows, their number per sequence and the token to go on with, as pace_draft_accept does.  (The rejected ones leave
        the cache, and no scale stands for them any more; what a large one has cost tokens of the same 16 slots when it was appended stays lost.)"""
        if self._tree is None:
            raise ValueError("nothing has been drafted")
        cu, parents = self._tree
        rows, counts, after = P.pace_draft_accept(tokens, parents, picked, cu)
        self.lens.copy_(P.pace_kv_compact(self.cache, cu, self.lens, self.table, rows=rows, counts=counts))
        self._tree, self._loose = None, True
        return rows, counts, after

    def prune(self, rows: torch.Tensor, cu_rows: Sequence[int]) -> None:
        """Of every sequence's tokens keeps cu_rows[b + 1] - cu_rows[b], those that rows (device int32) lists: numbers in the batch of all
        sequences one after the other, as pace_prune_index gives them, ascending."""
        if len(cu_rows) != self.B + 1:
            raise ValueError(f"cu_rows: expected a prefix of {self.B} numbers of rows")
        self._require([0] * self.B, "a prune")
        cu = [0]
        for n in self._lengths():
            cu.append(cu[-1] + n)
        self.lens.copy_(P.pace_kv_compact(self.cache, cu, self.lens, self.table, cu_rows=cu_rows, rows=rows))
        self._of_prompts = [int(b) - int(a) - self._steps for a, b in zip(cu_rows, cu_rows[1:])]

    def fork(self, source: int, to: Sequence[int]) -> None:
        """Copies sequence `source` to the (other) sequences `to`, which lose what they had."""
        to = [int(b) for b in to]
        if source in to or len(set(to)) != len(to) or any(b < 0 or b >= self.B for b in [source, *to]):
            raise ValueError("expected other sequences, each once")
        self._require([0] * self.B, "a fork")
        n = self._lengths()[source]
        at = torch.tensor(to, dtype=torch.int64, device=self.lens.device)
        lens = self.lens[source].repeat(len(to))
        self.lens[at] = P.pace_kv_compact(self.cache, list(range(0, n * len(to) + 1, n)) if n else [0] * (len(to) + 1), lens,
                                          self.table[source].repeat(len(to), 1), dst_table=self.table[at])
        for b in to:
            self._of_prompts[b] = self._of_prompts[source]

    def capture_step(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, positions: torch.Tensor) -> CapturedStep:
        """A graph of step() on these tensors; a replay reads what they hold then.  (Capturing runs nothing.)"""
        graph = CapturedStep()
        graph.layer = self
        with torch.cuda.graph(graph):
            self._step(K, V, Q, positions)
        return graph


def _tokens(n: int, heads: int, seed: int, device) -> torch.Tensor:
    g = torch.Generator(device=device).manual_seed(seed)
    return torch.randn(n, heads, synth.LLM_DIM, generator=g, device=device).to(torch.bfloat16)


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--visual", type=int, default=10549, help="visual tokens of the prompt")
    ap.add_argument("--keep", type=float, default=0.4, help="share of them that is kept")
    ap.add_argument("--steps", type=int, default=200, help="decode steps")
    ap.add_argument("--nodes", type=int, default=0, help="drafted tokens of a tree (0: none are drafted)")
    args = ap.parse_args(argv)
    dev, text = "cuda", 20
    n_vis = args.visual
    n = n_vis + 2 * text
    k = P.pace_budget(n_vis, args.keep)
    # which visual tokens stay: top k of the fused importance
    g = torch.Generator(device=dev).manual_seed(1)
    s_llm, s_vis = torch.rand(n_vis, generator=g, device=dev), torch.rand(n_vis, generator=g, device=dev)
    _, _, kept = P.pace_ddae_select(s_llm, s_vis, [0, n_vis], [0, k])
    rows = P.pace_prune_index([0, n], [text], [0, n_vis], [0, k], kept)
    # ids: text counts on, a visual token has its row and column
    i = torch.arange(n, device=dev)
    wide = max(1, int(n_vis ** 0.5))
    seen, j = (i >= text) & (i < text + n_vis), (i - text).clamp(0, n_vis - 1)
    after = text + wide + i - text - n_vis
    ids = torch.stack([torch.where(seen, text + 0 * i, torch.where(i < text, i, after)),
                       torch.where(seen, text + j // wide, torch.where(i < text, i, after)),
                       torch.where(seen, text + j % wide, torch.where(i < text, i, after))]).to(torch.int32)
    rounds = 20 if args.nodes > 0 else 0
    most = args.steps + (rounds + 1) * args.nodes
    layer = ServeLayer(1, len(rows) + most + 1, max_positions=n + most + 1)
    K, V, Q = _tokens(n, synth.LLM_KVHEADS, 2, dev), _tokens(n, synth.LLM_KVHEADS, 3, dev), _tokens(n, synth.LLM_QHEADS, 4, dev)
    layer.prompt(K, V, Q, [0, len(rows)], ids, rows=rows)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    layer.reset()
    layer.prompt(K, V, Q, [0, len(rows)], ids, rows=rows)
    torch.cuda.synchronize()
    prompt_us = 1e6 * (time.perf_counter() - t0)
    k1, v1, q1 = _tokens(1, synth.LLM_KVHEADS, 5, dev), _tokens(1, synth.LLM_KVHEADS, 6, dev), _tokens(1, synth.LLM_QHEADS, 7, dev)
    pos = torch.full((3, 1), int(after[-1]) + 1, dtype=torch.int32, device=dev)
    graph = layer.capture_step(k1, v1, q1, pos)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    graph.replay()
    start.record()
    for _ in range(args.steps - 1):
        pos += 1
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    layer.check()
    print(f"prompt: {len(rows)} of {n} tokens appended and attended in {prompt_us:.0f} us; "
          f"then {args.steps - 1} decode steps, {1e3 * start.elapsed_time(end) / max(args.steps - 1, 1):.1f} us each; "
          f"{int(layer.lens[0])} slots in use")

    if rounds == 0:
        return
    # trees of drafted tokens: each node a child of a random one before it, tokens and picks out of few, so that some agree
    m = args.nodes
    parents = [-1] + [int(torch.randint(0, t, (1,), generator=torch.Generator().manual_seed(t))) for t in range(1, m)]
    depth = [0] * m
    for t in range(1, m):
        depth[t] = depth[parents[t]] + 1
    depth, parents = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (depth, parents))
    k1, v1, q1 = _tokens(m, synth.LLM_KVHEADS, 8, dev), _tokens(m, synth.LLM_KVHEADS, 9, dev), _tokens(m, synth.LLM_QHEADS, 10, dev)
    before, at = layer.lens.clone(), int(pos[0, 0]) + 1
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for r in range(rounds):
        layer.draft(k1, v1, q1, parents, [0, m], (depth + at).repeat(3, 1))
        tokens, picked = (torch.randint(0, 3, (m,), generator=g, device=dev).to(torch.int32) for _ in range(2))
        layer.accept(tokens, picked)
        at += 1
    layer.check()
    print(f"{rounds} trees of {m} drafted tokens, {1e6 * (time.perf_counter() - t0) / rounds:.0f} us each; "
          f"{int(layer.lens[0] - before[0])} tokens accepted")


if __name__ == "__main__":
    main()
