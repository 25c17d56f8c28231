"""The attention of one decoder layer while a pruned prompt is answered.

ServeLayer owns a layer's paged 8-bit cache, its block table, lengths and scratch, and issues the
calls of a serving loop:

    prompt  append the prompt's kept rows (as pace_prune_index lists them) and attend, every token
    step    append one token per sequence and attend: a decode step

Everything is allocated once, and what a step needs is on the device, lengths included, so a step
can be captured in a CUDA graph and replayed while the sequences grow.  The host counts along: a call
or a replay that would take a sequence past max_len raises before it issues anything.  What the
kernels report (numbers out of range, values that are not finite) shows in check().

    python -m paper_2608_27206_gb300.serve

prunes the visual tokens of a 4K image (10549 of them) to 40 %, fills the cache with what is left
and times decode steps.
"""
from __future__ import annotations

import argparse
import time
from typing import Optional, Sequence

import torch

from . import pace as P
from . import synth


class CapturedStep(torch.cuda.CUDAGraph):
    """A captured step of a ServeLayer, whose replays count like its steps."""

    layer: "ServeLayer"

    def replay(self) -> None:
        self.layer._take_one()
        super().replay()


class ServeLayer:
    """max_len bounds a sequence's slots; sections are the pairs that each row of position ids turns.

    lens, on the device, are the sequences' lengths: prompt, step, replay and reset change them, nobody else may."""

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
        self.rope = P.pace_rope_table(max_positions or max_len, head_dim, rope_base, device=device)
        self.one = list(range(max_seqs + 1))
        self.q = torch.empty((max_seqs, n_q_heads, head_dim), dtype=torch.bfloat16, device=device)
        self.out = torch.empty_like(self.q)
        n = P.pace_kv_attention_workspace_size(self.cache, self.one, n_q_heads, max_len)
        self.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)

    def _take_one(self) -> None:
        if max(self._of_prompts) + self._steps >= self.max_len:
            raise ValueError(f"a step past max_len ({self.max_len})")
        self._steps += 1

    def reset(self) -> None:
        """Empties the sequences."""
        self.lens.zero_()
        self._of_prompts, self._steps = [0] * self.B, 0

    def check(self) -> None:
        """Waits for the device and raises if a call since the last check has reported an error."""
        code, where = P.pace_device_status(clear=True)
        if code != P.PACE_OK:
            raise RuntimeError(f"{P.status_string(code)} (device status {code} from kernel {where})")

    def prompt(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, cu_new: Sequence[int], positions: torch.Tensor,
               rows: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Appends cu_new[b + 1] - cu_new[b] tokens to every sequence b (0: none) and attends from each of them: a whole prompt, a
        chunk of one or a chat's next turn.  rows picks the tokens out of K, V, Q and positions.  bf16 [cu_new[-1], heads, D]."""
        new = [int(b) - int(a) for a, b in zip(cu_new, cu_new[1:])]
        if len(new) != self.B or min(new) < 0:
            raise ValueError(f"cu_new: expected a prefix of {self.B} numbers of tokens")
        taken = [a + b for a, b in zip(self._of_prompts, new)]
        if max(taken) + self._steps > self.max_len:
            raise ValueError(f"a prompt past max_len ({self.max_len})")
        self._of_prompts = taken
        self.lens += torch.tensor(new, dtype=torch.int32, device=self.lens.device)
        q = P.pace_kv_append(self.cache, K, V, cu_new, self.lens, self.table, rows=rows, rope=self.rope, positions=positions,
                             sections=self.sections, q=Q)
        return P.pace_kv_attention(self.cache, q, cu_new, self.lens, self.table, self.max_len, window=self.window, sinks=self.sinks)

    def step(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """One token for every sequence: row b of K, V, Q and of the position ids.  The result is overwritten by the next step."""
        self._take_one()
        return self._step(K, V, Q, positions)

    def _step(self, K: torch.Tensor, V: torch.Tensor, Q: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        self.lens += 1
        P.pace_kv_append(self.cache, K, V, self.one, self.lens, self.table, rope=self.rope, positions=positions,
                         sections=self.sections, q=Q, q_out=self.q)
        return P.pace_kv_attention(self.cache, self.q, self.one, self.lens, self.table, self.max_len, window=self.window,
                                   sinks=self.sinks, out=self.out, ws=self.ws)

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
    layer = ServeLayer(1, len(rows) + args.steps + 1, max_positions=n + args.steps + 1)
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


if __name__ == "__main__":
    main()
