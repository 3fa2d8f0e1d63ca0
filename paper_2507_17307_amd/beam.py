"""Beam search on a model whose cache is in pages.

Every prompt has n_beams slots of the model.  A step is one rs_decode_step for all beams of all prompts, rs_beam_select on its logits, and
rs_pages_fork, after which each beam's page table row holds its parent's state: whole pages are shared, a part-filled last one is copied where two
beams go on from it.  A beam that ended, or is not there, takes over nothing: its logits are not looked at any more, so it holds no page, the decode step skips
it, and what it wrote is in the steps' tokens.  rs_pages_reserve then hands out what the next position of the others needs.  All of it is
enqueued; the host reads the steps' parents and tokens once, at the end (and, now and then, whether all beams have ended).
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding as B


@dataclass
class Beam:
    tokens: List[int]            # what follows the prompt, up to and with eos
    score: float                 # sum of the tokens' log probabilities (in order of score / length^length_penalty)
    ended: bool


class BeamSearch:
    def __init__(self, model: B.PagedModel, n_prompts: int, n_beams: int, eos: int = -1, length_penalty: float = 0.0, logit_scale: float = 1.0):
        """Takes over the model's pages (PagedModel.page_pool).  n_prompts * n_beams <= the model's max_seqs and max_rows.  The search's
        slots are 0 .. n_prompts * n_beams - 1.  Every generate empties the slots of all searches made on the model (the most rows of any); it leaves
        the slots beyond them and their pages as they are."""
        cfg, rows = model.cfg, n_prompts * n_beams
        if n_prompts < 1 or n_beams < 1 or rows > cfg.max_seqs or rows > cfg.max_rows:
            raise ValueError(f"{n_prompts} x {n_beams} beams do not fit {cfg.max_seqs} slots / {cfg.max_rows} rows")
        if not -1 <= eos < cfg.vocab or not 0 <= length_penalty <= 30 or not 0 < logit_scale < float("inf"):
            raise ValueError("need eos -1 or a token, length_penalty in 0..30 and a positive logit_scale")
        n = B.rs_beam_select_scratch_bytes(n_prompts, n_beams, cfg.vocab, n_beams)
        if n == 0:
            raise ValueError(f"more than 64 beams of a prompt: {n_prompts} x {n_beams}")
        self.model, self.n_prompts, self.n_beams, self.eos, self.length_penalty, self.rows = model, n_prompts, n_beams, eos, length_penalty, rows
        dev = model.device
        self.pool = model.page_pool()
        model.search_slots = max(model.search_slots, rows)
        self.stream = torch.cuda.Stream(device=dev)          # a capturable (non-default) stream: repeated steps are replayed as a graph

        def ints(n: int, value: int = 0) -> torch.Tensor:
            return torch.full((n,), value, dtype=torch.int32, device=dev)
        # buffers of a step, at fixed addresses
        self.slot = torch.arange(cfg.max_seqs, dtype=torch.int32, device=dev)
        self.pos, self.end, self.token, self.length = ints(rows), ints(rows), ints(rows), ints(rows)
        self.score = torch.zeros(rows, dtype=torch.float64, device=dev)      # (sums over all steps: fp32 would round each of them)
        self.scale = torch.full((rows,), logit_scale, device=dev)
        self.logits = torch.zeros(rows, cfg.vocab, device=dev)
        self.record = B.new_route_out(rows, dev)
        self.flags, self.bad_rows = ints(rows), ints(rows)
        self.everything = ints(cfg.max_seqs, model.page_size * model.page_table.shape[1])
        self.pool_scratch = torch.empty(B.rs_pages_scratch_bytes(self.pool, rows), dtype=torch.uint8, device=dev)
        self.scratch = torch.empty(n, dtype=torch.uint8, device=dev)
        torch.cuda.synchronize(dev)

    def _prefill(self, prompts: Sequence[Sequence[int]]) -> None:
        """Every prompt into the slot of its first beam; the logits behind it into that beam's row."""
        mr, model = self.model.cfg.max_rows, self.model
        for g, prompt in enumerate(prompts):
            r = g * self.n_beams
            for at in range(0, len(prompt), mr):
                chunk = list(prompt[at:at + mr])
                span = torch.tensor(chunk + [0, len(chunk), at], dtype=torch.int32, device=model.device)
                logits = self.logits[r:r + 1] if at + mr >= len(prompt) else None
                B.rs_catchup_prefill(model.handle, 1, len(chunk), self.slot[r:], span, span[len(chunk):], span[len(chunk) + 2:], None, 0.5, B.RS_LLM,
                                     self.record, logits, self.stream)

    def _select(self, parent: torch.Tensor) -> None:
        """parent: where the parents of the step go."""
        B.rs_beam_select(self.logits, self.n_prompts, self.n_beams, self.scale, self.score, self.token, self.eos, self.length_penalty, self.length, self.n_beams,
                         parent, self.token, self.score, self.length, self.scratch, self.bad_rows, self.stream)
        heir = parent if self.eos < 0 else parent.masked_fill(self.token == self.eos, -1)      # (a beam that is not there has parent -1 already)
        B.rs_pages_fork(self.pool, self.n_prompts, self.n_beams, self.slot, heir, self.end, self.pos, self.pool_scratch, self.flags, self.stream)

    def generate(self, prompts: Sequence[Sequence[int]], n_tokens: int, check_every: int = 16) -> List[List[Beam]]:
        """The n_beams best continuations of every prompt by n_tokens tokens (or up to eos), best first.  check_every: how often, in steps,
        the host looks whether all beams have ended (0: never)."""
        cfg, nb = self.model.cfg, self.n_beams
        if len(prompts) != self.n_prompts or any(len(p) < 1 for p in prompts) or n_tokens < 1:
            raise ValueError("one prompt of at least one token each, and at least one token to generate")
        if any(not 0 <= t < cfg.vocab for p in prompts for t in p):
            raise ValueError("a prompt's token is out of range")
        if max(len(p) for p in prompts) + n_tokens - 1 > cfg.max_ctx:
            raise ValueError("prompt + tokens exceed max_ctx")
        parents = torch.zeros(n_tokens, self.rows, dtype=torch.int32, device=self.model.device)
        tokens = torch.zeros_like(parents)
        self.stream.wait_stream(torch.cuda.current_stream(self.model.device))
        with torch.cuda.stream(self.stream):
            # the searches' slots give back what they hold; only the first beam of every prompt is there yet
            B.rs_pages_release(self.pool, self.model.search_slots, self.slot, None, self.everything)
            self.flags.zero_(), self.bad_rows.zero_(), self.pos.zero_(), self.length.zero_(), self.token.fill_(-1)
            self.score.fill_(float("-inf"))
            self.score[::nb] = 0.0
            self.pos[::nb] = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=self.model.device)
            self.end.copy_(self.pos)
            B.rs_pages_reserve(self.pool, self.rows, self.slot, None, self.pos, self.pool_scratch, self.flags)
            self._prefill(prompts)
            done = n_tokens
            for t in range(n_tokens):
                if t > 0:
                    torch.add(self.pos, self.pos > 0, out=self.end)           # (rows that do not run hold 0 positions and get none: no page, and so no decode step)
                    B.rs_pages_reserve(self.pool, self.rows, self.slot, self.pos, self.end, self.pool_scratch, self.flags)
                    B.rs_decode_step(self.model.handle, self.rows, self.slot, self.token, self.pos, None, 0.5, B.RS_LLM, self.record, self.logits, self.stream)
                self._select(parents[t])
                tokens[t] = self.token
                if self.eos >= 0 and check_every and (t + 1) % check_every == 0 and bool(((self.token == self.eos) | (self.token < 0)).all()):
                    done = t + 1
                    break
        self.stream.synchronize()
        if bool((self.flags != 0).any()):
            raise B.RsError(-2, f"not enough pages for the beams: flags {self.flags.tolist()}")
        if bool((self.bad_rows != 0).any()):
            raise RuntimeError(f"logits that are no numbers: flags {self.bad_rows.tolist()}")
        return self._read(parents[:done].tolist(), tokens[:done].tolist(), self.score.tolist())

    def _read(self, parents: List[List[int]], tokens: List[List[int]], scores: List[float]) -> List[List[Beam]]:
        out: List[List[Beam]] = []
        for g in range(self.n_prompts):
            found = []
            for b in range(self.n_beams):
                at, back = b, []
                for t in range(len(tokens) - 1, -1, -1):
                    r = g * self.n_beams + at
                    if tokens[t][r] < 0:
                        break
                    back.append(tokens[t][r])
                    at = parents[t][r]
                else:
                    line = back[::-1]
                    ended = self.eos >= 0 and self.eos in line
                    found.append(Beam(line[:line.index(self.eos) + 1] if ended else line, scores[g * self.n_beams + b], ended))
            out.append(found)
        return out
