"""A language model service's two tasks on one GPU, measured and given to the gap fill.

  python -m paper_2311_10359_amd.service [--layers 4] [--requests 32] [--steps 20] [--rotary 128] [--beams 4] ...

The attention stack of a decoder (random weights; per layer a product to queries, keys and values, attention, a product back)
serves requests: their prompts first, then one token each per step.  Two tasks result that share the GPU in such a service:

  high priority   decode steps: short launches, idle time behind each step while the host picks what comes next
  low priority    a batch of prompts: longer launches, nobody waits for a single one

Every call's start and end are measured with events, as in the measurement phase, and written as launch records (a call
stands for its launches; its identity is its name and the sizes it was called with).  `fikit_profile_gapfill` then tells how
much of the prompts' work fits into the decode steps' idle times.

With `--rotary` heads are normed and rotated by position in front of the cache.  With `--beams` a request is continued by several beams:
every step scores their alternatives, and the best ones fork the requests, whose whole blocks they share.
"""
from __future__ import annotations

import argparse
import math
import random
import time
from typing import List, NamedTuple, Optional

import numpy as np
import torch

from . import binding, traces


class Sizes(NamedTuple):
    layers: int = 4
    q_heads: int = 32
    kv_heads: int = 8
    dim: int = 128
    block: int = 64
    blocks: int = 4096         # of the cache, per layer
    vocabulary: int = 8192
    rotary: int = 0            # dimensions of a head that are rotated; 0: heads are neither normed nor rotated

    @property
    def hidden(self) -> int:
        return self.q_heads * self.dim


class Recorder:
    """Launch records of one task: one per call."""

    def __init__(self):
        self.names: List[str] = []
        self.calls = []
        self.base = torch.cuda.Event(enable_timing=True)
        self.base.record()
        self.run = 0

    def __call__(self, name, sizes, f, *args, **more):
        if name not in self.names:
            self.names.append(name)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        got = f(*args, **more)
        end.record()
        self.calls.append((self.names.index(name), sizes, begin, end, self.run))
        return got

    def records(self) -> np.ndarray:
        torch.cuda.synchronize()
        rec = np.zeros(len(self.calls), dtype=traces.LAUNCH_DTYPE)
        for i, (name, sizes, begin, end, run) in enumerate(self.calls):
            rec[i]["name_id"], rec[i]["grid"], rec[i]["block"], rec[i]["run"] = name, sizes, (256, 1, 1), run
            rec[i]["start_ns"] = round(self.base.elapsed_time(begin) * 1e6)
            rec[i]["end_ns"] = max(rec[i]["start_ns"], round(self.base.elapsed_time(end) * 1e6))
        return rec


class Service:
    def __init__(self, sizes: Sizes, requests: int, longest: int, device="cuda:0", seed: int = 0):
        self.sizes, self.device = sizes, device
        gen = torch.Generator(device=device).manual_seed(seed)
        heads = sizes.q_heads + 2 * sizes.kv_heads

        def weight(rows, cols):
            return torch.randn((rows, cols), generator=gen, device=device, dtype=torch.float32).div_(math.sqrt(rows)).to(torch.bfloat16)
        self.w_qkv = [weight(sizes.hidden, heads * sizes.dim) for _ in range(sizes.layers)]
        self.w_out = [weight(sizes.hidden, sizes.hidden) for _ in range(sizes.layers)]
        self.w_tokens = weight(sizes.hidden, sizes.vocabulary)
        shape = (sizes.blocks, sizes.kv_heads, sizes.block, sizes.dim)
        self.caches = [[torch.zeros(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)] +
                       [torch.ones(shape[:2], dtype=torch.uint8, device=device) for _ in range(2)] for _ in range(sizes.layers)]
        self.table = torch.full((requests, -(-longest // sizes.block)), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(requests, dtype=torch.int32, device=device)
        self.free = torch.randperm(sizes.blocks, generator=gen, device=device).to(torch.int32)
        self.taken = 0                                  # blocks, from the front of `free`
        self.longest = 0
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        if sizes.rotary:
            self.frequencies = (10000.0 ** (-torch.arange(0, sizes.rotary, 2, device=device, dtype=torch.float64) / sizes.rotary)).float()
            self.norms = [[(1 + 0.1 * torch.randn(sizes.dim, generator=gen, device=device)).to(torch.bfloat16) for _ in range(2)] for _ in range(sizes.layers)]

    def _plan(self, record, added: List[int]) -> binding.CachePlan:
        n, sizes = sum(added), self.sizes
        return record("plan", (len(added), 1, 1), binding.fikit_cache_plan, self.lengths,
                      torch.tensor(added, dtype=torch.int32).to(self.device, non_blocking=True), n, sizes.block, self.table,
                      self.free[self.taken:], self.status, want_slots=False)

    def _layer(self, record, x, layer, attend, plan, positions):
        sizes, n = self.sizes, x.shape[0]
        qkv = record("to queries, keys, values", (n, 1, 1), torch.mm, x, self.w_qkv[layer]).view(n, -1, sizes.dim)
        q, k, v = qkv.split((sizes.q_heads, sizes.kv_heads, sizes.kv_heads), 1)
        if sizes.rotary:
            record("rotate", (n, 1, 1), binding.fikit_rotate_heads, q, k, positions, self.frequencies, self.status, q_weight=self.norms[layer][0],
                   k_weight=self.norms[layer][1], out=binding.RotatedHeads(q, k))
        record("append", (n, 1, 1), binding.fikit_cache_append, *self.caches[layer], k, v, plan.pieces, self.status)
        out = attend(q, k, v, layer)
        return x + record("back", (n, 1, 1), torch.mm, out.view(n, -1), self.w_out[layer])

    def prompts(self, record, x: torch.Tensor, lengths: List[int]) -> torch.Tensor:
        """x: [sum of lengths, hidden], the prompts one behind the other; returns the last layer's output.  They come first, or where every
        request has ended: prompt attention sees the new tokens only, so prompts behind tokens in the cache are refused."""
        if self.longest > 0:
            raise ValueError("prompts of requests that have no tokens in the cache")
        plan = self._plan(record, lengths)
        scale = 1 / math.sqrt(self.sizes.dim)
        positions = None
        if self.sizes.rotary:
            positions = torch.from_numpy(np.concatenate([np.arange(n, dtype=np.int32) for n in lengths])).to(self.device, non_blocking=True)
        for layer in range(self.sizes.layers):
            x = self._layer(record, x, layer, lambda q, k, v, _: record(
                "prompt attention", (q.shape[0], len(lengths), 1), binding.fikit_prompt_attention, q, k, v, plan.token_offsets, scale,
                self.status, want_lse=False).out, plan, positions)
        self._settle(plan, max(lengths))
        return x

    def step(self, record, x: torch.Tensor) -> torch.Tensor:
        """x: [requests, hidden], one new token per request; returns the logits of the next."""
        n = x.shape[0]
        plan = self._plan(record, [1] * n)
        scale = 1 / math.sqrt(self.sizes.dim)
        for layer in range(self.sizes.layers):
            x = self._layer(record, x, layer, lambda q, k, v, at: record(
                "cache attention", (n, 1, 1), binding.fikit_cache_attention, q, *self.caches[at], self.table, plan.lengths, scale,
                self.status, max_length=self.longest + 1, want_lse=False).out, plan, self.lengths)
        logits = record("to tokens", (n, 1, 1), torch.mm, x, self.w_tokens)
        self._settle(plan, 1)
        return logits

    def tokens(self, tokens: torch.Tensor) -> torch.Tensor:
        """What goes in for tokens, [n, hidden]: of a size that leaves the next token open.  A negative token is none, and zeros go in."""
        return torch.where(tokens[:, None] < 0, 0, self.w_tokens.t()[tokens.clamp(min=0).long()] * 4)

    def score(self, record, logits: torch.Tensor, n_top: int, tokens: Optional[torch.Tensor] = None) -> binding.TokenScores:
        return record("score", (logits.shape[0], 1, 1), binding.fikit_token_scores, logits, tokens, self.status, n_top=n_top)

    def fork(self, record, parents: torch.Tensor) -> None:
        """parents: int32 [n].  Request i is from now on the continuation of what was request parents[i], or an empty one for -1; requests that
        are nobody's parent end."""
        sizes = self.sizes
        fork = record("fork", (parents.numel(), 1, 1), binding.fikit_cache_fork, self.table, self.lengths, parents, sizes.block, sizes.blocks,
                      self.free[self.taken:], self.status)
        record("copy", (parents.numel(), 1, 1), binding.fikit_cache_copy, self.caches, fork.copies, self.status)
        self._check()
        self.table, self.lengths = fork.block_table, fork.lengths
        self.free, self.taken = fork.free_blocks[:int(fork.counts[2])], 0
        self.longest = max(fork.lengths.tolist(), default=0)          # (the longest one may have ended)

    def compact(self, record) -> int:
        """Moves the blocks in use together; returns the number of blocks behind the last of them."""
        sizes = self.sizes
        compaction = record("compact", (self.lengths.numel(), 1, 1), binding.fikit_cache_compact, self.table, self.lengths, sizes.block, sizes.blocks,
                            self.free[self.taken:], self.status)
        record("copy", (self.lengths.numel(), 1, 1), binding.fikit_cache_copy, self.caches, compaction.copies, self.status)
        self._check()
        self.table, self.free, self.taken = compaction.block_table, compaction.free_blocks, 0
        return sizes.blocks - int(compaction.counts[1])

    def _check(self) -> None:
        try:
            binding.fikit_check_status(self.status)
        except binding.FikitError:
            self.status.zero_()           # nothing of the step counts, and it can be tried again
            raise

    def _settle(self, plan, most_added) -> None:
        """What the host does at the end of a step, when it waits for the outputs anyway."""
        self._check()
        self.lengths = plan.lengths
        self.taken += int(plan.counts[0])
        self.longest += most_added


class Beams:
    """Beam search: every request is continued by the `width` most probable of its beams' alternatives.  Where less are left, the other beams are
    empty requests: of token -1, minus infinity for a log probability and no parent."""

    MOST = 32                  # alternatives that a score lists

    def __init__(self, service: Service, record, logits: torch.Tensor, width: int):
        """logits: [requests, vocabulary] behind the prompts."""
        if not 1 <= width <= min(self.MOST, logits.shape[1]):
            raise ValueError(f"width: from 1 to {self.MOST} and no more than tokens")
        self.service, self.width = service, width
        top = self._alternatives(record, logits)
        n = logits.shape[0]
        self._continue(record, top.top_logprob.reshape(-1), top.top_tokens.reshape(-1), torch.arange(n, device=logits.device).repeat_interleave(width))

    def _alternatives(self, record, logits: torch.Tensor) -> binding.TokenScores:
        top = self.service.score(record, logits, self.width)
        if bool(top.top_logprob.isnan().any()):            # (they would be sorted in front of those that are)
            raise FloatingPointError("logits that are not numbers, or infinite")
        return top

    def _continue(self, record, logprob, tokens, parents) -> torch.Tensor:
        none = logprob == -math.inf
        parents = torch.where(none, -1, parents).to(torch.int32)
        self.service.fork(record, parents)
        self.tokens, self.logprob = torch.where(none, -1, tokens), logprob
        return parents

    def step(self, record) -> torch.Tensor:
        """One more token for each beam; returns the parents, by the beams before."""
        width = self.width
        logits = self.service.step(record, self.service.tokens(self.tokens))
        top = self._alternatives(record, logits)
        # a request's width x width continuations, of which width are kept
        all_of = (self.logprob[:, None] + top.top_logprob).reshape(-1, width * width)
        logprob, best = (t.reshape(-1) for t in torch.topk(all_of, width, 1))
        request = torch.arange(all_of.shape[0], device=best.device).repeat_interleave(width)
        return self._continue(record, logprob, top.top_tokens.reshape(-1)[request * width * width + best], request * width + best // width)


def measure(sizes: Sizes = Sizes(), requests: int = 32, longest_prompt: int = 256, steps: int = 20, host_ms: float = 0.5, seed: int = 0,
            beams: int = 1):
    """Records of the two tasks (decode steps, prompts) and the services' last outputs."""
    rng = random.Random(seed)
    lengths = [rng.randint(1, longest_prompt) for _ in range(requests)]
    gen = torch.Generator(device="cuda:0").manual_seed(seed + 1)

    def tokens(n):
        return torch.randn((n, sizes.hidden), generator=gen, device="cuda:0", dtype=torch.float32).to(torch.bfloat16)
    got, records = {}, {}
    for task in ("warm-up", "decode", "prompts"):
        service = Service(sizes, requests, longest_prompt + steps, seed=seed)
        record = Recorder()
        got["prompts"] = service.prompts(record, tokens(sum(lengths)), lengths)
        if task != "prompts":
            record = Recorder()
            if beams > 1:
                last = torch.from_numpy(np.cumsum(lengths) - 1).to("cuda:0")
                search = Beams(service, record, torch.mm(got["prompts"][last], service.w_tokens), beams)
            for i in range(steps):
                record.run = i
                if beams > 1:
                    search.step(record)
                    got["step"] = search.logprob
                else:
                    got["step"] = service.step(record, tokens(requests))
                time.sleep(host_ms * 1e-3)
        records[task] = (record.records(), record.names)
    return records["decode"], records["prompts"], got, service


def main(argv=None) -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--requests", type=int, default=32)
    p.add_argument("--longest-prompt", type=int, default=256)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--host-ms", type=float, default=0.5, help="the host's time between two steps")
    p.add_argument("--rotary", type=int, default=0, help="dimensions of a head that are rotated by position; 0: no norm and no rotation")
    p.add_argument("--beams", type=int, default=1, help=f"beams of a request, up to {Beams.MOST}")
    a = p.parse_args(argv)
    if not 1 <= a.beams <= Beams.MOST:
        p.error(f"--beams: from 1 to {Beams.MOST}")
    (decode, names), (prompts, _), _, _ = measure(Sizes(layers=a.layers, rotary=a.rotary), a.requests, a.longest_prompt, a.steps, a.host_ms, beams=a.beams)
    decode["run"] = 0                                   # one trace: the idle times between steps are what is filled
    rec = np.concatenate([decode, prompts])
    off = np.array([0, decode.size, rec.size], dtype=np.uint64)
    hp, lp = np.array([0], dtype=np.uint32), np.array([1], dtype=np.uint32)
    dev = "cuda:0"
    profile, fill = binding.fikit_profile_gapfill(
        binding.to_device_records(rec, dev), binding.to_device_u64(off, dev), binding.to_device_u32(hp, dev), binding.to_device_u32(lp, dev),
        binding.to_device_u64(traces.gap_offsets(off, hp), dev), margin_ns=500, min_gap_ns=0, predictor=binding.FIKIT_PREDICT_MEAN)
    rows = binding.rows_to_numpy(profile.rows)
    print(f"{decode.size} calls in {a.steps} decode steps of {a.requests * a.beams} requests, {prompts.size} calls for {a.requests} prompts, {rows.size} kernels")
    for task, title in ((0, "decode"), (1, "prompts")):
        mine = rows[rows["task"] == task]
        print(f"  {title}: {mine['exec']['sum'].sum() / 1e6:.2f} ms busy, {mine['gap']['sum'].sum() / 1e6:.2f} ms idle")
    idle = rows[rows["task"] == 0]["gap"]["sum"].sum()
    print(f"prompt calls that fit the decode steps' idle times: {int(fill.lp_placed[0])} of {prompts.size}, "
          f"{int(fill.filled_ns.sum()) / 1e6:.2f} ms = {100 * int(fill.filled_ns.sum()) / max(1, int(idle)):.0f} % of the idle time")


if __name__ == "__main__":
    main()
