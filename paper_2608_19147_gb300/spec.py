"""Speculative decoding over pipeline shards with mask-based KV rewind (Section
5.2): greedy, with the final stage's top-1 head (Section 6.7), and on trees of
drafts with greedy or sampled tokens (TreeDecoder).

Host orchestration only, as the paper's coordinator does it: every forward
runs in the library's kernels through the C ABI -- one `shard_step_host` per
pipeline stage (the hidden states are handed from stage to stage, Section
3.3) and `head_top1_host` on the last stage's output -- while the host keeps
the per-request rewind state (a valid bit per physical cache entry and the
logical position, Section 5.2) and makes the greedy acceptance decision, a
token-id comparison (Section 5.2, greedy decoding only).

A verify step feeds [current token, d_1 .. d_k]: the target's greedy token
after input i is targets[i]; the longest prefix of drafts with
d_{i+1} == targets[i] is accepted (a tokens), the emitted tokens are
d_1 .. d_a followed by the correction targets[a], the rejected entries
d_{a+1} .. d_k stay in the cache but are masked out on every later forward,
and the logical position advances by 1 + a.  The emitted sequence equals
plain greedy decoding's (Section 5.3, 5.4).
"""
from __future__ import annotations

from typing import Callable, List, Optional, Sequence, Tuple

import numpy as np

from . import (SHARD_MAX_REQUESTS, SHARD_MAX_TOKENS, SHARD_MAX_TREE, SHARD_MAX_TREE_NODES, head_sample, head_top1_host, kv_state_alloc, kv_state_free,
               kv_state_length, kv_trim, shard_prefill, shard_step_host, shard_step_tree, shard_sync_status, shard_tree_accept)

# forward(token_ids [n] int32, position_ids [n] int32, mask [L + n] uint8) -> greedy tokens [n] int32
Forward = Callable[[np.ndarray, np.ndarray, np.ndarray], np.ndarray]


def greedy_accept(drafts: Sequence[int], targets: Sequence[int]) -> Tuple[int, List[int]]:
    """Greedy acceptance of one verify block.  targets has one more entry
    than drafts (targets[i] is the target's token after input i of
    [current, d_1 .. d_k]).  Returns (a, emitted): a = the number of leading
    drafts the target agrees with, emitted = drafts[:a] + [targets[a]]."""
    k = len(drafts)
    if len(targets) != k + 1:
        raise ValueError("need len(targets) == len(drafts) + 1, got %d and %d" % (len(targets), k))
    a = 0
    while a < k and int(drafts[a]) == int(targets[a]):
        a += 1
    return a, [int(d) for d in drafts[:a]] + [int(targets[a])]


class MaskedRequest:
    """Rewind state of one request row (Section 5.2): cache entries are
    appended in order and never removed; `valid[j]` says whether entry j
    still takes part in attention, `position` is the logical length (the
    next position id, which RoPE uses)."""

    def __init__(self, cached: int = 0):
        self.valid: List[int] = [1] * cached
        self.position = cached

    @property
    def physical(self) -> int:
        return len(self.valid)

    def inputs(self, n: int) -> Tuple[np.ndarray, np.ndarray]:
        """position_ids and attention mask for n new entries (all visible)."""
        pos = np.arange(self.position, self.position + n, dtype=np.int32)
        mask = np.array(self.valid + [1] * n, dtype=np.uint8)
        return pos, mask

    def commit(self, n_fed: int, n_kept: int) -> None:
        """n_fed entries were appended; the first n_kept stay visible."""
        if not 0 <= n_kept <= n_fed:
            raise ValueError("kept %d of %d" % (n_kept, n_fed))
        self.valid += [1] * n_kept + [0] * (n_fed - n_kept)
        self.position += n_kept


class GreedySpecDecoder:
    """Greedy (speculative) decoding of one request over a forward function.

    `prefill(prompt)` feeds the prompt in blocks of at most
    SHARD_MAX_TOKENS tokens and returns the first generated token;
    `step(drafts)` runs one verify block and returns the emitted tokens
    (`step([])` is one plain greedy step)."""

    def __init__(self, forward: Forward, max_block: int = SHARD_MAX_TOKENS):
        self.forward = forward
        self.max_block = max_block
        self.req = MaskedRequest(0)
        self.current: Optional[int] = None
        self.accepted = 0
        self.proposed = 0
        self.steps = 0

    def prefill(self, prompt: Sequence[int]) -> int:
        prompt = [int(t) for t in prompt]
        if not prompt:
            raise ValueError("empty prompt")
        last = None
        for i in range(0, len(prompt), self.max_block):
            block = np.array(prompt[i:i + self.max_block], dtype=np.int32)
            pos, mask = self.req.inputs(block.size)
            out = np.asarray(self.forward(block, pos, mask))
            self.req.commit(block.size, block.size)
            last = int(out[-1])
        self.current = last
        return last

    def step(self, drafts: Sequence[int] = ()) -> List[int]:
        if self.current is None:
            raise RuntimeError("prefill first")
        drafts = [int(d) for d in drafts]
        if len(drafts) + 1 > self.max_block:
            raise ValueError("at most %d drafts per step" % (self.max_block - 1))
        feed = np.array([self.current] + drafts, dtype=np.int32)
        pos, mask = self.req.inputs(feed.size)
        targets = np.asarray(self.forward(feed, pos, mask))
        a, emitted = greedy_accept(drafts, targets)
        self.req.commit(feed.size, 1 + a)
        self.current = emitted[-1]
        self.accepted += a
        self.proposed += len(drafts)
        self.steps += 1
        return emitted


class ShardPipeline:
    """A forward function over pipeline stages and a top-1 head through the
    C ABI: stage 0 takes token ids (it owns the embedding), every later
    stage the previous stage's fp16 hidden states; the head returns the
    greedy tokens.  One request row per stage state.

    stages: shard handles in pipeline order; hidden: their hidden width;
    head: a head handle; capacity: cache entries per stage state (prompt,
    generated tokens and rejected drafts)."""

    def __init__(self, stages: Sequence[int], hidden: int, head: int, capacity: int, stream: int = 0):
        self.stages = list(stages)
        self.hidden = hidden
        self.head = head
        self.stream = stream
        self.states = [kv_state_alloc(s, 1, capacity) for s in self.stages]
        self.capacity = capacity

    def __call__(self, tokens: np.ndarray, positions: np.ndarray, mask: np.ndarray) -> np.ndarray:
        n = int(tokens.size)
        h = np.empty((n, self.hidden), dtype=np.uint16)
        for i, (sh, st) in enumerate(zip(self.stages, self.states)):
            out = np.empty((n, self.hidden), dtype=np.uint16)
            shard_step_host(sh, st, None if i == 0 else h, tokens if i == 0 else None, [n], positions,
                            mask.reshape(1, -1), None, out, self.stream)
            h = out
        tok, _ = head_top1_host(self.head, h, self.stream)
        return tok

    def close(self) -> None:
        for st in self.states:
            kv_state_free(st)
        self.states = []


def tree_depths(parents: Sequence[int]) -> List[int]:
    """Depth of every node of one drafted tree: 0 for node 0, its parent's + 1 for the others."""
    depth: List[int] = []
    for i, p in enumerate(parents):
        if (p != -1) if i == 0 else not 0 <= p < i:
            raise ValueError("node %d has parent %d: node 0 is the root, and every other node's parent comes before it" % (i, p))
        depth.append(0 if i == 0 else depth[p] + 1)
    return depth


class TreeDecoder:
    """Speculative decoding of B requests on drafted trees, over pipeline
    stages and a head, on the GPU: one shard_step_tree per stage, a draw at every
    node (head_sample), and the acceptance with the mask-based rewind
    (shard_tree_accept).  Only the kept tokens come to the host.

    A request's tree is (drafts, parents): the drafted tokens behind its current
    token, and each one's parent among [current, drafts ..], an index of at least 0
    that is below the draft's own.  A draw from the model's distribution at
    every node of the kept path makes the emitted tokens draws of the model,
    whatever was drafted; with temperature 0 they are the greedy tokens.

    Every node of a step keeps its entry of the cache, kept or not (the rewind is
    a mask), so `capacity` counts all nodes that are ever verified.

    stages, hidden, head as in ShardPipeline; B at most SHARD_MAX_REQUESTS;
    settings: temperature, top_k, top_p and min_p of all requests; draws(n) gives
    n random numbers in [0, 1).  Where the head has no token for a request
    (logits that are not numbers, draws out of range, or a device wait that gave
    up, after which the head is to be created again), prefill and step raise
    RuntimeError and leave the decoder as it was before."""

    def __init__(self, stages: Sequence[int], hidden: int, head: int, B: int, capacity: int, temperature: float = 1.0,
                 top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0, draws: Optional[Callable[[int], np.ndarray]] = None):
        t, p, low = np.float32(temperature), np.float32(top_p), np.float32(min_p)
        if not (0 <= t < np.inf and top_k >= 0 and 0 < p <= 1 and 0 <= low <= 1):
            raise ValueError("temperature %r, top_k %r, top_p %r or min_p %r out of range" % (temperature, top_k, top_p, min_p))
        if not 1 <= B <= SHARD_MAX_REQUESTS:
            raise ValueError("%d requests outside [1, %d]" % (B, SHARD_MAX_REQUESTS))
        import torch

        self.torch = torch
        self.stages, self.hidden, self.head, self.B, self.capacity = list(stages), hidden, head, B, capacity
        self.states: List[int] = []
        self.mask = torch.zeros((B, capacity), dtype=torch.uint8, device="cuda")
        self.length = [0] * B    # entries, kept or not
        self.position = [0] * B  # of the current token
        self.current: List[Optional[int]] = [None] * B
        self.draws = draws or np.random.default_rng().random
        self.accepted = self.proposed = self.steps = 0
        n = SHARD_MAX_TOKENS
        self.settings = dict(temperature=torch.full((n,), float(temperature), device="cuda"),
                             top_k=torch.full((n,), int(top_k), dtype=torch.int32, device="cuda"),
                             top_p=torch.full((n,), float(top_p), device="cuda"),
                             min_p=torch.full((n,), float(min_p), device="cuda"))
        try:
            for sh in self.stages:
                self.states.append(kv_state_alloc(sh, B, capacity))
        except Exception:
            self.close()
            raise

    def _dev(self, values, dtype):
        return self.torch.from_numpy(np.ascontiguousarray(values, dtype=dtype)).to("cuda")

    def _numbers(self, n: int) -> np.ndarray:
        """n random numbers, before anything runs on them."""
        u = np.asarray(self.draws(n), np.float32)
        if u.shape != (n,):
            raise ValueError("draws(%d) gave numbers of shape %r" % (n, u.shape))
        return np.minimum(u, np.float32(1 - 2.0 ** -24))

    def _sample(self, h, numbers: np.ndarray):
        """A draw from the model's distribution after each hidden row, one per number (device int32 [n])."""
        torch, stream, n = self.torch, self.torch.cuda.current_stream().cuda_stream, numbers.size
        token = torch.empty(n, dtype=torch.int32, device="cuda")
        u = self._dev(numbers, np.float32)
        for i in range(0, n, SHARD_MAX_TOKENS):
            head_sample(self.head, h[i:].data_ptr(), min(SHARD_MAX_TOKENS, n - i), u[i:].data_ptr(), token[i:].data_ptr(),
                        **{k: v.data_ptr() for k, v in self.settings.items()}, stream=stream)
        return token

    def _require(self, tokens: Sequence[Sequence[int]]) -> None:
        """Where a request has no token: its and all others' entries behind the lengths taken back, and an error."""
        bad = [b for b, t in enumerate(tokens) if any(x < 0 for x in t)]
        if not bad:
            return
        for st in self.states:
            for b in range(self.B):
                n = kv_state_length(st, b)
                if n > self.length[b]:
                    kv_trim(st, b, np.arange(n) < self.length[b])
        raise RuntimeError("head %d has no token for request %s: logits that are not numbers, draws outside [0, 1), or a device wait that "
                           "gave up" % (self.head, ", ".join(map(str, bad))))

    def prefill(self, prompts: Sequence[Sequence[int]]) -> List[int]:
        """Runs each request's prompt through the stages; the first generated token of each."""
        if len(prompts) != self.B or any(len(p) == 0 for p in prompts):
            raise ValueError("one prompt of at least one token for each request")
        for b, prompt in enumerate(prompts):
            if self.length[b] + len(prompt) > self.capacity:
                raise ValueError("request %d would hold %d entries > %d" % (b, self.length[b] + len(prompt), self.capacity))
        numbers = self._numbers(self.B)
        torch, stream = self.torch, self.torch.cuda.current_stream().cuda_stream
        last = torch.empty((self.B, self.hidden), dtype=torch.int16, device="cuda")
        for b, prompt in enumerate(prompts):
            n, at = len(prompt), self.length[b]
            ids, pos = self._dev(prompt, np.int32), self._dev(np.arange(self.position[b], self.position[b] + n), np.int32)
            self.mask[b, at:at + n] = 1
            h = None
            for sh, st in zip(self.stages, self.states):
                out = torch.empty((n, self.hidden), dtype=torch.int16, device="cuda")
                shard_prefill(sh, st, b, None if h is None else h.data_ptr(), ids.data_ptr() if h is None else None, n, pos.data_ptr(),
                              self.mask[b].data_ptr(), self.capacity, out.data_ptr(), stream)
                h = out
            last[b] = h[n - 1]
        token = self._sample(last, numbers)
        for sh in self.stages:
            shard_sync_status(sh, stream)
        first = token.tolist()
        self._require([[t] for t in first])
        for b, prompt in enumerate(prompts):
            self.length[b] += len(prompt)
            self.position[b] += len(prompt)
        self.current = first
        return list(first)

    def step(self, trees: Optional[Sequence[Tuple[Sequence[int], Sequence[int]]]] = None) -> List[List[int]]:
        """Verifies one tree per request, (drafts, parents) each, or decodes plainly (None); the emitted tokens of each."""
        if any(c is None for c in self.current):
            raise RuntimeError("prefill first")
        trees = [((), ()) for _ in range(self.B)] if trees is None else trees
        if len(trees) != self.B or any(len(d) != len(p) for d, p in trees):
            raise ValueError("one tree for each request, a parent for each draft")
        tokens = [[c] + [int(t) for t in d] for c, (d, _) in zip(self.current, trees)]
        parents = [[-1] + [int(i) for i in p] for _, p in trees]
        n = [len(t) for t in tokens]
        depths = [tree_depths(p) for p in parents]
        for b in range(self.B):
            if n[b] > SHARD_MAX_TREE or self.length[b] + n[b] > self.capacity:
                raise ValueError("request %d: a tree of %d nodes behind %d entries (at most %d, capacity %d)"
                                 % (b, n[b], self.length[b], SHARD_MAX_TREE, self.capacity))
        torch, stream, N = self.torch, self.torch.cuda.current_stream().cuda_stream, sum(n)
        if N > SHARD_MAX_TREE_NODES:
            raise ValueError("%d nodes in all > %d" % (N, SHARD_MAX_TREE_NODES))
        numbers = self._numbers(N)
        start = self._dev(np.concatenate([[0], np.cumsum(n)]), np.int32)
        ids, up = self._dev(sum(tokens, []), np.int32), self._dev(sum(parents, []), np.int32)
        pos = self._dev([self.position[b] + d for b in range(self.B) for d in depths[b]], np.int32)
        lens = self._dev(self.length, np.int32)
        for b in range(self.B):
            self.mask[b, self.length[b]:self.length[b] + n[b]] = 1
        h = None
        for sh, st in zip(self.stages, self.states):
            out = torch.empty((N, self.hidden), dtype=torch.int16, device="cuda")
            shard_step_tree(sh, st, None if h is None else h.data_ptr(), ids.data_ptr() if h is None else None, n, up.data_ptr(),
                            pos.data_ptr(), self.mask.data_ptr(), self.capacity, out.data_ptr(), stream)
            h = out
        target = self._sample(h, numbers)
        path, emitted = (torch.empty((self.B, max(n)), dtype=torch.int32, device="cuda") for _ in range(2))
        count = torch.empty(self.B, dtype=torch.int32, device="cuda")
        shard_tree_accept(self.B, N, start.data_ptr(), up.data_ptr(), ids.data_ptr(), target.data_ptr(), max(n), path.data_ptr(),
                          emitted.data_ptr(), count.data_ptr(), lens=lens.data_ptr(), attention_mask=self.mask.data_ptr(),
                          mask_stride=self.capacity, stream=stream)
        for sh in self.stages:
            shard_sync_status(sh, stream)
        kept, tok = count.tolist(), emitted.tolist()
        out = [tok[b][:kept[b]] for b in range(self.B)]
        self._require(out)
        for b in range(self.B):
            self.length[b] += n[b]
            self.position[b] += kept[b]
            self.current[b] = out[b][-1]
        self.steps += 1
        self.proposed += N - self.B
        self.accepted += sum(kept) - self.B
        return out

    def close(self) -> None:
        for st in self.states:
            kv_state_free(st)
        self.states = []
