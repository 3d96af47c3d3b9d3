"""Prompts taken in by chunks, then verification steps, on caches that are kept within a budget of tokens.

The loop runs the library's entry points around prompts and bounded caches together as a serving process does:

  a chunk's rows of all requests: heads normalised and turned    `spec_qk_norm_rope`, at the tokens' own positions
                                  into the cache                 `spec_kv_append` or `spec_kv8_append`
                                  attention                      `spec_prompt_attn`, with each row's log-sum-exp
  a prompt's last rows say which of its tokens matter            `spec_kv_weight`
  a request with more tokens than the budget loses some          `spec_kv_evict`, into pages of its own; the old ones are free again
  every step: the same with k + 1 rows a request, then
              verification of the drafts                         `spec_reject_sample`
              and what the rows that stay look at is added       `spec_kv_weight` (`accepted_only`; otherwise what all rows look at, before it)

Positions go on counting when a cache has lost tokens.  There is no model around the steps: projections are Gaussian, the drafts
and both models' logits are made as in the control loop.

    python -m paper_2406_14066_amd.prompt_loop [--requests 8] [--prompt 4000] [--chunk 1024] [--budget 1024] [--k 4] [--steps 12] [--kv bf16]

prints one JSON line: tokens taken in and kept, the cache's bytes with and without the budget, the attention's time of the prompts and of
a step.  This module only generates inputs, marshals arguments and calls the library's entry points.
"""
from __future__ import annotations

import argparse
import json
import sys

import numpy as np

from . import spec_verify as sv


class PromptLoop:
    """`requests` requests with prompts of prompt[0] .. prompt[1] tokens; `budget` tokens stay of each, the first `first` and the last `recent` among them.
    `accepted_only`: a step's weights are of the rows that verification leaves; otherwise of all its rows, rejected drafts' among them, before verification."""

    def __init__(self, requests, prompt, *, budget, chunk=1024, window=32, first=4, recent=64, k=4, steps=12, Hq=32, Hkv=8, d=128, V=4096, kv="bf16",
                 layout=sv.KV_MFMA, sigma=0.773, seed=1, timed=False, accepted_only=False, device="cuda"):
        import torch
        if min(requests, prompt[0], chunk, budget, window) < 1 or min(first, recent, k, steps) < 0 or prompt[1] < prompt[0]:
            raise ValueError("requests, prompts, chunk, budget and window must be positive, first, recent, k and steps not negative")
        self.torch, self.device, self.seed, self.timed, self.accepted_only = torch, device, seed, timed, accepted_only
        self.B, self.chunk, self.window, self.first, self.recent, self.budget, self.k = requests, chunk, window, first, recent, budget, k
        self.Hq, self.Hkv, self.d, self.V, self.sigma, self.kv, self.layout = Hq, Hkv, d, V, sigma, kv, layout
        rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        self.prompt = rng.integers(prompt[0], prompt[1] + 1, requests).astype(np.int32)
        self.position = np.zeros(requests, dtype=np.int64)       # tokens that have been there
        self.kept = np.zeros(requests, dtype=np.int32)           # cached tokens (host copy)
        # pages: room for every prompt, for what an eviction fills while the old pages are still there, and for the steps
        most = int(self.prompt.max()) + steps * (k + 1)
        self.columns = (most + sv.BLOCK_SIZE - 1) // sv.BLOCK_SIZE
        self.num_blocks = requests * (self.columns + (budget + sv.BLOCK_SIZE - 1) // sv.BLOCK_SIZE + 1)
        self.free = [int(x) for x in rng.permutation(self.num_blocks)]
        self.table = np.zeros((requests, self.columns), dtype=np.int32)
        self.pages = np.zeros(requests, dtype=np.int32)          # of a request
        if kv == "bf16":
            self.k_cache, self.v_cache = (torch.zeros((self.num_blocks, Hkv, sv.BLOCK_SIZE, d), dtype=torch.bfloat16, device=device) for _ in range(2))
            self.kv_scale = None
        else:
            self.k_cache, self.v_cache, self.kv_scale = sv.alloc_kv8_pools(self.num_blocks, Hkv, d, torch.int8 if kv == "int8" else torch.float8_e4m3fn, device)
        self.weight = sv.alloc_kv_weight(self.num_blocks, Hkv, device)
        self.inv_freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(device)
        self.q_weight, self.k_weight = (1 + 0.2 * torch.randn(d, generator=self.gen, device=device) for _ in range(2))
        self.errors = torch.zeros(1, dtype=torch.int64, device=device)
        self.counters = torch.zeros(sv.NUM_COUNTERS, dtype=torch.int64, device=device)
        self.accepted = torch.zeros(requests, dtype=torch.int32, device=device)
        self.next_token, self.new_kv_len = torch.zeros_like(self.accepted), torch.zeros_like(self.accepted)
        self.step_index, self.evicted = 0, 0
        self.prompt_seconds, self.step_seconds = [], []

    def _int32(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(self.device)

    def _grow(self, lengths):
        """Pages for requests of `lengths` tokens."""
        for b, n in enumerate(lengths):
            while self.pages[b] * sv.BLOCK_SIZE < n:
                self.table[b, self.pages[b]] = self.free.pop()
                self.pages[b] += 1

    def _call(self, call, seconds):
        if not self.timed:
            return call()
        start, stop = (self.torch.cuda.Event(enable_timing=True) for _ in range(2))
        call()
        start.record()
        call()
        stop.record()
        stop.synchronize()
        seconds.append(start.elapsed_time(stop) * 1e-3)

    def _forward(self, counts, seconds):
        """Rows of the next `counts` tokens of every request into the cache, and their attention: (out, lse, rows' offsets)."""
        torch, Hq, Hkv = self.torch, self.Hq, self.Hkv
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.host_len = (self.kept + counts).astype(np.int32)
        self._grow(self.host_len)
        table, kv_len, dev_cu = self._int32(self.table), self._int32(self.host_len), self._int32(cu)
        self.positions = np.concatenate([np.arange(p, p + n) for p, n in zip(self.position, counts)])
        # queries and keys are turned in place, as slices of one fused projection
        self.raw = torch.randn((int(cu[-1]), Hq + 2 * Hkv, self.d), generator=self.gen, device=self.device).to(torch.bfloat16)
        rows = self.raw.clone()
        q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        rope, keep_r = sv.make_qk_norm_rope_args(q, k, q, k, self._int32(self.positions), self.inv_freq, q_weight=self.q_weight, k_weight=self.k_weight)
        sv.spec_qk_norm_rope(rope)
        if self.kv == "bf16":
            on = np.nonzero(counts)[0]      # (this append has no room for requests without rows)
            offsets, lengths = np.append(cu[on], cu[-1]).astype(np.int32), self.host_len[on]
            sv.spec_kv_append(k.contiguous(), v.contiguous(), self.k_cache, self.v_cache, self._int32(self.table[on]), self._int32(lengths), self._int32(offsets),
                              lengths, offsets, kv_layout=self.layout, error_count=self.errors)
        else:
            append, keep_a = sv.make_kv8_append_args(k, v, self.k_cache, self.v_cache, self.kv_scale, table, kv_len, dev_cu, self.host_len, cu, error_count=self.errors)
            sv.spec_kv8_append(append)
        out = torch.empty((int(cu[-1]), Hq, self.d), dtype=torch.bfloat16, device=self.device)
        lse = torch.empty((int(cu[-1]), Hq), dtype=torch.float32, device=self.device)
        attn, keep = sv.make_prompt_attn_args(q, self.k_cache, self.v_cache, table, kv_len, dev_cu, out, self.host_len, cu, lse=lse, kv_scale=self.kv_scale,
                                              kv_layout=self.layout, error_count=self.errors)
        workspace = sv.alloc_workspace(sv.spec_prompt_attn_workspace_bytes(attn), self.device)
        self._call(lambda: sv.spec_prompt_attn(attn, workspace), seconds)
        self.q, self.cu = q, cu
        return out, lse

    def _weigh(self, q, lse, lengths, cu, add):
        """The tokens' weights as the given rows see them, or those added to what they have."""
        args, keep = sv.make_kv_weight_args(q, lse, self.k_cache, self._int32(self.table), self._int32(lengths), self._int32(cu), self.weight, lengths, cu,
                                            weight_in=self.weight if add else None, kv_scale=self.kv_scale, kv_layout=self.layout, error_count=self.errors)
        sv.spec_kv_weight(args)

    def take_prompts(self):
        """All prompts, a chunk of every request at a time; returns the last chunk's (out, lse)."""
        torch = self.torch
        while (self.position < self.prompt).any():
            counts = np.minimum(self.prompt - self.position, self.chunk).astype(np.int32)
            out, lse = self._forward(counts, self.prompt_seconds)
            self.kept = self.host_len.copy()
            self.position += counts
            ends = np.nonzero((self.position == self.prompt) & (counts > 0))[0]
            if len(ends):      # what the last rows of the prompts that end here look at
                seen = np.zeros(self.B, dtype=np.int32)
                seen[ends] = np.minimum(counts[ends], self.window)
                rows = torch.from_numpy(np.concatenate([np.arange(self.cu[b + 1] - seen[b], self.cu[b + 1]) for b in range(self.B)])).to(self.device)
                self._weigh(self.q[rows], lse[rows], self.kept, np.concatenate([[0], np.cumsum(seen)]).astype(np.int32), False)
        return out, lse

    def evict(self):
        """Cuts every request with more than `budget` tokens down to it; returns the kept tokens' indices, a row per such request, and the requests."""
        torch = self.torch
        long = np.nonzero(self.kept > self.budget)[0]
        if not len(long):
            return None, long
        width = (self.budget + sv.BLOCK_SIZE - 1) // sv.BLOCK_SIZE
        new = np.array([[self.free.pop() for _ in range(width)] for _ in long], dtype=np.int32)
        kept = torch.empty((len(long), width * sv.BLOCK_SIZE), dtype=torch.int32, device=self.device)
        lengths = torch.empty(len(long), dtype=torch.int32, device=self.device)
        args, keep = sv.make_kv_evict_args(self.k_cache, self.v_cache, self.weight, self._int32(self.table[long]), self._int32(self.kept[long]),
                                           self._int32(np.full(len(long), self.budget)), self._int32(new), lengths, self.kept[long], kept=kept, first=self.first,
                                           recent=self.recent, kv_scale=self.kv_scale, kv_layout=self.layout, error_count=self.errors)
        sv.spec_kv_evict(args, sv.alloc_workspace(sv.spec_kv_evict_workspace_bytes(args), self.device))
        for i, b in enumerate(long):
            self.free.extend(int(x) for x in self.table[b, :self.pages[b]])
            self.table[b] = 0
            self.table[b, :width] = new[i]
            self.pages[b] = width
        self.evicted += int((self.kept[long] - self.budget).sum())
        self.kept[long] = lengths.cpu().numpy()
        return kept, long

    def step(self):
        """One verification step of all requests: (out, lse) of its rows."""
        torch, B, k = self.torch, self.B, self.k
        T = B * (k + 1)
        out, lse = self._forward(np.full(B, k + 1, dtype=np.int32), self.step_seconds)
        if not self.accepted_only:
            self._weigh(self.q, lse, self.host_len, self.cu, True)
        logits = torch.randn((T, self.V), generator=self.gen, device=self.device) * 3.0
        target = logits + torch.randn((T, self.V), generator=self.gen, device=self.device) * self.sigma
        drafts = logits[(torch.arange(T, device=self.device) + 1) % (k + 1) != 0]       # (a request's last row seeds its extra target row)
        gumbel = -torch.log(-torch.log(torch.rand(drafts.shape, generator=self.gen, device=self.device).clamp_(1e-12, 1.0)).clamp_(min=1e-30))
        tokens = torch.argmax(drafts + gumbel, dim=1).to(torch.int32)
        reject, keep_r = sv.make_reject_args(target, drafts if k else None, tokens if k else None, self._int32(self.cu), self.cu, self.accepted, self.next_token,
                                             self.counters, philox_seed=self.seed, philox_step=self.step_index, kv_len=self._int32(self.host_len),
                                             new_kv_len=self.new_kv_len)
        sv.spec_reject_sample(reject, sv.alloc_workspace(sv.spec_verify_workspace_bytes(None, reject), self.device))
        kept = self.new_kv_len.cpu().numpy().astype(np.int32)
        stay = kept - self.kept
        if self.accepted_only:      # (the tokens of rejected drafts are overwritten by the next step's, and their rows are in no sequence)
            rows = torch.from_numpy(np.concatenate([np.arange(self.cu[b], self.cu[b] + stay[b]) for b in range(B)])).to(self.device)
            self._weigh(self.q[rows], lse[rows], kept, np.concatenate([[0], np.cumsum(stay)]).astype(np.int32), True)
        self.position += stay
        self.kept = kept
        self.step_index += 1
        return out, lse

    def cache_bytes(self, bounded=True):
        """Bytes of the requests' tokens in the cache, or of all the tokens that have been there."""
        tokens = int(self.kept.sum() if bounded else self.position.sum())
        return tokens * self.Hkv * (4 * self.d if self.kv == "bf16" else 2 * self.d + 8)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=4000)
    ap.add_argument("--chunk", type=int, default=1024)
    ap.add_argument("--budget", type=int, default=1024)
    ap.add_argument("--k", type=int, default=4)
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--kv", choices=["bf16", "e4m3", "int8"], default="bf16")
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        print("prompt_loop: no GPU visible", file=sys.stderr)
        sys.exit(2)
    loop = PromptLoop(args.requests, ((args.prompt + 1) // 2, args.prompt), budget=args.budget, chunk=args.chunk, k=args.k, steps=args.steps, kv=args.kv, timed=True, accepted_only=True)
    loop.take_prompts()
    loop.evict()
    for _ in range(args.steps):
        loop.step()
        loop.evict()
    counters = loop.counters.cpu().numpy()
    print(json.dumps({
        "requests": loop.B, "prompt_tokens": int(loop.prompt.sum()), "budget": args.budget, "k": args.k, "steps": args.steps, "kv": args.kv,
        "tokens_kept": int(loop.kept.sum()), "tokens_evicted": loop.evicted, "accepted": int(counters[1]), "attempted": int(counters[2]), "emitted": int(counters[3]),
        "cache_bytes": loop.cache_bytes(), "cache_bytes_unbounded": loop.cache_bytes(bounded=False),
        "prompt_attention_us": 1e6 * float(np.sum(loop.prompt_seconds)), "step_attention_us": 1e6 * float(np.median(loop.step_seconds)),
        "errors": int(loop.errors.item()),
    }))


if __name__ == "__main__":
    main()
