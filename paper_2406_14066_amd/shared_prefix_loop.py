"""Verification steps of requests behind shared prompts, on the 8-bit KV cache.

Tenants' requests begin with their tenant's prompt, whose pages are in the cache once.  The loop runs the library's cache and
attention entry points together as a serving process does:

  prompts and questions enter the cache       `spec_kv8_append`, a tenant's prompt as rows of its own
  every step: k + 1 new K/V rows a request    `spec_kv8_append`
              lookahead attention             `spec_prefix_attn`, groups of requests behind their prompts
              verification of the drafts      `spec_reject_sample`, whose new lengths are the next step's
  a request leaves for another worker         `spec_kv8_read`, its own tokens as bf16 rows

`unshared_attention` is the same step's attention with `spec_kv8_attn`, which walks every request's whole context.  There is
no model around the steps: queries, keys and values are Gaussian, the drafts and both models' logits are made as in the control
loop (draft tokens drawn from the draft logits, target logits = draft logits + N(0, sigma^2)).

    python -m paper_2406_14066_amd.shared_prefix_loop [--tenants 4] [--requests 16] [--prompt 2048] [--k 4] [--steps 12] [--kv e4m3]

prints one JSON line: tokens kept, the cache's bytes with and without sharing, and the attention's time both ways.
This module only generates inputs, marshals arguments and calls the library's entry points.
"""
from __future__ import annotations

import argparse
import json
import sys

import numpy as np

from . import spec_verify as sv


class SharedPrefixLoop:
    """`tenants` groups of `requests` requests each, behind a prompt of `prompt` tokens (a multiple of the page) per group."""

    def __init__(self, tenants, requests, prompt, *, question=(8, 64), k=4, steps=12, Hq=32, Hkv=8, d=128, V=4096, kv="e4m3", sigma=0.773,
                 seed=1, timed=False, device="cuda"):
        import torch
        if prompt % sv.BLOCK_SIZE != 0:
            raise ValueError("prompt must be a multiple of %d" % sv.BLOCK_SIZE)
        self.torch, self.device, self.seed = torch, device, seed
        self.G, self.B, self.prompt, self.k, self.Hq, self.Hkv, self.d, self.V, self.sigma = tenants, tenants * requests, prompt, k, Hq, Hkv, d, V, sigma
        rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        asked = rng.integers(question[0], question[1] + 1, self.B).astype(np.int32)
        self.kept = (prompt + asked).astype(np.int32)                 # cached tokens of a request (host copy)
        self.max_kv_len = int(self.kept.max()) + steps * (k + 1)
        # block table: a tenant's prompt pages are in the first columns of all of its requests
        own = (self.max_kv_len - prompt + sv.BLOCK_SIZE - 1) // sv.BLOCK_SIZE
        shared = prompt // sv.BLOCK_SIZE
        self.num_blocks = tenants * shared + self.B * own
        pages = rng.permutation(self.num_blocks).astype(np.int32)
        head = pages[:tenants * shared].reshape(tenants, shared)
        self.table = torch.from_numpy(np.concatenate([np.repeat(head, requests, axis=0), pages[tenants * shared:].reshape(self.B, own)], axis=1)).to(device)
        self.k_cache, self.v_cache, self.kv_scale = sv.alloc_kv8_pools(self.num_blocks, Hkv, d, torch.int8 if kv == "int8" else torch.float8_e4m3fn, device)
        self.host_group = (np.arange(tenants + 1) * requests).astype(np.int32)
        self.host_prefix = np.full(tenants, prompt, dtype=np.int32)
        self.group, self.prefix = torch.from_numpy(self.host_group).to(device), torch.from_numpy(self.host_prefix).to(device)
        self.errors = torch.zeros(1, dtype=torch.int64, device=device)
        self.counters = torch.zeros(sv.NUM_COUNTERS, dtype=torch.int64, device=device)
        self.accepted = torch.zeros(self.B, dtype=torch.int32, device=device)
        self.next_token, self.new_kv_len = torch.zeros_like(self.accepted), torch.zeros_like(self.accepted)
        self.step_index = 0
        self.timed, self.attention_seconds = timed, []
        # prompts: one append for all tenants, through the first request's table row of each
        if prompt:
            self._append(np.full(tenants, prompt), np.full(tenants, prompt), self.table[:: requests].contiguous())
        self._append(asked, self.kept, self.table)

    def _int32(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(self.device)

    def _rows(self, *shape):
        return self.torch.randn(shape, generator=self.gen, device=self.device).to(self.torch.bfloat16)

    def _append(self, counts, lengths, table):
        """New K/V rows, the last `counts` of the requests' `lengths` tokens, as slices of one fused projection."""
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        rows = self._rows(int(cu[-1]), 2 * self.Hkv, self.d)
        args, keep = sv.make_kv8_append_args(rows[:, :self.Hkv], rows[:, self.Hkv:], self.k_cache, self.v_cache, self.kv_scale, table, self._int32(lengths),
                                             self._int32(cu), np.asarray(lengths, dtype=np.int32), cu, error_count=self.errors)
        sv.spec_kv8_append(args)
        return rows

    def _timed(self, call, times=10):
        """Seconds of a call among others (the attention may be repeated: its output is the same)."""
        start, stop = (self.torch.cuda.Event(enable_timing=True) for _ in range(2))
        call()
        start.record()
        for _ in range(times):
            call()
        stop.record()
        stop.synchronize()
        return start.elapsed_time(stop) * 1e-3 / times

    def step(self):
        """One verification step of all requests; returns the attention's output [T, Hq, d]."""
        torch, B, k = self.torch, self.B, self.k
        T = B * (k + 1)
        self.host_len = (self.kept + k + 1).astype(np.int32)
        self.host_cu = (np.arange(B + 1) * (k + 1)).astype(np.int32)
        self.kv_len, self.cu = self._int32(self.host_len), self._int32(self.host_cu)
        self._append(np.full(B, k + 1), self.host_len, self.table)

        self.q = self._rows(T, self.Hq, self.d)
        out = torch.empty_like(self.q)
        attn, keep_a = sv.make_prefix_attn_args(self.q, self.k_cache, self.v_cache, self.table, self.kv_len, self.cu, self.group, self.prefix, out,
                                                self.host_len, self.host_cu, self.host_group, self.host_prefix, kv_scale=self.kv_scale,
                                                max_kv_len=self.max_kv_len, error_count=self.errors)
        workspace = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(attn), self.device)
        if self.timed:
            self.attention_seconds.append(self._timed(lambda: sv.spec_prefix_attn(attn, workspace)))
        else:
            sv.spec_prefix_attn(attn, workspace)

        logits = torch.randn((T, self.V), generator=self.gen, device=self.device) * 3.0
        target = logits + torch.randn((T, self.V), generator=self.gen, device=self.device) * self.sigma
        drafts = logits[(torch.arange(T, device=self.device) + 1) % (k + 1) != 0]       # (a request's last row seeds its extra target row)
        gumbel = -torch.log(-torch.log(torch.rand(drafts.shape, generator=self.gen, device=self.device).clamp_(1e-12, 1.0)).clamp_(min=1e-30))
        tokens = torch.argmax(drafts + gumbel, dim=1).to(torch.int32)
        reject, keep_r = sv.make_reject_args(target, drafts if k else None, tokens if k else None, self.cu, self.host_cu, self.accepted, self.next_token,
                                             self.counters, philox_seed=self.seed, philox_step=self.step_index, kv_len=self.kv_len,
                                             new_kv_len=self.new_kv_len)
        sv.spec_reject_sample(reject, sv.alloc_workspace(sv.spec_verify_workspace_bytes(None, reject), self.device))
        self.kept = self.new_kv_len.cpu().numpy().astype(np.int32)
        self.step_index += 1
        return out

    def unshared_attention(self):
        """The last step's attention again, every request on its own: (output, seconds)."""
        out = self.torch.empty_like(self.q)
        attn, keep = sv.make_kv8_attn_args(self.q, self.k_cache, self.v_cache, self.kv_scale, self.table, self.kv_len, self.cu, out, self.host_len,
                                           self.host_cu, max_kv_len=self.max_kv_len, error_count=self.errors)
        workspace = sv.alloc_workspace(sv.spec_kv8_attn_workspace_bytes(attn), self.device)
        return out, self._timed(lambda: sv.spec_kv8_attn(attn, workspace))

    def hand_over(self, b):
        """Request b's own tokens as bf16 rows: (keys, values) [tokens, Hkv, d]."""
        n = int(self.kept[b]) - self.prompt
        out = [self.torch.empty((n, self.Hkv, self.d), dtype=self.torch.bfloat16, device=self.device) for _ in range(2)]
        cu = np.array([0, n], dtype=np.int32)
        args, keep = sv.make_kv8_read_args(out[0], out[1], self.k_cache, self.v_cache, self.kv_scale, self.table[b:b + 1], self._int32([self.prompt]),
                                           self._int32(cu), cu, error_count=self.errors)
        sv.spec_kv8_read(args)
        return out

    def cache_bytes(self, shared=True):
        """Bytes of the requests' tokens in the cache: 8-bit codes and two scales a token and KV head."""
        tokens = int((self.kept - self.prompt).sum()) + self.prompt * (self.G if shared else self.B)
        return tokens * self.Hkv * (2 * self.d + 8)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tenants", type=int, default=4)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--k", type=int, default=4)
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--kv", choices=["e4m3", "int8"], default="e4m3")
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        print("shared_prefix_loop: no GPU visible", file=sys.stderr)
        sys.exit(2)
    loop = SharedPrefixLoop(args.tenants, args.requests, args.prompt, k=args.k, steps=args.steps, kv=args.kv, timed=True)
    for _ in range(args.steps):
        out = loop.step()
    alone, alone_seconds = loop.unshared_attention()
    rows = loop.hand_over(0)[0].shape[0]
    counters = loop.counters.cpu().numpy()
    print(json.dumps({
        "tenants": args.tenants, "requests": loop.B, "prompt": args.prompt, "k": args.k, "steps": args.steps, "kv": args.kv,
        "tokens_kept": int(loop.kept.sum()), "accepted": int(counters[1]), "attempted": int(counters[2]), "emitted": int(counters[3]),
        "cache_bytes": loop.cache_bytes(), "cache_bytes_unshared": loop.cache_bytes(shared=False),
        "attention_us": 1e6 * float(np.median(loop.attention_seconds)), "attention_unshared_us": 1e6 * alone_seconds,
        "largest_difference": float((out.float() - alone.float()).abs().max()), "handed_over_tokens": rows, "errors": int(loop.errors.item()),
    }))


if __name__ == "__main__":
    main()
