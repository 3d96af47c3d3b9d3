"""The cache attention's workspace: it may hold anything when a call begins, also what other calls and other operators left in it."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_kv8 import Cache, _bf16, _table

pytestmark = pytest.mark.gpu


def _split_requests(rng, B, tokens, Hq, Hkv, d, kv="int8", q_len=2):
    """Requests of as many tokens as a block cannot walk alone, in the same pages: (a function of a workspace that gives the output,
    the workspace's size)."""
    kv_len = np.full(B, tokens, dtype=np.int32)
    cu = (np.arange(B + 1) * q_len).astype(np.int32)
    table, nb = _table(rng, kv_len[:1])
    k, v, sc = Cache(rng, nb, Hkv, d, kv).device()
    q = _bf16(rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)).cuda()
    out = torch.zeros(q.shape, device="cuda")
    dev = [torch.from_numpy(x).cuda() for x in (np.repeat(table, B, axis=0), kv_len, cu)]
    args, keep = sv.make_kv8_attn_args(q, k, v, sc, *dev, out, kv_len, cu)

    def run(ws):
        out.fill_(7.0)
        sv.spec_kv8_attn(args, ws)
        return out.clone()

    run.keep = (args, keep)
    return run, sv.spec_kv8_attn_workspace_bytes(args)


def test_numbers_that_partial_results_are_do_not_pass_for_tickets():
    """Every number from 2 on, in steps of an fp32 ulp: what a differently planned call may have left where the tickets are now."""
    rng = np.random.default_rng(41)
    run, need = _split_requests(rng, 64, 4200, 8, 8, 64)
    ws = sv.alloc_workspace(need).zero_()
    want = run(ws)
    assert bool((want != 7.0).any(-1).all())
    words, n = ws.view(torch.int64), 64 * 8     # as many tickets: one per (request, KV head)
    index = torch.arange(words.numel(), device="cuda") % n
    wrong = []
    for call in range(128):
        words.copy_(((0x40000000 + call * (n - 1) + index) << 32) | 0x3F800000)
        if not torch.equal(run(ws), want):
            wrong.append(call)
    assert wrong == []
