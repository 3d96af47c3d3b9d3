"""The cache attention's workspace: it may hold anything when a call begins, also what other calls and other operators left in it."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from paper_2406_14066_amd import harness as H
from paper_2406_14066_amd import workloads as W
from test_gpu_kv8 import Cache, _bf16, _table
from test_gpu_prefix_attn import _batch, _cache

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


def _kv8(rng, lens, q_len=3, Hq=16, Hkv=2, d=64):
    """spec_kv8_attn of requests that share pages: (run(workspace) -> output, size, largest |v|)."""
    kv_len = np.asarray(lens, dtype=np.int32)
    B = len(kv_len)
    cu = (np.arange(B + 1) * q_len).astype(np.int32)
    table, nb = _table(rng, [int(kv_len.max())])
    cache = Cache(rng, nb, Hkv, d, "e4m3")
    k, v, sc = cache.device()
    q = _bf16(rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)).cuda()
    out = torch.zeros(q.shape, device="cuda")
    args, keep = sv.make_kv8_attn_args(q, k, v, sc, torch.from_numpy(np.repeat(table, B, axis=0)).cuda(), torch.from_numpy(kv_len).cuda(),
                                       torch.from_numpy(cu).cuda(), out, kv_len, cu)

    def run(ws):
        out.fill_(7.0)
        sv.spec_kv8_attn(args, ws)
        return out.clone()

    run.keep = (args, keep)
    return run, sv.spec_kv8_attn_workspace_bytes(args), 448 * float(cache.scales.max())


def _prefix(rng, kind, requests, prefix_len, own, q_len=3, Hq=16, Hkv=2, d=64):
    """The same of spec_prefix_attn: one group."""
    _, kv_len, cu, cg, prefix, table, _, nb = _batch(rng, [(prefix_len, [(q_len, own)] * requests)])
    cache = _cache(rng, nb, Hkv, d, kind)
    k, v, sc = cache.device()
    q = _bf16(rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)).cuda()
    out = torch.zeros(q.shape, device="cuda")
    args, keep = sv.make_prefix_attn_args(q, k, v, *(torch.from_numpy(x).cuda() for x in (table, kv_len, cu, cg, prefix)), out, kv_len, cu, cg, prefix,
                                          kv_scale=sc, kv_layout=sv.KV_TOKEN_MAJOR if kind == "tokens" else sv.KV_MFMA)

    def run(ws):
        out.fill_(7.0)
        sv.spec_prefix_attn(args, ws)
        return out.clone()

    run.keep = (args, keep)
    most = 448 * float(cache.scales.max()) if sc is not None else max(float(np.abs(x).max()) for x in cache.values)
    return run, sv.spec_prefix_attn_workspace_bytes(args), most


def _serves(size, run, need, most):
    """`run` on a workspace of `size` bytes gives what it gives on one of its own, and stays inside."""
    want = run(sv.alloc_workspace(need).fill_(0xA5))
    assert bool((want != 7.0).any(-1).all())
    space = sv.alloc_workspace(size + 8192).fill_(0x5A)
    got = run(space[4096:4096 + size])
    torch.cuda.synchronize()
    assert bool((space[:4096] == 0x5A).all()) and bool((space[4096 + size:] == 0x5A).all())
    assert float((got - want).abs().max()) <= 2 * 2e-5 * most        # (the bound of each against 64 bits)


def test_a_workspace_of_the_largest_batch_serves_smaller_ones():
    rng = np.random.default_rng(42)
    for large, small in (([1024] * 256, [1000] * 3), ([4096] * 64, [4090] * 2), ([9000] * 8, [9000]), ([9000] * 40, [8000, 20, 5000])):
        _, size, _ = _kv8(rng, large)
        run, need, most = _kv8(rng, small)
        _serves(size, run, need, most)
    run, need, _ = _kv8(rng, [9000])
    with pytest.raises(sv.SpecVerifyError):
        run(sv.alloc_workspace(256))


@pytest.mark.parametrize("kind", ["tiles", "tokens", "e4m3"])
@pytest.mark.parametrize("shared", [None, 1, 0])
def test_a_workspace_of_the_largest_batch_serves_smaller_ones_behind_a_prefix(shared, kind, tuning):
    if shared is not None:
        tuning("SPEC_VERIFY_PREFIX_SHARED", shared)
    rng = np.random.default_rng(43)
    for large, small in (((64, 4096, 300), (2, 4096, 300)), ((40, 4400, 700), (30, 4400, 650)), ((3, 9008, 40), (2, 8000, 20)),
                         ((64, 2048, 100), (1, 2000, 90))):
        _, size, _ = _prefix(rng, kind, *large)
        run, need, most = _prefix(rng, kind, *small)
        _serves(size, run, need, most)


def test_operators_and_plans_take_turns_on_one_workspace():
    """Splits of different sizes, prefixes, and a verification step's attention, one after the other, twice, without a wait between them."""
    rng = np.random.default_rng(44)
    jobs = [_kv8(rng, [9000] * 8), _kv8(rng, [700]), _prefix(rng, "tiles", 20, 4096, 300), _kv8(rng, [5000, 40, 8000]), _prefix(rng, "e4m3", 3, 9008, 40),
            _prefix(rng, "tokens", 64, 2048, 100), _kv8(rng, [4200] * 64)]
    w = W.make_workload("turns", B=4, Hq=8, Hkv=2, d=128, V=64, dtype="bf16", kv_len=[3000, 17, 900, 2500], k=[2] * 4, draft_std=3.0, sigma=0.8, data_seed=1,
                        philox_seed=2)
    step = H.DeviceStep(w, kv_layout=sv.KV_TOKEN_MAJOR)
    jobs.append((lambda ws: (sv.spec_verify_attn(step.attn_args, ws), step.out.clone())[1], sv.spec_verify_workspace_bytes(step.attn_args, None), 0.0))
    want = [run(sv.alloc_workspace(need)) for run, need, _ in jobs]
    shared = sv.alloc_workspace(max(need for _, need, _ in jobs))
    torch.cuda.synchronize()
    for order in (range(len(jobs)), reversed(range(len(jobs)))):
        order = list(order)
        got = [jobs[i][0](shared) for i in order]
        torch.cuda.synchronize()
        for i, x in zip(order, got):
            assert torch.equal(x, want[i]), i
