"""Row offsets in device memory that are not prefix sums: they are found out before anything is addressed with them."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_cache_batches import _want
from test_gpu_kv8 import Cache, _bf16, check
from test_gpu_prefix_attn import _batch, _cache

pytestmark = pytest.mark.gpu

ODD = [-(2 ** 31), -5, 2 ** 31 - 1, 1000]
B, N, HKV, D = 4, 10, 2, 64


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("at", [0, 2, 4])
def test_append_and_read_stay_inside_their_arrays(at, odd):
    cu = (np.arange(B + 1) * N).astype(np.int32)
    bad = cu.copy()
    bad[at] = odd
    rng = np.random.default_rng(71)
    cache = Cache(rng, 2 * B, HKV, D, "int8")
    k, v, scale = cache.device()
    table = torch.arange(2 * B, dtype=torch.int32, device="cuda").reshape(B, 2)
    lens = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    rows = torch.randn((B * N, HKV, D), device="cuda")
    args, keep = sv.make_kv8_append_args(rows, rows, k, v, scale, table, lens, torch.from_numpy(bad).cuda(), None, cu)
    sv.spec_kv8_append(args)
    torch.cuda.synchronize()
    untouched = np.delete(np.arange(32), np.arange(10, 20))        # slots of a request's two pages: only tokens 10 .. 19 are new
    got = scale.cpu().numpy().transpose(0, 3, 1, 2).reshape(B, 32, HKV, 2)
    want = cache.scales.transpose(0, 3, 1, 2).reshape(B, 32, HKV, 2)
    np.testing.assert_array_equal(got[:, untouched], want[:, untouched])
    wide = [torch.full((3 * B * N, HKV, D), 7.0, device="cuda") for _ in range(2)]
    outs = [x[B * N:2 * B * N] for x in wide]
    args, keep2 = sv.make_kv8_read_args(outs[0], outs[1], k, v, scale, table, None, torch.from_numpy(bad).cuda(), cu)
    sv.spec_kv8_read(args)
    torch.cuda.synchronize()
    for x in wide:
        assert bool((x[:B * N] == 7.0).all()) and bool((x[2 * B * N:] == 7.0).all())


@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("groups", [1, 3, 80])
@pytest.mark.parametrize("requests", [2, 20], ids=["few_rows", "many_rows"])
@pytest.mark.parametrize("kind", ["tiles", "e4m3"])
def test_attention_stays_inside_its_arrays(kind, requests, groups, odd, tuning):
    """Nothing is written outside the output and the workspace; a request without a prefix, between valid offsets of its own, is right."""
    if groups * requests > 400:
        requests = 4
    tuning("SPEC_VERIFY_PREFIX_SHARED", 1)
    rng = np.random.default_rng(72)
    _, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, [(64, [(2, 20)] * requests)] * groups + [(0, [(2, 20)])])
    cache = _cache(rng, nb, 2, 128, kind)
    k, v, scale = cache.device()
    q = _bf16(rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)).cuda()
    bad = cu.copy()
    bad[cg[1]] = odd
    n = int(cu[-1])
    wide = torch.full((3 * n, 8, 128), 7.0, device="cuda")
    args, keep = sv.make_prefix_attn_args(
        q, k, v, torch.from_numpy(table).cuda(), torch.from_numpy(kv_len).cuda(), torch.from_numpy(bad).cuda(), torch.from_numpy(cg).cuda(),
        torch.from_numpy(prefix).cuda(), wide[n:2 * n], kv_len, cu, cg, prefix, kv_scale=scale)
    need = sv.spec_prefix_attn_workspace_bytes(args)
    space = sv.alloc_workspace(need + 8192)
    space.fill_(0x5A)
    sv.spec_prefix_attn(args, space[4096:4096 + need])
    torch.cuda.synchronize()
    assert bool((wide[:n] == 7.0).all()) and bool((wide[2 * n:] == 7.0).all())
    assert bool((space[:4096] == 0x5A).all()) and bool((space[4096 + need:] == 0x5A).all())
    want, most = _want(cache, q.float().cpu().numpy(), whole, kv_len, cu)
    got = wide[n:2 * n].cpu().numpy()
    last = slice(int(cu[-2]), n)                                    # the request without a prefix
    if groups == 1:                                                 # (it begins at the odd offset, and is left out)
        assert (got[last] == 7.0).all()
    else:
        check(got[last], want[last], "f32", most)
