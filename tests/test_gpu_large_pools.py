"""Pools of more than 4 GiB: pages whose byte offsets do not fit 32 bits give what the same pages of a small pool give, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_kv8 import _bf16
from test_gpu_prefix_attn import _batch, _cache

pytestmark = pytest.mark.gpu

BYTES = (4 << 30) + (1 << 28)


def _large(small, at):
    """A pool of BYTES with the small one's pages from page `at` on (`at` counted from the end)."""
    n = BYTES // (small[0].numel() * small.element_size())
    large = torch.empty((n,) + small.shape[1:], dtype=small.dtype, device="cuda")
    large[n - at:n - at + small.shape[0]] = small
    return large


@pytest.mark.parametrize("shared", [0, 1], ids=["whole", "shared"])
@pytest.mark.parametrize("kind", ["tiles", "tokens", "e4m3", "int8"])
def test_attention(kind, shared, tuning):
    tuning("SPEC_VERIFY_PREFIX_SHARED", shared)
    rng = np.random.default_rng(12)
    Hkv, d = 8, 128
    for groups in ([(96, [(3, 40), (3, 77)]), (0, [(2, 300)])], [(320, [(4, 20)] * 9)]):     # few rows, many rows
        _, kv_len, cu, cg, prefix, table, _, nb = _batch(rng, groups)
        k, v, scale = _cache(rng, nb, Hkv, d, kind).device()
        q = _bf16(rng.standard_normal((int(cu[-1]), 16, d)).astype(np.float32)).cuda()
        outs = []
        for big in (False, True):
            pools, shift = (k, v), 0
            if big:
                pools = (_large(k, nb), _large(v, nb))
                shift = pools[0].shape[0] - nb
            sc = scale
            if big and scale is not None:
                sc = torch.empty((pools[0].shape[0],) + scale.shape[1:], device="cuda")
                sc[shift:] = scale
            out = torch.zeros(q.shape, dtype=torch.float32, device="cuda")
            errors = torch.zeros(1, dtype=torch.int64, device="cuda")
            args, keep = sv.make_prefix_attn_args(
                q, pools[0], pools[1], torch.from_numpy(np.where(table >= 0, table + shift, table).astype(np.int32)).cuda(), torch.from_numpy(kv_len).cuda(),
                torch.from_numpy(cu).cuda(), torch.from_numpy(cg).cuda(), torch.from_numpy(prefix).cuda(), out, kv_len, cu, cg, prefix, kv_scale=sc,
                kv_layout=sv.KV_TOKEN_MAJOR if kind == "tokens" else sv.KV_MFMA, error_count=errors)
            ws = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(args))
            sv.spec_prefix_attn(args, ws)
            torch.cuda.synchronize()
            assert int(errors.item()) == 0
            outs.append(out)
        assert torch.equal(outs[0], outs[1]) and bool(outs[0].abs().sum() > 0)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_append_and_read(kind):
    rng = np.random.default_rng(13)
    Hkv, d, n = 8, 128, np.array([37, 5, 100])
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    kv_len = (n + np.array([3, 11, 0])).astype(np.int32)
    start = torch.from_numpy((kv_len - n).astype(np.int32)).cuda()
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn
    nb = BYTES // (Hkv * 16 * d)
    pools = sv.alloc_kv8_pools(nb, Hkv, d, dtype)
    table = (nb - 1 - rng.permutation(3 * 7).reshape(3, 7)).astype(np.int32)
    rows = torch.randn((int(cu[-1]), 2 * Hkv, d), device="cuda")
    out = [torch.zeros((int(cu[-1]), Hkv, d), device="cuda") for _ in range(4)]
    for pool, tab, to in ((pools, table, out[:2]), (sv.alloc_kv8_pools(21, Hkv, d, dtype), nb - 1 - table, out[2:])):
        td, cud = torch.from_numpy(tab.astype(np.int32)).cuda(), torch.from_numpy(cu).cuda()
        args, keep = sv.make_kv8_append_args(rows[:, :Hkv], rows[:, Hkv:], *pool, td, torch.from_numpy(kv_len).cuda(), cud, kv_len, cu)
        sv.spec_kv8_append(args)
        args, keep2 = sv.make_kv8_read_args(to[0], to[1], *pool, td, start, cud, cu)
        sv.spec_kv8_read(args)
        torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    assert float((out[0] - rows[:, :Hkv]).abs().max()) < 0.2
