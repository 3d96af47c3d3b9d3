"""Row offsets in device memory that do not fit the launch: the request is left out and counted, and nothing is written outside the arrays."""
import numpy as np
import pytest
import torch

import prompt_reference as R
import test_gpu_kv_weight as W
import test_gpu_prompt_attn as P
from paper_2406_14066_amd import spec_verify as sv

pytestmark = pytest.mark.gpu

ODD = [-(2 ** 31), -5, 2 ** 31 - 1, 1000]


def _left_out(cu, T):
    """Requests with rows that lie outside the packed ones."""
    return [b for b in range(len(cu) - 1) if cu[b] != cu[b + 1] and (cu[b] < 0 or cu[b + 1] < cu[b] or cu[b + 1] > T)]


def _batch(kind, d, q_len, kv_len):
    rng = np.random.default_rng(81)
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, 2, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), 8, d))
    return cache, table, cu, q


@pytest.mark.parametrize("at", [0, 2, 4])
@pytest.mark.parametrize("odd", ODD)
@pytest.mark.parametrize("out,workspace", [("f32", 256), ("bf16", None)])
def test_attention(out, workspace, odd, at):
    q_len, kv_len = [20, 50, 3, 40], [4000, 50, 30, 70]
    cache, table, cu, q = _batch("tiles", 128, q_len, kv_len)
    bad = cu.copy()
    bad[at] = odd
    T = int(cu[-1])
    args, keep, ws, o, lse, errors = P.run(cache, q, table, kv_len, cu, out, args_only=True)
    need = sv.spec_prompt_attn_workspace_bytes(args) if workspace is None else workspace
    wide = torch.full((3 * T, 8, 128), 7.0, dtype=o.dtype, device="cuda")
    args.out = wide[T:2 * T].data_ptr()
    space = sv.alloc_workspace(need + 8192)
    space.fill_(0x5A)
    [t for t in keep if hasattr(t, "is_cuda") and tuple(t.shape) == (5,)][0].copy_(torch.from_numpy(bad))
    sv.spec_prompt_attn(args, space[4096:4096 + need])
    torch.cuda.synchronize()
    assert bool((wide[:T] == 7.0).all()) and bool((wide[2 * T:] == 7.0).all())
    assert bool((space[:4096] == 0x5A).all()) and bool((space[4096 + need:] == 0x5A).all())
    assert int(errors.item()) == len(_left_out(bad, T)) > 0
    if at == 4:       # the requests before it are found as ever
        want = P.reference(cache, q, table, kv_len, cu)
        rest = slice(0, int(cu[3]))
        P.check(wide[T:2 * T][rest].float().cpu().numpy(), lse.cpu().numpy()[rest], tuple(w[rest] for w in want), out, "tiles", 128)
        assert bool((wide[T:2 * T][int(cu[3]):] == 7.0).all())


@pytest.mark.parametrize("at", [0, 2, 4])
@pytest.mark.parametrize("odd", ODD)
def test_weights(odd, at):
    q_len, kv_len = [20, 50, 3, 40], [200, 50, 30, 70]
    cache, table, cu, q = _batch("int8", 64, q_len, kv_len)
    bad = cu.copy()
    bad[at] = odd
    T = int(cu[-1])
    _, lse, _, steep, _ = P.reference(cache, q, table, kv_len, cu)
    args, keep, weight, errors = W.run(cache, q, lse, table, kv_len, cu, args_only=True)
    [t for t in keep if hasattr(t, "is_cuda") and tuple(t.shape) == (5,)][0].copy_(torch.from_numpy(bad))
    sv.spec_kv_weight(args)
    torch.cuda.synchronize()
    out = _left_out(bad, T)
    assert int(errors.item()) == len(out) > 0
    got = weight.cpu().numpy()
    for b in out:
        assert (got[table[b, :(kv_len[b] + 15) // 16]] == 7.0).all()


def test_requests_without_rows_are_none_of_them():
    """Slots without rows are no findings, wherever their offsets lie."""
    q_len, kv_len = [20, 0, 3], [200, 50, 30]
    cache, table, cu, q = _batch("tiles", 64, q_len, kv_len)
    got, lse, errors = P.run(cache, q, table, kv_len, cu)
    assert errors == 0
    _, errors = W.run(cache, q, lse, table, kv_len, cu)
    assert errors == 0
