"""Row offsets in device memory that are not the ones planned with: requests whose prefix results are not there are left out and counted."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_cache_batches import _want
from test_gpu_kv8 import _bf16, check
from test_gpu_prefix_attn import _batch, _cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests", [2, 20], ids=["few_rows", "many_rows"])
@pytest.mark.parametrize("kind", ["tiles", "e4m3"])
def test_a_group_whose_end_is_not_valid(kind, requests, tuning):
    """The first group's end is past the last row: its prefix launch has no rows to take, so none of its requests has a result."""
    tuning("SPEC_VERIFY_PREFIX_SHARED", 1)
    rng = np.random.default_rng(61)
    groups = [(320, [(2, 20)] * requests), (640, [(2, 30)] * requests), (0, [(2, 50)])]
    _, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, 2, 128, kind)
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    bad = cu.copy()
    bad[requests] = cu[-1] + 5          # the last request of the first group, and the first of the second
    k, v, scale = cache.device()
    out = torch.full(q.shape, 7.0, device="cuda")
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    args, keep = sv.make_prefix_attn_args(
        _bf16(q).cuda(), k, v, torch.from_numpy(table).cuda(), torch.from_numpy(kv_len).cuda(), torch.from_numpy(bad).cuda(), torch.from_numpy(cg).cuda(),
        torch.from_numpy(prefix).cuda(), out, kv_len, cu, cg, prefix, kv_scale=scale, error_count=errors)
    ws = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(args))
    ws.fill_(0xA5)
    sv.spec_prefix_attn(args, ws)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert (got[:cu[2 * requests]] == 7.0).all()
    assert int(errors.item()) == 2 * requests
    want, most = _want(cache, q, whole, kv_len, cu)
    check(got[cu[2 * requests]:], want[cu[2 * requests]:], "f32", most)
