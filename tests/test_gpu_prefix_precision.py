"""What a bf16 output may differ by, as a whole, and partial results of a prefix over the number range."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_cache_batches import _want
from test_gpu_prefix_attn import Bf16Cache, _batch, _bf16, _cache, _run

pytestmark = pytest.mark.gpu

KINDS = ["tiles", "tokens", "e4m3", "int8"]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["tiles", "tokens"])
def test_tokens_with_tiny_weights_and_the_only_values(kind, out, tuning):
    """V is zero in the prefix but for a few tokens, whose weights are 2^-124: the rows' own tokens are what counts."""
    tuning("SPEC_VERIFY_PREFIX_SHARED", 1)
    rng = np.random.default_rng(52)
    groups = [(4096, [(4, 20)] * 20)]
    _, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = Bf16Cache(rng, nb, 2, 128, kind)
    keys, values = cache.values
    keys[:] = 0.0
    shared = whole[0, :256]
    values[shared] = 0.0
    for page in shared[::8]:
        values[page, :, 11] = 1.0
        keys[page, :, 11, 0] = -86.0
    q = np.zeros((int(cu[-1]), 8, 128), dtype=np.float32)
    q[:, :, 0] = np.sqrt(128.0)
    got, errors = _run(cache, q, table, kv_len, cu, cg, prefix, out)
    want, _ = _want(cache, q, whole, kv_len, cu)
    assert errors == 0 and np.abs(want).max() > 1e-3
    # the output's rounding and the weights', 2^-8 and 2^-9 of what they multiply: up to 20 own values of up to 5, over 4096 tokens
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * 20 * 5 / 4096).all()
