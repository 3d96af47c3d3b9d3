"""What a bf16 output may differ by, as a whole, and partial results of a prefix over the number range."""
import numpy as np
import pytest
import torch

from paper_2406_14066_amd import spec_verify as sv
from test_gpu_cache_batches import _want
from test_gpu_prefix_attn import Bf16Cache, _batch, _bf16, _cache, _run

pytestmark = pytest.mark.gpu

KINDS = ["tiles", "tokens", "e4m3", "int8"]


@pytest.mark.parametrize("shared", [1, 0], ids=["shared", "whole"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("requests,d", [(20, 128), (20, 64), (3, 128), (3, 64)])
def test_a_bf16_output_is_as_exact_as_its_rounding(requests, d, kind, shared, tuning):
    """Many tokens cancel to small outputs: the error is relative to those.  Besides the output's rounding there are only weights of 11
    bits or more, a rounding of 2^-12 each beside 2^-9, which adds (1/8)^2 / 2 of it, and fp32's: together less than a twentieth."""
    tuning("SPEC_VERIFY_PREFIX_SHARED", shared)
    rng = np.random.default_rng(51)
    groups = [(3008, [(4, int(n)) for n in rng.integers(4, 120, requests)])]
    _, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, 2, d, kind)
    q = rng.standard_normal((int(cu[-1]), 8, d)).astype(np.float32)
    got, errors = _run(cache, q, table, kv_len, cu, cg, prefix, "bf16")
    want, _ = _want(cache, q, whole, kv_len, cu)
    assert errors == 0
    rounding = np.linalg.norm(torch.from_numpy(want).to(torch.bfloat16).double().numpy() - want)
    error = np.linalg.norm(got - want)
    assert error <= 1.05 * rounding, error / rounding


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
