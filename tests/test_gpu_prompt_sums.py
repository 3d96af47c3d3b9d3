"""Sums of very many nearly equal terms: softmax denominators over long contexts that are not split."""
import numpy as np
import pytest

import prompt_reference as R
import test_gpu_prompt_attn as P

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


def _one_large_key(rng, n, kind, d, scores):
    """A cache of n tokens in order whose keys are zero but token 0's, which a query of ones in dim 0 gives `scores`."""
    cache = R.Cache(rng, n // 16, 1, d, kind)
    cache.pool[0][:] = 0
    cache.value[0][:] = 0.0
    if kind in R.MOST:
        code = 1 if kind == "int8" else 0x38                    # the value 1
        cache.pool[0][0, 0, R.cells(kind, d, 0)[0, 0]] = code
        cache.scale[:, :, 0] = 1.0
        cache.scale[0, 0, 0, 0] = scores
        cache.value[0][0, 0, 0, 0] = np.float32(scores)
    else:
        cache.put(0, 0, 0, 0, 0, scores)
        cache.value[0][0, 0, 0, 0] = P.bf16([scores]).float().item()
    return cache, np.arange(n // 16, dtype=np.int32)[None]


@pytest.mark.parametrize("workspace", [256, None], ids=["whole", "planned"])
@pytest.mark.parametrize("n,scores,d", [(16384, 2.296875, 64), (65536, 1.203125, 128), (65536, 0.51171875, 64)])
@pytest.mark.parametrize("kind", R.KINDS)
def test_a_long_row_of_equal_keys(kind, n, scores, d, workspace):
    """All but the first of n tokens have e^-scores of its weight.

    A lane's weights of a step are summed in a few levels and the steps' sums with what each addition loses kept, so that neither lse nor the
    division has an error that grows with n: the allowance of the other tests holds.  The sums of weights times V are fp32 sums, a page (and a
    term of its weights, up to three) at a time: as the values differ, what their additions lose is a random walk, four times which is allowed."""
    print("case long row", kind, n, scores, d, workspace, flush=True)
    rng = np.random.default_rng(61)
    cache, table = _one_large_key(rng, n, kind, d, scores)
    q = np.zeros((3, 2, d))
    q[:, :, 0] = 1.0
    cu = R.prefix_sum([3])
    want = P.reference(cache, q, table, [n], cu, 1.0)
    got, lse, errors = P.run(cache, q, table, [n], cu, "f32", scale=1.0, workspace=workspace)
    assert errors == 0
    score = (d + 8) * STEP * want[3]
    assert (np.abs(lse - want[1]) <= score + 2.0 ** -22 * (np.abs(want[1]) + (20 if kind in R.MOST else 4))).all(), np.abs(lse - want[1]).max()
    sums = 4 * np.sqrt((2 if kind in R.MOST else 3) * n / 16) * STEP       # of the sum of weight * |V|
    limit = STEP * np.abs(want[0]) + want[2] * (2 * score[..., None] + 2.0 ** -20 + 2.0 ** -21 + 16 * STEP + sums)
    if kind in R.MOST:
        limit = limit + 2.0 ** -32 * want[4][:, None, None]
    err = np.abs(got - want[0])
    print("out off by %.2g of the sum of weights, lse by %.2g" % ((err / want[2]).max(), np.abs(lse - want[1]).max()), flush=True)
    assert (err <= limit).all(), (err / limit).max()
