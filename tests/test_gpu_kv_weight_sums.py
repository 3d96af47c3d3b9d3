"""A cached token's weight over very many rows: sums of nearly equal terms."""
import numpy as np
import pytest

import prompt_reference as R
import test_gpu_kv_weight as W

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


@pytest.mark.parametrize("rows,past,Hq,Hkv,d,value", [
    (12000, 40, 8, 1, 64, 2.296875),      # a block for each 32 tokens, four wavefronts share the rows
    (6000, 33, 32, 4, 64, 1.203125),      # 32 tokens for each wavefront
    (3000, 100, 32, 2, 128, 3.0),
])
@pytest.mark.parametrize("kind", ["tiles", "tokens", "int8"])
def test_a_token_that_all_of_many_rows_look_at_alike(kind, rows, past, Hq, Hkv, d, value):
    """Scores of zero and one lse: a token's weight is the number of (row, head) pairs that see it times e^-lse.

    A term's exponent is off by a few steps of 2^-24 of lse and 2^-22 for the exponential (the same for all terms); sixteen terms are summed in
    five levels, and tiles with what each addition loses kept: no part of the bound grows with the rows."""
    print("case many rows", kind, rows, past, Hq, Hkv, d, flush=True)
    rng = np.random.default_rng(62)
    n = past + rows
    table, nb = R.tables(rng, [n])
    cache = R.Cache(rng, nb, Hkv, d, kind)
    q = np.zeros((rows, Hq, d))
    lse = np.full((rows, Hq), value)
    got, errors = W.run(cache, q, lse, table, [n], R.prefix_sum([rows]))
    assert errors == 0
    t = np.arange(n)
    seen_by = np.minimum(n - t, rows) * (Hq // Hkv)
    want = seen_by * np.exp(-np.float64(np.float32(value)))
    have = got[table[0, t // 16], :, t % 16].astype(np.float64)
    err = np.abs(have / want[:, None] - 1).max()
    print("off by %.2g" % err, flush=True)
    assert err <= 2.0 ** -22 * (value + 4) + 16 * STEP


def test_weights_beyond_the_range_are_infinite():
    """Rows whose lse is far below their scores: a sum that overflows is an infinity, in few rows and in many."""
    rng = np.random.default_rng(63)
    for rows in (3, 300):
        table, nb = R.tables(rng, [400])
        cache = R.Cache(rng, nb, 1, 64, "tiles")
        lse = np.full((rows, 8), -70.0)
        lse[0] = -80.0
        lse[1, 0] = -100.0
        got, _ = W.run(cache, np.zeros((rows, 8, 64)), lse, table, [400], R.prefix_sum([rows]))
        t = np.arange(400 - rows + 2)
        assert np.isposinf(got[table[0, t // 16], :, t % 16]).all()
