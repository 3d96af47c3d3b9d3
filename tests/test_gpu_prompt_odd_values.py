"""Infinities in V as they are, and V scales of any size, in the attention of prompts."""
import numpy as np
import pytest

import prompt_reference as R
import test_gpu_prompt_attn as P

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tiles", "tokens"])
@pytest.mark.parametrize("q_len,kv_len,d", [([200, 3], [330, 400], 128), ([5], [300], 128), ([150, 9, 1], [150, 200, 129], 64), ([2], [4000], 64)])
def test_an_infinity_stays_one(q_len, kv_len, d, kind, out):
    """Rows that see +inf in a dim of V are +inf there whether their block sees the step whole or not, and -inf likewise; both, or a NaN: NaN."""
    print("case infinities", q_len, kv_len, d, kind, out, flush=True)
    rng = np.random.default_rng(71)
    Hq, Hkv = 8, 2
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    for b in range(len(q_len)):
        for t, dim, head, value in ((3, 5, 0, INF), (17, 60, 1, -INF), (90, 33, 0, NAN), (91, 1, 1, INF), (100, 1, 1, -INF), (kv_len[b] - 1, 40, 0, -INF), (64, 0, 0, INF)):
            cache.put(1, table[b, t // 16], head, t % 16, dim, value)
    want = P.reference(cache, q, table, kv_len, cu)
    assert np.isposinf(want[0]).any() and np.isneginf(want[0]).any() and np.isnan(want[0]).any()
    got, lse, _ = P.run(cache, q, table, kv_len, cu, out)
    P.check(got, lse, want, out, kind, d)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("power", [-60, 0, 60, 119])
@pytest.mark.parametrize("rows,workspace", [(3, 256), (3, None), (90, None)])
def test_small_weights_count_whatever_the_scale_of_v(rows, workspace, power, kind, out):
    """Every other 512 tokens hold one with 2^16 times the weight of each of the others, whose sum is about a hundredth of the whole.  V's scales: 2^power."""
    print("case scales", rows, workspace, power, kind, out, flush=True)
    rng = np.random.default_rng(72)
    n, d = 8192, 64
    cache = R.Cache(rng, n // 16, 1, d, kind)
    cells = R.cells(kind, d, 0)
    cache.pool[0][:] = 0
    cache.pool[0][:, 0, cells[:, 0]] = 1 if kind == "int8" else 0x38              # K is 1 in the first dim, and its scale the score
    cache.scale[:, :, 0] = 0.0
    code = cache.value[1] / cache.scale[:, :, 1].astype(np.float64)[..., None]
    cache.scale[:, :, 1] = 2.0 ** power
    cache.value[1] = np.round(code * 512) / 512 * 2.0 ** power
    high = np.arange(n // 16) % 64 < 2
    cache.scale[high, :, 0, 5] = 16 * np.log(2.0)
    q = np.zeros((rows, 1, d))
    q[:, :, 0] = 1.0
    table = np.arange(n // 16, dtype=np.int32)[None]
    got, lse, errors = P.run(cache, q, table, [n], R.prefix_sum([rows]), out, scale=1.0, workspace=workspace)
    weight = np.ones(n)
    weight.reshape(-1, 16)[high, 5] = np.exp(np.float64(np.float32(16 * np.log(2.0))))
    value = cache.value[1][:, 0].reshape(n, d)
    assert errors == 0
    most = np.abs(value).max()
    # fp32 output: sums of n / 16 pages in two terms and runs (2^-24 of the largest V each at worst), exponents of 11 known to 2^-24 x 8 of it;
    # fp16 weights below 2^-14 are off by 2^-25 (see the other tests); bf16: its own rounding and the weights', 2^-11
    for j in range(rows):
        see = n - rows + j + 1
        want = (weight[:see, None] * value[:see]).sum(0) / weight[:see].sum()
        limit = most * (2.0 ** -24 * 2 * 512 + 2.0 ** -20 + 2.0 ** -32 * n) if out == "f32" else 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * most
        assert (np.abs(got[j, 0] - want) <= limit).all(), np.abs(got[j, 0] - want).max() / most
        # (a reference that includes V's scale, up to 119 + 16, known to 2^-23 of itself)
        assert abs(lse[j, 0] - np.log(weight[:see].sum())) <= 2.0 ** -21 * (abs(power) + 40)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tiles", "tokens"])
@pytest.mark.parametrize("workspace", [None, 256], ids=["split", "whole"])
def test_odd_values_of_tokens_with_tiny_weights(workspace, kind, out):
    """The first 1000 tokens have weights of e^-200, below fp32's range, in chunks of their own where the tokens are split: an infinity or NaN of
    their V reaches the rows all the same (as itself or as NaN), and what else they hold counts nothing."""
    print("case tiny weights", workspace, kind, out, flush=True)
    rng = np.random.default_rng(73)
    q_len, kv_len, Hq, Hkv, d = [3], [8000], 8, 1, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    q = np.zeros((3, Hq, d))
    q[:, :, 0] = 1.0
    for page in range(nb):
        for slot in range(16):
            cache.put(0, page, 0, slot, 0, 0.0)
    for t in range(1000):
        cache.put(0, table[0, t // 16], 0, t % 16, 0, -200.0)
    cu = R.prefix_sum(q_len)
    plain = P.reference(cache, q, table, kv_len, cu, 1.0)
    for t, dim, value in ((10, 3, INF), (500, 77, -INF), (600, 90, NAN)):
        cache.put(1, table[0, t // 16], 0, t % 16, dim, value)
    got, lse, errors = P.run(cache, q, table, kv_len, cu, out, scale=1.0, workspace=workspace)
    odd = np.zeros(d, dtype=bool)
    odd[[3, 77, 90]] = True
    assert errors == 0 and not np.isfinite(got[..., odd]).any()
    assert not np.isposinf(got[..., 77]).any() and not np.isneginf(got[..., 3]).any() and np.isnan(got[..., 90]).all()
    P.check(got[..., ~odd], lse, (plain[0][..., ~odd], plain[1], plain[2][..., ~odd], plain[3], plain[4]), out, kind, d)
