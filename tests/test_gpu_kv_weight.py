"""The attention weight that cached tokens get from given rows, against the definition in 64 bits."""
import numpy as np
import pytest

import prompt_reference as R
from paper_2406_14066_amd import spec_verify as sv
from test_gpu_prompt_attn import _i32, bf16, reference

pytestmark = pytest.mark.gpu


def run(cache, q, lse, table, kv_len, cu, before=None, *, scale=0.0, bucket=0, host_kv=True, stride=0, in_place=False, args_only=False):
    """(weight pool, findings) of a call; the pool held 7 before, or `before` if in place."""
    import torch
    k, _, sc = cache.device()
    qd = bf16(q).cuda()
    if stride:
        wide = torch.full((q.shape[0], q.shape[1] + stride, q.shape[2]), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :q.shape[1]] = qd
        qd = wide[:, :q.shape[1]]
    weight = sv.alloc_kv_weight(cache.nb, cache.Hkv).fill_(7.0)
    given = None if before is None else torch.from_numpy(before).cuda()
    if in_place:
        weight.copy_(given)
        given = weight
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    hk = np.asarray(kv_len, dtype=np.int32)
    args, keep = sv.make_kv_weight_args(qd, torch.from_numpy(np.ascontiguousarray(lse, dtype=np.float32)).cuda(), k, _i32(table), _i32(hk), _i32(cu), weight,
                                        hk if host_kv else None, cu, weight_in=given, kv_scale=sc,
                                        kv_layout=sv.KV_TOKEN_MAJOR if cache.kind == "tokens" else sv.KV_MFMA, softmax_scale=scale, max_kv_len=bucket,
                                        error_count=errors)
    if args_only:
        return args, keep, weight, errors
    sv.spec_kv_weight(args)
    torch.cuda.synchronize()
    return weight.cpu().numpy(), int(errors.item())


def check(got, cache, q, lse, table, kv_len, cu, before, steep, scale=0.0, else_value=None):
    """A term's exponent is a score (a sum of d products) less the row's lse: a few steps of 2^-24 of either, 2^-22 for the exponential;
    a token's sum adds a step for each row in the worst order."""
    qv = bf16(q).float().numpy().astype(np.float64)
    lse = np.asarray(lse, dtype=np.float32).astype(np.float64)
    want = np.full(got.shape, 7.0) if else_value is None else else_value.astype(np.float64).copy()
    limit = np.zeros(got.shape)
    for b in range(len(cu) - 1):
        m, n = int(cu[b + 1] - cu[b]), int(kv_len[b])
        if m == 0:
            continue
        at = slice(cu[b], cu[b + 1])
        sums = R.token_weights(qv[at], lse[at], cache.rows(0, table[b], n), n, scale or None)
        finite = np.where(np.isfinite(lse[at]), np.abs(lse[at]), 0)
        off = (cache.d + 8) * 2.0 ** -24 * steep[at].max() + 2.0 ** -22 * (finite.max() + steep[at].max() + 4)
        for t in range(n):
            page, slot = table[b, t // 16], t % 16
            if not 0 <= page < cache.nb:
                continue
            old = before[page, :, slot].astype(np.float64) if before is not None and t < n - m else 0.0
            want[page, :, slot] = old + sums[t]
            limit[page, :, slot] = sums[t] * (off + m * q.shape[1] // cache.Hkv * 2.0 ** -24) + 2.0 ** -23 * want[page, :, slot] + 1e-30
    err = np.abs(got - want)
    assert (err <= limit).all(), "largest excess %.3g" % (err - limit).max()


CASES = [
    # (name, q_len, kv_len, Hq, Hkv, d, softmax scale)
    ("one_key", [1], [1], 4, 4, 128, 0.0),
    ("steps", [5, 1, 9, 3], [64, 65, 300, 3], 16, 2, 128, 0.0),
    ("window", [32, 32], [500, 40], 8, 1, 128, 0.0),
    ("prompts", [100, 257, 64], [100, 257, 64], 4, 2, 128, 0.0),
    ("d64", [70, 31], [150, 31], 6, 2, 64, 0.0),
    ("empty_rows", [3, 70, 0, 1, 2], [0, 2, 50, 0, 2], 8, 4, 128, 0.0),
    ("group_16", [20], [333], 16, 1, 64, 0.0),
    ("sharp", [40], [140], 4, 4, 128, 3.0),
    # tokens enough for wavefronts with tokens of their own: rows that all stay in LDS, for several groups of tokens, and more rows
    ("some_rows", [100, 37, 0, 128, 1], [1100, 1025, 40, 128, 33], 32, 16, 128, 0.0),
    ("some_rows_groups", [20, 40], [9000, 7533], 32, 16, 64, 0.0),
    ("many_rows", [300, 20, 129], [1100, 1025, 700], 32, 16, 64, 0.0),
    ("many_rows_d128", [520], [1101], 20, 20, 128, 0.0),
]


@pytest.mark.parametrize("kind", R.KINDS)
@pytest.mark.parametrize("name,q_len,kv_len,Hq,Hkv,d,scale", CASES, ids=[c[0] for c in CASES])
def test_matches_the_definition(name, q_len, kv_len, Hq, Hkv, d, scale, kind):
    print("case kv_weight", name, kind, flush=True)
    rng = np.random.default_rng(31)
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    _, lse, _, steep, _ = reference(cache, q, table, kv_len, cu, scale)
    before = rng.random((nb, Hkv, 16)).astype(np.float32)
    got, errors = run(cache, q, lse, table, kv_len, cu, scale=scale)
    check(got, cache, q, lse, table, kv_len, cu, None, steep, scale)
    assert errors == 0
    # weights of a row sum to one over the tokens it sees
    rows = sum(min(m, n) for m, n in zip(q_len, kv_len)) * Hq
    total = sum(got[table[b, t // 16], :, t % 16].astype(np.float64).sum() for b in range(len(q_len)) if q_len[b] for t in range(kv_len[b]))
    assert abs(total - rows) <= 1e-4 * rows
    more, _ = run(cache, q, lse, table, kv_len, cu, before, scale=scale, stride=2)
    check(more, cache, q, lse, table, kv_len, cu, before, steep, scale)
    again, _ = run(cache, q, lse, table, kv_len, cu, before, scale=scale, in_place=True)
    check(again, cache, q, lse, table, kv_len, cu, before, steep, scale, else_value=before)


def test_rows_without_a_finite_lse_count_nothing():
    rng = np.random.default_rng(32)
    q_len, kv_len, Hq, Hkv, d = [50], [90], 4, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((50, Hq, d))
    page, slot = table[0, 4], 6                  # token 70 of KV head 1: rows from 30 on are NaN
    cache.put(0, page, 1, slot, 5, float("nan"))
    _, lse, _, steep, _ = reference(cache, q, table, kv_len, cu)
    assert np.isnan(lse[30:, 2:]).all() and not np.isnan(lse[:30]).any()
    lse[7, 1], lse[8, 0] = np.inf, -np.inf
    got, _ = run(cache, q, lse, table, kv_len, cu)
    steep = np.where(np.isfinite(steep), steep, 0)
    assert np.isfinite(got[table[0]]).all()
    check(got, cache, q, lse, table, kv_len, cu, None, steep)


def test_findings_and_a_bucket():
    import torch
    rng = np.random.default_rng(33)
    q_len, kv_len, Hq, Hkv, d, bound = [4, 3, 2], [50, 64, 200], 4, 2, 64, 208
    table, nb = R.tables(rng, kv_len, columns=13)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    table[2, 5], table[2, 12] = nb, -3
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((9, Hq, d))
    _, lse, _, steep, _ = reference(cache, q, table, kv_len, cu)
    args, keep, weight, errors = run(cache, q, lse, table, kv_len, cu, bucket=bound, host_kv=False, args_only=True)
    device_len = [t for t in keep if hasattr(t, "is_cuda") and tuple(t.shape) == (3,)][0]
    device_len.copy_(_i32([50, bound + 1, 200]))
    sv.spec_kv_weight(args)
    torch.cuda.synchronize()
    got = weight.cpu().numpy()
    assert (got[table[1, :4]] == 7.0).all() and int(errors.item()) == 3
    check(got, cache, q, lse, table, [50, 0, 200], cu, None, steep)


def test_more_rows_than_planned_are_left_out_and_counted():
    """Few rows are planned for by the host's offsets; a request to which those in device memory give more than fit is left out."""
    import torch
    rng = np.random.default_rng(35)
    planned, q_len, kv_len, Hq, Hkv, d = [12, 12], [2, 22], [150, 200], 8, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((24, Hq, d))
    _, lse, _, steep, _ = reference(cache, q, table, kv_len, cu)
    args, keep, weight, errors = run(cache, q, lse, table, kv_len, R.prefix_sum(planned), args_only=True)
    device_cu = [t for t in keep if hasattr(t, "is_cuda") and tuple(t.shape) == (3,)][0]
    device_cu.copy_(_i32(cu))
    sv.spec_kv_weight(args)
    torch.cuda.synchronize()
    got = weight.cpu().numpy()
    assert (got[table[1]] == 7.0).all() and int(errors.item()) == 1
    check(got, cache, q[:2], lse[:2], table[:1], kv_len[:1], cu[:2], None, steep[:2])


def test_two_calls_at_once():
    """Two calls on two streams: as one after the other."""
    import torch
    rng = np.random.default_rng(36)
    calls = []
    for Hq, n in ((8, 9000), (16, 300)):
        q_len = [40]
        table, nb = R.tables(rng, [n])
        cache = R.Cache(rng, nb, 2, 128, "tiles")
        q, cu = rng.standard_normal((40, Hq, 128)), R.prefix_sum(q_len)
        lse = reference(cache, q, table, [n], cu)[1]
        want, _ = run(cache, q, lse, table, [n], cu)
        calls.append((want,) + tuple(run(cache, q, lse, table, [n], cu, args_only=True)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for call in calls:
            call[3].fill_(7.0)
        torch.cuda.synchronize()
        for stream, call in zip(streams, calls):
            sv.spec_kv_weight(call[1], stream)
        torch.cuda.synchronize()
        for call in calls:
            assert (call[3].cpu().numpy() == call[0]).all()


def test_a_graph_and_repeats():
    import torch
    rng = np.random.default_rng(34)
    q_len, kv_len, Hq, Hkv, d = [5, 5], [400, 77], 8, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "e4m3")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((10, Hq, d))
    lse = reference(cache, q, table, kv_len, cu)[1]
    one, _ = run(cache, q, lse, table, kv_len, cu)
    args, keep, weight, errors = run(cache, q, lse, table, kv_len, cu, args_only=True)
    sv.spec_kv_weight(args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_kv_weight(args)
    for _ in range(3):
        weight.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert (weight.cpu().numpy() == one).all()
