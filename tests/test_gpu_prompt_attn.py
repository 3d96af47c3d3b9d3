"""Attention of any number of rows per request over a paged cache, against the definition in 64 bits."""
import numpy as np
import pytest

import prompt_reference as R
from paper_2406_14066_amd import spec_verify as sv

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def _i32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def run(cache, q, table, kv_len, cu, out="bf16", *, scale=0.0, bucket=0, host_kv=True, stride=0, workspace=None, lse=True, num_blocks=None, fill=0xA5,
        args_only=False):
    """(out, lse, findings) of a call whose outputs held 7 before."""
    import torch
    k, v, sc = cache.device()
    T, Hq, d = q.shape
    qd = bf16(q).cuda()
    if stride:
        wide = torch.full((T, Hq + stride, d), NAN, dtype=torch.bfloat16, device="cuda")
        wide[:, :Hq] = qd
        qd = wide[:, :Hq]
    o = torch.full((T, Hq, d), 7.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    ls = torch.full((T, Hq), 7.0, device="cuda") if lse else None
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    hk = np.asarray(kv_len, dtype=np.int32)
    args, keep = sv.make_prompt_attn_args(qd, k, v, _i32(table), _i32(hk), _i32(cu), o, hk if host_kv else None, cu, lse=ls, kv_scale=sc,
                                          kv_layout=sv.KV_TOKEN_MAJOR if cache.kind == "tokens" else sv.KV_MFMA, softmax_scale=scale, max_kv_len=bucket,
                                          error_count=errors)
    need = sv.spec_prompt_attn_workspace_bytes(args)
    ws = sv.alloc_workspace(need if workspace is None else workspace)
    ws.fill_(fill)      # its contents need no initialisation
    if args_only:
        return args, keep, ws, o, ls, errors
    sv.spec_prompt_attn(args, ws)
    torch.cuda.synchronize()
    return o.float().cpu().numpy(), ls.cpu().numpy() if lse else None, int(errors.item())


def reference(cache, q, table, kv_len, cu, scale=0.0):
    """R.attention's answers, and each row's tokens times the largest |V|."""
    qv = bf16(q).float().numpy().astype(np.float64)
    T, Hq, d = q.shape
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, steep, far = np.full((T, Hq), -np.inf), np.zeros((T, Hq)), np.zeros(T)
    for b in range(len(cu) - 1):
        if cu[b + 1] > cu[b]:
            n = int(kv_len[b])
            at, values = slice(cu[b], cu[b + 1]), cache.rows(1, table[b], n)
            out[at], lse[at], size[at], steep[at] = R.attention(qv[at], cache.rows(0, table[b], n), values, n, scale or None)
            far[at] = n * np.abs(values[np.isfinite(values)]).max(initial=0.0)
    return out, lse, size, steep, far


def check(got, got_lse, want, out, kind, d):
    """A score is a sum of d products and a few steps of 2^-24 of it; weights and their sum are off by e^(2 x that), and by 2^-22 for each of
    the fp32 steps around the exponential.  Weights of bf16 outputs enter the product with 8 bits (bf16 pages: half a step is 2^-8 of each
    weight) or 11 (8-bit pages); of fp32 outputs with 22 or more.  The output is rounded once.
    lse is a reference and a logarithm, each known to 2^-23 of itself.  8-bit pages: both are further from it by the scales' logarithm (here at most 9, itself
    known to 2^-23) and 7.
    8-bit pages: fp16 weights below 2^-14 are multiples of 2^-24 and off by 2^-25.  The reference is at least 7 below the largest exponent, so the
    sum of w_t / v_t that divides is at least 2^7 / v of that token, and each token's code c is off by 2^-25 c v / 2^7 <= 2^-32 of the largest |V|."""
    value, lse, size, steep, far = want
    score = (d + 8) * 2.0 ** -24 * steep
    soft = 2 * score[..., None] + 2.0 ** -20
    if out == "bf16":
        limit = 2.0 ** -8 * np.abs(value) + size * (soft + (2.0 ** -8 if kind in ("tiles", "tokens") else 2.0 ** -11)) * (1 + 2.0 ** -8)
    else:
        limit = 2.0 ** -24 * np.abs(value) + size * (soft + 2.0 ** -21)
    if kind in R.MOST:
        limit = limit + 2.0 ** -32 * far[:, None, None]
    ok = np.isfinite(value)
    assert (np.isnan(got) == np.isnan(value)).all() and (np.isposinf(got) == np.isposinf(value)).all() and (np.isneginf(got) == np.isneginf(value)).all()
    err = np.abs(np.where(ok, got, 0) - np.where(ok, value, 0))
    allowed = np.where(ok & np.isfinite(limit), limit, np.inf)
    assert (err <= allowed).all(), "largest excess %.3g" % (err - allowed).max()
    if got_lse is None:
        return
    fine = np.isfinite(lse)
    assert (np.isneginf(got_lse) == np.isneginf(lse)).all() and (np.isnan(got_lse) == np.isnan(lse)).all()
    err = np.abs(np.where(fine, got_lse, 0) - np.where(fine, lse, 0))
    assert (err <= np.where(fine, score + 2.0 ** -22 * (np.abs(np.where(fine, lse, 0)) + (20 if kind in R.MOST else 4)), 0)).all(), "lse off by %.3g" % err.max()


CASES = [
    # (name, q_len, kv_len, Hq, Hkv, d, softmax scale)
    ("one_key", [1], [1], 4, 4, 128, 0.0),
    ("single_tokens", [1, 1, 1, 1], [15, 16, 17, 700], 8, 2, 128, 0.0),
    ("edges", [31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65], 2, 2, 128, 0.0),
    ("edges_behind", [127, 128, 129, 1], [130, 400, 129, 129], 4, 2, 128, 0.0),
    ("rows_255_257", [255, 256, 257], [255, 300, 257], 1, 1, 128, 0.0),
    ("d64", [5, 300, 70, 128], [5, 300, 333, 128], 6, 2, 64, 0.0),
    ("empty_rows", [3, 70, 0, 1, 2, 40], [0, 2, 0, 0, 2, 39], 8, 4, 128, 0.0),
    ("padded_slots", [0, 130, 0, 1, 0], [77, 140, 0, 5, 3], 4, 1, 64, 0.0),
    ("group_3", [100, 9], [150, 77], 9, 3, 128, 0.0),
    ("group_16", [40, 70], [300, 70], 16, 1, 64, 0.0),
    ("sharp", [60, 4], [200, 90], 4, 4, 128, 3.0),
    ("flat", [90], [200], 2, 1, 128, 1e-3),
    ("split", [3, 1], [5000, 1234], 8, 1, 128, 0.0),
    ("split_d64", [20, 2], [2600, 3000], 4, 2, 64, 0.5),
]


@pytest.mark.parametrize("kind", R.KINDS)
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("name,q_len,kv_len,Hq,Hkv,d,scale", CASES, ids=[c[0] for c in CASES])
def test_matches_the_definition(name, q_len, kv_len, Hq, Hkv, d, scale, out, kind):
    print("case prompt_attn", name, out, kind, flush=True)
    rng = np.random.default_rng(11)
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    want = reference(cache, q, table, kv_len, cu, scale)
    for stride in (0, 3):
        got, lse, errors = run(cache, q, table, kv_len, cu, out, scale=scale, stride=stride)
        check(got, lse, want, out, kind, d)
        assert errors == 0


@pytest.mark.parametrize("kind", ["tiles", "e4m3"])
def test_a_long_prompt(kind):
    """Whole, in two chunks behind each other, and its last row alone: rows of 3000 tokens, a few of them against the definition."""
    rng = np.random.default_rng(12)
    n, Hq, Hkv, d = 3001, 4, 1, 128
    table, nb = R.tables(rng, [n])
    cache = R.Cache(rng, nb, Hkv, d, kind)
    q = rng.standard_normal((n, Hq, d))
    whole, lse, _ = run(cache, q, table, [n], R.prefix_sum([n]))
    for rows in (slice(0, 70), slice(1470, 1540), slice(n - 70, n)):
        want = reference(cache, q[rows], table, [rows.stop], R.prefix_sum([rows.stop - rows.start]))
        check(whole[rows], lse[rows], want, "bf16", kind, d)
    cut = 1777
    parts = [run(cache, q[:cut], table, [cut], R.prefix_sum([cut])), run(cache, q[cut:], table, [n], R.prefix_sum([n - cut]))]
    got, got_lse = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
    want = reference(cache, q[cut - 40:cut + 40], table, [cut + 40], R.prefix_sum([80]))
    check(got[cut - 40:cut + 40], got_lse[cut - 40:cut + 40], want, "bf16", kind, d)
    # (rows that the two ways cut alike agree to a rounding of the output)
    assert np.abs(got - whole).max() <= 2.0 ** -6 * np.abs(whole).max()


@pytest.mark.parametrize("kind", R.KINDS)
def test_what_lies_behind_the_last_token_is_not_read_into_results(kind):
    """Slots past the end hold NaN (8-bit: codes and scales), and so do pages that no request has."""
    import torch
    rng = np.random.default_rng(13)
    q_len, kv_len, Hq, Hkv, d = [40, 7, 130], [41, 100, 130], 4, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    want = reference(cache, q, table, kv_len, cu)
    used = np.zeros((nb, 16), dtype=bool)
    for b, n in enumerate(kv_len):
        for t in range(n):
            used[table[b, t // 16], t % 16] = True
    odd = {1: 0x7F, 2: 0x7FC0}[cache.pool[0].dtype.itemsize]
    for w in range(2):
        at = R.cells(kind, d, w)
        for page, slot in zip(*np.nonzero(~used)):
            cache.pool[w][page][:, at[slot]] = odd
            if cache.scale is not None:
                cache.scale[page, :, w, slot] = np.nan
    for out in ("bf16", "f32"):
        got, lse, _ = run(cache, q, table, kv_len, cu, out)
        check(got, lse, want, out, kind, d)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tiles", "tokens"])
def test_odd_values_reach_the_rows_that_see_them(kind, out):
    """An infinity or a NaN of a token's K or V: rows before the token are as without it."""
    rng = np.random.default_rng(14)
    q_len, kv_len, Hq, Hkv, d = [150, 200], [170, 200], 4, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))

    def place(b, t):
        return table[b, t // 16], t % 16

    for b, t, dim, head, value in ((0, 100, 5, 0, INF), (0, 101, 5, 0, -INF), (0, 60, 77, 1, NAN), (1, 199, 3, 0, NAN), (1, 64, 127, 1, -INF), (1, 65, 0, 1, INF)):
        page, slot = place(b, t)
        cache.put(1, page, head, slot, dim, value)
    page, slot = place(1, 120)
    cache.put(0, page, 1, slot, 9, NAN)
    want = reference(cache, q, table, kv_len, cu)
    assert np.isnan(want[0]).any() and np.isposinf(want[0]).any() and np.isneginf(want[0]).any()
    got, lse, _ = run(cache, q, table, kv_len, cu, out)
    value = want[0]
    # a weight in several terms may have a zero or a negative one, which makes NaN of an infinity: not finite all the same
    if out == "f32":
        odd = np.isinf(value) & np.isnan(got)
        value = np.where(odd, np.nan, value)
    check(got, lse, (value,) + want[1:], out, kind, d)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_rows_that_could_not_be_quantised(kind):
    """A scale of NaN (K's or V's) makes the rows that see the token NaN, and no others."""
    rng = np.random.default_rng(15)
    q_len, kv_len, Hq, Hkv, d = [90], [90], 2, 1, 128
    table, nb = R.tables(rng, kv_len)
    for w in (0, 1):
        cache = R.Cache(rng, nb, Hkv, d, kind)
        cu = R.prefix_sum(q_len)
        q = rng.standard_normal((90, Hq, d))
        page, slot = table[0, 70 // 16], 70 % 16
        cache.scale[page, 0, w, slot] = np.nan
        cache.pool[w][page, 0, R.cells(kind, d, w)[slot]] = 0
        cache.value[w][page, 0, slot] = np.nan
        want = reference(cache, q, table, kv_len, cu)
        got, _, _ = run(cache, q, table, kv_len, cu)
        check(got, None, want, "bf16", kind, d)
        assert np.isnan(got[70:]).all() and not np.isnan(got[:70]).any()


@pytest.mark.parametrize("kind", ["tiles", "int8"])
def test_a_bucket_serves_other_lengths_in_a_graph(kind):
    """One captured launch while the lengths change, with the program's own work between the replays; each replay against a call of its own."""
    import torch
    rng = np.random.default_rng(16)
    B, Hq, Hkv, d, bound = 3, 8, 2, 128, 2048
    q_len = [5, 1, 9]
    lens = [[700, 16, 2048], [5, 1, 9], [2048, 2047, 1025], [64, 2, 1000]]
    table, nb = R.tables(rng, [bound] * B)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    args, keep, ws, out, lse, errors = run(cache, q, table, lens[0], cu, "f32", bucket=bound, args_only=True)
    kv_len = [t for t in keep if hasattr(t, "shape") and tuple(t.shape) == (B,) and hasattr(t, "is_cuda")][0]
    sv.spec_prompt_attn(args, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_prompt_attn(args, ws)
    for n in lens:
        kv_len.copy_(_i32(n))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = reference(cache, q, table, n, cu)
        check(out.cpu().numpy(), lse.cpu().numpy(), want, "f32", kind, d)
        torch.randn(1000, device="cuda").sum()
    assert int(errors.item()) == 0


def test_two_graphs_share_a_workspace_and_two_streams_have_their_own():
    """Two captured calls with one workspace (both split tokens), replayed in turn on a stream; then both at once, a stream and a workspace each."""
    import torch
    rng = np.random.default_rng(23)
    calls = []
    for kind, q_len, kv_len, Hq, Hkv, d in (("tiles", [3, 1], [5000, 1234], 8, 1, 128), ("e4m3", [20, 2], [2600, 3000], 4, 2, 64)):
        table, nb = R.tables(rng, kv_len)
        cache = R.Cache(rng, nb, Hkv, d, kind)
        cu = R.prefix_sum(q_len)
        q = rng.standard_normal((int(cu[-1]), Hq, d))
        want = run(cache, q, table, kv_len, cu, "f32")
        assert want[2] == 0
        calls.append((want,) + tuple(run(cache, q, table, kv_len, cu, "f32", args_only=True)))
    shared = sv.alloc_workspace(max(sv.spec_prompt_attn_workspace_bytes(c[1]) for c in calls))
    assert shared.numel() > 256
    graphs = []
    for _, args, keep, ws, out, lse, errors in calls:
        sv.spec_prompt_attn(args, shared)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sv.spec_prompt_attn(args, shared)

    def clear():
        for c in calls:
            c[4].fill_(7.0)
            c[5].fill_(7.0)

    def same():
        torch.cuda.synchronize()
        for want, args, keep, ws, out, lse, errors in calls:
            assert (out.cpu().numpy() == want[0]).all() and (lse.cpu().numpy() == want[1]).all() and int(errors.item()) == 0

    for order in ((0, 1), (1, 0), (0, 1)):
        clear()
        for i in order:
            graphs[i].replay()
        same()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        clear()
        torch.cuda.synchronize()
        for stream, (want, args, keep, ws, out, lse, errors) in zip(streams, calls):
            sv.spec_prompt_attn(args, ws, stream)
        same()


def test_requests_that_do_not_fit_are_left_out_and_counted():
    import torch
    rng = np.random.default_rng(17)
    q_len, kv_len, Hq, Hkv, d, bound = [40, 3, 300, 2], [50, 64, 300, 16], 4, 2, 64, 304
    table, nb = R.tables(rng, kv_len, columns=19)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    want = reference(cache, q, table, kv_len, cu)
    args, keep, ws, out, lse, errors = run(cache, q, table, kv_len, cu, "f32", bucket=bound, host_kv=False, args_only=True)
    device_len = [t for t in keep if hasattr(t, "is_cuda") and tuple(t.shape) == (4,)][0]
    device_len.copy_(_i32([50, -1, bound + 1, 16]))
    sv.spec_prompt_attn(args, ws)
    torch.cuda.synchronize()
    got, got_lse = out.cpu().numpy(), lse.cpu().numpy()
    left_out = np.r_[cu[1]:cu[3]]
    assert (got[left_out] == 7.0).all() and (got_lse[left_out] == 7.0).all() and int(errors.item()) == 2
    rest = np.r_[0:cu[1], cu[3]:cu[4]]
    check(got[rest], got_lse[rest], tuple(w[rest] for w in want), "f32", "tiles", d)


@pytest.mark.parametrize("kind", R.KINDS)
def test_pages_outside_the_pool_read_as_zeros_and_are_counted(kind):
    rng = np.random.default_rng(18)
    q_len, kv_len, Hq, Hkv, d = [200, 2], [200, 3000], 8, 2, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    table[0, 3], table[0, 12], table[1, 100], table[1, 187] = nb, -1, nb + 12345, -2147483648
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    want = reference(cache, q, table, kv_len, cu)
    got, lse, errors = run(cache, q, table, kv_len, cu, "f32")
    check(got, lse, want, "f32", kind, d)
    assert errors == 4


def test_a_smaller_workspace_serves_and_results_repeat():
    import torch
    rng = np.random.default_rng(19)
    q_len, kv_len, Hq, Hkv, d = [4, 2], [6000, 3333], 8, 1, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    want = reference(cache, q, table, kv_len, cu)
    split = run(cache, q, table, kv_len, cu, "f32")
    again = run(cache, q, table, kv_len, cu, "f32", fill=0xFF)
    whole = run(cache, q, table, kv_len, cu, "f32", workspace=256)
    assert (split[0] == again[0]).all() and (split[1] == again[1]).all()
    assert not (split[0] == whole[0]).all()       # (the split changes the order of the sums)
    for got in (split, whole):
        check(got[0], got[1], want, "f32", "tiles", d)
    args, keep, ws, out, lse, errors = run(cache, q, table, kv_len, cu, args_only=True)
    with pytest.raises(sv.SpecVerifyError) as e:
        sv.spec_prompt_attn(args, torch.empty(128, dtype=torch.uint8, device="cuda"))
    assert e.value.status == sv.SPEC_EWORKSPACE


def test_without_lse_and_without_rows():
    import torch
    rng = np.random.default_rng(20)
    table, nb = R.tables(rng, [50, 20])
    cache = R.Cache(rng, nb, 2, 64, "tokens")
    q = rng.standard_normal((30, 4, 64))
    cu = R.prefix_sum([30, 0])
    want = reference(cache, q, table, [50, 20], cu)
    got, _, _ = run(cache, q, table, [50, 20], cu, lse=False)
    check(got, None, want, "bf16", "tokens", 64)
    args, keep, ws, out, lse, errors = run(cache, q[:0], table, [50, 20], R.prefix_sum([0, 0]), args_only=True)
    sv.spec_prompt_attn(args, ws)
    torch.cuda.synchronize()


def test_a_batch_that_fills_the_device():
    """Many requests of all lengths: every row block of the grid is found, with more than 64 requests and empty slots among them."""
    rng = np.random.default_rng(21)
    B, Hq, Hkv, d = 150, 4, 2, 64
    q_len = rng.integers(0, 150, B)
    q_len[rng.random(B) < 0.2] = 0
    kv_len = q_len + rng.integers(0, 60, B)
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    got, lse, errors = run(cache, q, table, kv_len, cu)
    check(got, lse, reference(cache, q, table, kv_len, cu), "bf16", "tiles", d)
    assert errors == 0


@pytest.mark.parametrize("kind,out", [("tiles", "f32"), ("e4m3", "bf16")])
def test_one_request_much_longer_than_the_others(kind, out):
    """On a device of 256 units its rows' tokens are cut in a whole chunk and a rest, which units without a block take."""
    rng = np.random.default_rng(24)
    q_len, kv_len, Hq, Hkv, d = [256, 250, 256, 256, 251, 255, 256], [1597, 1000, 1100, 1080, 900, 1100, 1050], 32, 8, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu = R.prefix_sum(q_len)
    q = rng.standard_normal((int(cu[-1]), Hq, d))
    got, lse, errors = run(cache, q, table, kv_len, cu, out)
    check(got, lse, reference(cache, q, table, kv_len, cu), out, kind, d)
    assert errors == 0


@pytest.mark.parametrize("scale", [1e3, 1e7])
def test_very_negative_scores(scale):
    """The softmax is that of the differences."""
    rng = np.random.default_rng(22)
    n, d = 100, 128
    table, nb = R.tables(rng, [n])
    cache = R.Cache(rng, nb, 1, d, "tiles")
    q = np.zeros((n, 1, d))
    q[:, 0, 0] = scale
    for t in range(n):
        page, slot = table[0, t // 16], t % 16
        cache.put(0, page, 0, slot, 0, -1.0 - (t % 7))
    want = reference(cache, q, table, [n], R.prefix_sum([n]), 1.0)
    got, lse, _ = run(cache, q, table, [n], R.prefix_sum([n]), "f32", scale=1.0)
    assert np.isfinite(got).all() and np.abs(got - want[0]).max() < 1e-4 * np.abs(want[0]).max()
    np.testing.assert_allclose(lse, want[1], rtol=1e-6)


def test_pools_of_more_than_4_gib():
    import torch
    rng = np.random.default_rng(23)
    q_len, kv_len, Hq, Hkv, d = [130, 3], [140, 700], 16, 8, 128
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    cu = R.prefix_sum(q_len)
    q = bf16(rng.standard_normal((int(cu[-1]), Hq, d))).cuda()
    k, v, _ = cache.device()
    outs = []
    for big in (False, True):
        pools, shift = [k, v], 0
        if big:
            total = ((4 << 30) + (1 << 28)) // (k[0].numel() * 2)
            shift = total - nb
            pools = []
            for small in (k, v):
                large = torch.empty((total,) + small.shape[1:], dtype=small.dtype, device="cuda")
                large[shift:] = small
                pools.append(large)
        out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
        args, keep = sv.make_prompt_attn_args(q, pools[0], pools[1], _i32(table + shift), _i32(kv_len), _i32(cu), out, kv_len, cu)
        sv.spec_prompt_attn(args, sv.alloc_workspace(sv.spec_prompt_attn_workspace_bytes(args)))
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
