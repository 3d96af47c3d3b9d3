"""The 8-bit KV cache on the GPU: quantising rows as they enter the pages, reading them back, and attention over
the pages, against the 64-bit reference."""
import numpy as np
import pytest

import kv8_reference as R
from paper_2406_14066_amd import spec_verify as sv

pytestmark = pytest.mark.gpu

KINDS = ["e4m3", "int8"]


def _torch_type(kv):
    import torch
    return torch.float8_e4m3fn if kv == "e4m3" else torch.int8


def _bytes(pool):
    import torch
    return pool.view(torch.uint8).cpu().numpy().reshape(pool.shape[0], pool.shape[1], -1)


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def _table(rng, lens, spare=3, columns=None):
    counts = [(n + 15) // 16 for n in lens]
    order = rng.permutation(sum(counts) + spare)
    table = np.zeros((len(lens), columns or max(max(counts), 1)), dtype=np.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


class Cache:
    """Pools filled with random codes and scales (every slot, also those that hold no visible token)."""

    def __init__(self, rng, nb, Hkv, d, kv):
        import torch
        self.kv, self.Hkv, self.d = kv, Hkv, d
        code = rng.integers(0, 256, size=(2, nb, Hkv, 16 * d)).astype(np.uint8)
        if kv == "e4m3":    # no NaN codes
            code[(code & 127) == 127] = 0x7E
        self.pools = [code[0], code[1]]
        self.scales = (rng.uniform(0.5, 2.0, size=(nb, Hkv, 2, 16)) / R.MOST[kv]).astype(np.float32)
        self.torch = torch

    def device(self):
        t = self.torch
        pools = [t.from_numpy(p.view(np.int8).reshape(p.shape[0], self.Hkv, 16, self.d).copy()).cuda().view(_torch_type(self.kv))
                 for p in self.pools]
        return pools[0], pools[1], t.from_numpy(self.scales.copy()).cuda()


APPENDS = [
    ("one_token", [1], [687], 8, 128, "bf16"),
    ("steps", [5, 3, 1, 9, 2], [37, 16, 1, 300, 129], 4, 128, "bf16"),
    ("steps_d64_f32", [4, 4, 4], [4, 20, 33], 3, 64, "f32"),
    ("prompts", [200, 0, 17, 33, 1], [200, 40, 32, 50, 16], 2, 128, "bf16"),
    ("prompts_f32", [77, 160], [90, 161], 5, 128, "f32"),
]


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("strided", [False, True], ids=["rows", "slices"])
@pytest.mark.parametrize("name,q_len,kv_len,Hkv,d,src", APPENDS, ids=[a[0] for a in APPENDS])
def test_append_writes_the_codes_and_nothing_else(name, q_len, kv_len, Hkv, d, src, strided, kv):
    import torch
    print("case kv8 append", name, kv, flush=True)
    rng = np.random.default_rng(7)
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    T = int(cu[-1])
    table, nb = _table(rng, kv_len)
    cache = Cache(rng, nb, Hkv, d, kv)
    rows = (rng.standard_normal((T, 2 * Hkv + 3, d)) * np.exp(rng.standard_normal((T, 2 * Hkv + 3, 1)))).astype(np.float32)
    rows[0, 3] = 0.0                              # a row of zeros
    if T > 1:
        rows[1, 3] *= np.float32(1e-25)           # smaller than the smallest scale is made for
        rows[T - 1, 4, 5] = np.inf
        rows[T // 2, 3 + Hkv, 0] = np.nan
    dev = torch.from_numpy(rows).cuda()
    dev = dev.to(torch.bfloat16) if src == "bf16" else dev
    new_k, new_v = dev[:, 3:3 + Hkv], dev[:, 3 + Hkv:]
    if not strided:
        new_k, new_v = new_k.contiguous(), new_v.contiguous()
    k, v, sc = cache.device()
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    hk = np.array(kv_len, dtype=np.int32)
    args, keep = sv.make_kv8_append_args(new_k, new_v, k, v, sc, torch.from_numpy(table).cuda(), torch.from_numpy(hk).cuda(),
                                         torch.from_numpy(cu).cuda(), hk, cu, error_count=errors)
    sv.spec_kv8_append(args)
    torch.cuda.synchronize()
    want_k, want_v, want_s = cache.pools[0].copy(), cache.pools[1].copy(), cache.scales.copy()
    assert R.append(new_k.float().cpu().numpy(), want_k, want_s, 0, table, kv_len, cu, kv) == 0
    assert R.append(new_v.float().cpu().numpy(), want_v, want_s, 1, table, kv_len, cu, kv) == 0
    np.testing.assert_array_equal(sc.cpu().numpy(), want_s)
    for got, want in ((k, want_k), (v, want_v)):
        got = _bytes(got)
        if kv == "e4m3":    # the two zeros are one value
            got, want = np.where(got == 128, 0, got), np.where(want == 128, 0, want)
        np.testing.assert_array_equal(got, want)
    assert int(errors.item()) == 0


def test_append_leaves_out_rows_that_do_not_fit():
    """Positions before the first token or past the table's row, and pages outside the pool, are counted and not written."""
    import torch
    rng = np.random.default_rng(8)
    q_len, kv_len, Hkv, d, kv = [5, 20, 3], [3, 40, 3], 2, 64, "int8"     # request 0: two rows before token 0
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table = np.array([[1, 2], [3, 9], [-1, 0]], dtype=np.int32)           # request 1 needs three columns; page 9 is none; page -1 neither
    cache = Cache(rng, 5, Hkv, d, kv)
    rows = rng.standard_normal((2, int(cu[-1]), Hkv, d)).astype(np.float32)
    k, v, sc = cache.device()
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    args, keep = sv.make_kv8_append_args(torch.from_numpy(rows[0]).cuda(), torch.from_numpy(rows[1]).cuda(), k, v, sc,
                                         torch.from_numpy(table).cuda(), torch.tensor(kv_len, dtype=torch.int32).cuda(),
                                         torch.from_numpy(cu).cuda(), None, cu, error_count=errors)
    sv.spec_kv8_append(args)
    torch.cuda.synchronize()
    want_k, want_v, want_s = cache.pools[0].copy(), cache.pools[1].copy(), cache.scales.copy()
    left_out = R.append(rows[0], want_k, want_s, 0, table, kv_len, cu, kv)
    assert left_out == R.append(rows[1], want_v, want_s, 1, table, kv_len, cu, kv) == 2 + 20 + 3
    np.testing.assert_array_equal(_bytes(k), want_k)
    np.testing.assert_array_equal(_bytes(v), want_v)
    np.testing.assert_array_equal(sc.cpu().numpy(), want_s)
    assert int(errors.item()) == left_out


@pytest.mark.parametrize("kv", KINDS)
def test_codes_are_within_half_a_step(kv):
    """What a row reads back as, against the row itself: half a step of the type, plus fp32's roundings (2^-22 relative)."""
    import torch
    rng = np.random.default_rng(9)
    T, Hkv, d = 40, 4, 128
    x = (rng.standard_normal((T, Hkv, d)) * np.exp(2 * rng.standard_normal((T, Hkv, 1)))).astype(np.float32)
    k, v, sc = sv.alloc_kv8_pools(4, Hkv, d, _torch_type(kv))
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32).cuda()
    cu = np.array([0, T], dtype=np.int32)
    dev, cud = torch.from_numpy(x).cuda(), torch.from_numpy(cu).cuda()
    args, keep = sv.make_kv8_append_args(dev, -dev, k, v, sc, table, cud[1:], cud, cu[1:], cu)
    sv.spec_kv8_append(args)
    out_k, out_v = torch.empty_like(dev), torch.empty_like(dev)
    args, keep2 = sv.make_kv8_read_args(out_k, out_v, k, v, sc, table, None, cud, cu)
    sv.spec_kv8_read(args)
    got = out_k.cpu().numpy().astype(np.float64)
    np.testing.assert_array_equal(out_v.cpu().numpy(), -out_k.cpu().numpy())
    scale = np.abs(x.astype(np.float64)).max(-1, keepdims=True) / R.MOST[kv]
    step = scale if kv == "int8" else scale * 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x / scale), 2.0 ** -6))) - 3)
    assert (np.abs(got - x) <= 0.5 * step * (1 + 1e-6) + np.abs(x) * 2.0 ** -22).all()


READS = [
    ("one", [1], [0], 8, 128), ("ragged", [37, 0, 16, 1, 200], [0, 5, 16, 31, 90], 3, 128), ("d64", [333, 15], [0, 17], 5, 64),
]


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,count,start,Hkv,d", READS, ids=[r[0] for r in READS])
def test_read_gives_the_values(name, count, start, Hkv, d, out, kv):
    import torch
    print("case kv8 read", name, out, kv, flush=True)
    rng = np.random.default_rng(10)
    lens = [a + n for a, n in zip(start, count)]
    table, nb = _table(rng, lens)
    cache = Cache(rng, nb, Hkv, d, kv)
    bad = len(lens) - 1
    if lens[bad] > 64:      # a page outside the pool in the middle of a range
        table[bad, 6] = nb + 4
    cu = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
    dtype = torch.float32 if out == "f32" else torch.bfloat16
    outs = [torch.full((int(cu[-1]) + 2, Hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    k, v, sc = cache.device()
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    args, keep = sv.make_kv8_read_args(outs[0][:int(cu[-1])], outs[1][:int(cu[-1])], k, v, sc, torch.from_numpy(table).cuda(),
                                       torch.tensor(start, dtype=torch.int32).cuda(), torch.from_numpy(cu).cuda(), cu, error_count=errors)
    sv.spec_kv8_read(args)
    torch.cuda.synchronize()
    for which in (0, 1):
        want = np.concatenate([R.read(cache.pools[which], cache.scales, which, table[b], start[b], count[b], kv) for b in range(len(count))])
        got = outs[which].float().cpu().numpy()
        assert (got[int(cu[-1]):] == 7.0).all()
        # code * scale rounded once: the same rounding here
        want = torch.from_numpy(want).float().to(dtype).float().numpy()
        np.testing.assert_array_equal(got[:int(cu[-1])], want)
    assert int(errors.item()) == (16 if (table[bad] == nb + 4).any() else 0)


# ------------------------------------------------------------------------------------------ attention
def bound(out, v_most, ref, bf16_cache=False):
    """Largest error of an output element.  fp32 output: 2e-5 of the largest |v| (scores of up to some ten in fp32, weights of
    22 bits or more).  bf16 output: its own rounding (2^-9 of the value) and that of the softmax weights (2^-9 as bf16, 2^-12 as
    fp16, of the largest |v|), each taken twice."""
    if out == "f32":
        return 2e-5 * v_most
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 if bf16_cache else 2.0 ** -11) * v_most


def check(got, want, out, v_most, bf16_cache=False):
    assert (np.isnan(got) == np.isnan(want)).all()
    ok = ~np.isnan(want)
    err = np.abs(np.where(ok, got, 0) - np.where(ok, want, 0))
    limit = bound(out, v_most, np.where(ok, want, 0), bf16_cache)
    assert (err <= limit).all(), "largest error %.3g, allowed there %.3g" % (err.max(), np.broadcast_to(limit, err.shape).flat[err.argmax()])


ATTNS = [
    # (name, q_len, kv_len, Hq, Hkv, d, softmax scale)
    ("one_key", [1], [1], 4, 4, 128, 0.0),
    ("edges", [1, 2, 3, 4, 5, 6, 7, 8, 9], [15, 16, 17, 31, 32, 33, 127, 128, 129], 8, 2, 128, 0.0),
    ("edges_d64", [9, 1, 4, 2], [9, 255, 256, 257], 6, 2, 64, 0.0),
    ("empty_rows", [3, 5, 0, 1, 2], [0, 2, 0, 0, 2], 8, 4, 128, 0.0),
    ("padded_slots", [0, 2, 0, 1], [77, 40, 0, 5], 4, 1, 64, 0.0),
    ("wide_group", [9, 8], [300, 1000], 32, 2, 128, 0.0),
    ("wide_group_d64", [9], [700], 16, 1, 64, 0.0),
    ("sharp", [4, 4], [600, 900], 8, 8, 128, 3.0),
    ("long", [2], [9001], 8, 1, 128, 0.0),
    ("long_d64", [5, 1], [6000, 20], 8, 2, 64, 0.5),
]


def _run_attn(cache, q, table, kv_len, cu, out_dtype, scale=0.0, max_kv_len=0, host_kv=True, stride=0):
    import torch
    k, v, sc = cache.device()
    T, Hq, d = q.shape
    qd = _bf16(q).cuda()
    if stride:
        wide = torch.full((T, Hq + stride, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :Hq] = qd
        qd = wide[:, :Hq]
    out = torch.full((T, Hq, d), 7.0, dtype=torch.float32 if out_dtype == "f32" else torch.bfloat16, device="cuda")
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    hk = np.asarray(kv_len, dtype=np.int32)
    args, keep = sv.make_kv8_attn_args(qd, k, v, sc, torch.from_numpy(table).cuda(), torch.from_numpy(hk).cuda(),
                                       torch.from_numpy(cu).cuda(), out, hk if host_kv else None, cu, softmax_scale=scale,
                                       max_kv_len=max_kv_len, error_count=errors)
    ws = sv.alloc_workspace(sv.spec_kv8_attn_workspace_bytes(args))
    ws.fill_(0xA5)      # its contents need no initialisation
    sv.spec_kv8_attn(args, ws)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), int(errors.item())


def _reference(cache, q, table, kv_len, cu, scale=0.0):
    import torch
    qv = _bf16(q).float().numpy().astype(np.float64)
    out = np.zeros(q.shape)
    most = 0.0
    for b in range(len(cu) - 1):
        n = int(kv_len[b])
        keys, values = (R.read(cache.pools[w], cache.scales, w, table[b], 0, n, cache.kv) for w in (0, 1))
        most = max(most, float(np.nanmax(np.abs(values), initial=0.0)))
        out[cu[b]:cu[b + 1]] = R.attention(qv[cu[b]:cu[b + 1]], keys, values, n, scale or None)
    return out, most


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,q_len,kv_len,Hq,Hkv,d,scale", ATTNS, ids=[a[0] for a in ATTNS])
def test_attention_matches_the_definition(name, q_len, kv_len, Hq, Hkv, d, scale, out, kv):
    print("case kv8 attn", name, out, kv, flush=True)
    rng = np.random.default_rng(11)
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table, nb = _table(rng, kv_len)
    cache = Cache(rng, nb, Hkv, d, kv)
    for b, n in enumerate(kv_len):      # slots past the end hold anything
        if n % 16:
            cache.scales[table[b, n // 16], :, :, n % 16:] = np.nan
            for which in (0, 1):
                for slot in range(n % 16, 16):
                    cache.pools[which][table[b, n // 16]][:, R.cell(slot, np.arange(d), which)] = 0x7F
    q = rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)
    want, most = _reference(cache, q, table, kv_len, cu, scale)
    got, errors = _run_attn(cache, q, table, kv_len, cu, out, scale, stride=3 if name == "edges" else 0)
    assert errors == 0
    check(got, want, out, most)
    for b in range(len(q_len)):         # rows before the first key
        hidden = max(min(q_len[b] - kv_len[b], q_len[b]), 0)
        assert (got[cu[b]:cu[b] + hidden] == 0).all()


@pytest.mark.parametrize("kv", KINDS)
def test_a_bucket_serves_other_lengths(kv):
    """The launch is planned from the bound alone; the lengths come from the device."""
    rng = np.random.default_rng(12)
    q_len, lens, bucket = [3, 3, 3], [5, 400, 2000], 2048
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table, nb = _table(rng, lens, columns=bucket // 16)
    cache = Cache(rng, nb, 2, 128, kv)
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    for kv_len in (lens, [0, 1, 3], [16, 257, 1999]):
        want, most = _reference(cache, q, table, kv_len, cu)
        got, errors = _run_attn(cache, q, table, kv_len, cu, "f32", max_kv_len=bucket, host_kv=False)
        assert errors == 0
        check(got, want, "f32", most)


def test_requests_that_do_not_fit_are_left_out_and_counted():
    rng = np.random.default_rng(13)
    q_len, lens, bucket = [2, 2, 2, 2], [300, 100, 50, 40], 320
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table, nb = _table(rng, lens, columns=bucket // 16)
    cache = Cache(rng, nb, 2, 64, "int8")
    q = rng.standard_normal((int(cu[-1]), 4, 64)).astype(np.float32)
    kv_len = [321, 100, -1, 40]
    table[3, 1] = -5            # reads as zeros: score 0, value 0
    got, errors = _run_attn(cache, q, table, kv_len, cu, "f32", max_kv_len=bucket, host_kv=False)
    assert (got[cu[0]:cu[1]] == 7.0).all() and (got[cu[2]:cu[3]] == 7.0).all()
    assert errors == 2 + 1
    want, most = _reference(cache, q, table, [0, 100, 0, 40], cu)
    check(got[cu[1]:cu[2]], want[cu[1]:cu[2]], "f32", most)
    check(got[cu[3]:cu[4]], want[cu[3]:cu[4]], "f32", most)


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_scales_of_any_size(kv, out):
    """Scales of neighbouring tokens that differ by many orders of magnitude, zeros among them (an unwritten page)."""
    rng = np.random.default_rng(14)
    q_len, kv_len = [4, 4], [100, 333]
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table, nb = _table(rng, kv_len)
    cache = Cache(rng, nb, 2, 128, kv)
    cache.scales[:, :, 1] *= np.exp(rng.uniform(-30, 30, size=cache.scales[:, :, 1].shape)).astype(np.float32)
    cache.scales[table[0, 2]] = 0.0
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    want, most = _reference(cache, q, table, kv_len, cu)
    got, errors = _run_attn(cache, q, table, kv_len, cu, out)
    check(got, want, out, most)
    # all of a request's values tiny: relative to those
    cache.scales[:, :, 1] = np.float32(2.0 ** -68)
    want, most = _reference(cache, q, table, kv_len, cu)
    got, errors = _run_attn(cache, q, table, kv_len, cu, out)
    check(got, want, out, most)


@pytest.mark.parametrize("kv", KINDS)
def test_rows_with_nan_reach_only_the_rows_that_see_them(kv):
    rng = np.random.default_rng(15)
    q_len, kv_len = [5, 5], [130, 37]
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    table, nb = _table(rng, kv_len)
    cache = Cache(rng, nb, 2, 128, kv)
    for b, n in enumerate(kv_len):      # the last two draft tokens are poisoned as an append of NaN leaves them
        for t in (n - 2, n - 1):
            cache.scales[table[b, t // 16], :, b, t % 16] = np.nan      # K's for request 0, V's for request 1
            cache.pools[b][table[b, t // 16]][:, R.cell(t % 16, np.arange(128), b)] = 0
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    want, most = _reference(cache, q, table, kv_len, cu)
    assert np.isnan(want[3:5]).all() and np.isfinite(want[:3]).all()
    for out in ("f32", "bf16"):
        got, errors = _run_attn(cache, q, table, kv_len, cu, out)
        check(got, want, out, most)


def test_replays_of_a_graph_and_another_stream():
    """A captured append and attention on a stream of their own, replayed with other lengths and rows in between eager work."""
    import torch
    rng = np.random.default_rng(16)
    B, q, Hq, Hkv, d, bucket = 6, 3, 16, 2, 128, 3008
    cu = (np.arange(B + 1) * q).astype(np.int32)
    lens = [2900, 1500, 700, 300, 40, 3]
    table, nb = _table(rng, [bucket] * B)
    k, v, sc = sv.alloc_kv8_pools(nb, Hkv, d, torch.float8_e4m3fn)
    fill = torch.randn((B * bucket, Hkv, d), device="cuda")
    cub = (np.arange(B + 1) * bucket).astype(np.int32)
    tb, cud = torch.from_numpy(table).cuda(), torch.from_numpy(cu).cuda()
    args, keep = sv.make_kv8_append_args(fill, fill * 0.5, k, v, sc, tb, torch.full((B,), bucket, dtype=torch.int32, device="cuda"),
                                         torch.from_numpy(cub).cuda(), None, cub)
    sv.spec_kv8_append(args)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    new = torch.randn((B * q, Hkv, d), device="cuda").to(torch.bfloat16)
    queries = torch.randn((B * q, Hq, d), device="cuda").to(torch.bfloat16)
    out = torch.zeros((B * q, Hq, d), device="cuda")
    app, keep1 = sv.make_kv8_append_args(new, new, k, v, sc, tb, kv_len, cud, None, cu)
    att, keep2 = sv.make_kv8_attn_args(queries, k, v, sc, tb, kv_len, cud, out, None, cu, max_kv_len=bucket)
    ws = sv.alloc_workspace(sv.spec_kv8_attn_workspace_bytes(att))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        sv.spec_kv8_append(app)
        sv.spec_kv8_attn(att, ws)
    for step in range(4):
        kv_len.copy_(torch.tensor([max(n - 7 * step, 3) for n in lens], dtype=torch.int32))
        new.copy_(torch.randn(new.shape, device="cuda"))
        queries.copy_(torch.randn(queries.shape, device="cuda"))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        with torch.cuda.stream(stream):
            sv.spec_kv8_append(app)
            sv.spec_kv8_attn(att, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(out.abs().sum() > 0)
