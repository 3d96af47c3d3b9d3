"""Attention of groups of requests that share a prefix, against the 64-bit reference over each request's whole context."""
import numpy as np
import pytest

import kv8_reference as R
from paper_2406_14066_amd import spec_verify as sv
from test_gpu_kv8 import Cache, _bf16, check

pytestmark = pytest.mark.gpu

KINDS = ["tiles", "tokens", "e4m3", "int8"]


class Bf16Cache:
    """bf16 pools: logical values [nb, Hkv, 16, d] in 64 bits, and their bytes in either layout."""

    def __init__(self, rng, nb, Hkv, d, layout):
        self.layout, self.Hkv, self.d = layout, Hkv, d
        self.values = [_bf16(rng.standard_normal((nb, Hkv, 16, d))).float().numpy() for _ in range(2)]

    def device(self):
        out = []
        for which, x in enumerate(self.values):
            nb, Hkv, _, d = x.shape
            if self.layout == "tiles" and which == 0:
                x = x.reshape(nb, Hkv, 16, d // 8, 8).transpose(0, 1, 3, 2, 4)
            elif self.layout == "tiles":
                x = x.reshape(nb, Hkv, 4, 4, d // 32, 2, 16).transpose(0, 1, 4, 2, 6, 5, 3)
            out.append(_bf16(np.ascontiguousarray(x).reshape(nb, Hkv, 16, d)).cuda())
        return out[0], out[1], None

    def read(self, which, pages, n):
        nb = self.values[which].shape[0]
        rows = [self.values[which][pages[t // 16], :, t % 16] if 0 <= pages[t // 16] < nb else np.zeros((self.Hkv, self.d)) for t in range(n)]
        return np.array(rows, dtype=np.float64).reshape(n, self.Hkv, self.d)


def _cache(rng, nb, Hkv, d, kind):
    return Cache(rng, nb, Hkv, d, kind) if kind in ("e4m3", "int8") else Bf16Cache(rng, nb, Hkv, d, kind)


def _tokens(cache, which, pages, n):
    if isinstance(cache, Bf16Cache):
        return cache.read(which, pages, n)
    return R.read(cache.pools[which], cache.scales, which, pages, 0, n, cache.kv)


def _batch(rng, groups, columns=None):
    """groups: (prefix_len, [(q_len, own tokens), ...]).  The table's prefix entries of all but a group's first request are not valid."""
    q_len = [q for _, rs in groups for q, _ in rs]
    kv_len = [p + n for p, rs in groups for _, n in rs]
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    cg = np.concatenate([[0], np.cumsum([len(rs) for _, rs in groups])]).astype(np.int32)
    prefix = np.array([p for p, _ in groups], dtype=np.int32)
    pages = sum(p // 16 + sum((n + 15) // 16 for _, n in rs) for p, rs in groups)
    order = rng.permutation(pages + 3)
    width = columns or max(max((n + 15) // 16 for n in kv_len), 1)
    table = np.full((len(q_len), width), -7, dtype=np.int32)
    whole = table.copy()        # with the prefix everywhere: what the reference walks
    at = b = 0
    for p, rs in groups:
        shared = order[at:at + p // 16]
        at += p // 16
        table[b, :p // 16] = shared
        for _, n in rs:
            whole[b, :p // 16] = shared
            mine = order[at:at + (n + 15) // 16]
            at += len(mine)
            table[b, p // 16:p // 16 + len(mine)] = whole[b, p // 16:p // 16 + len(mine)] = mine
            b += 1
    return q_len, np.array(kv_len, dtype=np.int32), cu, cg, prefix, table, whole, len(order)


def _run(cache, q, table, kv_len, cu, cg, prefix, out, *, scale=0.0, max_kv_len=0, host_kv=True, device_prefix=None, host_kv_len=None):
    import torch
    k, v, sc = cache.device()
    qd = _bf16(q).cuda()
    o = torch.full(q.shape, 7.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    layout = sv.KV_TOKEN_MAJOR if getattr(cache, "layout", "") == "tokens" else sv.KV_MFMA
    args, keep = sv.make_prefix_attn_args(
        qd, k, v, torch.from_numpy(table).cuda(), torch.from_numpy(kv_len).cuda(), torch.from_numpy(cu).cuda(), torch.from_numpy(cg).cuda(),
        torch.from_numpy(prefix if device_prefix is None else device_prefix).cuda(), o, (kv_len if host_kv_len is None else host_kv_len) if host_kv else None,
        cu, cg, prefix, kv_scale=sc, kv_layout=layout, softmax_scale=scale, max_kv_len=max_kv_len, error_count=errors)
    ws = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(args))
    ws.fill_(0xA5)
    sv.spec_prefix_attn(args, ws)
    torch.cuda.synchronize()
    return o.float().cpu().numpy(), int(errors.item())


def _reference(cache, q, whole, kv_len, cu, scale=0.0):
    qv = _bf16(q).float().numpy().astype(np.float64)
    out, most = np.zeros(q.shape), 0.0
    for b in range(len(cu) - 1):
        n = int(kv_len[b])
        keys, values = (_tokens(cache, w, whole[b], n) for w in (0, 1))
        most = max(most, float(np.max(np.abs(values[np.isfinite(values)]), initial=0.0)))
        out[cu[b]:cu[b + 1]] = R.attention(qv[cu[b]:cu[b + 1]], keys, values, n, scale or None)
    return out, most


CASES = [
    # (name, groups, Hq, Hkv, d, scale)
    ("two_requests", [(32, [(3, 5), (3, 20)])], 4, 2, 128, 0.0),
    ("single_page", [(16, [(1, 1), (1, 1), (1, 1)])], 2, 2, 64, 0.0),
    ("alone_and_without_prefix", [(48, [(2, 17)]), (0, [(3, 40), (1, 1)]), (160, [(9, 9), (1, 33), (4, 64)])], 8, 2, 128, 0.0),
    ("no_prefix_at_all", [(0, [(3, 40)]), (0, [(2, 7), (5, 100)])], 8, 4, 64, 0.0),
    ("padded_slots", [(64, [(0, 0), (2, 9), (0, 5)]), (32, [(0, 0)]), (16, [(0, 0), (1, 1)])], 4, 1, 128, 0.0),
    ("many_rows", [(208, [(9, 30)] * 7 + [(1, 1)])], 32, 2, 128, 0.0),
    ("many_rows_d64", [(336, [(5, 12)] * 9), (80, [(5, 5)] * 3)], 16, 2, 64, 0.0),
    ("sharp", [(320, [(4, 90)] * 5)], 8, 2, 128, 2.0),
    ("long_prefix", [(4400, [(3, 10), (3, 600)])], 8, 1, 128, 0.0),
    ("long_prefix_many_rows", [(2512, [(4, 4)] * 9), (16, [(4, 30)])], 16, 1, 128, 0.0),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,groups,Hq,Hkv,d,scale", CASES, ids=[c[0] for c in CASES])
def test_matches_the_definition(name, groups, Hq, Hkv, d, scale, out, kind):
    print("case prefix attn", name, out, kind, flush=True)
    rng = np.random.default_rng(21)
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, Hkv, d, kind)
    q = rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)
    want, most = _reference(cache, q, whole, kv_len, cu, scale)
    got, errors = _run(cache, q, table, kv_len, cu, cg, prefix, out, scale=scale)
    assert errors == 0
    check(got, want, out, most, kind in ("tiles", "tokens"))


@pytest.mark.parametrize("kind", KINDS)
def test_many_groups(kind):
    """More groups than lanes of a wavefront."""
    rng = np.random.default_rng(22)
    groups = [(16 * (g % 4), [(1 + g % 3, 1 + g % 3 + g % 20)] * (1 + g % 2)) for g in range(150)]
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, 2, 64, kind)
    q = rng.standard_normal((int(cu[-1]), 4, 64)).astype(np.float32)
    want, most = _reference(cache, q, whole, kv_len, cu)
    got, errors = _run(cache, q, table, kv_len, cu, cg, prefix, "f32")
    assert errors == 0
    check(got, want, "f32", most)


@pytest.mark.parametrize("kind", KINDS)
def test_a_bucket_serves_other_lengths(kind):
    rng = np.random.default_rng(23)
    groups = [(640, [(3, 5), (3, 900)]), (0, [(3, 1400)]), (1200, [(3, 3)] * 4)]
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups, columns=2048 // 16)
    cache = _cache(rng, nb, 2, 128, kind)
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    for less in (0, 3, 500):
        lens = np.maximum(kv_len - less, np.repeat(prefix, np.diff(cg)) + 3).astype(np.int32)
        want, most = _reference(cache, q, whole, lens, cu)
        got, errors = _run(cache, q, table, lens, cu, cg, prefix, "f32", max_kv_len=2048, host_kv=False)
        assert errors == 0
        check(got, want, "f32", most)


def test_what_does_not_fit_is_left_out_and_counted():
    rng = np.random.default_rng(24)
    groups = [(64, [(2, 20), (2, 30)]), (128, [(2, 5), (2, 9)]), (32, [(2, 40)])]
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups, columns=20)
    cache = _cache(rng, nb, 2, 128, "tiles")
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    lens = kv_len.copy()
    lens[1] = 65            # its own two rows do not both lie after the prefix
    bad_prefix = prefix.copy()
    bad_prefix[1] = 72      # not whole pages: the group is left out
    got, errors = _run(cache, q, table, lens, cu, cg, prefix, "f32", max_kv_len=300, host_kv=False, device_prefix=bad_prefix)
    assert (got[2:4] == 7.0).all() and (got[4:8] == 7.0).all()
    assert errors == 1 + 2
    want, most = _reference(cache, q, whole, kv_len, cu)
    check(got[:2], want[:2], "f32", most)
    check(got[8:], want[8:], "f32", most)


@pytest.mark.parametrize("kind", ["tiles", "tokens"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_infinities_and_nan_where_rows_do_not_see_them(kind, out):
    """Hidden draft tokens and slots past the end hold infinities and NaN; visible ones reach the rows that see them."""
    rng = np.random.default_rng(25)
    groups = [(64, [(5, 37), (5, 5), (4, 64)]), (0, [(3, 18)])]
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups)
    cache = Bf16Cache(rng, nb, 2, 128, kind)
    for b, n in enumerate(kv_len):
        if n % 16:
            for which in (0, 1):
                cache.values[which][whole[b, n // 16], :, n % 16:] = np.nan
        t = int(n) - 2          # seen by the last two rows
        cache.values[1][whole[b, t // 16], 0, t % 16, 7] = np.inf
        cache.values[1][whole[b, t // 16], 1, t % 16, 100] = np.nan
        t = int(n) - 1          # seen by the last row
        cache.values[0][whole[b, t // 16], 1, t % 16, 3] = np.nan
    q = rng.standard_normal((int(cu[-1]), 8, 128)).astype(np.float32)
    want, most = _reference(cache, q, whole, kv_len, cu)
    got, errors = _run(cache, q, table, kv_len, cu, cg, prefix, out)
    inf = np.isinf(want)
    assert inf.any() and (got[inf] == want[inf]).all()
    check(np.where(inf, 0, got), np.where(inf, 0, want), out, most, True)


@pytest.mark.parametrize("kind", KINDS)
def test_replays_of_a_graph(kind):
    import torch
    rng = np.random.default_rng(26)
    groups = [(1600, [(4, 900)] * 5), (160, [(4, 200)] * 2), (0, [(4, 1000)])]
    q_len, kv_len, cu, cg, prefix, table, whole, nb = _batch(rng, groups, columns=2560 // 16)
    cache = _cache(rng, nb, 2, 128, kind)
    k, v, sc = cache.device()
    q = torch.randn((int(cu[-1]), 16, 128), device="cuda").to(torch.bfloat16)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    kl = torch.from_numpy(kv_len).cuda()
    args, keep = sv.make_prefix_attn_args(q, k, v, torch.from_numpy(table).cuda(), kl, torch.from_numpy(cu).cuda(), torch.from_numpy(cg).cuda(),
                                          torch.from_numpy(prefix).cuda(), out, None, cu, cg, prefix, kv_scale=sc, max_kv_len=2560,
                                          kv_layout=sv.KV_TOKEN_MAJOR if kind == "tokens" else sv.KV_MFMA)
    ws = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(args))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sv.spec_prefix_attn(args, ws)
    for step in range(4):
        kl.copy_(torch.from_numpy(kv_len - 11 * step))
        q.copy_(torch.randn(q.shape, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        sv.spec_prefix_attn(args, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(out.float().abs().sum() > 0)
