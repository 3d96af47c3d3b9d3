"""Batches that fill the device, against 64-bit attention: they take the row tiles, splits and pieces that small ones do not (two and
three row tiles a block, split requests of several tiles, prefixes in many pieces, more than 64 groups)."""
import numpy as np
import pytest

import kv8_reference as R
from paper_2406_14066_amd import spec_verify as sv
from test_gpu_kv8 import Cache, _bf16, _run_attn, check
from test_gpu_prefix_attn import Bf16Cache, _batch, _cache, _run

pytestmark = pytest.mark.gpu

KINDS = ["tiles", "tokens", "e4m3", "int8"]


def _values(cache):
    """The cache's keys and values [num_blocks, Hkv, 16, d] in 64 bits."""
    if isinstance(cache, Bf16Cache):
        return [np.asarray(x, dtype=np.float64) for x in cache.values]
    table = np.array([R.code_value(c, cache.kv) for c in range(256)], dtype=np.float64)
    out = []
    for which in (0, 1):
        pool = np.asarray(cache.pools[which])
        nb, Hkv = pool.shape[:2]
        d = pool[0, 0].size // 16
        flat = table[pool.reshape(nb, Hkv, 16 * d)]
        where = np.array([[R.cell(slot, dim, which) for dim in range(d)] for slot in range(16)])
        out.append(flat[:, :, where] * np.asarray(cache.scales, dtype=np.float64).reshape(nb, Hkv, 2, 16)[:, :, which, :, None])
    return out


def _want(cache, q, table, kv_len, cu):
    import torch
    keys, values = (torch.from_numpy(x) for x in _values(cache))
    qv = _bf16(q).double()
    out, most = np.zeros(q.shape), 0.0
    for b in range(len(cu) - 1):
        n, m = int(kv_len[b]), int(cu[b + 1] - cu[b])
        pages = torch.from_numpy(table[b][:(n + 15) // 16].astype(np.int64))
        k, v = (x[pages].permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :n] for x in (keys, values))
        Hkv, d = k.shape[0], k.shape[2]
        rows = qv[cu[b]:cu[b + 1]].reshape(m, Hkv, -1, d).permute(1, 2, 0, 3)            # [Hkv, group, m, d]
        s = torch.matmul(rows, k[:, None].transpose(2, 3).contiguous()) / np.sqrt(d)
        seen = torch.arange(n)[None, :] <= (n - m + torch.arange(m))[:, None]
        w = torch.softmax(s.masked_fill(~seen, -np.inf), dim=-1)
        out[cu[b]:cu[b + 1]] = torch.matmul(w, v[:, None]).permute(2, 0, 1, 3).reshape(m, -1, d).numpy()
        most = max(most, float(v.abs().max()))
    return out, most


BATCHES = [
    # (name, requests, q_len, shortest, longest, Hq, Hkv, d)
    ("three_tiles", 48, 5, 20, 120, 64, 8, 128),
    ("two_tiles", 48, 4, 20, 120, 64, 8, 128),
    ("three_tiles_d64", 48, 9, 20, 120, 32, 8, 64),
    ("two_tiles_d64", 40, 7, 20, 120, 32, 8, 64),
    ("two_row_blocks", 12, 9, 300, 900, 40, 8, 128),
    ("two_tiles_split", 14, 7, 500, 1800, 32, 8, 128),
    ("three_tiles_split", 9, 5, 1200, 2600, 64, 8, 128),
    ("three_tiles_split_d64", 16, 5, 1000, 1600, 64, 8, 64),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("name,B,q_len,lo,hi,Hq,Hkv,d", BATCHES, ids=[b[0] for b in BATCHES])
def test_a_full_device(name, B, q_len, lo, hi, Hq, Hkv, d, kind, out):
    rng = np.random.default_rng(len(name))
    kv_len = rng.integers(lo, hi, B)
    _, kv_len, cu, _, _, table, _, nb = _batch(rng, [(0, [(q_len, int(n)) for n in kv_len])])
    cache = Cache(rng, nb, Hkv, d, kind)
    q = rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)
    got, errors = _run_attn(cache, q, table, kv_len, cu, out)
    want, most = _want(cache, q, table, kv_len, cu)
    assert errors == 0
    check(got, want, out, most)


GROUPS = [
    # (name, groups, requests of one, prefix, q_len, own tokens, Hq, Hkv, d)
    ("few_rows_three_tiles", 40, 2, 64, 3, 40, 32, 4, 128),
    ("few_rows_two_tiles_split", 24, 2, 2000, 2, 30, 32, 4, 128),
    ("few_rows_three_tiles_d64", 40, 2, 96, 5, 40, 16, 4, 64),
    ("many_groups_many_rows", 70, 3, 48, 3, 30, 32, 4, 128),
    ("sixteen_pieces", 3, 9, 5008, 4, 20, 16, 1, 128),
    ("thirteen_pieces", 1, 20, 4160, 5, 25, 32, 8, 128),
    ("pieces_d64", 2, 12, 3024, 6, 18, 16, 4, 64),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name,G,n,prefix,q_len,own,Hq,Hkv,d", GROUPS, ids=[g[0] for g in GROUPS])
def test_groups_that_fill_the_device(name, G, n, prefix, q_len, own, Hq, Hkv, d, kind, out):
    rng = np.random.default_rng(len(name))
    groups = [(max(prefix // 16 - int(rng.integers(0, 4)), 1) * 16, [(q_len, int(rng.integers(q_len, own))) for _ in range(n)]) for _ in range(G)]
    _, kv_len, cu, cg, lens, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, Hkv, d, kind)
    q = rng.standard_normal((int(cu[-1]), Hq, d)).astype(np.float32)
    got, errors = _run(cache, q, table, kv_len, cu, cg, lens, out)
    want, most = _want(cache, q, whole, kv_len, cu)
    assert errors == 0
    check(got, want, out, most, bf16_cache=kind in ("tiles", "tokens"))


@pytest.mark.parametrize("kind", ["tiles", "e4m3"])
def test_two_runs_agree_to_the_bit(kind):
    """Split requests are joined in chunk order whichever block comes last, and pieces in theirs."""
    rng = np.random.default_rng(3)
    groups = [(1600, [(4, int(n)) for n in rng.integers(4, 2500, 5)]), (320, [(2, 900), (5, 1700)])]
    _, kv_len, cu, cg, lens, table, whole, nb = _batch(rng, groups)
    cache = _cache(rng, nb, 2, 128, kind)
    q = rng.standard_normal((int(cu[-1]), 16, 128)).astype(np.float32)
    runs = [_run(cache, q, table, kv_len, cu, cg, lens, "f32")[0] for _ in range(3)]
    np.testing.assert_array_equal(runs[0], runs[1])
    np.testing.assert_array_equal(runs[0], runs[2])


def test_a_table_entry_outside_the_pool_reads_as_zeros_anywhere():
    """In pages that every row sees whole, too, and in a prefix."""
    rng = np.random.default_rng(4)
    groups = [(640, [(3, 700) for _ in range(8)])]
    _, kv_len, cu, cg, lens, table, whole, nb = _batch(rng, groups)
    for kind in KINDS:
        cache = _cache(rng, nb, 2, 128, kind)
        bad, bad_whole = table.copy(), whole.copy()
        bad[0, 7] = nb + 5
        bad[2, 44] = -3
        bad_whole[:, 7] = nb
        bad_whole[2, 44] = nb
        values = _values(cache)     # page nb: zeros
        zeros = [np.concatenate([x, np.zeros_like(x[:1])]) for x in values]
        q = rng.standard_normal((int(cu[-1]), 16, 128)).astype(np.float32)
        got, errors = _run(cache, q, bad, kv_len, cu, cg, lens, "f32")
        plain = Bf16Cache.__new__(Bf16Cache)
        plain.values = zeros
        want, most = _want(plain, q, bad_whole, kv_len, cu)
        assert errors == 2
        check(got, want, "f32", most)


@pytest.mark.parametrize("counts", ["alike", "ragged", "one_long", "mostly_empty"])
def test_append_finds_every_request_of_a_large_batch(counts):
    """More requests than lanes of a wavefront, alike and not: every row goes where its request's table says, and comes back."""
    import torch
    rng = np.random.default_rng(9)
    B, Hkv, d = 333, 2, 64
    n = {"alike": np.full(B, 5), "ragged": rng.integers(0, 40, B), "one_long": np.where(np.arange(B) == 200, 3000, 1),
         "mostly_empty": np.where(rng.random(B) < 0.03, 17, 0)}[counts]
    before = rng.integers(0, 50, B)
    kv_len = (before + n).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    pages = (kv_len + 15) // 16
    nb = int(pages.sum()) + 1
    order = rng.permutation(nb)[:int(pages.sum())]
    table = np.zeros((B, int(pages.max())), dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    rows = torch.randint(-127, 128, (int(cu[-1]), 2 * Hkv, d), device="cuda").float()
    rows[:, :, 0] = 127.0        # scale 1: every value comes back as it is
    k, v, scale = sv.alloc_kv8_pools(nb, Hkv, d, torch.int8)
    dev = [torch.from_numpy(x).cuda() for x in (table, kv_len, cu, before.astype(np.int32))]
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    args, keep = sv.make_kv8_append_args(rows[:, :Hkv], rows[:, Hkv:], k, v, scale, dev[0], dev[1], dev[2], kv_len, cu, error_count=errors)
    sv.spec_kv8_append(args)
    out = [torch.zeros((int(cu[-1]), Hkv, d), device="cuda") for _ in range(2)]
    args, keep2 = sv.make_kv8_read_args(out[0], out[1], k, v, scale, dev[0], dev[3], dev[2], cu, error_count=errors)
    sv.spec_kv8_read(args)
    torch.cuda.synchronize()
    assert torch.equal(out[0], rows[:, :Hkv]) and torch.equal(out[1], rows[:, Hkv:]) and int(errors.item()) == 0


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_codes_and_scales_are_those_of_fp32_tensor_arithmetic(kv):
    """Bit for bit, ties included: M / a and a / M are products with rounded reciprocals in both."""
    import torch
    T, Hkv, d = 16 * 512, 8, 128
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    x = torch.randn((T, Hkv, d), generator=gen, device="cuda")
    k, v, scale = sv.alloc_kv8_pools(T // 16, Hkv, d, torch.int8 if kv == "int8" else torch.float8_e4m3fn)
    table = torch.arange(T // 16, dtype=torch.int32, device="cuda")[None]
    cu = np.array([0, T], dtype=np.int32)
    cud = torch.from_numpy(cu).cuda()
    args, keep = sv.make_kv8_append_args(x, -x, k, v, scale, table, cud[1:], cud, cu[1:], cu)
    sv.spec_kv8_append(args)
    most = float(R.MOST[kv])
    a = x.abs().amax(-1)
    code = x * (most / a)[..., None]
    code = torch.round(code).to(torch.int8) if kv == "int8" else code.clamp(-most, most).to(torch.float8_e4m3fn).view(torch.int8)
    got = k.view(torch.int8).view(T // 16, Hkv, d // 16, 16, 16).permute(0, 3, 1, 2, 4).reshape(T, Hkv, d)
    assert torch.equal(got, code)
    assert torch.equal(scale[:, :, 0].permute(0, 2, 1).reshape(T, Hkv), a / most)
