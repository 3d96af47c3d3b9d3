"""The operators around prompts and bounded caches together: prompts by chunks, eviction, verification steps, against the definitions at each call."""
import numpy as np
import pytest

import prompt_reference as R
from paper_2406_14066_amd import spec_verify as sv
from paper_2406_14066_amd.prompt_loop import PromptLoop
from test_gpu_prompt_attn import check

pytestmark = pytest.mark.gpu


class Pools:
    """What a loop's pools hold now, in 64 bits."""

    def __init__(self, loop):
        kind = loop.kv if loop.kv != "bf16" else "tokens" if loop.layout == sv.KV_TOKEN_MAJOR else "tiles"
        self.kind, self.nb, self.Hkv, self.d = kind, loop.num_blocks, loop.Hkv, loop.d
        self.value = []
        for w, pool in enumerate((loop.k_cache, loop.v_cache)):
            flat = pool.float().cpu().numpy().astype(np.float64).reshape(self.nb, self.Hkv, -1)
            rows = flat[:, :, R.cells(kind, self.d, w)]
            if loop.kv_scale is not None:
                rows = rows * loop.kv_scale[:, :, w].cpu().numpy().astype(np.float64)[..., None]
            self.value.append(rows)

    def rows(self, w, pages, n):
        t = np.arange(n)
        return self.value[w][np.asarray(pages)[t // 16], :, t % 16]


def _check_rows(loop, before_kept, out, lse, raw, positions):
    """The rows of the last call: turned as the definition says, in the cache behind what was there, and their attention."""
    pools = Pools(loop)
    Hq, Hkv, d = loop.Hq, loop.Hkv, loop.d
    freq = loop.inv_freq.cpu().numpy()
    raw = raw.float().cpu().numpy()
    q = loop.q.float().cpu().numpy().astype(np.float64)
    want_q, size = R.norm_rope(raw[:, :Hq], loop.q_weight.cpu().numpy(), positions, freq, 1e-6, False)
    assert (np.abs(q - want_q) <= 2.0 ** -8 * np.abs(want_q) + 2.0 ** -16 * size).all()
    want_k, size_k = R.norm_rope(raw[:, Hq:Hq + Hkv], loop.k_weight.cpu().numpy(), positions, freq, 1e-6, False)
    for b in range(loop.B):
        lo, hi, n = loop.cu[b], loop.cu[b + 1], int(loop.host_len[b])
        if hi == lo:
            continue
        keys, values = (pools.rows(w, loop.table[b], n) for w in (0, 1))
        assert n - (hi - lo) == before_kept[b]
        # (8-bit rows: half a step of the row's largest value, e4m3's of the value itself or of its smallest normal number)
        for got, want, more in ((keys[before_kept[b]:], want_k[lo:hi], 2.0 ** -16 * size_k[lo:hi]), (values[before_kept[b]:], raw[lo:hi, Hq + Hkv:].astype(np.float64), 0.0)):
            most = np.abs(want).max(-1, keepdims=True) * 1.01
            step = {"bf16": 2.0 ** -8 * np.abs(want), "int8": most / 127 * 0.51 + 2.0 ** -8 * np.abs(want),
                    "e4m3": 2.0 ** -4 * 1.1 * np.abs(want) + most * 2.0 ** -17 + 2.0 ** -8 * np.abs(want)}[loop.kv]
            assert (np.abs(got - want) <= step + more).all()
        answer = R.attention(q[lo:hi], keys, values, n) + (np.full(hi - lo, n * np.abs(values).max()),)
        check(out[lo:hi].float().cpu().numpy(), lse[lo:hi].cpu().numpy(), answer, "bf16", pools.kind, d)
    return pools


CASES = [
    # (kv, layout, requests, prompt, chunk, budget, k, Hq, Hkv, d)
    ("bf16", sv.KV_MFMA, 3, (40, 210), 64, 90, 4, 8, 2, 128),
    ("bf16", sv.KV_TOKEN_MAJOR, 2, (30, 150), 200, 64, 0, 4, 4, 64),
    ("e4m3", sv.KV_MFMA, 3, (60, 190), 77, 100, 2, 4, 1, 64),
    ("int8", sv.KV_MFMA, 2, (100, 300), 128, 48, 8, 8, 2, 128),
]


@pytest.mark.parametrize("kv,layout,requests,prompt,chunk,budget,k,Hq,Hkv,d", CASES, ids=["tiles", "tokens", "e4m3", "int8"])
def test_prompts_eviction_and_steps(kv, layout, requests, prompt, chunk, budget, k, Hq, Hkv, d, monkeypatch):
    loop = PromptLoop(requests, prompt, budget=budget, chunk=chunk, window=9, first=3, recent=10, k=k, steps=5, Hq=Hq, Hkv=Hkv, d=d, V=256, kv=kv, layout=layout, seed=8)
    calls = []
    real = PromptLoop._forward

    def forward(self, counts, seconds):
        before = self.kept.copy()
        out, lse = real(self, counts, seconds)
        calls.append((before, _check_rows(self, before, out, lse, self.raw, self.positions)))
        return out, lse

    monkeypatch.setattr(PromptLoop, "_forward", forward)

    def check_weights(before, rows_of):
        """`before` plus what the given rows look at."""
        pools, got = Pools(loop), loop.weight.cpu().numpy()
        for b, (q, lse, n, m) in rows_of.items():
            want = R.token_weights(q, lse, pools.rows(0, loop.table[b], n), n)
            t = np.arange(n)
            if before is not None:
                want[:n - m] += before[loop.table[b][t // 16], :, t % 16].astype(np.float64)[:n - m]
            have = got[loop.table[b][t // 16], :, t % 16]
            assert (np.abs(have - want) <= 2.0 ** -13 * want + 1e-30).all()      # (exponents of up to some ten: 2^-20 each; up to 72 rows)

    def check_eviction():
        weight, table, lengths, pools = loop.weight.cpu().numpy(), loop.table.copy(), loop.kept.copy(), Pools(loop)
        kept, long = loop.evict()
        assert list(long) == list(np.nonzero(lengths > budget)[0])
        after, new_weight = Pools(loop), loop.weight.cpu().numpy()
        for i, b in enumerate(long):
            stay = R.choose(weight, table[b], int(lengths[b]), budget, loop.first, loop.recent, loop.num_blocks)
            got = kept[i].cpu().numpy()
            assert list(got[:budget]) == stay and (got[budget:] == -1).all() and loop.kept[b] == budget
            t = np.arange(budget)
            for w in (0, 1):
                np.testing.assert_array_equal(after.rows(w, loop.table[b], budget), pools.rows(w, table[b], int(lengths[b]))[stay])
            old_t = np.array(stay)
            np.testing.assert_array_equal(new_weight[loop.table[b][t // 16], :, t % 16], weight[table[b][old_t // 16], :, old_t % 16])
        used = [int(p) for b in range(loop.B) for p in loop.table[b, :loop.pages[b]]]
        assert len(set(used)) == len(used) and not set(used) & set(loop.free) and len(used) + len(loop.free) == loop.num_blocks

    out, lse = loop.take_prompts()
    assert (loop.kept == loop.prompt).all() and (loop.position == loop.prompt).all()
    assert (loop.weight.cpu().numpy() >= 0).all()
    check_eviction()
    for _ in range(4):
        before = loop.weight.cpu().numpy()
        out, lse = loop.step()
        q, ls = loop.q.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        check_weights(before, {b: (q[loop.cu[b]:loop.cu[b + 1]], ls[loop.cu[b]:loop.cu[b + 1]], int(loop.host_len[b]), k + 1) for b in range(loop.B)})
        check_eviction()
    assert (loop.kept <= budget).all() and (loop.position >= loop.prompt + 4).all()
    assert int(loop.errors.item()) == 0 and loop.cache_bytes() <= loop.cache_bytes(bounded=False)


@pytest.mark.parametrize("kind,d", [("tiles", 128), ("tokens", 64), ("f32", 64)])
def test_prompts_enter_plain_caches(kind, d):
    """`spec_kv_append` with prompts of any length beside steps."""
    import torch
    rng = np.random.default_rng(9)
    q_len, kv_len, Hkv = [300, 1, 17, 1000, 9], [310, 40, 17, 1000, 100], 3
    table, nb = R.tables(rng, kv_len)
    cache = R.Cache(rng, nb, Hkv, d, kind)
    cu, lens = R.prefix_sum(q_len), np.array(kv_len, dtype=np.int32)
    new = [torch.from_numpy(rng.standard_normal((int(cu[-1]), Hkv, d)).astype(np.float32)).to(cache.type) for _ in range(2)]
    k, v, _ = cache.device()
    to = lambda x: torch.from_numpy(x).cuda()
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    sv.spec_kv_append(new[0].cuda(), new[1].cuda(), k, v, to(table), to(lens), to(cu), lens, cu, kv_layout=sv.KV_MFMA if kind == "tiles" else sv.KV_TOKEN_MAJOR,
                      error_count=errors)
    torch.cuda.synchronize()
    for w, (pool, rows) in enumerate(zip((k, v), new)):
        want = cache.pool[w].copy()
        bits = rows.view(torch.int32 if kind == "f32" else torch.int16).numpy()
        at = R.cells(kind, d, w)
        for b in range(len(q_len)):
            for j in range(q_len[b]):
                pos = kv_len[b] - q_len[b] + j
                want[table[b, pos // 16]][:, at[pos % 16]] = bits[cu[b] + j]
        got = pool.view(torch.int32 if kind == "f32" else torch.int16).cpu().numpy().reshape(want.shape)
        assert (got == want).all()
    assert int(errors.item()) == 0
