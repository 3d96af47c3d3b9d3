"""The operators of the 8-bit cache together: steps of requests behind shared prompts, against a cache kept in 64 bits beside them."""
import numpy as np
import pytest

import kv8_reference as R
from paper_2406_14066_amd import spec_verify as sv
from paper_2406_14066_amd.shared_prefix_loop import SharedPrefixLoop
from test_gpu_kv8 import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("tenants,requests,prompt,k,d,Hq,Hkv", [(2, 3, 96, 4, 128, 8, 2), (3, 2, 32, 0, 64, 4, 4), (1, 9, 272, 8, 64, 16, 2), (2, 2, 0, 2, 128, 4, 1)])
def test_steps_of_the_loop(tenants, requests, prompt, k, d, Hq, Hkv, kv, monkeypatch):
    # what enters the cache, quantised by the definition, by (table row, position)
    cache, appended = {}, []
    real = SharedPrefixLoop._append

    def append(self, counts, lengths, table):
        rows = real(self, counts, lengths, table)
        appended.append((np.asarray(counts), np.asarray(lengths), table.cpu().numpy(), rows.float().cpu().numpy()))
        return rows

    monkeypatch.setattr(SharedPrefixLoop, "_append", append)
    loop = SharedPrefixLoop(tenants, requests, prompt, question=(1, 30), k=k, steps=4, Hq=Hq, Hkv=Hkv, d=d, V=512, kv=kv, seed=5)

    def keep():
        for counts, lengths, table, rows in appended:
            at = 0
            for b, (n, length) in enumerate(zip(counts, lengths)):
                for pos in range(length - n, length):
                    for h in range(2 * Hkv):
                        codes, scale = R.quantise(rows[at, h], kv)
                        cache[(int(table[b, pos // 16]), pos % 16, h)] = np.array([R.code_value(c, kv) for c in codes]) * float(scale)
                    at += 1
        appended.clear()

    table = loop.table.cpu().numpy()
    own = lambda b, n, first=0: [np.array([[cache[(int(table[b, t // 16]), t % 16, w * Hkv + h)] for h in range(Hkv)] for t in range(first, n)]) for w in (0, 1)]
    for _ in range(4):
        before = loop.kept.copy()
        out = loop.step().float().cpu().numpy()
        keep()
        q = loop.q.double().cpu().numpy()
        want, most = np.zeros(q.shape), 0.0
        for b in range(loop.B):
            n = int(loop.host_len[b])
            keys, values = own(b, n)
            most = max(most, float(np.abs(values).max()))
            want[b * (k + 1):(b + 1) * (k + 1)] = R.attention(q[b * (k + 1):(b + 1) * (k + 1)], keys, values, n)
        check(out, want, "bf16", most)
        alone, _ = loop.unshared_attention()
        check(alone.float().cpu().numpy(), want, "bf16", most)
        accepted = loop.accepted.cpu().numpy()
        assert ((0 <= accepted) & (accepted <= k)).all()
        np.testing.assert_array_equal(loop.kept, before + 1 + accepted)
    for b in (0, loop.B - 1):
        got = loop.hand_over(b)
        for g, w in zip(got, own(b, int(loop.kept[b]), prompt)):
            # (bf16 of fp32 codes times scales)
            assert (np.abs(g.float().cpu().numpy() - w) <= 2.0 ** -8 * np.abs(w)).all()
    assert int(loop.errors.item()) == 0
    assert loop.cache_bytes() <= loop.cache_bytes(shared=False)
