"""A step's token weights are those of the rows that verification leaves."""
import numpy as np
import pytest

import prompt_reference as R
from paper_2406_14066_amd import spec_verify as sv
from paper_2406_14066_amd.prompt_loop import PromptLoop
from test_gpu_prompt_loop import Pools

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,layout,k,Hq,Hkv,d", [("bf16", sv.KV_MFMA, 4, 8, 2, 128), ("bf16", sv.KV_TOKEN_MAJOR, 8, 4, 4, 64), ("int8", sv.KV_MFMA, 8, 8, 2, 128)])
def test_rejected_drafts_leave_no_weight(kv, layout, k, Hq, Hkv, d):
    loop = PromptLoop(4, (40, 120), budget=70, chunk=64, window=9, first=3, recent=10, k=k, steps=7, Hq=Hq, Hkv=Hkv, d=d, V=256, kv=kv, layout=layout, sigma=2.0,
                      seed=5, accepted_only=True)
    loop.take_prompts()
    loop.evict()
    rejected = 0
    for _ in range(6):
        before, kept = loop.weight.cpu().numpy(), loop.kept.copy()
        out, lse = loop.step()
        q, ls = loop.q.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        got, pools = loop.weight.cpu().numpy(), Pools(loop)
        for b in range(loop.B):
            n, m = int(loop.kept[b]), int(loop.kept[b] - kept[b])
            assert 1 <= m <= k + 1 and n - m == kept[b]
            rejected += k + 1 - m
            rows = slice(loop.cu[b], loop.cu[b] + m)
            want = R.token_weights(q[rows], ls[rows], pools.rows(0, loop.table[b], n), n)
            t = np.arange(n)
            want[:n - m] += before[loop.table[b][t // 16], :, t % 16].astype(np.float64)[:n - m]
            have = got[loop.table[b][t // 16], :, t % 16]
            assert (np.abs(have - want) <= 2.0 ** -13 * want + 1e-30).all()      # (exponents of up to some ten: 2^-20 each; up to 72 rows)
        loop.evict()
    assert rejected > 0 and int(loop.errors.item()) == 0


def test_all_rows_of_a_step_look_before_verification_otherwise():
    """Without the choice, rejected rows count: more weight than the rows that stay give."""
    sums = []
    for accepted_only in (False, True):
        loop = PromptLoop(3, (40, 90), budget=200, chunk=64, k=8, steps=2, Hq=4, Hkv=2, d=64, V=256, sigma=2.0, seed=6, accepted_only=accepted_only)
        loop.take_prompts()
        before = loop.weight.cpu().numpy().astype(np.float64).sum()
        loop.step()
        sums.append(loop.weight.cpu().numpy().astype(np.float64).sum() - before)
        stay = int((loop.kept - loop.prompt).sum())
    assert stay < 27
    # a row's weights sum to one over the tokens it sees, for each of its heads
    assert abs(sums[0] - 27 * 4) <= 1e-3 * 27 * 4 and abs(sums[1] - stay * 4) <= 1e-3 * 27 * 4
