"""Sizes at the limits of the cache attention's 32-bit offsets: refused on the host, nothing is launched."""
import ctypes as C

import pytest

from paper_2406_14066_amd import spec_verify as sv
from test_kv8_host import FAKE, _attn


def _call(a, prefix):
    name = "spec_prefix_attn" if prefix else "spec_kv8_attn"
    return getattr(sv.lib(), name)(C.byref(a), FAKE << 20, 1 << 50, None)


@pytest.mark.parametrize("prefix", [False, True], ids=["kv8", "prefix"])
def test_partial_results_of_a_request_past_32_bits(prefix):
    """9 * 2048 rows, 128 dims, 512 chunks of 4096 tokens: 4.8 GB of one request's partial results, addressed with 32-bit offsets."""
    a = _attn(prefix, kv_len=(1 << 21, 50, 20), q_len=(9, 2, 0), prefixes=(0, 0))
    a.Hq, a.Hkv, a.max_blocks_per_req = 2048, 128, 1 << 17
    assert _call(a, prefix) == sv.SPEC_EUNSUPPORTED
