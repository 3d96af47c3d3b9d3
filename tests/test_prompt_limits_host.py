"""Sizes that the 32-bit places in the kernels do not hold are refused before anything is launched."""
import ctypes as C

import pytest

from paper_2406_14066_amd import spec_verify as sv
from test_prompt_host import U, _call, _host, _prompt, _rope, _weight


@pytest.mark.parametrize("make", [_prompt, _weight])
@pytest.mark.parametrize("tokens", [2 ** 30 + 1, 2 ** 31 - 63, 2 ** 31 - 1])
@pytest.mark.parametrize("bucket", [True, False])
def test_contexts_beyond_2_30_tokens(make, tokens, bucket):
    a = make(kv_len=(60, 60), q_len=(1, 1))
    a.Hq = a.Hkv = 1
    a.max_blocks_per_req = 1 << 27
    if bucket:
        a.max_kv_len, a.host_kv_len = tokens, None
    else:
        _host("host_kv_len", [60, tokens])(a)
    if make is _prompt:
        assert sv.lib().spec_prompt_attn_workspace_bytes(C.byref(a)) == 0
    assert _call(a) == U


def test_the_longest_contexts_are_planned_for():
    a = _prompt(kv_len=(60, 60), q_len=(1, 1))
    a.max_blocks_per_req, a.max_kv_len, a.host_kv_len = 1 << 26, 2 ** 30, None
    assert sv.lib().spec_prompt_attn_workspace_bytes(C.byref(a)) > 256


@pytest.mark.parametrize("Hq,Hkv,d", [(1 << 24, 1, 128), (1, 1 << 24, 128), (1 << 25, 0, 64), ((1 << 23), 1 << 23, 128)])
def test_tokens_of_2_31_elements(Hq, Hkv, d):
    a = _rope()
    a.T, a.Hq, a.Hkv, a.d, a.rot_dim = 1, Hq, Hkv, d, 64
    assert _call(a) == U
