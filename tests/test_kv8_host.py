"""Refusals of the 8-bit cache's entry points and of the shared-prefix attention: host checks, nothing is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2406_14066_amd import spec_verify as sv

FAKE = 0x1000   # non-null, aligned, never dereferenced


def _append():
    a = sv.Kv8AppendArgs()
    hc, hk = np.array([0, 3, 5], dtype=np.int32), np.array([40, 20], dtype=np.int32)
    a.B, a.Hkv, a.d, a.num_blocks, a.max_blocks_per_req, a.T = 2, 2, 128, 16, 4, 5
    a.src_dtype, a.kv_dtype = sv.SPEC_BF16, sv.SPEC_E4M3
    for f in ("new_k", "new_v", "k_cache", "v_cache", "kv_scale", "block_table", "kv_len", "cu_q_len"):
        setattr(a, f, FAKE)
    a.host_kv_len, a.host_cu_q_len = hk.ctypes.data, hc.ctypes.data
    a._keep = (hk, hc)
    return a


def _read():
    a = sv.Kv8ReadArgs()
    hc = np.array([0, 30, 30, 35], dtype=np.int32)
    a.B, a.Hkv, a.d, a.num_blocks, a.max_blocks_per_req, a.T = 3, 2, 64, 16, 4, 35
    a.kv_dtype, a.out_dtype = sv.SPEC_INT8, sv.SPEC_F32
    for f in ("k_cache", "v_cache", "kv_scale", "block_table", "cu_len", "out_k", "out_v"):
        setattr(a, f, FAKE)
    a.host_cu_len = hc.ctypes.data
    a._keep = (hc,)
    return a


def _attn(prefix=False, kv_len=(60, 50, 20), q_len=(3, 2, 0), groups=(0, 2, 3), prefixes=(48, 0), bucket=0):
    a = sv.PrefixAttnArgs() if prefix else sv.Kv8AttnArgs()
    hk = np.array(kv_len, dtype=np.int32)
    hc = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    hg, hp = np.array(groups, dtype=np.int32), np.array(prefixes, dtype=np.int32)
    a.B, a.Hq, a.Hkv, a.d, a.num_blocks, a.max_blocks_per_req, a.T = len(kv_len), 8, 2, 128, 16, 4, int(hc[-1])
    a.kv_dtype, a.out_dtype, a.max_kv_len = sv.SPEC_E4M3, sv.SPEC_BF16, bucket
    for f in ("q", "k_cache", "v_cache", "kv_scale", "block_table", "kv_len", "cu_q_len", "out"):
        setattr(a, f, FAKE)
    a.host_kv_len, a.host_cu_q_len = hk.ctypes.data, hc.ctypes.data
    if prefix:
        a.G, a.kv_layout = len(prefixes), sv.KV_MFMA
        a.cu_group = a.prefix_len = FAKE
        a.host_cu_group, a.host_prefix_len = hg.ctypes.data, hp.ctypes.data
    a._keep = (hk, hc, hg, hp)
    return a


def _set(**kw):
    def go(a):
        for k, v in kw.items():
            setattr(a, k, v)
    return go


def _host(field, values):
    def go(a):
        x = np.array(values, dtype=np.int32)
        setattr(a, field, x.ctypes.data)
        a._keep += (x,)
    return go


@pytest.mark.parametrize("mutate,status", [
    (_set(new_k=None), sv.SPEC_EINVAL), (_set(kv_scale=None), sv.SPEC_EINVAL), (_set(host_cu_q_len=None), sv.SPEC_EINVAL),
    (_set(B=0), sv.SPEC_EINVAL), (_set(T=6), sv.SPEC_EINVAL), (_set(src_dtype=sv.SPEC_E4M3), sv.SPEC_EINVAL),
    (_set(kv_dtype=sv.SPEC_BF16), sv.SPEC_EINVAL), (_set(k_cache=FAKE + 16), sv.SPEC_EINVAL), (_set(new_v=FAKE + 8), sv.SPEC_EINVAL),
    (_set(token_stride=255), sv.SPEC_EINVAL), (_set(token_stride=260), sv.SPEC_EINVAL),      # shorter than a row; not 16-byte rows
    (_set(max_blocks_per_req=2), sv.SPEC_EINVAL), (_host("host_kv_len", [40, 1]), sv.SPEC_EINVAL),
    (_host("host_cu_q_len", [0, 6, 5]), sv.SPEC_EINVAL), (_host("host_cu_q_len", [1, 3, 5]), sv.SPEC_EINVAL),
    (_set(d=96), sv.SPEC_EUNSUPPORTED),
])
def test_append_refuses(mutate, status):
    a = _append()
    mutate(a)
    assert sv.lib().spec_kv8_append(C.byref(a), None) == status


@pytest.mark.parametrize("mutate,status", [
    (_set(out_v=None), sv.SPEC_EINVAL), (_set(cu_len=None), sv.SPEC_EINVAL), (_set(T=36), sv.SPEC_EINVAL),
    (_set(kv_dtype=sv.SPEC_F32), sv.SPEC_EINVAL), (_set(out_dtype=sv.SPEC_INT8), sv.SPEC_EINVAL), (_set(out_k=FAKE + 16), sv.SPEC_EINVAL),
    (_host("host_cu_len", [0, 30, 29, 35]), sv.SPEC_EINVAL), (_set(d=32), sv.SPEC_EUNSUPPORTED),
])
def test_read_refuses(mutate, status):
    a = _read()
    mutate(a)
    assert sv.lib().spec_kv8_read(C.byref(a), None) == status


ATTN = [
    (_set(q=None), sv.SPEC_EINVAL), (_set(out=None), sv.SPEC_EINVAL), (_set(host_kv_len=None), sv.SPEC_EINVAL),
    (_set(Hkv=3), sv.SPEC_EINVAL), (_set(T=6), sv.SPEC_EINVAL), (_set(kv_dtype=sv.SPEC_F32), sv.SPEC_EINVAL),
    (_set(out_dtype=sv.SPEC_E4M3), sv.SPEC_EINVAL), (_set(kv_scale=None), sv.SPEC_EINVAL), (_set(q=FAKE + 8), sv.SPEC_EINVAL),
    (_set(out=FAKE + 16), sv.SPEC_EINVAL), (_set(softmax_scale=-1.0), sv.SPEC_EINVAL), (_set(softmax_scale=float("nan")), sv.SPEC_EINVAL),
    (_set(softmax_scale=float("inf")), sv.SPEC_EINVAL), (_set(q_token_stride=1000), sv.SPEC_EINVAL), (_set(q_token_stride=1028), sv.SPEC_EINVAL),
    (_set(max_blocks_per_req=3), sv.SPEC_EINVAL), (_set(max_kv_len=65), sv.SPEC_EINVAL), (_set(max_kv_len=59), sv.SPEC_EINVAL),
    (_set(max_kv_len=-1), sv.SPEC_EINVAL), (_host("host_cu_q_len", [0, 10, 12, 5]), sv.SPEC_EINVAL),
    (_set(d=96), sv.SPEC_EUNSUPPORTED), (_set(Hq=34), sv.SPEC_EUNSUPPORTED),
]


@pytest.mark.parametrize("prefix", [False, True], ids=["kv8", "prefix"])
@pytest.mark.parametrize("mutate,status", ATTN)
def test_attention_refuses(mutate, status, prefix):
    a = _attn(prefix)
    name = "spec_prefix_attn" if prefix else "spec_kv8_attn"
    assert getattr(sv.lib(), name + "_workspace_bytes")(C.byref(a)) > 0
    mutate(a)
    assert getattr(sv.lib(), name + "_workspace_bytes")(C.byref(a)) == 0
    assert getattr(sv.lib(), name)(C.byref(a), FAKE, 1 << 40, None) == status


@pytest.mark.parametrize("prefix", [False, True], ids=["kv8", "prefix"])
def test_attention_limits(prefix):
    fn = "spec_prefix_attn" if prefix else "spec_kv8_attn"

    def ok(**kw):
        return getattr(sv.lib(), fn + "_workspace_bytes")(C.byref(_attn(prefix, **kw))) > 0

    assert ok(q_len=(9, 2, 0)) and not ok(q_len=(10, 2, 0))
    assert ok(bucket=64)
    assert not ok(kv_len=(60, 65, 20))                  # beyond the table's row
    if prefix:
        assert not ok(kv_len=(50, 50, 20))              # the first request's three rows do not all follow the prefix
    else:
        assert ok(kv_len=(2, 0, 0))                     # rows that see no key


@pytest.mark.parametrize("mutate", [
    _set(G=0), _set(G=4), _set(cu_group=None), _set(prefix_len=None), _set(host_cu_group=None), _set(host_prefix_len=None),
    _host("host_prefix_len", [47, 0]), _host("host_prefix_len", [-16, 0]), _host("host_prefix_len", [80, 0]),
    _host("host_prefix_len", [48, 80]), _host("host_cu_group", [0, 0, 3]), _host("host_cu_group", [0, 2, 2]),
    _set(kv_layout=sv.KV_TOKEN_MAJOR),                  # 8-bit pools have one layout
    _set(kv_dtype=sv.SPEC_BF16),                        # ... and bf16 pools no scales
])
def test_prefix_attention_refuses(mutate):
    a = _attn(True)
    mutate(a)
    assert sv.lib().spec_prefix_attn(C.byref(a), FAKE, 1 << 40, None) == sv.SPEC_EINVAL


@pytest.mark.parametrize("prefix", [False, True], ids=["kv8", "prefix"])
def test_workspace_is_checked(prefix):
    name = "spec_prefix_attn" if prefix else "spec_kv8_attn"
    a = _attn(prefix)
    need = getattr(sv.lib(), name + "_workspace_bytes")(C.byref(a))
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert getattr(sv.lib(), name)(C.byref(a), ws, size, None) == sv.SPEC_EWORKSPACE


def test_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    k, v, sc = sv.alloc_kv8_pools(4, 2, 64, torch.int8, device="cpu")
    rows, table = torch.zeros((3, 2, 64)), torch.zeros((1, 2), dtype=torch.int32)
    lens, cu = torch.tensor([3], dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)

    def make(new_k=rows, new_v=rows, k=k, v=v, sc=sc):
        return sv.make_kv8_append_args(new_k, new_v, k, v, sc, table, lens, cu, [3], [0, 3])

    make()
    make(torch.zeros((3, 7, 64))[:, 1:3], torch.zeros((3, 7, 64))[:, 3:5])      # slices of a projection
    with pytest.raises(TypeError):
        make(rows.half(), rows.half())
    with pytest.raises(TypeError):
        make(k=k.float(), v=v.float())
    for bad in (dict(new_k=rows[:, :1]), dict(new_v=torch.zeros((3, 4, 64))[:, :2]), dict(new_k=torch.zeros((3, 64, 2)).transpose(1, 2)),
                dict(sc=sc[:3]), dict(sc=sc.double()), dict(v=v[:3])):
        with pytest.raises(ValueError):
            make(**bad)
