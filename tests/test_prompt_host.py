"""Refusals of the entry points around prompts and bounded caches, and of their binding: host checks, nothing is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2406_14066_amd import spec_verify as sv

torch = pytest.importorskip("torch")

FAKE = 0x1000   # non-null, aligned, never dereferenced
WORKSPACE = 1 << 40


def _fake(a, *fields):
    for f in fields:
        setattr(a, f, FAKE)


def _rope():
    a = sv.QkNormRopeArgs()
    a.T, a.Hq, a.Hkv, a.d, a.dtype, a.weight_dtype, a.rot_dim = 5, 8, 2, 128, sv.SPEC_BF16, sv.SPEC_F32, 128
    _fake(a, "q", "k", "out_q", "out_k", "q_weight", "k_weight", "positions", "inv_freq")
    a.eps = 1e-6
    return a


def _rows(cls, kv_len=(60, 50, 20), q_len=(30, 2, 0), bucket=0):
    a = cls()
    hk, hc = np.array(kv_len, dtype=np.int32), np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    a.B, a.Hq, a.Hkv, a.d, a.num_blocks, a.max_blocks_per_req, a.T = len(kv_len), 8, 2, 128, 16, 4, int(hc[-1])
    a.kv_dtype, a.kv_layout, a.max_kv_len = sv.SPEC_E4M3, sv.KV_MFMA, bucket
    _fake(a, "q", "k_cache", "kv_scale", "block_table", "kv_len", "cu_q_len", "lse")
    a.host_kv_len, a.host_cu_q_len = hk.ctypes.data, hc.ctypes.data
    a._keep = (hk, hc)
    return a


def _prompt(**kw):
    a = _rows(sv.PromptAttnArgs, **kw)
    _fake(a, "v_cache", "out")
    a.out_dtype = sv.SPEC_BF16
    return a


def _weight(**kw):
    a = _rows(sv.KvWeightArgs, **kw)
    _fake(a, "weight", "weight_in")
    return a


def _evict():
    a = sv.KvEvictArgs()
    hk = np.array([60, 50], dtype=np.int32)
    a.B, a.Hkv, a.d, a.num_blocks, a.max_blocks_per_req, a.dst_max_blocks, a.first, a.recent = 2, 2, 128, 16, 4, 2, 4, 8
    a.kv_dtype, a.kv_layout = sv.SPEC_INT8, sv.KV_MFMA
    _fake(a, "k_cache", "v_cache", "kv_scale", "weight", "block_table", "kv_len", "keep", "kept")
    a.dst_block_table, a.new_kv_len = FAKE * 2, FAKE << 8
    a.host_kv_len = hk.ctypes.data
    a._keep = (hk,)
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


def _call(a, workspace=WORKSPACE, at=FAKE):
    L = sv.lib()
    if isinstance(a, sv.QkNormRopeArgs):
        return L.spec_qk_norm_rope(C.byref(a), None)
    if isinstance(a, sv.PromptAttnArgs):
        return L.spec_prompt_attn(C.byref(a), at, workspace, None)
    if isinstance(a, sv.KvWeightArgs):
        return L.spec_kv_weight(C.byref(a), None)
    return L.spec_kv_evict(C.byref(a), at, workspace, None)


E, U = sv.SPEC_EINVAL, sv.SPEC_EUNSUPPORTED


@pytest.mark.parametrize("mutate,status", [
    (_set(T=-1), E), (_set(Hq=0, Hkv=0), E), (_set(d=0), E), (_set(dtype=sv.SPEC_E4M3), E), (_set(weight_dtype=sv.SPEC_INT8), E), (_set(rot_dim=130), E),
    (_set(rot_dim=-16), E), (_set(interleaved=2), E), (_set(eps=-1e-6), E), (_set(eps=float("nan")), E), (_set(scale=float("inf")), E), (_set(q=None), E),
    (_set(out_k=None), E), (_set(positions=None), E), (_set(inv_freq=None), E), (_set(q=FAKE + 8), E), (_set(out_q=FAKE + 4), E), (_set(k_weight=FAKE + 2), E),
    (_set(q_stride=1023), E), (_set(q_stride=1028), E), (_set(out_k_stride=128), E), (_set(d=96, rot_dim=96), U), (_set(rot_dim=24), U),
    (_set(T=1 << 30), U), (_set(T=(1 << 25) + 1, Hq=1, Hkv=1), U),
    (_set(out_q_stride=1032), E), (_set(q_stride=2048), E), (_set(k_stride=1024), E), (_set(k_stride=1024, out_k_stride=1032), E),   # (in place, but other tokens apart)
])
def test_rope_refuses(mutate, status):
    a = _rope()
    mutate(a)
    assert _call(a) == status


ROWS = [
    (_set(B=0), E), (_set(Hq=7), E), (_set(Hkv=0), E), (_set(num_blocks=0), E), (_set(T=33), E), (_set(T=-1), E), (_set(q=None), E), (_set(k_cache=None), E),
    (_set(block_table=None), E), (_set(kv_len=None), E), (_set(cu_q_len=None), E), (_set(host_cu_q_len=None), E), (_set(kv_dtype=sv.SPEC_F32), E),
    (_set(kv_scale=None), E), (_set(kv_dtype=sv.SPEC_BF16), E), (_set(kv_layout=sv.KV_TOKEN_MAJOR), E), (_set(kv_layout=2, kv_dtype=sv.SPEC_BF16, kv_scale=None), E),
    (_set(k_cache=FAKE + 16), E), (_set(q=FAKE + 8), E), (_set(max_kv_len=-1), E), (_set(host_kv_len=None), E), (_set(max_kv_len=80), E), (_set(max_kv_len=59), E),
    (_host("host_kv_len", [60, -1, 0]), E), (_host("host_kv_len", [65, 50, 20]), E), (_host("host_cu_q_len", [0, 33, 32, 32]), E),
    (_host("host_cu_q_len", [1, 30, 32, 32]), E), (_set(softmax_scale=-1.0), E), (_set(softmax_scale=float("nan")), E), (_set(softmax_scale=float("inf")), E),
    (_set(q_token_stride=1023), E), (_set(q_token_stride=1028), E), (_set(d=96), U), (_set(Hq=34), U),
]


@pytest.mark.parametrize("mutate,status", ROWS + [
    (_set(v_cache=None), E), (_set(out=None), E), (_set(out_dtype=sv.SPEC_E4M3), E), (_set(v_cache=FAKE + 16), E), (_set(out=FAKE + 8), E), (_set(lse=FAKE + 2), E),
])
def test_prompt_attn_refuses(mutate, status):
    a = _prompt()
    mutate(a)
    assert sv.lib().spec_prompt_attn_workspace_bytes(C.byref(a)) == 0
    assert _call(a) == status


@pytest.mark.parametrize("mutate,status", ROWS + [
    (_set(weight=None), E), (_set(lse=None), E), (_set(weight=FAKE + 8), E), (_set(weight_in=FAKE + 8), E), (_set(lse=FAKE + 1), E),
    (_set(weight_in=FAKE + 16 * 2 * 64 - 32), E), (_set(weight_in=FAKE - 32), E),
])
def test_kv_weight_refuses(mutate, status):
    a = _weight()
    mutate(a)
    assert _call(a) == status


@pytest.mark.parametrize("mutate,status", [
    (_set(new_kv_len=FAKE), E), (_set(new_kv_len=FAKE + 4), E), (_set(kv_len=(FAKE << 8) + 4), E), (_set(keep=FAKE << 8), E),   # (lengths out over lengths in)
    (_set(B=0), E), (_set(Hkv=0), E), (_set(num_blocks=0), E), (_set(dst_max_blocks=0), E), (_set(first=-1), E), (_set(recent=-1), E), (_set(k_cache=None), E),
    (_set(weight=None), E), (_set(keep=None), E), (_set(new_kv_len=None), E), (_set(dst_block_table=None), E), (_set(dst_block_table=FAKE), E),
    (_set(kv_scale=None), E), (_set(kv_dtype=sv.SPEC_BF16), E), (_set(kv_dtype=sv.SPEC_F32, kv_scale=None), E), (_set(kv_dtype=7), E),
    (_set(kv_layout=sv.KV_TOKEN_MAJOR), E), (_set(v_cache=FAKE + 16), E), (_set(weight=FAKE + 4), E), (_set(host_kv_len=None), E), (_set(max_kv_len=65), E),
    (_host("host_kv_len", [60, 65]), E), (_host("host_kv_len", [-1, 50]), E), (_set(max_kv_len=59), E), (_set(d=32), U), (_set(B=65536, host_kv_len=None, max_kv_len=60), U),
])
def test_kv_evict_refuses(mutate, status):
    a = _evict()
    mutate(a)
    assert sv.lib().spec_kv_evict_workspace_bytes(C.byref(a)) == 0
    assert _call(a) == status


@pytest.mark.parametrize("make", [_prompt, _weight])
def test_more_rows_than_a_kv_head_can_have_are_refused(make):
    """T tokens times the group: 2^28 is one too many, whatever the requests are."""
    a = make(kv_len=(60, 60), q_len=(1, 1))
    a.Hq, a.Hkv, a.T = 16, 1, 1 << 24
    _host("host_cu_q_len", [0, 1 << 23, 1 << 24])(a)
    assert _call(a) == U
    a.T -= 1
    _host("host_cu_q_len", [0, 1 << 23, (1 << 24) - 1])(a)
    if make is _prompt:
        assert sv.lib().spec_prompt_attn_workspace_bytes(C.byref(a)) == 256      # (rows like these are not split)


def test_null_arguments_and_workspaces():
    L = sv.lib()
    assert L.spec_qk_norm_rope(None, None) == E and L.spec_prompt_attn(None, FAKE, WORKSPACE, None) == E
    assert L.spec_kv_weight(None, None) == E and L.spec_kv_evict(None, FAKE, WORKSPACE, None) == E
    assert L.spec_prompt_attn_workspace_bytes(None) == 0 and L.spec_kv_evict_workspace_bytes(None) == 0
    for make in (_prompt, _evict):
        for at, size in ((None, WORKSPACE), (FAKE + 128, WORKSPACE), (FAKE, 128)):
            assert _call(make(), size, at) == sv.SPEC_EWORKSPACE


def test_workspaces_depend_on_shapes_and_lengths_alone():
    L = sv.lib()
    whole = _prompt(kv_len=(60, 50, 20))
    assert L.spec_prompt_attn_workspace_bytes(C.byref(whole)) == 256            # nothing is split
    long = _prompt(kv_len=(60000, 50, 20), q_len=(2, 2, 0))
    long.max_blocks_per_req = 4000
    split = L.spec_prompt_attn_workspace_bytes(C.byref(long))
    assert split > 256
    bucket = _prompt(kv_len=(60, 50, 20), q_len=(2, 2, 0), bucket=60000)
    bucket.max_blocks_per_req = 4000
    bucket.host_kv_len = None
    assert L.spec_prompt_attn_workspace_bytes(C.byref(bucket)) > 256
    e = _evict()
    assert L.spec_kv_evict_workspace_bytes(C.byref(e)) == 256                   # places of 2 x 32 tokens; no scores are handed over
    e.max_blocks_per_req, e.max_kv_len, e.host_kv_len = 600, 9000, None
    assert L.spec_kv_evict_workspace_bytes(C.byref(e)) == 2 * 16384 * 4 + 256


def test_a_batch_without_rows_is_nothing_to_do():
    for make in (_prompt, _weight):
        a = make(q_len=(0, 0, 0))
        a.q = a.lse = None
        if make is _prompt:
            a.out = None
        assert _call(a) == sv.SPEC_OK
    a = _rope()
    a.T = 0
    a.q = a.k = a.out_q = a.out_k = a.positions = None
    assert _call(a) == sv.SPEC_OK


# ------------------------------------------------------------------------------------------ the binding
def _i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_rope_binding_refuses():
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    pos, freq, w = _i32(0, 1, 2), torch.zeros(32), torch.zeros(64)

    def make(q=x, k=x, out_q=x, out_k=x, positions=pos, inv_freq=freq, **kw):
        return sv.make_qk_norm_rope_args(q, k, out_q, out_k, positions, inv_freq, **kw)

    args, _ = make(q_weight=w, k_weight=w)
    assert (args.T, args.Hq, args.Hkv, args.d, args.rot_dim) == (3, 2, 2, 64, 64)
    assert make(x, None, x, None)[0].Hkv == 0
    for kw in (dict(q=None, k=None, out_q=None, out_k=None), dict(out_q=None), dict(out_k=x.float()), dict(k=x[:2], out_k=x[:2]), dict(q=x.expand(3, 2, 64)[:, :, ::2]),
               dict(positions=pos.long()), dict(positions=_i32(0, 1)), dict(inv_freq=freq.double()), dict(q_weight=w[:32]), dict(q_weight=w, k_weight=w.bfloat16()),
               dict(q=x[:1].expand(3, 2, 64))):
        with pytest.raises((ValueError, TypeError)):
            make(**kw)
    with pytest.raises(TypeError):
        make(*(x.half(),) * 4)


def _cache(kind="int8", Hkv=2, d=64):
    if kind == "bf16":
        return torch.zeros((4, Hkv, 16, d), dtype=torch.bfloat16), torch.zeros((4, Hkv, 16, d), dtype=torch.bfloat16), None
    return sv.alloc_kv8_pools(4, Hkv, d, torch.int8, device="cpu")


def test_row_bindings_refuse():
    k, v, scale = _cache()
    q = torch.zeros((30, 4, 64), dtype=torch.bfloat16)
    base = dict(q=q, table=torch.zeros((1, 2), dtype=torch.int32), lens=_i32(30), cu=_i32(0, 30), out=torch.zeros_like(q), lse=torch.zeros((30, 4)),
                weight=sv.alloc_kv_weight(4, 2, "cpu"), weight_in=None, scale=scale, errors=torch.zeros(1, dtype=torch.int64))

    def prompt(**kw):
        a = dict(base, **kw)
        return sv.make_prompt_attn_args(a["q"], k, v, a["table"], a["lens"], a["cu"], a["out"], [30], [0, 30], lse=a["lse"], kv_scale=a["scale"], error_count=a["errors"])

    def weight(**kw):
        a = dict(base, **kw)
        return sv.make_kv_weight_args(a["q"], a["lse"], k, a["table"], a["lens"], a["cu"], a["weight"], [30], [0, 30], weight_in=a["weight_in"], kv_scale=a["scale"],
                                      error_count=a["errors"])

    both = [dict(q=q.float()), dict(q=q[:, :, ::2]), dict(q=q[:1].expand(30, 4, 64)), dict(table=base["table"].long()), dict(table=base["table"][0]), dict(lens=_i32()), dict(cu=_i32(0)),
            dict(lse=base["lse"].double()), dict(lse=base["lse"][:, :3]), dict(lse=torch.zeros((30, 8))[:, ::2]), dict(errors=_i32(0)), dict(scale=scale.double())]
    for make, more in ((prompt, [dict(out=base["out"].half()), dict(out=base["out"][:20])]),
                       (weight, [dict(lse=None), dict(weight=base["weight"].double()), dict(weight=base["weight"][:3]), dict(weight_in=base["weight"][:, :1])])):
        make()
        for kw in both + more:
            with pytest.raises((ValueError, TypeError)):
                make(**kw)
    assert prompt(lse=None)[0].lse is None


def test_evict_binding_refuses():
    k, v, _ = _cache("bf16")
    base = dict(weight=sv.alloc_kv_weight(4, 2, "cpu"), table=torch.zeros((2, 2), dtype=torch.int32), lens=_i32(20, 20), keep=_i32(3, 3),
                dst=torch.zeros((2, 1), dtype=torch.int32), new=_i32(0, 0), kept=torch.zeros((2, 16), dtype=torch.int32), k=k)

    def make(**kw):
        a = dict(base, **kw)
        return sv.make_kv_evict_args(a["k"], v, a["weight"], a["table"], a["lens"], a["keep"], a["dst"], a["new"], [20, 20], kept=a["kept"])

    assert make()[0].dst_max_blocks == 1 and make(kept=None)[0].kept is None
    for kw in (dict(weight=None), dict(weight=base["weight"][:2]), dict(lens=_i32(20)), dict(keep=base["keep"].long()), dict(dst=base["dst"][0]), dict(dst=base["dst"][:1]),
               dict(new=_i32(0)), dict(kept=torch.zeros((2, 17), dtype=torch.int32)), dict(kept=torch.zeros((1, 16), dtype=torch.int32)), dict(k=k[:, :, :8])):
        with pytest.raises((ValueError, TypeError)):
            make(**kw)


@pytest.mark.parametrize("wrong", [dict(requests=0), dict(prompt=(0, 9)), dict(prompt=(9, 8)), dict(chunk=0), dict(budget=0), dict(window=0), dict(first=-1), dict(k=-1)])
def test_prompt_loop_refuses(wrong):
    from paper_2406_14066_amd.prompt_loop import PromptLoop
    given = dict(requests=1, prompt=(8, 9), budget=4, chunk=8)
    given.update(wrong)
    with pytest.raises(ValueError):
        PromptLoop(given.pop("requests"), given.pop("prompt"), device="cpu", **given)
