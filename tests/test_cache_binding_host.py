"""What the Python binding of the cache operators refuses before it makes an argument struct: nothing is launched."""
import numpy as np
import pytest

from paper_2406_14066_amd import spec_verify as sv

torch = pytest.importorskip("torch")


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def _pools(Hkv=2, d=64):
    return sv.alloc_kv8_pools(4, Hkv, d, torch.int8, device="cpu")


def _append(new_k, new_v=None, Hkv=2):
    T = new_k.shape[0]
    return sv.make_kv8_append_args(new_k, new_k if new_v is None else new_v, *_pools(Hkv), torch.zeros((1, 2), dtype=torch.int32), _i32(T), _i32(0, T), [T], [0, T])


def _attn(q, prefix=False):
    T = q.shape[0]
    k, v, scale = _pools()
    table, out = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(q.shape, dtype=torch.bfloat16)
    if prefix:
        return sv.make_prefix_attn_args(q, k, v, table, _i32(20), _i32(0, T), _i32(0, 1), _i32(16), out, [20], [0, T], [0, 1], [16], kv_scale=scale)
    return sv.make_kv8_attn_args(q, k, v, scale, table, _i32(20), _i32(0, T), out, [20], [0, T])


@pytest.mark.parametrize("make", [_append, _attn, lambda q: _attn(q, True)], ids=["append", "kv8", "prefix"])
def test_rows_that_lie_on_each_other_are_refused(make):
    """An expanded tensor's token stride is 0, which the argument structs take for packed rows: T rows would be read where one is."""
    row = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    make(row.repeat(3, 1, 1))
    make(row)                                           # (one token: its stride says nothing)
    with pytest.raises(ValueError):
        make(row.expand(3, 2, 64))
    with pytest.raises(ValueError):                     # tokens half a row apart
        make(torch.zeros(1024, dtype=torch.bfloat16).as_strided((3, 2, 64), (64, 64, 1)))


def _all(which, **other):
    """Arguments of one binding with every array it reads, some of them replaced: three requests in two groups, five rows."""
    k, v, scale = _pools()
    a = dict(table=torch.zeros((3, 2), dtype=torch.int32), lens=_i32(20, 20, 20), cu=_i32(0, 2, 4, 5), start=_i32(0, 0, 0), groups=_i32(0, 2, 3),
             prefix=_i32(16, 0), errors=torch.zeros(1, dtype=torch.int64), host_lens=[20, 20, 20], host_cu=[0, 2, 4, 5], rows=torch.zeros((5, 2, 64)),
             out=torch.zeros((5, 2, 64)), host_groups=[0, 2, 3], host_prefix=[16, 0], scale=scale, **{})
    a.update(other)
    q = a["rows"].to(torch.bfloat16)
    if which == "append":
        return sv.make_kv8_append_args(a["rows"], a["rows"], k, v, a["scale"], a["table"], a["lens"], a["cu"], a["host_lens"], a["host_cu"], error_count=a["errors"])
    if which == "read":
        return sv.make_kv8_read_args(a["out"], a["out"], k, v, a["scale"], a["table"], a["start"], a["cu"], a["host_cu"], error_count=a["errors"])
    if which == "kv8":
        return sv.make_kv8_attn_args(q, k, v, a["scale"], a["table"], a["lens"], a["cu"], a["out"], a["host_lens"], a["host_cu"], error_count=a["errors"])
    return sv.make_prefix_attn_args(q, k, v, a["table"], a["lens"], a["cu"], a["groups"], a["prefix"], a["out"], a["host_lens"], a["host_cu"], a["host_groups"],
                                    a["host_prefix"], kv_scale=a["scale"], error_count=a["errors"])


ARRAYS = {"append": ("table", "lens", "cu", "errors"), "read": ("table", "start", "cu", "errors"), "kv8": ("table", "lens", "cu", "errors"),
          "prefix": ("table", "lens", "cu", "groups", "prefix", "errors")}


@pytest.mark.parametrize("which,name", [(w, n) for w, names in ARRAYS.items() for n in names])
def test_index_arrays_are_what_the_kernels_read(which, name):
    """The kernels read 32-bit entries (the counter: 64) one after another, as many as there are requests or groups."""
    good = {"table": torch.zeros((3, 2), dtype=torch.int32), "lens": _i32(20, 20, 20), "cu": _i32(0, 2, 4, 5), "start": _i32(0, 0, 0),
            "groups": _i32(0, 2, 3), "prefix": _i32(16, 0), "errors": torch.zeros(1, dtype=torch.int64)}[name]
    _all(which)
    _all(which, **{name: good})
    wide = torch.stack([good, good], -1)
    bad = [good.to(torch.int32 if name == "errors" else torch.int64), good[:-1], good.to("meta")]
    bad += [wide[..., 0]] if good.numel() > 1 else []
    if name == "table":
        bad += [torch.zeros((3, 5), dtype=torch.int32)[:, :2], good[0]]
    for x in bad:
        with pytest.raises(ValueError):
            _all(which, **{name: x})


@pytest.mark.parametrize("which,name,bad", [("append", "host_lens", [20, 20]), ("kv8", "host_lens", [20, 20]), ("prefix", "host_lens", [20]),
                                            ("prefix", "host_groups", [0, 3])])
def test_host_arrays_are_long_enough(which, name, bad):
    with pytest.raises(ValueError):
        _all(which, **{name: bad})


@pytest.mark.parametrize("which", list(ARRAYS))
def test_tensors_of_another_device_are_refused(which):
    for name in ("scale", "out" if which != "append" else "rows"):
        x = _pools()[2] if name == "scale" else torch.zeros((5, 2, 64))
        with pytest.raises(ValueError):
            _all(which, **{name: x.to("meta")})


def test_an_append_and_a_read_of_no_rows_do_nothing():
    """An empty tensor has no address."""
    empty = torch.zeros((0, 2, 64))
    args, keep = _append(empty)
    assert args.new_k is None
    sv.spec_kv8_append(args, stream=_NoStream())
    k, v, scale = _pools()
    args, keep = sv.make_kv8_read_args(empty, empty, k, v, scale, torch.zeros((1, 2), dtype=torch.int32), None, _i32(0, 0), [0, 0])
    assert args.out_k is None
    sv.spec_kv8_read(args, stream=_NoStream())


class _NoStream:
    cuda_stream = 0
