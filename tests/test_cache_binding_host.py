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
