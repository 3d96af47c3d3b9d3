"""The 8-bit cache at the ends of the number range."""
import numpy as np
import pytest
import torch

import kv8_reference as R
from paper_2406_14066_amd import spec_verify as sv

pytestmark = pytest.mark.gpu

KINDS = ["e4m3", "int8"]


def _type(kv):
    return torch.int8 if kv == "int8" else torch.float8_e4m3fn


def _appended(rows, kv):
    """rows [T, Hkv, d] through spec_kv8_append: (codes of K [T, Hkv, d] as bytes, K's scales [T, Hkv], rows read back in fp32)."""
    T, Hkv, d = rows.shape
    k, v, scale = sv.alloc_kv8_pools((T + 15) // 16, Hkv, d, _type(kv))
    table = torch.arange((T + 15) // 16, dtype=torch.int32, device="cuda")[None]
    cu = np.array([0, T], dtype=np.int32)
    cud = torch.from_numpy(cu).cuda()
    args, keep = sv.make_kv8_append_args(rows, rows, k, v, scale, table, cud[1:], cud, cu[1:], cu)
    sv.spec_kv8_append(args)
    out = [torch.empty((T, Hkv, d), device="cuda") for _ in range(2)]
    args, keep2 = sv.make_kv8_read_args(out[0], out[1], k, v, scale, table, None, cud, cu)
    sv.spec_kv8_read(args)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(scale[:, :, 0], scale[:, :, 1])
    codes = k.view(torch.int8).view(-1, Hkv, d // 16, 16, 16).permute(0, 3, 1, 2, 4).reshape(-1, Hkv, d)[:T]
    return codes.cpu().numpy(), scale[:, :, 0].permute(0, 2, 1).reshape(-1, Hkv)[:T].cpu().numpy(), out[0].cpu().numpy()


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("kv", KINDS)
def test_codes_do_not_depend_on_the_magnitude_of_the_row(kv, src):
    """A power of two goes into the scale and leaves the codes as they are, up to the largest finite row."""
    rng = np.random.default_rng(31)
    T, Hkv, d = 32, 2, 128
    x = rng.uniform(-1, 1, (T, Hkv, d)).astype(np.float32)
    x[:, :, 3] = rng.uniform(1.0, 1.99, (T, Hkv))        # the largest element: 2^0 up to 2^1
    x[0, :, 3] = np.float32(2) - np.float32(2.0 ** -7)   # ... up to the largest finite value of the type
    if src == "f32":
        x[1, :, 3] = np.float32(2) - np.float32(2.0 ** -23)
    dev = torch.from_numpy(x).cuda().to(torch.float32 if src == "f32" else torch.bfloat16)
    codes, scales, _ = _appended(dev, kv)
    assert np.abs(codes[:, :, 3].astype(np.int64)).min() == (126 if kv == "e4m3" else 127)
    for up in (60, 100, 124, 125, 126, 127):
        big = (dev.double() * 2.0 ** up).to(dev.dtype)
        assert bool(torch.isfinite(big).all())
        got, got_scales, back = _appended(big, kv)
        np.testing.assert_array_equal(got, codes, err_msg="2^%d" % up)
        np.testing.assert_array_equal(got_scales, scales * np.float32(2.0 ** up))
        value = R.code_value(codes.view(np.uint8), kv) * got_scales.astype(np.float64)[..., None]
        np.testing.assert_array_equal(back, value.astype(np.float32))
        assert np.isfinite(back).all()


@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_tokens_that_do_not_exist_read_as_zeros_whatever_the_pool_holds(kv, out):
    """Every byte of the pool is a code, NaN's among them: a page outside the pool is not some other page times zero."""
    Hkv, d, n = 3, 128, 40
    pools = [torch.full((4, Hkv, 16, d), 0x7F, dtype=torch.int8, device="cuda").view(_type(kv)) for _ in range(2)]
    scale = torch.full((4, Hkv, 2, 16), float("inf"), device="cuda")
    table = torch.tensor([[9, -1, 4]], dtype=torch.int32, device="cuda")
    cu = np.array([0, n], dtype=np.int32)
    outs = [torch.full((n, Hkv, d), 7.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda") for _ in range(2)]
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    args, keep = sv.make_kv8_read_args(*outs, *pools, scale, table, None, torch.from_numpy(cu).cuda(), cu, error_count=errors)
    sv.spec_kv8_read(args)
    torch.cuda.synchronize()
    assert int(errors.item()) == n
    assert bool((outs[0] == 0).all()) and bool((outs[1] == 0).all())
