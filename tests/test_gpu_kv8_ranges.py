"""The 8-bit cache at the ends of the number range: rows of any finite magnitude, V scales of any size, pools that hold anything."""
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


@pytest.mark.parametrize("shared", [None, 1, 0], ids=["kv8", "shared", "whole"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kv", KINDS)
@pytest.mark.parametrize("power", [-60, 0, 60, 119])
@pytest.mark.parametrize("rows", [30, 60], ids=["few", "many"])
def test_small_weights_count_whatever_the_scale_of_v(rows, kv, out, power, shared, tuning):
    """Every wavefront's pages hold a token with 2^16 times the weight of each of the others, whose sum is a thousandth of the whole."""
    if shared is not None:
        tuning("SPEC_VERIFY_PREFIX_SHARED", shared)
    Hq = Hkv = 2
    d, n, B = 64, 8192, rows
    pages = n // 16
    rng = np.random.default_rng(33)
    code = rng.integers(1, 127, size=(2, pages, Hkv, 16 * d)).astype(np.uint8)
    code[0] = 0
    one = 1 if kv == "int8" else 0x38                    # the value 1
    code[0][:, :, R.cell(np.arange(16), 0, 0)] = one     # K is 1 in the first dim, and its scale the score
    scales = np.full((pages, Hkv, 2, 16), 2.0 ** power, dtype=np.float32)
    scales[:, :, 0] = 0.0
    high = np.arange(pages) % 32 < 8
    scales[high, :, 0, 5] = 16 * np.log(2.0)
    dev = [torch.from_numpy(c.view(np.int8).reshape(pages, Hkv, 16, d)).cuda().view(_type(kv)) for c in code]
    cu = np.arange(B + 1, dtype=np.int32)
    kv_len = np.full(B, n, dtype=np.int32)
    q = torch.zeros((B, Hq, d), device="cuda")
    q[:, :, 0] = 1.0
    q = q.to(torch.bfloat16)
    o = torch.zeros((B, Hq, d), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(B, 1)
    arrays = (table, torch.from_numpy(kv_len).cuda(), torch.from_numpy(cu).cuda())
    if shared is None:
        args, keep = sv.make_kv8_attn_args(q, *dev, torch.from_numpy(scales).cuda(), *arrays, o, kv_len, cu, softmax_scale=1.0)
        ws = sv.alloc_workspace(sv.spec_kv8_attn_workspace_bytes(args))
        sv.spec_kv8_attn(args, ws)
    else:                                                # (the last page is not the prefix's, and the same for all)
        group, prefix = np.array([0, B], dtype=np.int32), np.array([n - 16], dtype=np.int32)
        args, keep = sv.make_prefix_attn_args(q, *dev, *arrays, torch.from_numpy(group).cuda(), torch.from_numpy(prefix).cuda(), o, kv_len, cu, group,
                                              prefix, kv_scale=torch.from_numpy(scales).cuda(), softmax_scale=1.0)
        ws = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(args))
        sv.spec_prefix_attn(args, ws)
    torch.cuda.synchronize()
    cache = np.moveaxis(np.array([R.token(code[1], scales, 1, t // 16, t % 16, kv) for t in range(n)]), 0, 1)     # [Hkv, n, d]
    weight = np.ones(n)
    weight.reshape(pages, 16)[high, 5] = 2.0 ** 16
    want = (weight[None, :, None] * cache).sum(1) / weight.sum()
    got = o.double().cpu().numpy()
    # fp32 output: sums of 8192 terms (2^-24 of the sum each, as a random walk 2^-17.5) and weights of 22 bits: 2^-16 of the largest |v|;
    # bf16: its own rounding (2^-8 of the value) and that of the weights as one fp16 (2^-11)
    most = np.abs(cache).max()
    limit = 2.0 ** -16 * most if out == "f32" else 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * most
    assert (np.abs(got - want[None]) <= limit).all(), np.abs(got / want[None] - 1).max()
