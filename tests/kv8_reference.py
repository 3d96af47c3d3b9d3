"""Plain 64-bit reference (numpy) of the 8-bit cache's operators and of attention over shared prefixes, written from
their definitions in include/spec_verify.h.  Pools are bytes [num_blocks, Hkv, 16 * d]; nothing here calls the library."""
import numpy as np

PAGE = 16
MOST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_value(code):
    """Value of 8-bit codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.asarray(code, dtype=np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


_E4M3 = e4m3_value(np.arange(256))
_INT8 = np.arange(256).astype(np.uint8).view(np.int8).astype(np.float64)


def code_value(code, kv):
    return (_E4M3 if kv == "e4m3" else _INT8)[np.asarray(code, dtype=np.uint8)]


def cell(slot, dim, which):
    """Byte of (token slot, dim) in one KV head's page of K (0) or V (1)."""
    if which == 0:
        return dim // 16 * 256 + slot * 16 + dim % 16
    return ((dim // 64 * 4 + slot // 4) * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + slot % 4


def quantise(row, kv):
    """(code bytes [.., d], scales [..]) of fp32 rows with the library's fp32 steps, which decide ties; the values they
    stand for are checked against 64 bits separately."""
    row = np.asarray(row, dtype=np.float32)
    a = np.maximum(np.abs(row).max(-1), np.float32(2.0 ** -60)).astype(np.float32)
    most = np.float32(MOST[kv])
    with np.errstate(invalid="ignore", over="ignore"):
        x = row * ((np.float32(1) / a) * most)[..., None]
    bad = ~np.isfinite(row).all(-1)
    if kv == "int8":
        code = np.clip(np.rint(np.where(bad[..., None], 0, x)), -127, 127).astype(np.int8).view(np.uint8)
    else:
        x = np.clip(np.where(bad[..., None], 0, x), -448, 448).astype(np.float64)
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
        v = np.rint(x / step) * step
        table = _E4M3[:127]
        code = np.searchsorted(table, np.abs(v)).astype(np.uint8)
        assert (table[code] == np.abs(v)).all()
        code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    scale = np.where(bad, np.float32(np.nan), (a * (np.float32(1) / most)).astype(np.float32))
    return code, scale


def append(new, pool, scales, which, table, kv_len, cu, kv):
    """`new` [T, Hkv, d] fp32 into pool bytes and scales [nb, Hkv, 2, 16], in place; returns the rows left out."""
    nb, Hkv, n = pool.shape
    d, left_out = n // PAGE, 0
    dims = np.arange(d)
    for b in range(len(cu) - 1):
        for r in range(cu[b], cu[b + 1]):
            pos = int(kv_len[b]) - int(cu[b + 1] - cu[b]) + r - int(cu[b])
            if pos < 0 or pos // PAGE >= table.shape[1] or not 0 <= table[b, pos // PAGE] < nb:
                left_out += 1
                continue
            page, slot = table[b, pos // PAGE], pos % PAGE
            code, scale = quantise(new[r], kv)
            pool[page][:, cell(slot, dims, which)] = code
            scales[page, :, which, slot] = scale
    return left_out


def token(pool, scales, which, page, slot, kv):
    """[Hkv, d] in 64 bits."""
    d = pool.shape[2] // PAGE
    return code_value(pool[page][:, cell(slot, np.arange(d), which)], kv) * scales[page, :, which, slot].astype(np.float64)[:, None]


def read(pool, scales, which, pages, first, count, kv):
    """[count, Hkv, d] in 64 bits; pages outside the pool read as zeros."""
    nb, Hkv, n = pool.shape
    out = np.zeros((count, Hkv, n // PAGE))
    for i in range(count):
        at = (first + i) // PAGE
        if 0 <= at < len(pages) and 0 <= pages[at] < nb:
            out[i] = token(pool, scales, which, pages[at], (first + i) % PAGE, kv)
    return out


def attention(q, keys, values, n, scale=None):
    """q [m, Hq, d]; keys, values [n, Hkv, d]; row j sees the keys up to n - m + j.  Rows that see none are zero."""
    m, Hq, d = q.shape
    group = Hq // keys.shape[1]
    out = np.zeros((m, Hq, d))
    for j in range(m):
        last = n - m + j
        if last < 0:
            continue
        for h in range(Hq):
            k, v = keys[:last + 1, h // group], values[:last + 1, h // group]
            with np.errstate(invalid="ignore", over="ignore"):
                s = k @ q[j, h] * (scale or 1.0 / np.sqrt(d))
                w = np.exp(s - s.max())
                out[j, h] = (w[:, None] * v).sum(0) / w.sum()
    return out
