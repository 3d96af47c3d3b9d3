"""Plain 64-bit reference (numpy) of the operators around prompts and bounded caches, written from their definitions in
include/spec_verify.h, and caches to run them on.  Nothing here calls the library."""
import numpy as np

PAGE = 16
MOST = {"e4m3": 448.0, "int8": 127.0}
KINDS = ["tiles", "tokens", "e4m3", "int8"]


def cells(kind, d, which):
    """[16, d]: place of (token slot, dim) in one KV head's page of K (0) or V (1)."""
    s, c = np.arange(PAGE)[:, None], np.arange(d)[None, :]
    if kind in ("tokens", "f32"):
        return s * d + c
    if kind == "tiles":
        return c // 8 * 128 + s * 8 + c % 8 if which == 0 else (((c // 32 * 4 + s // 4) * 16 + c % 16) * 2 + c // 16 % 2) * 4 + s % 4
    return c // 16 * 256 + s * 16 + c % 16 if which == 0 else ((c // 64 * 4 + s // 4) * 16 + c % 16) * 16 + c % 64 // 16 * 4 + s % 4


class Cache:
    """Random pools of a kind; every slot holds something.  `value[w]` [nb, Hkv, 16, d] is what K's (V's) slots stand for, in 64 bits."""

    def __init__(self, rng, nb, Hkv, d, kind, spread=1.0):
        import torch
        self.kind, self.Hkv, self.d, self.nb = kind, Hkv, d, nb
        self.pool, self.value, self.scale = [], [], None
        scales = []
        for w in range(2):
            rows = rng.standard_normal((nb, Hkv, PAGE, d)).astype(np.float32) * np.float32(spread)
            if kind in MOST:
                a = np.abs(rows).max(-1)
                code = torch.from_numpy(rows * (MOST[kind] / a)[..., None])
                code = code.round().to(torch.int8) if kind == "int8" else code.clamp(-448, 448).to(torch.float8_e4m3fn)
                scales.append((a / MOST[kind]).astype(np.float32))
                self.value.append(code.float().numpy().astype(np.float64) * scales[w].astype(np.float64)[..., None])
            else:
                code = torch.from_numpy(rows).to(torch.float32 if kind == "f32" else torch.bfloat16)
                self.value.append(code.float().numpy().astype(np.float64))
            raw = code.view(torch.uint8 if code.element_size() == 1 else torch.int16 if code.element_size() == 2 else torch.int32)
            self.type = code.dtype
            self.pool.append(self.arrange(raw.numpy(), w))
        if scales:
            self.scale = np.stack(scales, 2)

    def arrange(self, rows, w):
        out = np.empty((rows.shape[0], self.Hkv, PAGE * self.d), dtype=rows.dtype)
        out[:, :, cells(self.kind, self.d, w).ravel()] = rows.reshape(rows.shape[0], self.Hkv, -1)
        return out

    def put(self, w, page, head, slot, dim, value):
        """One element of a bf16 pool (every dim, head if None)."""
        import torch
        bits = torch.tensor([value], dtype=torch.float32).to(torch.bfloat16).view(torch.int16).numpy()[0]
        heads = range(self.Hkv) if head is None else [head]
        for h in heads:
            self.value[w][page, h, slot, dim] = value
            self.pool[w][page, h, cells(self.kind, self.d, w)[slot, dim]] = bits

    def device(self):
        import torch
        got = [torch.from_numpy(p.reshape(self.nb, self.Hkv, PAGE, self.d).copy()).cuda().view(self.type) for p in self.pool]
        return got[0], got[1], None if self.scale is None else torch.from_numpy(self.scale.copy()).cuda()

    def rows(self, w, pages, n):
        """[n, Hkv, d]; pages outside the pool are zeros."""
        out = np.zeros((n, self.Hkv, self.d))
        for t in range(n):
            page = pages[t // PAGE]
            if 0 <= page < self.nb:
                out[t] = self.value[w][page, :, t % PAGE]
        return out


def tables(rng, lens, spare=3, columns=None, more=()):
    """A shuffled block table for each of lens and more, over one pool."""
    groups, counts = [lens] + list(more), []
    for g in groups:
        counts.append([(n + PAGE - 1) // PAGE for n in g])
    order = rng.permutation(sum(map(sum, counts)) + spare).astype(np.int32)
    made, at = [], 0
    for c in counts:
        table = np.zeros((len(c), columns or max(max(c), 1)), dtype=np.int32)
        for b, n in enumerate(c):
            table[b, :n] = order[at:at + n]
            at += n
        made.append(table)
    return (made if more else made[0]), len(order)


def prefix_sum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int32)


def norm_rope(x, weight, positions, inv_freq, eps, interleaved, scale=1.0):
    """(rows in 64 bits, |y_a| + |y_b| of each element's pair)."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    half = len(inv_freq)
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    angle = positions.astype(np.float64)[:, None, None] * inv_freq.astype(np.float64)
    out, size = y.copy(), np.abs(y)
    out[..., a] = scale * (y[..., a] * np.cos(angle) - y[..., b] * np.sin(angle))
    out[..., b] = scale * (y[..., b] * np.cos(angle) + y[..., a] * np.sin(angle))
    size[..., a] = size[..., b] = abs(scale) * (np.abs(y[..., a]) + np.abs(y[..., b]))
    return out, size


def attention(q, keys, values, n, scale=None):
    """q [m, Hq, d], keys and values [n, Hkv, d] -> out, lse, and for bounds: sum of weight * |v|, largest scaled sum of |q k|.  Row j sees the keys
    up to n - m + j; infinities and NaN of V count for the rows that see them."""
    m, Hq, d = q.shape
    Hkv = keys.shape[1]
    out, size = np.zeros((m, Hq, d)), np.zeros((m, Hq, d))
    lse, steep = np.full((m, Hq), -np.inf), np.zeros((m, Hq))
    scale = scale or 1.0 / np.sqrt(d)
    for h in range(Hq):
        k, v = keys[:, h // (Hq // Hkv)], values[:, h // (Hq // Hkv)]
        with np.errstate(invalid="ignore", over="ignore"):
            s = q[:, h] @ k.T * scale
            mass = np.abs(q[:, h]) @ np.abs(k).T * scale
        for j in range(m):
            see = n - m + j + 1
            if see <= 0:
                continue
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                x = s[j, :see]
                w = np.exp(x - x.max())
                lse[j, h] = x.max() + np.log(w.sum())
                out[j, h] = (w[:, None] * v[:see]).sum(0) / w.sum()
                size[j, h] = (w[:, None] * np.abs(v[:see])).sum(0) / w.sum()
                steep[j, h] = mass[j, :see].max()
    return out, lse, size, steep


def token_weights(q, lse, keys, n, scale=None):
    """q [m, Hq, d], lse [m, Hq], keys [n, Hkv, d] -> [n, Hkv] sums over the rows that see a token."""
    m, Hq, d = q.shape
    Hkv = keys.shape[1]
    out = np.zeros((n, Hkv))
    scale = scale or 1.0 / np.sqrt(d)
    for h in range(Hq):
        with np.errstate(invalid="ignore", over="ignore"):
            s = q[:, h] @ keys[:, h // (Hq // Hkv)].T * scale
        for j in range(m):
            see = n - m + j + 1
            if see > 0 and np.isfinite(lse[j, h]):
                out[:see, h // (Hq // Hkv)] += np.exp(s[j, :see] - lse[j, h])
    return out


def choose(weight, pages, n, keep, first, recent, nb):
    """Indices of the tokens that stay, ascending; weight [nb, Hkv, 16] fp32."""
    keep = min(n, keep)
    first = min(first, keep)
    recent = min(recent, keep - first)
    score = np.full(n, -np.inf, dtype=np.float64)
    for t in range(n):
        page = pages[t // PAGE]
        if 0 <= page < nb:
            score[t] = np.float32(weight[page, :, t % PAGE].astype(np.float64).sum())
    none = np.isnan(score) | ~np.array([0 <= pages[t // PAGE] < nb for t in range(n)], dtype=bool)
    middle = [t for t in range(first, n - recent)]
    middle.sort(key=lambda t: (none[t], -score[t] if not none[t] else 0, t))
    return sorted(list(range(first)) + middle[:keep - first - recent] + list(range(n - recent, n))) if n else []
