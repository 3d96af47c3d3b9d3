"""Performance cases of the operators around an 8-bit KV cache and around a batch that shares a prefix.

A case is a dict of plain values.  `op` names the operator:

  append  spec_kv8_append: K/V rows are quantised (one scale per token and KV head) as they enter the paged cache
  read    spec_kv8_read: ranges of tokens of an 8-bit cache come back as plain rows
  attn    spec_kv8_attn: lookahead attention over an 8-bit cache
  prefix  spec_prefix_attn: lookahead attention of groups of requests that share their first pages,
          which are read and multiplied once per group (bf16 pages in either layout, or 8-bit ones)

With `own` false `run` computes the operators' plain form with elementary torch operations in 32 bits; with
`own` true it calls the library.  Lengths and group sizes are derived from the case alone, so that a case has
one amount of work; everything else is drawn from the seed.

Pages hold 16 tokens of one request for all KV heads.  An 8-bit page of a KV head is K [d/16][16 tokens][16 dims]
and V [d/64][4 token groups][16 dims][4 dim quarters][4 tokens]; its scales are [2][16] floats, K's and V's.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
MOST = {"e4m3": 448.0, "int8": 127.0}     # largest value of the type
POOL_TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
OUT_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SMALLEST_ROW = 2.0 ** -60                 # rows whose largest magnitude is below take the scale of this


def listed():
    append = dict(op="append", src="bf16", fused=False)
    attn = dict(op="attn", ragged_k=False, out="bf16", bucket=False)
    prefix = dict(op="prefix", ragged_k=False, out="bf16")
    return [
        # One interactive user without speculation: one token enters one layer's cache.  Latency only.
        dict(append, name="kv8_append_one", B=1, qmin=1, qmax=1, past_min=686, past_max=686, Hq=64, Hkv=8, d=128, kv="int8"),
        # The K/V rows of a full batch's verification step (k = 4) enter one layer's cache.
        dict(append, name="kv8_append_batch256", B=256, qmin=5, qmax=5, past_min=251, past_max=1019, Hq=64, Hkv=8, d=128, kv="e4m3"),
        # Prompts are taken in: long odd row counts, and the rows come as slices of a fused QKV projection.
        dict(append, name="kv8_append_prompts", B=6, qmin=700, qmax=5000, past_min=0, past_max=40, Hq=64, Hkv=8, d=128, kv="e4m3",
             fused=True),
        # A short request's cache is read back in fp32, as one checks a small model's cache.
        dict(op="read", name="kv8_read_one", B=1, nmin=333, nmax=333, start_max=0, Hkv=8, d=64, kv="int8", out="f32"),
        # A batch's cache moves to another worker, or to a bf16 pool.
        dict(op="read", name="kv8_read_handover", B=32, nmin=500, nmax=8000, start_max=100, Hkv=8, d=128, kv="e4m3", out="bf16"),
        # One interactive user of a 70B-shaped model under a length bucket: latency.
        dict(attn, name="kv8_attn_one_request", B=1, k=4, lmin=687, lmax=687, Hq=64, Hkv=8, d=128, kv="e4m3", bucket=True),
        # The full batch of a 70B-shaped model, ragged contexts of the length of chat and summarisation traces.
        dict(attn, name="kv8_attn_70b_batch256", B=256, k=2, lmin=256, lmax=1024, Hq=64, Hkv=8, d=128, kv="e4m3"),
        # A few long documents with draft lengths chosen per request, 32-bit output.
        dict(attn, name="kv8_attn_long_int8", B=4, k=8, ragged_k=True, lmin=6000, lmax=32768, Hq=32, Hkv=8, d=128, kv="int8", out="f32"),
        # Two users of the same short instructions: the smallest batch that shares anything.
        dict(prefix, name="prefix_two_requests", G=1, gmin=2, gmax=2, k=4, pmin=512, pmax=512, lmin=40, lmax=100, Hq=32, Hkv=8,
             d=128, kv="bf16", layout="tiles"),
        # A system prompt shared by a whole batch of a 70B-shaped model.
        dict(prefix, name="prefix_system_prompt", G=1, gmin=64, gmax=64, k=2, pmin=4096, pmax=4096, lmin=100, lmax=700, Hq=64, Hkv=8,
             d=128, kv="bf16", layout="tiles"),
        # Questions about a few long documents, an 8-bit cache.
        dict(prefix, name="prefix_documents_e4m3", G=3, gmin=5, gmax=30, k=4, ragged_k=True, pmin=6000, pmax=20000, lmin=30, lmax=900,
             Hq=64, Hkv=8, d=128, kv="e4m3", layout="tiles"),
        # A small grouped-head model on token-major pages: tenants with prompts of their own, some alone, some without a prompt.
        dict(prefix, name="prefix_tenants_d64", G=6, gmin=1, gmax=16, k=7, pmin=0, pmax=2000, lmin=20, lmax=600, Hq=32, Hkv=8, d=64,
             kv="bf16", layout="tokens", out="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attn", "attn", "prefix", "prefix"])
    Hq, Hkv, d = rng.choice([(32, 32, 128), (32, 8, 128), (64, 8, 128), (64, 4, 128), (16, 16, 64), (32, 8, 64)])
    kv = rng.choice(["e4m3", "int8"])
    spread = rng.choice([0.0, 0.3, 0.9])

    def around(mean, least):
        return max(least, int(mean * (1 - spread))), max(least, int(mean * (1 + spread)))

    if op == "append":
        B = _log_int(rng, 1, 256)
        if rng.random() < 0.5:
            qmin = qmax = rng.randint(1, 9)
        else:       # a prompt, or a chunk of one
            qmin, qmax = around(_log_int(rng, 1, max(2, min(8000, int(10e6 / (B * Hkv * d))))), 1)
        past_min, past_max = around(_log_int(rng, 1, 4000), 0)
        return dict(op=op, B=B, qmin=qmin, qmax=qmax, past_min=past_min, past_max=past_max, Hq=Hq, Hkv=Hkv, d=d, kv=kv,
                    src=rng.choice(["bf16", "bf16", "f32"]), fused=rng.random() < 0.4)
    if op == "read":
        B = _log_int(rng, 1, 128)
        nmin, nmax = around(_log_int(rng, 1, max(2, min(32768, int(60e6 / (B * Hkv * d))))), 1)
        return dict(op=op, B=B, nmin=nmin, nmax=nmax, start_max=rng.choice([0, 0, 37, 1000]), Hkv=Hkv, d=d, kv=kv,
                    out=rng.choice(["bf16", "bf16", "f32"]))
    k = rng.randint(0, 8)
    ragged_k = k > 1 and rng.random() < 0.4
    out = rng.choice(["bf16", "bf16", "f32"])
    if op == "attn":
        B = _log_int(rng, 1, 256)
        longest = min(80e6 / (B * Hkv * d), 16e9 / (4 * B * (k + 1) * Hq * d))
        lmin, lmax = around(_log_int(rng, 32, int(max(40, min(32768, longest)))), k + 1)
        return dict(op=op, B=B, k=k, ragged_k=ragged_k, lmin=lmin, lmax=lmax, Hq=Hq, Hkv=Hkv, d=d, kv=kv, out=out,
                    bucket=rng.random() < 0.3)
    G = _log_int(rng, 1, 8)
    gmin, gmax = around(_log_int(rng, 1, 64 // G), 1)
    rows = G * gmax * (k + 1) * Hq
    longest = min(20e6 / (G * Hkv * d), 20e9 / (4 * rows * d), 32768)
    pmin, pmax = around(_log_int(rng, 16, int(max(40, longest))), 0)
    lmin, lmax = around(_log_int(rng, k + 1, int(max(k + 2, min(1500, 20e6 / (G * gmax * Hkv * d))))), k + 1)
    kv = rng.choice(["bf16", "bf16", kv])
    layout = rng.choice(["tiles", "tokens"]) if kv == "bf16" else "tiles"
    return dict(op=op, G=G, gmin=gmin, gmax=gmax, k=k, ragged_k=ragged_k, pmin=pmin, pmax=pmax, lmin=lmin, lmax=lmax, Hq=Hq, Hkv=Hkv,
                d=d, kv=kv, layout=layout, out="bf16" if kv == "bf16" and d == 128 else out)


# --------------------------------------------------------------------------- lengths: from the case alone
def _some(salt, n, lo, hi):
    rng = random.Random("%s %d %d %d" % (salt, n, lo, hi))
    return [rng.randint(lo, hi) for _ in range(n)]


def _prefix_sum(values):
    sums = [0]
    for n in values:
        sums.append(sums[-1] + n)
    return sums


def _group_sizes(case):
    return _some("group", case["G"], case["gmin"], case["gmax"])


def _prefix_lens(case):
    """Whole pages: an engine shares a page or copies it."""
    return [n // PAGE * PAGE for n in _some("prefix", case["G"], case["pmin"], case["pmax"])]


def _batch(case):
    return sum(_group_sizes(case)) if case["op"] == "prefix" else case["B"]


def _q_lens(case):
    if case["op"] == "append":
        return _some("rows", case["B"], case["qmin"], case["qmax"])
    if case["ragged_k"]:
        return [n + 1 for n in _some("k", _batch(case), 1, case["k"])]
    return [case["k"] + 1] * _batch(case)


def _kv_lens(case):
    if case["op"] == "read":
        starts, counts = _read_ranges(case)
        return [a + n for a, n in zip(starts, counts)]
    q = _q_lens(case)
    if case["op"] == "append":
        return [a + n for a, n in zip(_some("past", case["B"], case["past_min"], case["past_max"]), q)]
    lens = [max(n, m) for n, m in zip(_some("kv", _batch(case), case["lmin"], case["lmax"]), q)]
    if case["op"] == "prefix":      # a request's own tokens follow its group's
        shared = [p for p, n in zip(_prefix_lens(case), _group_sizes(case)) for _ in range(n)]
        lens = [p + n for p, n in zip(shared, lens)]
    return lens


def _read_ranges(case):
    return _some("start", case["B"], 0, case["start_max"]), _some("count", case["B"], case["nmin"], case["nmax"])


def _pages(n):
    return (n + PAGE - 1) // PAGE


# --------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32)


def _values(shape, g):
    """Rows whose magnitude varies from token to token (a factor of e^(0.4 N(0, 1)), the last dimension is a row)."""
    x = torch.randn(shape, dtype=torch.float32, device="cuda", generator=g)
    return x * torch.exp(0.4 * torch.randn(shape[:-1] + (1,), dtype=torch.float32, device="cuda", generator=g))


def _table(case, g):
    """A shuffled block table over a pool with a quarter of its pages spare.  Requests of a group have its first pages in common."""
    counts = [_pages(n) for n in _kv_lens(case)]
    shared, owner = [0] * len(counts), list(range(len(counts)))
    if case["op"] == "prefix":
        shared, owner, b = [], [], 0
        for p, n in zip(_prefix_lens(case), _group_sizes(case)):
            shared += [p // PAGE] * n
            owner += [b] * n
            b += n
    index = np.zeros((len(counts), max(counts)), dtype=np.int64)
    need = 0
    for b, n in enumerate(counts):
        first = shared[b] if owner[b] != b else 0
        index[b, :first] = index[owner[b], :first]
        index[b, first:n] = np.arange(need, need + n - first)
        need += n - first
    blocks = need + (need + 3) // 4
    order = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)
    table = order[torch.from_numpy(index).cuda()]
    used = torch.arange(max(counts), device="cuda")[None, :] < torch.tensor(counts, device="cuda")[:, None]
    return torch.where(used, table, torch.zeros_like(table)), blocks


def _quantised(rows, kv):
    """(codes as fp32 values, scales) of rows of the last dimension."""
    most = torch.clamp(rows.abs().amax(-1), min=SMALLEST_ROW)
    codes = rows * (MOST[kv] / most)[..., None]
    codes = torch.round(codes).clamp(-127, 127) if kv == "int8" else codes.clamp(-448, 448).to(torch.float8_e4m3fn).float()
    return codes, most / MOST[kv]


def _k_to_pages8(codes):
    n, heads, _, d = codes.shape
    return codes.view(n, heads, PAGE, d // 16, 16).permute(0, 1, 3, 2, 4).reshape(n, heads, PAGE, d)


def _v_to_pages8(codes):
    n, heads, _, d = codes.shape
    return codes.view(n, heads, 4, 4, d // 64, 4, 16).permute(0, 1, 4, 2, 6, 5, 3).reshape(n, heads, PAGE, d)


def _k_from_pages8(pages):
    n, heads, _, d = pages.shape
    return pages.reshape(n, heads, d // 16, PAGE, 16).permute(0, 1, 3, 2, 4).reshape(n, heads, PAGE, d)


def _v_from_pages8(pages):
    n, heads, _, d = pages.shape
    return pages.reshape(n, heads, d // 64, 4, 16, 4, 4).permute(0, 1, 3, 6, 2, 5, 4).reshape(n, heads, PAGE, d)


def _k_from_tiles(pages):       # bf16 pages in matrix-operand order
    n, heads, _, d = pages.shape
    return pages.reshape(n, heads, d // 8, PAGE, 8).permute(0, 1, 3, 2, 4).reshape(n, heads, PAGE, d)


def _v_from_tiles(pages):
    n, heads, _, d = pages.shape
    return pages.reshape(n, heads, d // 32, 4, 16, 2, 4).permute(0, 1, 3, 6, 2, 5, 4).reshape(n, heads, PAGE, d)


class _State:
    pass


def _pools(s, case, blocks, g):
    """A pool whose every page holds tokens: the requests' and other requests'."""
    shape = (blocks, case["Hkv"], PAGE, case["d"])
    if case["kv"] == "bf16":        # normal values are normal values in either page layout
        s.k_cache, s.v_cache = (_values(shape, g).to(torch.bfloat16) for _ in range(2))
        s.kv_scale = None
        return
    pool = POOL_TYPE[case["kv"]]
    codes, k_scale = _quantised(_values(shape, g), case["kv"])
    s.k_cache = _k_to_pages8(codes).to(pool)
    codes, v_scale = _quantised(_values(shape, g), case["kv"])
    s.v_cache = _v_to_pages8(codes).to(pool)
    s.kv_scale = torch.stack([k_scale, v_scale], 2).contiguous()


def prepare(case, seed):
    s, g = _State(), _gen(seed, 1)
    s.case, s.handle = case, None
    s.table, blocks = _table(case, g)
    _pools(s, case, blocks, g)
    s.host_kv_len = np.array(_kv_lens(case), dtype=np.int32)
    s.kv_len = torch.from_numpy(s.host_kv_len).cuda()
    if case["op"] == "read":
        starts, counts = _read_ranges(case)
        s.host_cu = np.array(_prefix_sum(counts), dtype=np.int32)
        s.start, s.cu = _i32(starts).cuda(), torch.from_numpy(s.host_cu).cuda()
        s.out_k, s.out_v = (torch.zeros((int(s.host_cu[-1]), case["Hkv"], case["d"]), dtype=OUT_TYPE[case["out"]], device="cuda")
                            for _ in range(2))
        return s
    s.host_cu = np.array(_prefix_sum(_q_lens(case)), dtype=np.int32)
    s.cu = torch.from_numpy(s.host_cu).cuda()
    T, Hq, Hkv, d = int(s.host_cu[-1]), case["Hq"], case["Hkv"], case["d"]
    if case["op"] == "append":
        heads = Hq + 2 * Hkv if case["fused"] else 2 * Hkv
        rows = _values((T, heads, d), g).to(OUT_TYPE[case["src"]])
        s.new_k, s.new_v = rows[:, heads - 2 * Hkv:heads - Hkv], rows[:, heads - Hkv:]
        if not case["fused"]:
            s.new_k, s.new_v = s.new_k.contiguous(), s.new_v.contiguous()
        return s
    s.q = torch.randn((T, Hq, d), dtype=torch.float32, device="cuda", generator=g).to(torch.bfloat16)
    s.out = torch.zeros((T, Hq, d), dtype=OUT_TYPE[case["out"]], device="cuda")
    s.bound = 0
    if case.get("bucket"):      # a bucket's table has room for its longest request
        s.bound = (int(s.host_kv_len.max()) + 255) // 256 * 256
        s.table = torch.nn.functional.pad(s.table, (0, s.bound // PAGE - s.table.shape[1])).contiguous()
    if case["op"] == "prefix":
        s.host_groups = np.array(_prefix_sum(_group_sizes(case)), dtype=np.int32)
        s.host_prefix = np.array(_prefix_lens(case), dtype=np.int32)
        s.groups, s.prefix = torch.from_numpy(s.host_groups).cuda(), torch.from_numpy(s.host_prefix).cuda()
    return s


# --------------------------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_2406_14066_amd import spec_verify as sv
    op = s.case["op"]
    if s.handle is None:        # what a decode loop makes once for its buffers: argument structs and the workspace
        if op == "append":
            s.handle = sv.make_kv8_append_args(s.new_k, s.new_v, s.k_cache, s.v_cache, s.kv_scale, s.table, s.kv_len, s.cu,
                                               s.host_kv_len, s.host_cu)
        elif op == "read":
            s.handle = sv.make_kv8_read_args(s.out_k, s.out_v, s.k_cache, s.v_cache, s.kv_scale, s.table, s.start, s.cu, s.host_cu)
        elif op == "attn":
            s.handle = sv.make_kv8_attn_args(s.q, s.k_cache, s.v_cache, s.kv_scale, s.table, s.kv_len, s.cu, s.out, s.host_kv_len,
                                             s.host_cu, max_kv_len=s.bound)
            s.workspace = sv.alloc_workspace(sv.spec_kv8_attn_workspace_bytes(s.handle[0]))
        else:
            layout = sv.KV_TOKEN_MAJOR if s.case["layout"] == "tokens" else sv.KV_MFMA
            s.handle = sv.make_prefix_attn_args(s.q, s.k_cache, s.v_cache, s.table, s.kv_len, s.cu, s.groups, s.prefix, s.out,
                                                s.host_kv_len, s.host_cu, s.host_groups, s.host_prefix, kv_scale=s.kv_scale,
                                                kv_layout=layout)
            s.workspace = sv.alloc_workspace(sv.spec_prefix_attn_workspace_bytes(s.handle[0]))
    if op == "append":
        sv.spec_kv8_append(s.handle[0])
        return dict(k_cache=s.k_cache, v_cache=s.v_cache, kv_scale=s.kv_scale)
    if op == "read":
        sv.spec_kv8_read(s.handle[0])
        return dict(k=s.out_k, v=s.out_v)
    if op == "attn":
        sv.spec_kv8_attn(s.handle[0], s.workspace)
    else:
        sv.spec_prefix_attn(s.handle[0], s.workspace)
    return dict(out=s.out)


# --------------------------------------------------------------------------- the plain form
def _request_of_row(s, total):
    return torch.searchsorted(s.cu[1:].contiguous(), torch.arange(total, device="cuda", dtype=torch.int32), right=True)


def _plain_append(s):
    case = s.case
    d, T = case["d"], s.new_k.shape[0]
    b = _request_of_row(s, T)
    position = s.kv_len[b].long() - s.cu[1:][b].long() + torch.arange(T, device="cuda")
    page, slot = s.table[b, position // PAGE].long(), position % PAGE
    dim = torch.arange(d, device="cuda")
    k_at = (dim // 16 * 256 + dim % 16)[None, :] + slot[:, None] * 16
    v_at = (dim // 64 * 1024 + dim % 16 * 16 + dim % 64 // 16 * 4)[None, :] + (slot // 4 * 256 + slot % 4)[:, None]
    head = torch.arange(case["Hkv"], device="cuda")[None, :, None]
    for new, pool, at, which in ((s.new_k, s.k_cache, k_at, 0), (s.new_v, s.v_cache, v_at, 1)):
        codes, scale = _quantised(new.float(), case["kv"])
        bytes_ = codes.to(pool.dtype).view(torch.uint8)
        pool.view(torch.uint8).view(pool.shape[0], case["Hkv"], PAGE * d)[page[:, None, None], head, at[:, None, :]] = bytes_
        s.kv_scale[page[:, None], head[:, :, 0], which, slot[:, None]] = scale
    return dict(k_cache=s.k_cache, v_cache=s.v_cache, kv_scale=s.kv_scale)


def _dequantised(s, pages):
    """K and V of the pages, [..., Hkv, 16, d] in 32 bits."""
    flat = pages.reshape(-1).long()
    k, v = s.k_cache[flat].float(), s.v_cache[flat].float()
    if s.kv_scale is not None:
        scale = s.kv_scale[flat]
        k, v = _k_from_pages8(k) * scale[:, :, 0, :, None], _v_from_pages8(v) * scale[:, :, 1, :, None]
    elif s.case["layout"] == "tiles":
        k, v = _k_from_tiles(k), _v_from_tiles(v)
    return k.view(pages.shape + k.shape[1:]), v.view(pages.shape + v.shape[1:])


def _plain_read(s):
    T = s.out_k.shape[0]
    b = _request_of_row(s, T)
    position = s.start[b].long() + torch.arange(T, device="cuda") - s.cu[b].long()
    k, v = _dequantised(s, s.table)
    k, v = (x.transpose(2, 3)[b, position // PAGE, position % PAGE].to(s.out_k.dtype) for x in (k, v))
    return dict(k=k, v=v)


def _parts(s, q, pages, last):
    """Unnormalised attention over rows of pages: q [N, R, Hq, d] sees the tokens up to last [N, R] of pages [N, P].
    Returns the largest score, the sum of exponentials and their product with V."""
    N, R, Hq, d = q.shape
    Hkv = s.case["Hkv"]
    k, v = (x.permute(0, 2, 1, 3, 4).reshape(N, Hkv, -1, d) for x in _dequantised(s, pages))
    rows = q.view(N, R, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(N, Hkv, -1, d)
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    score = score.view(N, Hkv, R, Hq // Hkv, -1)
    hidden = torch.arange(score.shape[-1], device="cuda") > last[:, None, :, None, None]
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(-1)
    weight = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top)[..., None])
    out = torch.matmul(weight.view(N, Hkv, -1, weight.shape[-1]), v).view(N, Hkv, R, Hq // Hkv, d)
    top, total = (x.permute(0, 2, 1, 3).reshape(N, R, Hq) for x in (top, weight.sum(-1)))
    return top, total, out.permute(0, 2, 1, 3, 4).reshape(N, R, Hq, d)


def _padded(s, starts, ends, most):
    """Rows starts..ends-1 of the queries as [N, most, Hq, d] in 32 bits, and each row's index."""
    at = starts.long()[:, None] + torch.arange(most, device="cuda")[None, :]
    return s.q[torch.minimum(at, ends.long()[:, None] - 1)].float(), at


def _plain_attention(s):
    case = s.case
    T = s.q.shape[0]
    row = torch.arange(T, device="cuda")
    b = _request_of_row(s, T)
    q_len = s.cu[1:] - s.cu[:-1]
    q, at = _padded(s, s.cu[:-1], s.cu[1:], int(np.diff(s.host_cu).max()))
    last = s.kv_len.long()[:, None] - q_len.long()[:, None] + at - s.cu[:-1].long()[:, None]
    here = (b, row - s.cu[b].long())
    if case["op"] == "attn":
        _, total, out = (x[here] for x in _parts(s, q, s.table, last))
        return dict(out=(out / total[..., None]).to(s.out.dtype))
    # each request's own pages
    sizes = s.groups[1:] - s.groups[:-1]
    group = torch.repeat_interleave(torch.arange(case["G"], device="cuda"), sizes.long(), output_size=s.table.shape[0])
    shared = s.prefix[group].long()
    width = max(_pages(int(n)) - int(p) // PAGE for n, p in zip(s.host_kv_len, np.repeat(s.host_prefix, np.diff(s.host_groups))))
    column = (shared // PAGE)[:, None] + torch.arange(width, device="cuda")[None, :]
    pages = torch.gather(s.table, 1, column.clamp(max=s.table.shape[1] - 1))
    top, total, out = (x[here] for x in _parts(s, q, pages, last - shared[:, None]))
    # its group's
    if int(s.host_prefix.max()) > 0:
        starts, ends = s.cu[s.groups[:-1].long()], s.cu[s.groups[1:].long()]
        q, at = _padded(s, starts, ends, int(np.diff(s.host_cu[s.host_groups]).max()))
        pages = s.table[s.groups[:-1].long(), :int(s.host_prefix.max()) // PAGE]
        more = _parts(s, q, pages, (s.prefix.long() - 1)[:, None].expand(-1, q.shape[1]))
        g = group[b]
        top2, total2, out2 = (x[g, row - starts.long()[g]] for x in more)
        most = torch.maximum(top, top2)
        w1, w2 = torch.exp(top - most), torch.exp(top2 - most)
        total, out = total * w1 + total2 * w2, out * w1[..., None] + out2 * w2[..., None]
    return dict(out=(out / total[..., None]).to(s.out.dtype))


def run(s):
    if own:
        return _run_own(s)
    return {"append": _plain_append, "read": _plain_read, "attn": _plain_attention, "prefix": _plain_attention}[s.case["op"]](s)


# --------------------------------------------------------------------------- work
def work(case):
    """Each token of K and V once (a group's prefix once for all), codes and scales; queries, outputs and table entries."""
    d, Hkv = case["d"], case["Hkv"]
    token = 4 * d * Hkv if case["kv"] == "bf16" else (2 * d + 8) * Hkv
    if case["op"] == "read":
        n = sum(_read_ranges(case)[1])
        esz = 4 if case["out"] == "f32" else 2
        return {"bytes": n * token + 2 * n * Hkv * d * esz + 4 * sum(map(_pages, _kv_lens(case))), "flops": 2 * n * Hkv * d}
    q_lens, kv_lens = _q_lens(case), _kv_lens(case)
    T = sum(q_lens)
    if case["op"] == "append":
        esz = 4 if case["src"] == "f32" else 2
        return {"bytes": 2 * T * Hkv * d * esz + T * token + 4 * (T + 2 * case["B"]), "flops": 6 * T * Hkv * d}
    shared = sum(_prefix_lens(case)) if case["op"] == "prefix" else 0
    own_tokens = sum(kv_lens)
    if case["op"] == "prefix":
        own_tokens -= sum(p * n for p, n in zip(_prefix_lens(case), _group_sizes(case)))
    nbytes = (shared + own_tokens) * token + 4 * (shared + own_tokens) // PAGE
    nbytes += T * case["Hq"] * d * (2 + (4 if case["out"] == "f32" else 2))
    return {"bytes": nbytes, "flops": sum(4 * n * q * case["Hq"] * d for n, q in zip(kv_lens, q_lens))}


# --------------------------------------------------------------------------- 64 bits
def _round_e4m3(x):
    """The nearest of the type's values, ties to the even one: 3 bits after the leading one, spacing 2^-9 at the least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _cell(slot, dim, pool):
    """Place of (slot, dim) in a page of one KV head: 8-bit K, 8-bit V, bf16 tiles of K and of V, token rows."""
    if pool == "k8":
        return dim // 16 * 256 + slot * 16 + dim % 16
    if pool == "v8":
        return ((dim // 64 * 4 + slot // 4) * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + slot % 4
    if pool == "k16":
        return dim // 8 * 128 + slot * 8 + dim % 8
    if pool == "v16":
        return (((dim // 32 * 4 + slot // 4) * 16 + dim % 16) * 2 + dim // 16 % 2) * 4 + slot % 4
    return None


def _tokens(s, pages, first, count, which):
    """K (0) or V (1) of `count` tokens from position `first` on, [Hkv, count, d] in 64 bits."""
    case = s.case
    d = case["d"]
    position = torch.arange(first, first + count, device="cuda")
    page, slot = pages[position // PAGE].long(), position % PAGE
    pool = (s.k_cache, s.v_cache)[which]
    if case["kv"] == "bf16" and case["layout"] == "tokens":
        return pool[page, :, slot].double().transpose(0, 1)
    cell = _cell(slot[:, None], torch.arange(d, device="cuda")[None, :], ("k", "v")[which] + ("16" if case["kv"] == "bf16" else "8"))
    flat = pool.view(torch.int16 if case["kv"] == "bf16" else torch.int8).view(pool.shape[0], case["Hkv"], PAGE * d)
    got = flat[page[:, None], :, cell]                      # [count, d, Hkv]
    got = got.view(pool.dtype).double().permute(2, 0, 1)
    if case["kv"] != "bf16":
        got = got * s.kv_scale[page, :, which, slot].double().transpose(0, 1)[..., None]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    d, Hkv = case["d"], case["Hkv"]
    if case["op"] == "append":
        most = MOST[case["kv"]]
        answer = dict(kv_scale=s.kv_scale.double())
        pools = [x.double().view(x.shape[0], Hkv, PAGE * d) for x in (s.k_cache, s.v_cache)]
        for b, n in enumerate(_q_lens(case)):
            position = torch.arange(int(s.host_kv_len[b]) - n, int(s.host_kv_len[b]), device="cuda")
            page, slot = s.table[b][position // PAGE].long(), position % PAGE
            for which, new in enumerate((s.new_k, s.new_v)):
                x = new[int(s.host_cu[b]):int(s.host_cu[b + 1])].double()
                scale = x.abs().amax(-1).clamp(min=SMALLEST_ROW) / most
                answer["kv_scale"][page, :, which, slot] = scale
                cell = _cell(slot[:, None], torch.arange(d, device="cuda")[None, :], ("k8", "v8")[which])
                x = x / scale[..., None]
                x = torch.round(x) if case["kv"] == "int8" else _round_e4m3(x)
                pools[which][page[:, None], :, cell] = x.transpose(1, 2)
        for name, pool, like in zip(("k_cache", "v_cache"), pools, (s.k_cache, s.v_cache)):
            answer[name] = None if case["kv"] == "int8" else pool.view(like.shape)
        return answer
    if case["op"] == "read":
        starts, counts = _read_ranges(case)
        got = [torch.cat([_tokens(s, s.table[b], a, n, w).transpose(0, 1) for b, (a, n) in enumerate(zip(starts, counts))])
               for w in (0, 1)]
        return dict(k=got[0], v=got[1])
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    group = case["Hq"] // Hkv
    for b, n in enumerate(s.host_kv_len.tolist()):
        lo, hi = int(s.host_cu[b]), int(s.host_cu[b + 1])
        m = hi - lo
        keys, values = (_tokens(s, s.table[b], 0, n, w) for w in (0, 1))
        rows = s.q[lo:hi].double().reshape(m, Hkv, group, d).transpose(0, 1).reshape(Hkv, m * group, d)
        score = torch.matmul(rows, keys.transpose(1, 2).contiguous()) / math.sqrt(d)
        last = n - m + torch.arange(m, device="cuda").repeat_interleave(group)
        score.masked_fill_(torch.arange(n, device="cuda")[None, None, :] > last[None, :, None], -math.inf)
        answer = torch.matmul(torch.softmax(score, -1), values.contiguous())
        out[lo:hi] = answer.reshape(Hkv, m, group, d).transpose(0, 1).reshape(m, case["Hq"], d)
    return dict(out=out)
