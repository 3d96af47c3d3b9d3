"""Performance cases of the operators around prompts and bounded caches.

A case is a dict of plain values.  `op` names the operator:

  rope    spec_qk_norm_rope: root-mean-square norms of each query and key head and the rotation by position, in one pass
  prompt  spec_prompt_attn: causal attention of any number of query rows a request over the paged cache, with each row's log-sum-exp
  weight  spec_kv_weight: the attention weight that every cached token gets from the given query rows
  evict   spec_kv_evict: the tokens with the largest weights, the first and the latest ones go into other pages in their order

With `own` false `run` computes the operators' plain form with elementary torch operations; with `own` true it
calls the library.  Lengths are derived from the case alone, so that a case has one amount of work; everything else
is drawn from the seed.

Pages hold 16 tokens of one request for all KV heads.  bf16 pages are rows of tokens ("tokens") or lie in the order of
the matrix instructions' operands ("tiles"); 8-bit pages have a float scale for each token's K and V row.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
MOST = {"e4m3": 448.0, "int8": 127.0}     # largest value of the type
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def listed():
    rope = dict(op="rope", dtype="bf16", norm=True, interleaved=False, fused=True, theta=500000.0)
    prompt = dict(op="prompt", kv="bf16", layout="tiles", out="bf16", lse=True, bucket=False)
    weight = dict(op="weight", kv="bf16", layout="tiles", add=True)
    evict = dict(op="evict", kv="bf16", layout="tiles")
    return [
        # One interactive user's verification step, k = 4: latency only.
        dict(rope, name="rope_one_step", B=1, qmin=5, qmax=5, past_min=686, past_max=686, Hq=64, Hkv=8, d=128, rot=128),
        # Packed prompts as slices of a fused projection.
        dict(rope, name="rope_prompts", B=6, qmin=700, qmax=5000, past_min=0, past_max=40, Hq=64, Hkv=8, d=128, rot=128),
        # A short instruction of one user.
        dict(prompt, name="prompt_one_short", B=1, qmin=77, qmax=77, past_min=0, past_max=0, Hq=32, Hkv=8, d=128),
        # Packed prompts of different lengths.
        dict(prompt, name="prompt_packed", B=6, qmin=700, qmax=5000, past_min=0, past_max=0, Hq=64, Hkv=8, d=128),
        # One long document.
        dict(prompt, name="prompt_long", B=1, qmin=16384, qmax=16384, past_min=0, past_max=0, Hq=64, Hkv=8, d=128),
        # Chunks of prompts behind what is in an 8-bit cache already.
        dict(prompt, name="prompt_chunks_e4m3", B=4, qmin=300, qmax=512, past_min=3000, past_max=20000, Hq=32, Hkv=8, d=128, kv="e4m3"),
        # Short prompts of a small model on token rows, fp32 output.
        dict(prompt, name="prompt_d64_tokens", B=16, qmin=20, qmax=600, past_min=0, past_max=100, Hq=16, Hkv=16, d=64, layout="tokens",
             out="f32"),
        # The last tokens of chunked prompts and single tokens, behind long contexts, under a length bucket.
        dict(prompt, name="prompt_few_rows", B=8, qmin=1, qmax=9, past_min=2000, past_max=30000, Hq=32, Hkv=8, d=128, bucket=True),
        # Which tokens of long prompts matter: seen from their last 32 rows.
        dict(weight, name="weight_window", B=4, qmin=32, qmax=32, past_min=4000, past_max=12000, Hq=64, Hkv=8, d=128, add=False),
        # A batch's verification step adds to the weights of an 8-bit cache.
        dict(weight, name="weight_step_e4m3", B=64, qmin=5, qmax=5, past_min=1000, past_max=3000, Hq=32, Hkv=8, d=128, kv="e4m3"),
        # One request's cache is cut down.
        dict(evict, name="evict_one", B=1, lmin=2100, lmax=2100, keep=512, first=4, recent=64, Hkv=8, d=128),
        # A batch's 8-bit caches, long contexts.
        dict(evict, name="evict_batch_e4m3", B=16, lmin=6000, lmax=30000, keep=4096, first=4, recent=256, Hkv=8, d=128, kv="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "prompt", "prompt", "weight", "evict"])
    Hq, Hkv, d = rng.choice([(32, 32, 128), (32, 8, 128), (64, 8, 128), (64, 4, 128), (16, 16, 64), (32, 8, 64)])
    kv = rng.choice(["bf16", "bf16", "e4m3", "int8"])
    layout = rng.choice(["tiles", "tokens"]) if kv == "bf16" else "tiles"
    spread = rng.choice([0.0, 0.3, 0.9])

    def around(mean, least):
        return max(least, int(mean * (1 - spread))), max(least, int(mean * (1 + spread)))

    if op == "rope":
        B = _log_int(rng, 1, 256)
        qmin, qmax = around(_log_int(rng, 1, max(2, int(60e6 / (B * (Hq + Hkv) * d)))), 1)
        past_min, past_max = around(_log_int(rng, 1, 500000), 0)
        return dict(op=op, B=B, qmin=qmin, qmax=qmax, past_min=past_min, past_max=past_max, Hq=Hq, Hkv=Hkv, d=d,
                    rot=rng.choice([d, d, d // 2, d // 4]), dtype=rng.choice(["bf16", "bf16", "f32"]), norm=rng.random() < 0.6,
                    interleaved=rng.random() < 0.4, fused=rng.random() < 0.6, theta=rng.choice([10000.0, 500000.0]))
    if op == "evict":
        B = _log_int(rng, 1, 64)
        lmin, lmax = around(_log_int(rng, 64, max(80, min(32768, int(300e6 / (B * Hkv * d))))), 1)
        keep = _log_int(rng, 16, max(20, lmax))
        return dict(op=op, B=B, lmin=lmin, lmax=lmax, keep=keep, first=rng.choice([0, 1, 4, 20]), recent=rng.choice([0, 1, 64, 300]), Hkv=Hkv, d=d,
                    kv=kv, layout=layout)
    few = rng.random() < 0.35       # a step's rows, or the last ones of a prompt
    B = _log_int(rng, 1, 64)
    if few:
        qmin, qmax = around(rng.randint(1, 40), 1)
        past_min, past_max = around(_log_int(rng, 1, max(2, min(32768, int(60e6 / (B * Hkv * d))))), 0)
    else:       # pairs of tokens bounded: a long case is no more than half of the longest listed one
        pairs = 1.2e8 * 64 * 128 / (Hq * d) / 2 / (1 + spread) ** 2
        q = _log_int(rng, 8, int(max(16, min(12000, math.sqrt(pairs / B), 5e7 / (B * Hq * d) * 4))))
        qmin, qmax = around(q, 1)
        past_min, past_max = rng.choice([(0, 0), (0, 0), around(_log_int(rng, 1, max(2, min(20000, int(pairs / 2 / (B * q)), int(60e6 / (B * Hkv * d))))), 0)])
    case = dict(op=op, B=B, qmin=qmin, qmax=qmax, past_min=past_min, past_max=past_max, Hq=Hq, Hkv=Hkv, d=d, kv=kv, layout=layout)
    if op == "weight":
        return dict(case, add=rng.random() < 0.5)
    return dict(case, out=rng.choice(["bf16", "bf16", "f32"]), lse=rng.random() < 0.5, bucket=few and rng.random() < 0.4)


# --------------------------------------------------------------------------- lengths: from the case alone
def _some(salt, n, lo, hi):
    rng = random.Random("%s %d %d %d" % (salt, n, lo, hi))
    return [rng.randint(lo, hi) for _ in range(n)]


def _prefix_sum(values):
    sums = [0]
    for n in values:
        sums.append(sums[-1] + n)
    return sums


def _q_lens(case):
    return _some("rows", case["B"], case["qmin"], case["qmax"])


def _kv_lens(case):
    if case["op"] == "evict":
        return _some("kv", case["B"], case["lmin"], case["lmax"])
    return [a + n for a, n in zip(_some("past", case["B"], case["past_min"], case["past_max"]), _q_lens(case))]


def _pages(n):
    return (n + PAGE - 1) // PAGE


# --------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _values(shape, g):
    """Rows whose magnitude varies from token to token (a factor of e^(0.4 N(0, 1)), the last dimension is a row)."""
    x = torch.randn(shape, dtype=torch.float32, device="cuda", generator=g)
    return x * torch.exp(0.4 * torch.randn(shape[:-1] + (1,), dtype=torch.float32, device="cuda", generator=g))


def _codes(shape, kv, g):
    """8-bit rows and their scales.  Normal values are normal values in any order of a page's elements."""
    rows = _values(shape, g)
    most = rows.abs().amax(-1).clamp(min=1e-6)
    codes = rows * (MOST[kv] / most)[..., None]
    codes = torch.round(codes).clamp(-127, 127) if kv == "int8" else codes.clamp(-448, 448)
    return codes.to(TYPE[kv]), most / MOST[kv]


class _State:
    pass


def _tables(case, g):
    """Shuffled block tables over a pool with a quarter of its pages spare: the requests' pages, and those that an eviction fills."""
    counts = [_pages(n) for n in _kv_lens(case)]
    new = [_pages(min(n, case["keep"])) for n in _kv_lens(case)] if case["op"] == "evict" else []
    need = sum(counts) + sum(new)
    blocks = need + (need + 3) // 4
    order = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)
    tables, at = [], 0
    for rows in (counts, new):
        if not rows:
            continue
        starts = at + np.cumsum([0] + rows[:-1])
        index = torch.from_numpy(starts)[:, None] + torch.arange(max(rows))[None, :]
        used = torch.arange(max(rows))[None, :] < torch.tensor(rows)[:, None]
        tables.append(order[torch.where(used, index, 0).cuda()].contiguous())
        at += sum(rows)
    return tables, blocks


def _pools(s, case, blocks, g):
    """A pool whose every page holds tokens: the requests' and other requests'."""
    shape = (blocks, case["Hkv"], PAGE, case["d"])
    s.kv_scale = None
    if case["kv"] == "bf16":
        s.k_cache, s.v_cache = (_values(shape, g).to(torch.bfloat16) for _ in range(2))
    else:
        (s.k_cache, k_scale), (s.v_cache, v_scale) = (_codes(shape, case["kv"], g) for _ in range(2))
        s.kv_scale = torch.stack([k_scale, v_scale], 2).contiguous()


def prepare(case, seed):
    s, g = _State(), _gen(seed, 1)
    s.case, s.handle, s.workspace = case, None, None
    s.host_kv_len = np.array(_kv_lens(case), dtype=np.int32)
    s.kv_len = torch.from_numpy(s.host_kv_len).cuda()
    Hkv, d = case["Hkv"], case["d"]
    if case["op"] != "evict":
        s.host_cu = np.array(_prefix_sum(_q_lens(case)), dtype=np.int32)
        s.cu = torch.from_numpy(s.host_cu).cuda()
        T, Hq = int(s.host_cu[-1]), case["Hq"]
        b = torch.searchsorted(s.cu[1:].contiguous(), torch.arange(T, device="cuda", dtype=torch.int32), right=True)
        s.positions = (s.kv_len[b].long() - s.cu[1:][b].long() + torch.arange(T, device="cuda")).to(torch.int32)
    if case["op"] == "rope":
        heads = Hq + 2 * Hkv if case["fused"] else Hq + Hkv
        rows = _values((T, heads, d), g).to(TYPE[case["dtype"]])
        s.q, s.k = rows[:, :Hq], rows[:, Hq:Hq + Hkv]
        if not case["fused"]:
            s.q, s.k = s.q.contiguous(), s.k.contiguous()
        s.out_q, s.out_k = (torch.zeros((T, n, d), dtype=rows.dtype, device="cuda") for n in (Hq, Hkv))
        s.inv_freq = (case["theta"] ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])).float()
        s.q_weight = s.k_weight = None
        if case["norm"]:
            s.q_weight, s.k_weight = ((1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(rows.dtype) for _ in range(2))
        return s
    tables, blocks = _tables(case, g)
    s.table = tables[0]
    _pools(s, case, blocks, g)
    if case["op"] == "evict":
        # accumulated weights: a few tokens have most of it
        s.weight = torch.exp(1.5 * torch.randn((blocks, Hkv, PAGE), dtype=torch.float32, device="cuda", generator=g))
        s.new_table = tables[1]
        s.keep = torch.full((case["B"],), case["keep"], dtype=torch.int32, device="cuda")
        s.new_kv_len = torch.zeros_like(s.keep)
        s.kept = torch.zeros((case["B"], s.new_table.shape[1] * PAGE), dtype=torch.int32, device="cuda")
        return s
    s.q = torch.randn((T, Hq, d), dtype=torch.float32, device="cuda", generator=g).to(torch.bfloat16)
    if case["op"] == "weight":
        s.lse = _plain_attention(s, False)[1]
        s.weight = torch.zeros((blocks, Hkv, PAGE), dtype=torch.float32, device="cuda")
        s.before = torch.rand((blocks, Hkv, PAGE), dtype=torch.float32, device="cuda", generator=g) if case["add"] else None
        return s
    s.out = torch.zeros((T, Hq, d), dtype=TYPE[case["out"]], device="cuda")
    s.lse = torch.zeros((T, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
    s.bound = 0
    if case["bucket"]:      # a bucket's table has room for its longest request
        s.bound = (int(s.host_kv_len.max()) + 255) // 256 * 256
        s.table = torch.nn.functional.pad(s.table, (0, s.bound // PAGE - s.table.shape[1])).contiguous()
    return s


# --------------------------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_2406_14066_amd import spec_verify as sv
    case = s.case
    op = case["op"]
    if s.handle is None:        # what a serving loop makes once for its buffers: argument structs and the workspace
        layout = sv.KV_TOKEN_MAJOR if case.get("layout") == "tokens" else sv.KV_MFMA
        if op == "rope":
            s.handle = sv.make_qk_norm_rope_args(s.q, s.k, s.out_q, s.out_k, s.positions, s.inv_freq, q_weight=s.q_weight, k_weight=s.k_weight,
                                                 eps=1e-6, interleaved=case["interleaved"])
        elif op == "prompt":
            s.handle = sv.make_prompt_attn_args(s.q, s.k_cache, s.v_cache, s.table, s.kv_len, s.cu, s.out, s.host_kv_len, s.host_cu, lse=s.lse,
                                                kv_scale=s.kv_scale, kv_layout=layout, max_kv_len=s.bound)
            s.workspace = sv.alloc_workspace(sv.spec_prompt_attn_workspace_bytes(s.handle[0]))
        elif op == "weight":
            s.handle = sv.make_kv_weight_args(s.q, s.lse, s.k_cache, s.table, s.kv_len, s.cu, s.weight, s.host_kv_len, s.host_cu,
                                              weight_in=s.before, kv_scale=s.kv_scale, kv_layout=layout)
        else:
            s.handle = sv.make_kv_evict_args(s.k_cache, s.v_cache, s.weight, s.table, s.kv_len, s.keep, s.new_table, s.new_kv_len, s.host_kv_len,
                                             kept=s.kept, first=case["first"], recent=case["recent"], kv_scale=s.kv_scale, kv_layout=layout)
            s.workspace = sv.alloc_workspace(sv.spec_kv_evict_workspace_bytes(s.handle[0]))
    if op == "rope":
        sv.spec_qk_norm_rope(s.handle[0])
        return dict(q=s.out_q, k=s.out_k)
    if op == "prompt":
        sv.spec_prompt_attn(s.handle[0], s.workspace)
        return dict(out=s.out, lse=s.lse) if case["lse"] else dict(out=s.out)
    if op == "weight":
        sv.spec_kv_weight(s.handle[0])
        return dict(weight=s.weight)
    sv.spec_kv_evict(s.handle[0], s.workspace)
    return _evicted(s)


def _evicted(s):
    got = dict(new_kv_len=s.new_kv_len, kept=s.kept, k_cache=s.k_cache, v_cache=s.v_cache, weight=s.weight)
    return got if s.kv_scale is None else dict(got, kv_scale=s.kv_scale)


# --------------------------------------------------------------------------- the plain form
def _plain_rope(s):
    case = s.case
    rot, outs = case["rot"], []
    angle = s.positions.double()[:, None] * s.inv_freq.double()[None, :]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for x, weight in ((s.q, s.q_weight), (s.k, s.k_weight)):
        y = x.float()
        if case["norm"]:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
        turned, rest = y[..., :rot], y[..., rot:]
        if case["interleaved"]:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = turned[..., :rot // 2], turned[..., rot // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        outs.append(torch.cat([turned, rest], -1).to(x.dtype))
    return dict(q=outs[0], k=outs[1])


def _rows_of_pages(s, pool, which, pages):
    """K (0) or V (1) of the pages [..., P] as [..., Hkv, P * 16, d] in 32 bits."""
    case = s.case
    Hkv, d = case["Hkv"], case["d"]
    x = pool[pages.reshape(-1).long()].float()
    n = x.shape[0]
    if case["kv"] != "bf16":
        if which == 0:
            x = x.view(n, Hkv, d // 16, PAGE, 16).permute(0, 1, 3, 2, 4)
        else:
            x = x.view(n, Hkv, d // 64, 4, 16, 4, 4).permute(0, 1, 3, 6, 2, 5, 4)
        x = x.reshape(n, Hkv, PAGE, d) * s.kv_scale[pages.reshape(-1).long()][:, :, which, :, None]
    elif case["layout"] == "tiles":
        if which == 0:
            x = x.view(n, Hkv, d // 8, PAGE, 8).permute(0, 1, 3, 2, 4)
        else:
            x = x.view(n, Hkv, d // 32, 4, 16, 2, 4).permute(0, 1, 3, 6, 2, 5, 4)
    x = x.reshape(pages.shape + (Hkv, PAGE, d))
    return x.transpose(-4, -3).reshape(pages.shape[:-1] + (Hkv, -1, d)).contiguous()


def _scores(s, first, count, k):
    """Scores [B, Hkv, count * group, tokens] of the rows first .. first + count - 1 of every request, masked; and where those rows are."""
    case = s.case
    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    j = first + torch.arange(count, device="cuda")
    q_len = (s.cu[1:] - s.cu[:-1]).long()
    at = s.cu[:-1].long()[:, None] + torch.minimum(j[None, :], q_len[:, None] - 1)
    q = s.q[at].float().view(B, count, Hkv, Hq // Hkv, d).transpose(1, 2).reshape(B, Hkv, -1, d)
    score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    last = (s.kv_len.long() - q_len)[:, None] + j[None, :]
    hidden = torch.arange(k.shape[2], device="cuda")[None, None, :] > last[:, :, None]
    score.view(B, Hkv, count, Hq // Hkv, -1).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    return score, at, j[None, :] < q_len[:, None]


def _row_blocks(s, tokens):
    """Query rows go in blocks that keep the scores within memory."""
    most = int(np.diff(s.host_cu).max())
    step = max(1, min(most, int(2 ** 30 / (s.case["B"] * s.case["Hq"] * tokens))))
    return [(i, min(step, most - i)) for i in range(0, most, step)]


def _plain_attention(s, values=True):
    case = s.case
    B, Hq, Hkv, d, T = case["B"], case["Hq"], case["Hkv"], case["d"], s.q.shape[0]
    pages = s.table[:, :_pages(int(s.host_kv_len.max()))]
    k = _rows_of_pages(s, s.k_cache, 0, pages)
    v = _rows_of_pages(s, s.v_cache, 1, pages) if values else None
    out = torch.empty((T, Hq, d), dtype=torch.float32, device="cuda") if values else None
    lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
    for first, count in _row_blocks(s, k.shape[2]):
        score, at, real = _scores(s, first, count, k)
        top = score.amax(-1, keepdim=True)
        weight = score.sub_(top).exp_()
        total = weight.sum(-1, keepdim=True)

        def rows(x):
            return x.view(B, Hkv, count, Hq // Hkv, -1).transpose(1, 2).reshape(B, count, Hq, -1)[real]

        lse[at[real]] = rows(top + total.log())[..., 0]
        if values:
            out[at[real]] = rows(torch.matmul(weight, v) / total)
    return (out.to(s.out.dtype) if values else None), lse


def _plain_weight(s):
    case = s.case
    B, Hq, Hkv = case["B"], case["Hq"], case["Hkv"]
    k = _rows_of_pages(s, s.k_cache, 0, s.table)
    sums = torch.zeros((B, Hkv, k.shape[2]), dtype=torch.float32, device="cuda")
    for first, count in _row_blocks(s, k.shape[2]):
        score, at, real = _scores(s, first, count, k)
        lse = s.lse[at].masked_fill(~real[:, :, None], math.inf)
        lse = lse.view(B, count, Hkv, Hq // Hkv).transpose(1, 2).reshape(B, Hkv, -1, 1)
        sums += score.sub_(lse).exp_().sum(2)
    token = torch.arange(k.shape[2], device="cuda")
    b, t = torch.nonzero(token[None, :] < s.kv_len[:, None], as_tuple=True)
    page, slot, new = s.table[b, t // PAGE].long(), t % PAGE, sums[b, :, t]
    if s.before is not None:
        past = (s.kv_len - (s.cu[1:] - s.cu[:-1]))[b] > t
        new = new + torch.where(past[:, None], s.before[page, :, slot], 0.0)
    s.weight[page, :, slot] = new
    return dict(weight=s.weight)


def _cell(case, slot, dim, which):
    """Place of (slot, dim) in a KV head's page."""
    if case["kv"] != "bf16":
        return dim // 16 * 256 + slot * 16 + dim % 16 if which == 0 else ((dim // 64 * 4 + slot // 4) * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + slot % 4
    if case["layout"] == "tokens":
        return slot * case["d"] + dim
    return dim // 8 * 128 + slot * 8 + dim % 8 if which == 0 else (((dim // 32 * 4 + slot // 4) * 16 + dim % 16) * 2 + dim // 16 % 2) * 4 + slot % 4


def _bits(pool):
    return pool.view(torch.int16 if pool.element_size() == 2 else torch.uint8)


def _plain_evict(s):
    case = s.case
    B, Hkv, d, n = case["B"], case["Hkv"], case["d"], s.table.shape[1] * PAGE
    t = torch.arange(n, device="cuda")[None, :]
    kv_len, keep = s.kv_len.long()[:, None], s.keep.long()[:, None]
    first = keep.clamp(max=case["first"])
    recent = torch.minimum(keep - first, torch.full_like(keep, case["recent"]))
    score = s.weight[s.table.long()].double().sum(2).view(B, n).float()
    score = torch.where((t < first) | (t >= kv_len - recent), math.inf, score).masked_fill(t >= kv_len, -math.inf)
    order = torch.sort(score, dim=1, descending=True, stable=True).indices
    new_len = torch.minimum(kv_len, keep)
    chosen = torch.where(t < new_len, order, n)[:, :s.kept.shape[1]].sort(1).values
    s.kept.fill_(-1)
    s.kept[:, :chosen.shape[1]] = torch.where(chosen < n, chosen, -1)
    s.new_kv_len.copy_(new_len[:, 0])
    b, i = torch.nonzero(chosen < n, as_tuple=True)
    t = chosen[b, i]
    page, slot, new_page, new_slot = s.table[b, t // PAGE].long(), t % PAGE, s.new_table[b, i // PAGE].long(), i % PAGE
    dim, head = torch.arange(d, device="cuda")[None, None, :], torch.arange(Hkv, device="cuda")[None, :, None]
    for pool, which in ((s.k_cache, 0), (s.v_cache, 1)):
        flat = _bits(pool).view(pool.shape[0], Hkv, PAGE * d)
        flat[new_page[:, None, None], head, _cell(case, new_slot[:, None, None], dim, which)] = \
            flat[page[:, None, None], head, _cell(case, slot[:, None, None], dim, which)]
    s.weight[new_page, :, new_slot] = s.weight[page, :, slot]
    if s.kv_scale is not None:
        s.kv_scale[new_page, :, :, new_slot] = s.kv_scale[page, :, :, slot]
    return _evicted(s)


def run(s):
    if own:
        return _run_own(s)
    op = s.case["op"]
    if op == "prompt":
        out, lse = _plain_attention(s)
        return dict(out=out, lse=lse) if s.case["lse"] else dict(out=out)
    return {"rope": _plain_rope, "weight": _plain_weight, "evict": _plain_evict}[op](s)


# --------------------------------------------------------------------------- work
def work(case):
    """Each row, and each token of K and V (or of K alone), once; codes with their scales; products of visible pairs only."""
    d, Hkv, kv_lens = case["d"], case["Hkv"], _kv_lens(case)
    if case["op"] == "evict":
        token = (4 * d if case["kv"] == "bf16" else 2 * d + 8) + 4
        kept = sum(min(n, case["keep"]) for n in kv_lens)
        return {"bytes": sum(kv_lens) * (4 * Hkv + 0.25) + 2 * kept * Hkv * token + 4 * kept, "flops": sum(kv_lens) * Hkv}
    Hq, q_lens = case["Hq"], _q_lens(case)
    T = sum(q_lens)
    if case["op"] == "rope":
        elements = T * (Hq + Hkv) * d
        return {"bytes": 2 * elements * (4 if case["dtype"] == "f32" else 2) + 4 * T, "flops": elements * (8 if case["norm"] else 3)}
    pairs = sum(q * (n - q) + q * (q + 1) // 2 for q, n in zip(q_lens, kv_lens))
    row = 2 * d if case["kv"] == "bf16" else d + 4      # of K or V
    if case["op"] == "weight":
        return {"bytes": sum(kv_lens) * Hkv * (row + (8 if case["add"] else 4)) + T * Hq * (2 * d + 4), "flops": 2 * d * Hq * pairs}
    return {"bytes": sum(kv_lens) * Hkv * 2 * row + T * Hq * (2 * d + (4 if case["out"] == "f32" else 2) * d + (4 if case["lse"] else 0)),
            "flops": 4 * d * Hq * pairs}


# --------------------------------------------------------------------------- 64 bits
def _token_rows(s, b, which, first, last):
    """K (0) or V (1) of request b's tokens first .. last - 1, [Hkv, n, d] in 64 bits."""
    case = s.case
    pool = (s.k_cache, s.v_cache)[which]
    t = torch.arange(first, last, device="cuda")
    page, slot = s.table[b][t // PAGE].long(), t % PAGE
    flat = _bits(pool).view(pool.shape[0], case["Hkv"], PAGE * case["d"])
    got = flat[page[:, None], :, _cell(case, slot[:, None], torch.arange(case["d"], device="cuda")[None, :], which)]      # [n, d, Hkv]
    got = got.view(pool.dtype).double().permute(2, 0, 1)
    if case["kv"] != "bf16":
        got = got * s.kv_scale[page, :, which, slot].double().t()[..., None]
    return got.contiguous()


def _exact_rope(s):
    case, answer = s.case, {}
    half, T = case["rot"] // 2, s.positions.shape[0]
    turn = torch.polar(torch.ones((T, half), dtype=torch.float64, device="cuda"), s.positions.double()[:, None] * s.inv_freq.double())[:, None]
    index = torch.arange(half, device="cuda")
    one, two = (2 * index, 2 * index + 1) if case["interleaved"] else (index, index + half)
    for name, x, weight in (("q", s.q, s.q_weight), ("k", s.k, s.k_weight)):
        y = x.double()
        if weight is not None:
            y = y * (y.square().sum(-1, keepdim=True) / case["d"] + 1e-6).rsqrt() * weight.double()
        z = torch.complex(y[..., one], y[..., two]) * turn
        y = y.clone()
        y[..., one], y[..., two] = z.real, z.imag
        answer[name] = y
    return answer


def _exact_rows(s, b, first, count, keys):
    """Scores of `count` query rows of request b from its row `first` on, [Hkv, group, count, tokens] in 64 bits."""
    case = s.case
    lo, n, m = int(s.host_cu[b]) + first, int(s.host_kv_len[b]), int(s.host_cu[b + 1] - s.host_cu[b])
    q = s.q[lo:lo + count].double().permute(1, 0, 2).reshape(case["Hkv"], -1, case["d"])
    score = torch.matmul(q, keys.transpose(1, 2).contiguous()).view(case["Hkv"], -1, count, n) / math.sqrt(case["d"])
    late = torch.arange(n, device="cuda") > (n - m + first + torch.arange(count, device="cuda"))[:, None]
    return score.masked_fill_(late, -math.inf)


def _exact_evict(s):
    """The definition request by request: a token stays if it is protected or enough of the others weigh less."""
    case = s.case
    flats = [p.double().view(p.shape[0], case["Hkv"], -1) for p in (s.k_cache, s.v_cache)]
    weight, scale = s.weight.double(), None if s.kv_scale is None else s.kv_scale.double()
    dim = torch.arange(case["d"], device="cuda")[None, None, :]
    head = torch.arange(case["Hkv"], device="cuda")[None, :, None]
    moves = []
    for b, n in enumerate(s.host_kv_len.tolist()):
        keep = min(n, case["keep"])
        first = min(keep, case["first"])
        recent = min(keep - first, case["recent"])
        t = torch.arange(n, device="cuda")
        score = s.weight[s.table[b].long()].double().sum(1).reshape(-1)[:n].float().cpu().numpy()
        middle = np.arange(first, n - recent)
        best = middle[np.lexsort((middle, -score[middle]))][:keep - first - recent]
        t = torch.from_numpy(np.sort(np.concatenate([np.arange(first), best, np.arange(n - recent, n)]))).cuda()
        i = torch.arange(keep, device="cuda")
        moves.append((s.table[b][t // PAGE].long(), t % PAGE, s.new_table[b][i // PAGE].long(), i % PAGE))
    page, slot, new_page, new_slot = (torch.cat(x) for x in zip(*moves))
    for which, flat in enumerate(flats):
        flat[new_page[:, None, None], head, _cell(case, new_slot[:, None, None], dim, which)] = \
            flat[page[:, None, None], head, _cell(case, slot[:, None, None], dim, which)]
    weight[new_page, :, new_slot] = weight[page, :, slot]
    answer = dict(new_kv_len=None, kept=None, weight=weight)
    for name, flat, pool in zip(("k_cache", "v_cache"), flats, (s.k_cache, s.v_cache)):
        answer[name] = None if case["kv"] == "int8" else flat.view(pool.shape)
    if scale is not None:
        scale[new_page, :, :, new_slot] = scale[page, :, :, slot]
        answer["kv_scale"] = scale
    return answer


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(s)
    if case["op"] == "evict":
        return _exact_evict(s)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    if case["op"] == "weight":
        weight = s.weight.double()
    else:
        out, lse = (torch.empty(shape, dtype=torch.float64, device="cuda") for shape in (s.q.shape, s.q.shape[:2]))
    for b, n in enumerate(s.host_kv_len.tolist()):
        lo, m = int(s.host_cu[b]), int(s.host_cu[b + 1] - s.host_cu[b])
        keys = _token_rows(s, b, 0, 0, n)
        values = _token_rows(s, b, 1, 0, n) if case["op"] == "prompt" else None
        step = max(1, min(m, int(2 ** 28 / (Hq * n))))
        got = torch.zeros((Hkv, n), dtype=torch.float64, device="cuda")
        for first in range(0, m, step):
            count = min(step, m - first)
            score = _exact_rows(s, b, first, count, keys)
            rows = slice(lo + first, lo + first + count)
            if case["op"] == "weight":
                got += torch.exp(score - s.lse[rows].double().t().reshape(Hkv, -1, count, 1)).sum((1, 2))
                continue
            total = torch.logsumexp(score, -1, keepdim=True)
            lse[rows] = total.reshape(Hq, count).t()
            answer = torch.matmul(torch.exp(score - total).view(Hkv, -1, n), values)
            out[rows] = answer.view(Hq, count, d).transpose(0, 1)
        if case["op"] == "weight":
            t = torch.arange(n, device="cuda")
            page, slot = s.table[b][t // PAGE].long(), t % PAGE
            if s.before is not None:
                got[:, :n - m] += s.before[page, :, slot].double().t()[:, :n - m]
            weight[page, :, slot] = got.t()
    if case["op"] == "weight":
        return dict(weight=weight)
    return dict(out=out, lse=lse) if case["lse"] else dict(out=out)
