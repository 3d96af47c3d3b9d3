"""Eviction by accumulated weight: which tokens stay, and that everything of theirs goes with them and nothing else changes."""
import numpy as np
import pytest

import prompt_reference as R
from paper_2406_14066_amd import spec_verify as sv
from test_gpu_prompt_attn import _i32

pytestmark = pytest.mark.gpu

KINDS = R.KINDS + ["f32"]


def _raw(t):
    import torch
    n = t.element_size()
    return t.view(torch.uint8 if n == 1 else torch.int16 if n == 2 else torch.int32).cpu().numpy().reshape(t.shape[0], t.shape[1], -1).copy()


def run(cache, weight, table, kv_len, keep, new_table, first, recent, *, bucket=0, host_kv=True, kept=True, fill=0xA5, args_only=False):
    import torch
    k, v, sc = cache.device()
    w = torch.from_numpy(weight).cuda()
    B = len(kv_len)
    new_len = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    kp = torch.full((B, 16 * new_table.shape[1]), 77, dtype=torch.int32, device="cuda") if kept else None
    errors = torch.zeros(1, dtype=torch.int64, device="cuda")
    hk = np.asarray(kv_len, dtype=np.int32)
    args, keepalive = sv.make_kv_evict_args(k, v, w, _i32(table), _i32(hk), _i32(keep), _i32(new_table), new_len, hk if host_kv else None, kept=kp, first=first,
                                            recent=recent, kv_scale=sc, kv_layout=sv.KV_TOKEN_MAJOR if cache.kind in ("tokens", "f32") else sv.KV_MFMA,
                                            max_kv_len=bucket, error_count=errors)
    ws = sv.alloc_workspace(sv.spec_kv_evict_workspace_bytes(args))
    ws.fill_(fill)
    state = dict(k=k, v=v, scale=sc, weight=w, new_len=new_len, kept=kp, errors=errors)
    if args_only:
        return args, keepalive, ws, state
    sv.spec_kv_evict(args, ws)
    torch.cuda.synchronize()
    return state


def check(state, cache, weight, table, kv_len, keep, new_table, first, recent, left_out=()):
    """Bit for bit: the pools are what copying the chosen tokens by hand makes of them."""
    pools = [cache.pool[0].copy(), cache.pool[1].copy()]
    scale = None if cache.scale is None else cache.scale.copy()
    want_w = weight.copy()
    width = 16 * new_table.shape[1]
    want_len, want_kept = np.zeros(len(kv_len), dtype=np.int32), np.full((len(kv_len), width), -1, dtype=np.int32)
    for b, n in enumerate(kv_len):
        if b in left_out:
            want_len[b] = -1
            continue
        stay = R.choose(weight, table[b], n, keep[b], first, recent, cache.nb)
        want_len[b] = len(stay)
        want_kept[b, :len(stay)] = stay
        for i, t in enumerate(stay):
            src, dst = table[b, t // 16], new_table[b, i // 16]
            if not 0 <= dst < cache.nb:
                continue
            inside = 0 <= src < cache.nb
            for w in range(2):
                at = R.cells(cache.kind, cache.d, w)
                pools[w][dst][:, at[i % 16]] = cache.pool[w][src][:, at[t % 16]] if inside else 0
            want_w[dst, :, i % 16] = weight[src, :, t % 16] if inside else 0
            if scale is not None:
                scale[dst, :, :, i % 16] = cache.scale[src, :, :, t % 16] if inside else 0
    assert (state["new_len"].cpu().numpy() == want_len).all()
    if state["kept"] is not None:
        assert (state["kept"].cpu().numpy() == want_kept).all()
    for w, name in enumerate("kv"):
        assert (_raw(state[name]) == pools[w].view(_raw(state[name]).dtype)).all(), name
    np.testing.assert_array_equal(state["weight"].cpu().numpy(), want_w)
    if scale is not None:
        np.testing.assert_array_equal(state["scale"].cpu().numpy(), scale)


CASES = [
    # (name, kv_len, keep, first, recent, Hkv, d)
    ("one", [100], [37], 4, 8, 2, 128),
    ("edges", [16, 17, 31, 32, 33, 1, 0], [16, 16, 17, 1, 32, 1, 5], 1, 2, 1, 64),
    ("nothing_to_do", [20, 64, 5], [20, 100, 64], 4, 8, 3, 128),
    ("keep_none", [40, 50], [0, 3], 4, 8, 2, 64),
    ("protected_alone", [90, 70], [12, 20], 4, 8, 2, 128),
    ("protected_more_than_kept", [90, 70], [6, 3], 4, 100, 2, 64),
    ("no_protection", [500, 333], [100, 320], 0, 0, 4, 128),
    ("long", [5000, 9000], [1000, 8190], 16, 64, 1, 64),
]
LONG_CASES = [   # (lengths concern the choice alone: two kinds of pools)
    ("longer", [20000, 17], [300, 20], 4, 64, 1, 64),
    ("longest", [70001, 40000], [500, 33000], 4, 1000, 1, 64),      # the choice fetches scores again for each pass
]
EACH = [pytest.param(*c, kind, id="%s-%s" % (c[0], kind)) for c in CASES for kind in KINDS]
EACH += [pytest.param(*c, kind, id="%s-%s" % (c[0], kind)) for c in LONG_CASES for kind in ("tiles", "int8")]


@pytest.mark.parametrize("name,kv_len,keep,first,recent,Hkv,d,kind", EACH)
def test_matches_the_definition(name, kv_len, keep, first, recent, Hkv, d, kind):
    print("case kv_evict", name, kind, flush=True)
    rng = np.random.default_rng(41)
    (table, new_table), nb = R.tables(rng, kv_len, more=[[min(n, k) for n, k in zip(kv_len, keep)]])
    cache = R.Cache(rng, nb, Hkv, d, kind)
    weight = np.exp(1.5 * rng.standard_normal((nb, Hkv, 16))).astype(np.float32)
    check(run(cache, weight, table, kv_len, keep, new_table, first, recent), cache, weight, table, kv_len, keep, new_table, first, recent)
    check(run(cache, weight, table, kv_len, keep, new_table, first, recent, kept=False, fill=0xFF), cache, weight, table, kv_len, keep, new_table, first, recent)


@pytest.mark.parametrize("what", ["all_equal", "few_values", "zeros_of_both_signs", "negative", "odd", "tiny", "huge"])
def test_ties_and_odd_weights(what):
    """Equal scores: the earlier token stays.  NaN below everything, infinities above and below; scores below fp32's normal numbers are told apart."""
    rng = np.random.default_rng(42)
    kv_len, keep, Hkv, d = [3000, 200, 77], [700, 50, 30], 3, 64
    (table, new_table), nb = R.tables(rng, kv_len, more=[keep])
    cache = R.Cache(rng, nb, Hkv, d, "tokens")
    shape = (nb, Hkv, 16)
    weight = {
        "all_equal": lambda: np.full(shape, 0.25),
        "few_values": lambda: rng.integers(0, 3, shape) / 2.0,
        "zeros_of_both_signs": lambda: np.where(rng.random(shape) < 0.5, 0.0, -0.0) + (rng.random(shape) < 0.03),
        "negative": lambda: rng.standard_normal(shape),
        "odd": lambda: np.where(rng.random(shape) < 0.1, rng.choice([np.nan, np.inf, -np.inf], shape), rng.random(shape)),
        "tiny": lambda: rng.integers(0, 5, shape) * 2.0 ** -149,
        "huge": lambda: rng.random(shape) * 3e38,
    }[what]().astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        check(run(cache, weight, table, kv_len, keep, new_table, 2, 5), cache, weight, table, kv_len, keep, new_table, 2, 5)


def test_sums_are_in_64_bits_and_rounded_once():
    """2^24 + 1 + 1 + ..: in 32 bits the ones would be lost."""
    rng = np.random.default_rng(43)
    Hkv, d, kv_len, keep = 8, 64, [64], [16]
    (table, new_table), nb = R.tables(rng, kv_len, more=[keep])
    cache = R.Cache(rng, nb, Hkv, d, "tiles")
    weight = np.zeros((nb, Hkv, 16), dtype=np.float32)
    for t in range(64):
        weight[table[0, t // 16], 0, t % 16] = 2.0 ** 24
        weight[table[0, t // 16], 1:1 + t % 8, t % 16] = 1.0
    check(run(cache, weight, table, kv_len, keep, new_table, 0, 0), cache, weight, table, kv_len, keep, new_table, 0, 0)


def test_findings():
    """Lengths and budgets that do not fit leave a request out; bad pages are skipped or read as zeros, and counted by the token."""
    import torch
    rng = np.random.default_rng(44)
    kv_len, Hkv, d, bound = [100, 100, 100, 100, 100], 2, 64, 112
    keep = [40, 40, -1, 49, 40]
    (table, new_table), nb = R.tables(rng, kv_len, columns=7, more=[[48] * 5])
    new_table = np.ascontiguousarray(new_table[:, :3])
    cache = R.Cache(rng, nb, Hkv, d, "int8")
    weight = rng.random((nb, Hkv, 16)).astype(np.float32)
    table[0, 2] = nb + 5            # 16 tokens without a score; the first and last tokens are elsewhere
    new_table[4, 1] = -7
    args, keepalive, ws, state = run(cache, weight, table, kv_len, keep, new_table, 4, 8, bucket=bound, host_kv=False, args_only=True)
    lens = [t for t in keepalive if hasattr(t, "is_cuda") and tuple(t.shape) == (5,)]
    lens[0].copy_(_i32([100, bound + 1, 100, 100, 100]))
    sv.spec_kv_evict(args, ws)
    torch.cuda.synchronize()
    check(state, cache, weight, table, kv_len, keep, new_table, 4, 8, left_out=(1, 2, 3))
    assert int(state["errors"].item()) == 3 + 16
    # protected tokens of a page outside the pool are copied as zeros
    table[0, 0] = -1
    table[0, 2] = table[0, 1]
    state = run(cache, weight, table[:1], kv_len[:1], [40], new_table[:1], 4, 8)
    check(state, cache, weight, table[:1], kv_len[:1], [40], new_table[:1], 4, 8)
    assert int(state["errors"].item()) == 4


def test_a_bucket_in_a_graph():
    import torch
    rng = np.random.default_rng(45)
    B, Hkv, d, bound = 2, 2, 128, 640
    (table, new_table), nb = R.tables(rng, [bound] * B, more=[[100] * B])
    cache = R.Cache(rng, nb, Hkv, d, "e4m3")
    weight = rng.random((nb, Hkv, 16)).astype(np.float32)
    args, keepalive, ws, state = run(cache, weight, table, [bound] * B, [100] * B, new_table, 4, 8, bucket=bound, args_only=True)
    lens = [t for t in keepalive if hasattr(t, "is_cuda") and tuple(t.shape) == (B,)]
    sv.spec_kv_evict(args, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_kv_evict(args, ws)
    fresh = cache.device() + (torch.from_numpy(weight).cuda(),)
    for n, keep in (([640, 33], [100, 20]), ([0, 101], [5, 100]), ([500, 500], [0, 1])):
        for to, new in zip((state["k"].view(torch.uint8), state["v"].view(torch.uint8), state["scale"], state["weight"]), fresh):
            to.copy_(new.view(torch.uint8) if new.element_size() == 1 else new)
        lens[0].copy_(_i32(n))
        lens[1].copy_(_i32(keep))
        graph.replay()
        torch.cuda.synchronize()
        check(state, cache, weight, table, n, keep, new_table, 4, 8)


def test_another_stream_and_a_workspace_of_two_graphs():
    """Two captured calls with one workspace, a choice in one launch and one of scores handed over, replayed in turn; then each on a stream of its own."""
    import torch
    rng = np.random.default_rng(46)
    calls = []
    for kind, n, keep in (("tiles", 700, 300), ("int8", 6000, 2000)):
        (table, new_table), nb = R.tables(rng, [n], more=[[keep]])
        cache = R.Cache(rng, nb, 2, 64, kind)
        weight = rng.random((nb, 2, 16)).astype(np.float32)
        calls.append(((cache, weight, table, [n], [keep], new_table, 4, 8),) + tuple(run(cache, weight, table, [n], [keep], new_table, 4, 8, args_only=True)))
    shared = sv.alloc_workspace(max(sv.spec_kv_evict_workspace_bytes(c[1]) for c in calls))
    graphs = []
    for given, args, keepalive, ws, state in calls:
        sv.spec_kv_evict(args, shared)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sv.spec_kv_evict(args, shared)

    def clear():
        for given, args, keepalive, ws, state in calls:
            fresh = given[0].device()
            for name, new in zip(("k", "v", "scale", "weight"), fresh + (torch.from_numpy(given[1]).cuda(),)):
                if new is not None:
                    state[name].view(torch.uint8).copy_(new.view(torch.uint8))
            state["new_len"].fill_(77)
            state["kept"].fill_(77)
        torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        for given, args, keepalive, ws, state in calls:
            check(state, *given)

    for order in ((0, 1), (1, 0), (1, 0)):
        clear()
        for i in order:
            graphs[i].replay()
        same()
    clear()
    streams = [torch.cuda.Stream() for _ in calls]
    for stream, (given, args, keepalive, ws, state) in zip(streams, calls):
        sv.spec_kv_evict(args, ws, stream)
    same()
