"""Attention over the paged cache against the formulas in 64 bits, and a step's calls together: ragged batches from one token
on, every kind of workgroup, windows and sinks, pages of any size, poison where nothing may be read, workspaces, streams, graphs."""
import pytest
import torch

import attention_reference as ref
from paged_cases import Batch
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu

DECODE = [(1, 1), (1, 300), (0, 0), (1, 64), (1, 65), (0, 17), (1, 1300)]
MIXED = [(1, 700), (20, 20), (0, 0), (130, 400), (16, 900), (17, 33), (1, 1), (3, 2)]
CHUNK = [(300, 1000)]
PREFILL = [(257, 257), (64, 64)]

# lens, H, Hkv, D, page, window, sinks
CASES = [
    (DECODE, 4, 4, 64, 16, 0, 0),
    (DECODE, 16, 2, 128, 64, 0, 0),
    (DECODE, 12, 4, 128, 24, 100, 3),
    (DECODE, 8, 8, 64, 1, 0, 0),
    (DECODE, 40, 1, 64, 16, 0, 0),          # forty query heads to a kv head
    (DECODE, 80, 2, 128, 5, 33, 70),
    (MIXED, 8, 2, 64, 16, 0, 0),
    (MIXED, 8, 2, 128, 16, 64, 4),
    (MIXED, 5, 5, 128, 48, 0, 0),
    (MIXED, 6, 2, 64, 7, 65, 1),
    (MIXED, 4, 1, 128, 128, 1, 0),          # every token sees itself alone
    (CHUNK, 4, 4, 128, 64, 0, 0),
    (CHUNK, 3, 1, 64, 33, 200, 100),
    (CHUNK, 4, 4, 128, 32, 31, 0),
    (PREFILL, 4, 2, 64, 64, 0, 0),
    (PREFILL, 2, 2, 128, 10, 0, 0),
]
TYPES = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n", range(len(CASES)))
def test_batches(n, dtype, cache):
    lens, H, Hkv, D, page, window, sinks = CASES[n]
    b = Batch(lens, H, Hkv, D, page, dtype, cache, ("token", "head", "gaps")[n % 3], seed=n, before=n % 3, behind=(n + 1) % 3)
    want = b.reference(window, sinks)
    b.check(*b.attend(window, sinks), want)
    if window == 0 or n % 2:
        b.check(*b.attend(window, sinks, workspace=0), want)                       # in one piece
        piece = b.T * H * (D + 1) * 4
        b.check(*b.attend(window, sinks, workspace=3 * piece + 100, max_kv=64), want)   # a max_kv that is off


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("B", [65, 300])
def test_many_sequences(B, rows, dtype, cache):
    """More sequences than a wave has lanes, one in ten an empty slot, written, attended and read."""
    gen = torch.Generator().manual_seed(B + rows)
    draw = lambda n: int(torch.randint(n, (1,), generator=gen))
    lens = [(0, 0) if draw(10) == 0 else (1 + draw(rows), 40 + draw(90)) for _ in range(B)]
    b = Batch(lens, 2, 1, 64, 16, dtype, cache, seed=B, before=1, behind=2)
    b.check(*b.attend(), b.reference())
    b.check(*b.attend(30, 2), b.reference(30, 2))
    k, v = b.k.cuda(), b.v.cuda()
    binding.s2attn_cache_write(b.params(k=k, v=v))
    back = [torch.full_like(x, 5.0) for x in (k, v)]
    binding.s2attn_cache_read(b.params(k=back[0], v=back[1]))
    torch.cuda.synchronize()
    own = b.own.cuda()
    for x, y in zip((b.k, b.v), back):
        want = x
        if cache == "e4m3":
            values, e = ref.quantise(x)
            want = (values * 2.0 ** (e.double() - 127)[..., None]).to(x.dtype)
        assert torch.equal(y[own].cpu(), want[b.own]) and (y[~own] == 5).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_more_rows_than_tokens(window, sinks, dtype, cache):
    """Rows at negative positions see nothing, in every kind of workgroup."""
    b = Batch([(300, 100), (150, 149), (9, 3), (40, 0), (1, 0)], 4, 4, 128, 16, dtype, cache, seed=7)
    want = b.reference(window, sinks)
    assert torch.isinf(want["lse"][:, :200]).all()
    b.check(*b.attend(window, sinks), want)
    b = Batch([(1, 0), (12, 5)], 4, 2, 64, 8, dtype, cache, seed=8)
    b.check(*b.attend(window, sinks), b.reference(window, sinks))


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_many_query_heads_of_one_kv_head(dtype, cache):
    b = Batch([(1, 200), (0, 0), (1, 31)], 128, 1, 64, 16, dtype, cache, seed=3)
    b.check(*b.attend(), b.reference())
    b = Batch([(3, 200), (1, 90)], 96, 1, 128, 16, dtype, cache, seed=4)
    b.check(*b.attend(50, 1), b.reference(50, 1))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 40])
def test_long_chunk(cache, page):
    """Rows enough for eight waves to a workgroup: two kv heads out of many are compared."""
    b = Batch([(1100, 1600), (600, 600), (9, 800)], 80, 80, 128, page, "bf16", cache, seed=2)
    o, lse = b.attend(0, 0)
    some = [0, 43]
    sub = {n: x[:, :, some] if x is not None else None for n, x in b.host.items()}
    want = ref.paged_reference(b.q[:, some], sub["k"], sub["v"], sub["k_exp"], sub["v_exp"], b.row_start, b.kv_len, b.table, 0, 0)
    ref.hold("o", o[:, some], want)
    ref.hold("lse", lse[some], want)


def test_decode_over_many_tokens():
    """A long cache for one row: many pieces, joined."""
    for dtype, cache, H, Hkv, window, sinks in (("bf16", "e4m3", 8, 8, 0, 0), ("bf16", "bf16", 16, 2, 0, 0), ("f32", "f32", 4, 2, 0, 0), ("bf16", "bf16", 8, 1, 9000, 5)):
        b = Batch([(1, 20000), (1, 3)], H, Hkv, 128, 64, dtype, cache, seed=H)
        assert binding.paged_workspace_bytes(b.params(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"))) > 0
        b.check(*b.attend(window, sinks), b.reference(window, sinks))


def test_peaked_scores():
    for dtype, cache in TYPES:
        b = Batch(MIXED, 4, 2, 64, 16, dtype, cache, seed=4)
        b.q *= 6
        b.check(*b.attend(), b.reference())
        b.check(*b.attend(scale=0.5, window=50, sinks=2), b.reference(50, 2, 0.5))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "e4m3")])
@pytest.mark.parametrize("lens,page", [([(1, 100), (1, 90), (1, 200)], 16), ([(30, 100), (40, 90), (1, 200)], 16), ([(30, 100), (40, 90), (1, 200)], 9)])
def test_positions_without_a_page(dtype, cache, lens, page):
    """Keys of pages that do not exist are invisible; a sequence without any page sees nothing."""
    big = 2 ** 31 - 1
    bad = [(0, 1, -1), (0, 3, big)] + [(1, c, 10 ** 6 if c % 2 else -big - 1) for c in range(10)]
    b = Batch(lens, 4, 2, 64, page, dtype, cache, bad_pages=[x for x in bad if x[1] < -(-lens[x[0]][1] // page)], cols=12)
    want = b.reference()
    assert torch.isinf(want["lse"][:, b.row_start[1]:b.row_start[2]]).all()
    b.check(*b.attend(), want)
    b.check(*b.attend(workspace=0), want)
    b.check(*b.attend(37, 3), b.reference(37, 3))


def test_strides_of_rows_and_tables():
    """q as a slice of a packed projection, a page table that is a part of a wider one, no lse."""
    b = Batch(MIXED, 8, 8, 128, 16, seed=9)
    packed = torch.full((b.T, 3, 8, 128), float("nan"), dtype=b.dt, device="cuda")
    packed[:, 1] = b.q.cuda()
    wide = torch.full((len(MIXED), b.cols + 5), 10 ** 6, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + b.cols] = b.table.cuda()
    b.plan["page_table"] = wide[:, 2:2 + b.cols]
    want = b.reference()
    b.check(*b.attend(q=packed[:, 1]), want)
    o = torch.full((b.T, 8, 128), 5.0, dtype=b.dt, device="cuda")
    binding.s2attn_paged_fwd(b.params(q=packed[:, 1], o=o))
    ref.hold("o", o, want, b.own)


def test_shared_prefix():
    """Two sequences whose first pages are the same."""
    b = Batch([(4, 100), (4, 100)], 4, 2, 64, 16, seed=6)
    b.table[1, :5] = b.table[0, :5]
    b.plan["page_table"] = b.table.cuda()
    b.check(*b.attend(), b.reference())


def test_plans_that_make_no_sense_stay_inside():
    b = Batch([(10, 20), (6, 30)], 4, 2, 64, 16)
    for starts, lens in (([0, 10, 1000], [20, 30]), ([-50, 10, 16], [20, 30]), ([16, 16, 16], [20, 30]), ([12, 3, 16], [20, 30]),
                         ([0, 10, 16], [-5, 2 ** 31 - 1]), ([0, 10, 16], [-2 ** 31, 100000])):
        b.plan.update(row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        guard = torch.full((3 * b.T, 4, 64), 5.0, dtype=b.dt, device="cuda")
        lse = torch.full((3, 4, b.T), 7.0, device="cuda")
        kw = dict(q=b.q.cuda(), o=guard[b.T:2 * b.T], lse=lse[1])
        ws = torch.empty(max(256, binding.paged_workspace_bytes(b.params(**kw))), dtype=torch.uint8, device="cuda")
        binding.s2attn_paged_fwd(b.params(workspace=ws, **kw))
        torch.cuda.synchronize()
        assert (guard[:b.T] == 5).all() and (guard[2 * b.T:] == 5).all() and (lse[0] == 7).all() and (lse[2] == 7).all()


@pytest.mark.parametrize("lens", [DECODE, MIXED], ids=["decode", "mixed"])
@pytest.mark.parametrize("dtype,cache", [("bf16", "e4m3"), ("f32", "f32")])
def test_runs_repeat(dtype, cache, lens):
    b = Batch(lens, 8, 2, 64, 16, dtype, cache, seed=8)
    o, lse = b.attend()
    for _ in range(3):
        o2, lse2 = b.attend()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,cache,D", [("bf16", "bf16", 128), ("bf16", "e4m3", 64), ("f32", "f32", 64)])
def test_a_prompt_and_its_continuation(dtype, cache, D):
    """The calls as a server makes them: a prompt in chunks, then token by token in a graph that is replayed while lengths and
    rows change on the device; everything against one causal pass over the whole sequence."""
    H, Hkv, page, N, prompt, window, sinks = 8, 2, 16, 333, 300, 120, 4
    gen = torch.Generator().manual_seed(12)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = (torch.randn(N, h, D, generator=gen).to(dt) for h in (H, Hkv, Hkv))
    b = Batch([(N, N)], H, Hkv, D, page, dtype, cache, seed=13)
    if cache == "e4m3":      # what the cache holds
        hold_k, hold_v = ((y * 2.0 ** (e.double() - 127)[..., None]).to(dt) for y, e in (ref.quantise(x) for x in (k, v)))
    else:
        hold_k, hold_v = k, v
    want = ref.window_reference(q[None], hold_k[None], hold_v[None], None, window, sinks)
    o = torch.empty(N, H, D, dtype=dt, device="cuda")
    for s0, s1 in ((0, 100), (100, 101), (101, prompt)):
        b.plan.update(row_start=torch.tensor([0, s1 - s0], dtype=torch.int32, device="cuda"), kv_len=torch.tensor([s1], dtype=torch.int32, device="cuda"))
        rows = dict(q=q[s0:s1].cuda(), k=k[s0:s1].cuda(), v=v[s0:s1].cuda(), o=o[s0:s1])
        p = b.params(**rows, window=window, sinks=sinks)
        ws = torch.empty(binding.paged_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        p = b.params(**rows, window=window, sinks=sinks, workspace=ws)
        binding.s2attn_cache_write(p)
        binding.s2attn_paged_fwd(p)
        torch.cuda.synchronize()
    b.plan.update(row_start=torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    step = {n: torch.zeros(1, h, D, dtype=dt, device="cuda") for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("o", H))}
    p = b.params(**step, window=window, sinks=sinks)
    ws = torch.empty(max(256, binding.paged_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
    p = b.params(**step, window=window, sinks=sinks, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.s2attn_cache_write(p)
        binding.s2attn_paged_fwd(p)
    for t in range(prompt, N):
        b.plan["kv_len"].fill_(t + 1)
        for n, x in (("q", q), ("k", k), ("v", v)):
            step[n].copy_(x[t:t + 1])
        step["o"].fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        o[t] = step["o"][0]
    ref.hold("o", o[None], want)
    # the whole prefix back, and the pass over contiguous tensors on it
    back_k, back_v = (torch.empty(N, Hkv, D, dtype=dt, device="cuda") for _ in range(2))
    b.plan.update(row_start=torch.tensor([0, N], dtype=torch.int32, device="cuda"), kv_len=torch.tensor([N], dtype=torch.int32, device="cuda"))
    binding.s2attn_cache_read(b.params(k=back_k, v=back_v))
    torch.cuda.synchronize()
    assert torch.equal(back_k.cpu(), hold_k) and torch.equal(back_v.cpu(), hold_v)
    o2, lse2 = torch.empty(1, N, H, D, dtype=dt, device="cuda"), torch.empty(1, H, N, device="cuda")
    binding.s2attn_window_fwd(binding.make_params(q[None].cuda(), back_k[None], back_v[None], o2, lse2, 0), window, sinks)
    torch.cuda.synchronize()
    ref.hold("o", o2, want)
    ref.hold("lse", lse2, want)


def test_two_graphs_share_a_workspace():
    """Two layers captured with one workspace, replayed in turn with other work between, on a stream of their own."""
    layers = [Batch([(1, 2000), (1, 900), (1, 1)], 8, 2, 128, 16, "bf16", "e4m3", seed=s) for s in (20, 21)]
    outs, graphs = [], []
    kw = [dict(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"), lse=torch.empty(8, b.T, device="cuda")) for b in layers]
    ws = torch.empty(max(binding.paged_workspace_bytes(b.params(**x)) for b, x in zip(layers, kw)), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for b, x in zip(layers, kw):
        p = b.params(workspace=ws, **x)
        with torch.cuda.stream(stream):
            binding.s2attn_paged_fwd(p)      # eager, on that stream
        stream.synchronize()
        b.check_now = b.reference()
        ref.hold("o", x["o"], b.check_now)
        outs.append((x["o"].clone(), x["lse"].clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            binding.s2attn_paged_fwd(p)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        kw[i]["o"].fill_(float("nan"))
        ws.fill_(255)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(kw[i]["o"], outs[i][0]) and torch.equal(kw[i]["lse"], outs[i][1]), i


def test_two_calls_at_once():
    """Two steps on two streams, each with its own workspace: the bits of the same steps one after the other."""
    batches = [Batch([(1, 6000), (40, 3000), (1, 50)], 8, 2, 128, 16, "bf16", "e4m3", seed=31), Batch(MIXED, 8, 2, 64, 16, "f32", "f32", seed=32)]
    calls = []
    for b in batches:
        kw = dict(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"), lse=torch.empty(8, b.T, device="cuda"))
        ws = torch.empty(binding.paged_workspace_bytes(b.params(**kw)), dtype=torch.uint8, device="cuda")
        calls.append((b.params(workspace=ws, **kw), kw, ws))
    want = []
    for p, kw, _ in calls:
        binding.s2attn_paged_fwd(p)
        torch.cuda.synchronize()
        want.append((kw["o"].clone(), kw["lse"].clone()))
        kw["o"].fill_(float("nan"))
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for (p, _, _), s in zip(calls, streams):
            binding.s2attn_paged_fwd(p, stream=s)
    torch.cuda.synchronize()
    for b, (_, kw, _), (o, lse) in zip(batches, calls, want):
        own = b.own.cuda()
        assert torch.equal(kw["o"][own], o[own]) and torch.equal(kw["lse"][:, own], lse[:, own])
