"""Attention over the paged cache, kernel by kernel against the formulas in 64 bits: eight waves and four in one piece and in
several, two blocks of rows of single tokens, with windows, sinks, shared kv heads and pages that do not exist."""
import pytest
import torch

import attention_reference as ref
from paged_cases import Batch
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu


def check_heads(b, window, sinks, kv_heads, workspace="wanted"):
    """The query heads of some kv heads."""
    r = b.H // b.Hkv
    heads = [c * r + i for c in kv_heads for i in range(r)]
    sub = {n: x[:, :, kv_heads] if x is not None else None for n, x in b.host.items()}
    want = ref.paged_reference(b.q[:, heads], sub["k"], sub["v"], sub["k_exp"], sub["v_exp"], b.row_start, b.kv_len, b.table, window, sinks)
    o, lse = b.attend(window, sinks, workspace=workspace)
    own = b.own
    ref.hold("o", o[:, heads], want, own)
    ref.hold("lse", lse[heads], want, (slice(None), own))
    assert (o[~own.cuda()] == 5).all() and (lse[:, ~own.cuda()] == 7).all(), "rows of no sequence"
    assert torch.isfinite(o).all()


def pieces(b, window=0, sinks=0):
    """Pieces of all rows that the call asks room for."""
    n = binding.paged_workspace_bytes(b.params(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"), window=window, sinks=sinks))
    return n // (b.T * b.H * (b.D + 1) * 4)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 0), (257, 5), (64, 130)])
@pytest.mark.parametrize("page", [16, 48])
def test_eight_waves(page, window, sinks, cache):
    """1200 and 1040 rows of four query heads to a kv head, a page that does not exist, and one token beside them."""
    bad = [(0, 3, -1), (0, 11, 10 ** 6), (1, 0, -5)]
    b = Batch([(300, 900), (260, 1000), (1, 500)], 96, 24, 128, page, "bf16", cache, ("token", "head")[page == 48], seed=page, before=1, behind=2, bad_pages=bad)
    check_heads(b, window, sinks, [0, 17])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (12000, 10)])
def test_eight_waves_in_pieces(window, sinks, cache):
    b = Batch([(600, 16000)], 32, 8, 128, 16, "bf16", cache, "head", seed=6, bad_pages=[(0, 100, -1), (0, 700, 10 ** 6)])
    assert pieces(b, window, sinks) >= 2
    check_heads(b, window, sinks, [3])
    check_heads(b, window, sinks, [5], workspace=0)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2000, 7), (2900, 100)])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("D", [64, 128])
def test_four_waves_in_pieces(D, page, window, sinks, cache):
    """Tens of rows over some thousand keys, alone and beside single tokens."""
    for lens in ([(40, 3500)], [(40, 3500), (1, 3100), (70, 3300)]):
        b = Batch(lens, 8, 2, D, page, "bf16", cache, seed=D + page, bad_pages=[(0, 5, -1)])
        assert pieces(b, window, sinks) >= 2
        b.check(*b.attend(window, sinks), b.reference(window, sinks))


@pytest.mark.parametrize("D,page", [(128, 16), (128, 24), (64, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 3)])
@pytest.mark.parametrize("lens,H,Hkv", [([(1, 6000), (0, 0), (1, 33), (1, 1500)], 20, 1), ([(1, 6000), (1, 1)], 64, 2), ([(3, 5000)], 20, 2), ([(2, 900), (1, 4000)], 9, 1)])
def test_two_blocks_of_rows(lens, H, Hkv, window, sinks, D, page):
    """17 to 32 rows over e4m3, over many tiles and in pieces."""
    b = Batch(lens, H, Hkv, D, page, "bf16", "e4m3", ("token", "gaps")[Hkv - 1], seed=H, before=1, bad_pages=[(0, 7, -1)])
    want = b.reference(window, sinks)
    assert pieces(b, window, sinks) >= 2
    b.check(*b.attend(window, sinks), want)
    b.check(*b.attend(window, sinks, workspace=0), want)


def test_two_calls_at_once_from_poison():
    """Two steps on two streams, each with its own workspace, whose memory holds NaN before every turn: the bits of the same steps by
    themselves, which the formulas' bounds hold."""
    batches = [Batch([(1, 6000), (40, 3000), (1, 50)], 8, 2, 128, 16, "bf16", "e4m3", seed=31), Batch([(1, 700), (20, 2000), (0, 0), (130, 400), (3, 2)], 8, 2, 64, 16, "f32", "f32", seed=32)]
    calls = []

    def poison(kw, ws):
        for x in (kw["o"], kw["lse"]):
            x.fill_(float("nan"))
        ws.fill_(255)

    for b in batches:
        kw = dict(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"), lse=torch.empty(8, b.T, device="cuda"))
        n = binding.paged_workspace_bytes(b.params(**kw))
        assert n > 0
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        p = b.params(workspace=ws, **kw)
        poison(kw, ws)
        binding.s2attn_paged_fwd(p)
        want = b.reference()
        ref.hold("o", kw["o"], want)
        ref.hold("lse", kw["lse"], want)
        calls.append((p, kw, ws, kw["o"].clone(), kw["lse"].clone()))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(4):
        for _, kw, ws, _, _ in calls:
            poison(kw, ws)
        torch.cuda.synchronize()
        for (p, _, _, _, _), s in zip(calls, streams):
            binding.s2attn_paged_fwd(p, stream=s)
        torch.cuda.synchronize()
        for _, kw, _, o, lse in calls:
            assert torch.equal(kw["o"], o) and torch.equal(kw["lse"], lse)
