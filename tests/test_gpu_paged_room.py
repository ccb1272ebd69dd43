"""Pieces of few rows beside long prompts: slots of their own in the workspace, workspaces of any size, and the join over both."""
import pytest
import torch

import attention_reference as ref
from paged_cases import Batch
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")]


def wanted(b, **kw):
    return binding.paged_workspace_bytes(b.params(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"), **kw))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 24)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 7)])
def test_both_in_pieces(window, sinks, D, page, dtype, cache):
    lens = [(1, 6000), (300, 3000), (3, 4000), (0, 0), (16, 2000), (2, 2)]
    b = Batch(lens, 8, 2, D, page, dtype, cache, seed=D, before=1, behind=2)
    n, piece = wanted(b, window=window, sinks=sinks), b.T * b.H * (D + 1) * 4
    assert 2 * piece <= n and n % piece == 0
    want = b.reference(window, sinks)
    for ws in (n, n // 2, 3 * piece + 100, piece, piece // 3, 256, 0):
        b.check(*b.attend(window, sinks, workspace=ws), want)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("lens", [[(1100, 1500), (2, 5000), (1, 300)], [(1100, 1500), (620, 700), (2, 5000)]], ids=["four waves", "eight waves"])
def test_few_rows_alone_in_pieces(lens, dtype, cache):
    """Prompts that fill the chip in one piece: room for the short sequences' alone.  Two kv heads out of many are compared."""
    b = Batch(lens, 64, 64, 128, 16, dtype, cache, seed=3, before=2, behind=1)
    n, piece = wanted(b), b.T * b.H * 129 * 4
    assert 256 < n < 2 * piece          # less than all rows in two pieces
    some = [0, 43]
    sub = {m: x[:, :, some] if x is not None else None for m, x in b.host.items()}
    want = ref.paged_reference(b.q[:, some], sub["k"], sub["v"], sub["k_exp"], sub["v_exp"], b.row_start, b.kv_len, b.table, 0, 0)
    for ws in (n, n // 3, 0):
        o, lse = b.attend(workspace=ws)
        ref.hold("o", o[:, some], want, b.own)
        ref.hold("lse", lse[some], want, (slice(None), b.own))
        assert (o[~b.own.cuda()] == 5).all() and (lse[:, ~b.own.cuda()] == 7).all()


def test_many_heads_of_a_kv_head_beside_few():
    """20 heads to a kv head: one token is more rows than few workgroups take, all sequences go in chunks."""
    b = Batch([(1, 3000), (40, 2000), (2, 100)], 20, 1, 128, 16, "bf16", "e4m3", seed=4)
    b.check(*b.attend(), b.reference())
    b.check(*b.attend(100, 5), b.reference(100, 5))
