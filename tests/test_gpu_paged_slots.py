"""Batches of slots: as many sequences as rows, or more, of which some have no row and others several."""
import pytest
import torch

import attention_reference as ref
from paged_cases import Batch
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")]
IDLE = [(0, 50)]
# lens: no more rows than sequences
SLOTS = [
    IDLE * 3 + [(40, 700)] + IDLE * 50,                                                # one prompt among idle slots
    [(1, 90)] + IDLE + [(3, 200), (1, 20)] + IDLE * 2 + [(7, 7), (2, 1)] + IDLE * 9,   # single tokens beside drafts of several
    IDLE * 70 + [(5, 300)] + IDLE * 70 + [(66, 400), (1, 1)] + IDLE * 2,               # more slots than a wave has lanes
    [(1, 300)] * 5,                                                                    # the plain step
]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H,Hkv,D,page", [(2, 2, 64, 16), (10, 2, 128, 16), (16, 1, 64, 24), (24, 1, 128, 8)])
@pytest.mark.parametrize("n", range(len(SLOTS)))
def test_slots(n, H, Hkv, D, page, dtype, cache):
    """1, 5, 16 and 24 query heads to a kv head: 16, 3, 1 and (e4m3, fp32) 1 tokens to a workgroup."""
    b = Batch(SLOTS[n], H, Hkv, D, page, dtype, cache, seed=n, before=2 if n == 1 else 0, behind=1)
    assert b.T <= len(b.lens) + 3
    want = b.reference()
    b.check(*b.attend(), want)
    b.check(*b.attend(workspace=0), want)
    b.check(*b.attend(40, 3), b.reference(40, 3))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3")])
def test_slots_in_pieces(dtype, cache):
    """Keys enough for several pieces, joined."""
    b = Batch(IDLE * 4 + [(9, 6000)] + IDLE * 3 + [(2, 900)] + IDLE * 6, 12, 2, 128, 16, dtype, cache, seed=5)
    assert binding.paged_workspace_bytes(b.params(q=b.q.cuda(), o=torch.empty_like(b.q, device="cuda"))) > 0
    b.check(*b.attend(), b.reference())
    b.check(*b.attend(3000, 10), b.reference(3000, 10))


def test_a_prompt_among_idle_slots_takes_no_turns():
    """256 rows of one sequence: in 256 slots at most a few times what they take in one (by turns of one workgroup a kv head: 100 times)."""
    T, H, Hkv, D, kv = 256, 64, 8, 128, 8192
    kc, vc = (torch.randn(kv // 64, 64, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    table = torch.arange(kv // 64, dtype=torch.int32, device="cuda")[None]
    q = torch.randn(T, H, D, device="cuda").bfloat16()
    took, outs = [], []
    for B in (1, 256):
        at = 100 if B > 1 else 0
        plan = dict(row_start=torch.tensor([0] * (at + 1) + [T] * (B - at), dtype=torch.int32, device="cuda"),
                    kv_len=torch.full((B,), kv, dtype=torch.int32, device="cuda"), page_table=table.repeat(B, 1))
        o = torch.empty_like(q)
        p = binding.make_paged_params(**plan, k_cache=kc, v_cache=vc, q=q, o=o)
        ws = torch.empty(max(256, binding.paged_workspace_bytes(p)), dtype=torch.uint8, device="cuda")
        p = binding.make_paged_params(**plan, k_cache=kc, v_cache=vc, q=q, o=o, workspace=ws)
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            binding.s2attn_paged_fwd(p)
        e0.record()
        for _ in range(10):
            binding.s2attn_paged_fwd(p)
        e1.record()
        e1.synchronize()
        took.append(e0.elapsed_time(e1) / 10)
        outs.append(o.float())
    print("ms, in one slot and in 256:", took)
    # two roundings of P and o of values below 1 (an average of some thousand keys)
    assert (outs[0] - outs[1]).abs().max() < 4 * 2.0 ** -8
    assert took[1] < 20 * took[0], took
