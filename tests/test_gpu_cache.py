"""Writing the paged cache and reading it back, against the same in 64 bits, to the bit: types, memory orders, page sizes, rows
of no sequence, positions without a page, special values."""
import pytest
import torch

import attention_reference as ref
from paged_cases import TYPES, Batch
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu

LENS = [(5, 5), (0, 0), (1, 33), (40, 75), (0, 12), (2, 1)]   # whole, an empty slot, one token, a chunk, no rows, more rows than tokens


def written(b, k=None, v=None):
    """The caches on the host after the plan's rows were put there one by one."""
    out = {n: x.clone() if x is not None else None for n, x in b.host.items()}
    for name, rows in (("k", b.k if k is None else k), ("v", b.v if v is None else v)):
        bits = out[name].view(torch.uint8) if out[name].dtype == TYPES["e4m3"] else out[name]
        for s in range(len(b.lens)):
            s0, s1 = int(b.row_start[s]), int(b.row_start[s + 1])
            for t in range(s0, s1):
                pos = int(b.kv_len[s]) - (s1 - t)
                pg = int(b.table[s, pos // b.page]) if 0 <= pos and pos // b.page < b.cols else -1
                if not 0 <= pg < bits.shape[0]:
                    continue
                if out[name + "_exp"] is not None:
                    y, e = ref.quantise(rows[t])
                    bits[pg, pos % b.page] = y.float().to(TYPES["e4m3"]).view(torch.uint8)
                    out[name + "_exp"][pg, pos % b.page] = e
                else:
                    bits[pg, pos % b.page] = rows[t]
    return out


def same(got, want, name):
    if want.dtype == TYPES["e4m3"]:
        a, b = got.view(torch.uint8), want.view(torch.uint8)
        a, b = (torch.where((x & 0x7F) == 0x7F, 0x7F, x) for x in (a, b))    # NaN has two signs
    else:
        a, b = got.contiguous().view(torch.int16 if got.dtype == TYPES["bf16"] else torch.int32 if got.dtype == TYPES["f32"] else torch.uint8), \
               want.contiguous().view(torch.int16 if want.dtype == TYPES["bf16"] else torch.int32 if want.dtype == TYPES["f32"] else torch.uint8)
    assert torch.equal(a, b), (name, (a != b).nonzero()[:4].tolist())


def check_write(b, k=None, v=None):
    want = written(b, k, v)
    kk, vv = (b.k if k is None else k).cuda(), (b.v if v is None else v).cuda()
    binding.s2attn_cache_write(b.params(k=kk, v=vv))
    torch.cuda.synchronize()
    for name, x in want.items():
        if x is not None:
            same(b.dev[name].cpu(), x, name)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")])
@pytest.mark.parametrize("layout", ["token", "head", "gaps"])
@pytest.mark.parametrize("Hkv,D,page", [(1, 64, 1), (3, 128, 24), (8, 64, 16), (5, 128, 64)])
def test_write_and_read(dtype, cache, layout, Hkv, D, page):
    b = Batch(LENS, Hkv, Hkv, D, page, dtype, cache, layout, seed=Hkv + page, before=2, behind=3)
    check_write(b)
    # the rows of the call back, then all cached tokens but the unwritten ones' NaN
    k, v = (torch.full((b.T, Hkv, D), 5.0, dtype=b.dt, device="cuda") for _ in range(2))
    binding.s2attn_cache_read(b.params(k=k, v=v))
    host = {n: x.cpu() if x is not None else None for n, x in b.dev.items()}
    for name, got in (("k", k.cpu()), ("v", v.cpu())):
        want = torch.full((b.T, Hkv, D), 5.0, dtype=torch.float64)
        for s in range(len(b.lens)):
            s0, s1, kv = int(b.row_start[s]), int(b.row_start[s + 1]), int(b.kv_len[s])
            x, _ = ref.cached_rows(host[name], host[name + "_exp"], b.table[s], kv, page)
            n = min(s1 - s0, kv)
            want[s0:s1 - n] = 0
            want[s1 - n:s1] = x[kv - n:]
        assert torch.equal(got.double(), want), name     # bf16 and fp32 hold these values exactly


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_values_in_8_bits(dtype):
    """Zero rows, one large value, infinities and NaN, the ends of the exponents' range, and values that lie half way."""
    D, T = 64, 14
    x = torch.randn(T, 2, D, generator=torch.Generator().manual_seed(3))
    x[0] = 0.0
    x[1] = 1e-38
    x[2] = 3e38
    x[3, :, 5], x[3, :, 9] = float("inf"), -float("inf")
    x[4, :, 0] = float("nan")
    x[5] = float("nan")
    x[6], x[6, 0, 0] = 0.0, 448.0
    x[7], x[7, 0, 0] = 0.0, 2.0 ** -133          # less than any normal number
    x[8, :, 3] = 1e6
    x[9, :, :9] = torch.tensor([448.0, 1.0625, 1.1875, -1.0625, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 464.0, 2.0 ** -6])
    x[10] = 2.0 ** 119 * 448
    x[11] = 2.0 ** -110
    x[12] = -0.0
    x[13] = 449.0
    x = x.to(TYPES[dtype])
    b = Batch([(T, T)], 2, 2, D, 16, dtype, "e4m3")
    check_write(b, x, x.flip(0))
    k, v = (torch.empty(T, 2, D, dtype=b.dt, device="cuda") for _ in range(2))
    binding.s2attn_cache_read(b.params(k=k, v=v))
    got, fin = k.cpu().double(), torch.isfinite(x)
    assert torch.isnan(got[~fin]).all()
    # half a step of e4m3 relative to the value, or half the least one's step where the row's scale makes it small
    amax = torch.where(fin, x.double().abs(), 0.0).amax(-1, keepdim=True)
    room = torch.maximum(2.0 ** -4 * x.double().abs(), torch.maximum(amax / 224, torch.tensor(2.0 ** -110)) * 2.0 ** -10)
    assert ((got - x.double()).abs() <= room)[fin].all()
    host = {n: t.cpu() for n, t in b.dev.items()}
    want, _ = ref.cached_rows(host["k"], host["k_exp"], b.table[0], T, 16)
    assert torch.equal(torch.nan_to_num(got, nan=9.0), torch.nan_to_num(want.to(TYPES[dtype]).double(), nan=9.0))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_positions_without_a_page(cache):
    """Pages below zero and beyond the cache, and tokens beyond the table's columns: not written, read as zeros."""
    big = 2 ** 31 - 1
    b = Batch([(60, 60), (30, 30), (50, 100)], 4, 4, 64, 16, "bf16", cache, bad_pages=[(0, 1, -1), (0, 2, big), (1, 0, 1000), (1, 1, -big - 1)], cols=4)
    check_write(b)
    k, v = (torch.full((b.T, 4, 64), 5.0, dtype=b.dt, device="cuda") for _ in range(2))
    binding.s2attn_cache_read(b.params(k=k, v=v))
    k, v = k.cpu(), v.cpu()
    for x in (k, v):
        assert not x[16:48].any() and not x[60:90].any()          # no such pages
        assert not x[90 + 14:].any()                              # positions 64 on: beyond four pages of 16
        assert x[:16].abs().sum(-1).all() and x[48:60].abs().sum(-1).all() and x[90:104].abs().sum(-1).all()


def test_plans_that_make_no_sense_stay_inside():
    """Row starts that fall or lie outside the rows: every access stays in the tensors, rows of the sensible sequences are right."""
    b = Batch([(10, 20), (6, 30)], 2, 2, 64, 16)
    T = b.T
    for starts in ([0, 10, 1000], [-50, 10, 16], [16, 16, 16], [12, 3, 16]):
        plan = dict(b.plan, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        k, v = (torch.zeros(T, 2, 64, dtype=b.dt, device="cuda") for _ in range(2))
        guard = torch.full((3 * T, 2, 64), 5.0, dtype=b.dt, device="cuda")
        binding.s2attn_cache_read(binding.make_paged_params(**plan, **b.caches(), k=guard[T:2 * T], v=v))
        torch.cuda.synchronize()
        assert (guard[:T] == 5).all() and (guard[2 * T:] == 5).all()


def test_nothing_to_do():
    b = Batch([(0, 20), (0, 0)], 2, 2, 64, 16)
    before = b.dev["k"].clone()
    binding.s2attn_cache_write(b.params(k=b.k.cuda(), v=b.v.cuda()))
    binding.s2attn_cache_read(b.params(k=b.k.cuda(), v=b.v.cuda()))
    torch.cuda.synchronize()
    assert torch.equal(before.view(torch.int16), b.dev["k"].view(torch.int16))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_packed_rows(cache):
    """k and v as slices of a packed projection, written and read."""
    b = Batch([(70, 90)], 4, 4, 128, 16, "bf16", cache)
    x = torch.stack([b.k, b.k * 3, b.v], 1).cuda()
    binding.s2attn_cache_write(b.params(k=x[:, 0], v=x[:, 2]))
    y = torch.full_like(x, 5.0)
    binding.s2attn_cache_read(b.params(k=y[:, 0], v=y[:, 2]))
    k, v = (torch.empty(70, 4, 128, dtype=b.dt, device="cuda") for _ in range(2))
    binding.s2attn_cache_read(b.params(k=k, v=v))
    torch.cuda.synchronize()
    assert torch.equal(y[:, 0], k) and torch.equal(y[:, 2], v) and (y[:, 1] == 5).all()
    if cache == "bf16":
        assert torch.equal(k, x[:, 0]) and torch.equal(v, x[:, 2])


def test_offsets_beyond_32_bits():
    """A cache of over 2^32 bytes a tensor, rows in its last pages."""
    pages, page, Hkv, D = 70000, 64, 4, 128
    kc, vc = (torch.empty(pages, page, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    T = 150
    plan = dict(row_start=torch.tensor([0, T], dtype=torch.int32, device="cuda"), kv_len=torch.tensor([T], dtype=torch.int32, device="cuda"), page_table=table)
    k, v = (torch.randn(T, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    binding.s2attn_cache_write(binding.make_paged_params(**plan, k_cache=kc, v_cache=vc, k=k, v=v))
    for x, c in ((k, kc), (v, vc)):
        assert torch.equal(torch.cat([c[pages - 1], c[3], c[pages - 2][:T - 128]]), x)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    binding.s2attn_cache_read(binding.make_paged_params(**plan, k_cache=kc, v_cache=vc, k=k2, v=v2))
    assert torch.equal(k, k2) and torch.equal(v, v2)
    q = torch.randn(T, 8, D, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty(8, T, device="cuda")
    binding.s2attn_paged_fwd(binding.make_paged_params(**plan, k_cache=kc, v_cache=vc, q=q, o=o, lse=lse))
    want = ref.window_reference(q.cpu()[None], k.cpu()[None], v.cpu()[None], None, T, 0)
    ref.hold("o", o[None], want)
    ref.hold("lse", lse[None], want)
