"""Refusals of the paged cache's calls and of the binding in front of them, workspace sizes, and the reference of their
tests against torch's types; no GPU."""
import ctypes

import pytest
import torch

import attention_reference as ref
from paper_2309_12307_amd import binding
from paper_2309_12307_amd.binding import BF16, E4M3, F32

WRITE, READ, FWD = 0, 1, 2
FAKE = 0x10000


def block(**kw):
    d = dict(T=40, B=3, H=8, Hkv=4, D=128, pages=50, page_size=16, table_cols=20, dtype=BF16, cache_dtype=BF16, window=0, sinks=0, max_kv=0)
    d.update({n: FAKE for n in ("q", "o", "lse", "k", "v", "k_cache", "v_cache", "page_table", "row_start", "kv_len")})
    if kw.get("cache_dtype") == E4M3:
        d.update(k_exp=FAKE + 1, v_exp=FAKE + 3)
    d.update(kw)
    p = binding.S2AttnPagedParams()
    for n, x in d.items():
        setattr(p, n, (ctypes.c_longlong * len(x))(*x) if isinstance(x, tuple) else x)
    return p


def rc(call=FWD, **kw):
    return binding.check_paged_args(block(**kw), call)


@pytest.mark.parametrize("call", [WRITE, READ, FWD])
def test_accepts(call):
    for kw in (dict(), dict(T=0, q=None, o=None, k=None, v=None), dict(cache_dtype=E4M3), dict(dtype=F32, cache_dtype=F32), dict(dtype=F32, cache_dtype=E4M3),
               dict(page_size=1), dict(page_size=23), dict(H=4), dict(D=64, T=1), dict(H=260, Hkv=4), dict(table_stride=21),
               dict(B=100, T=3), dict(T=1, B=1, pages=1 << 24), dict(q_strides=(3 * 8 * 128, 128)), dict(k_strides=(2 * 4 * 128, 128)),
               dict(k_cache_strides=(2 * 4 * 16 * 128, 128, 16 * 128)), dict(cache_dtype=E4M3, k_exp_strides=(65, 1, 16))):
        assert rc(call, **kw) == 0, (kw, binding.strerror(rc(call, **kw)))
    assert rc(FWD, lse=None, k=None, v=None, workspace=None) == 0
    assert rc(WRITE, q=None, o=None, lse=None) == 0 == rc(READ, q=None, o=None, H=0)     # what a call does not read
    assert rc(FWD, window=2 ** 31 - 1, sinks=2 ** 31 - 1, max_kv=2 ** 31 - 1) == 0


@pytest.mark.parametrize("code,call,kw", [
    (-9, 3, dict()), (-9, -1, dict()), (-9, FWD, dict(dtype=E4M3)), (-9, FWD, dict(cache_dtype=F32)), (-9, WRITE, dict(dtype=F32, cache_dtype=BF16)),
    (-3, FWD, dict(B=0)), (-3, FWD, dict(T=-1)), (-3, READ, dict(pages=0)), (-3, WRITE, dict(page_size=0)), (-3, FWD, dict(table_cols=0)), (-3, FWD, dict(H=0)),
    (-5, FWD, dict(H=6)), (-6, WRITE, dict(D=96)), (-6, FWD, dict(D=256)),
    (-16, FWD, dict(window=-1)), (-16, FWD, dict(sinks=-1)), (-16, FWD, dict(max_kv=-1)),
    (-1, FWD, dict(q=None)), (-1, FWD, dict(o=None)), (-1, WRITE, dict(k=None)), (-1, READ, dict(v=None)), (-1, FWD, dict(page_table=None)),
    (-1, READ, dict(row_start=None)), (-1, WRITE, dict(kv_len=None)), (-1, FWD, dict(k_cache=None)), (-1, WRITE, dict(cache_dtype=E4M3, v_exp=None)),
    (-2, FWD, dict(q=FAKE + 8)), (-2, READ, dict(v=FAKE + 2)), (-2, FWD, dict(v_cache=FAKE + 8)), (-2, FWD, dict(kv_len=FAKE + 2)),
    (-2, FWD, dict(lse=FAKE + 1)), (-2, FWD, dict(workspace=FAKE + 16)),
    (-12, FWD, dict(table_cols=1 << 28)), (-12, FWD, dict(T=1 << 28)), (-12, WRITE, dict(T=1 << 27)), (-12, READ, dict(B=(1 << 24) + 1)),
    (-12, FWD, dict(B=1 << 24, H=64, Hkv=64)),
    (-13, FWD, dict(q_strides=(8 * 128, -128))), (-13, FWD, dict(q_strides=(8 * 128 + 4, 128))), (-13, FWD, dict(k_cache_strides=(8192, 512, 132))),
    (-13, WRITE, dict(k_cache_strides=(8192, 512, 64))), (-13, WRITE, dict(v_cache_strides=(0, 512, 128))), (-13, READ, dict(k_strides=(256, 128))),
    (-13, WRITE, dict(cache_dtype=E4M3, k_exp_strides=(64, 4, 0))), (-13, FWD, dict(table_stride=-20)), (-13, READ, dict(v_strides=(1 << 41, 128))),
])
def test_refuses(code, call, kw):
    assert rc(call, **kw) == code, (rc(call, **kw), binding.strerror(rc(call, **kw)))


def test_null_block():
    assert binding.lib().s2attn_check_paged_args(None, FWD) == -1
    assert binding.lib().s2attn_paged_workspace_bytes(None) == 0


def test_reading_calls_take_broadcast_views():
    """Heads or tokens of q, k, v and of the caches that lie on each other are fine where they are only read."""
    assert rc(FWD, q_strides=(0, 128)) == 0 and rc(WRITE, k_strides=(128, 0)) == 0
    assert rc(FWD, k_cache_strides=(0, 512, 128)) == 0 == rc(READ, v_cache_strides=(8192, 0, 128))


def test_workspace_sizes():
    size = lambda **kw: binding.paged_workspace_bytes(block(**kw))
    per_piece = lambda T, H, D: T * H * (D + 1) * 4
    for kw in (dict(T=1, B=1, table_cols=8000), dict(T=8, B=8, table_cols=600), dict(T=300, B=2, table_cols=2000)):
        n = size(**kw)
        assert n > 0 and n % per_piece(kw["T"], 8, 128) == 0
    assert size(T=0) == 0 and size(T=1, B=1, table_cols=1) == 0          # nothing to deal out
    assert size(T=1, B=1, table_cols=8000, max_kv=100) == 0
    assert size(T=1, B=1, table_cols=8000, window=100) < size(T=1, B=1, table_cols=8000)
    for kw in (dict(B=0), dict(H=6), dict(Hkv=0), dict(D=0), dict(T=-4), dict(pages=0), dict(page_size=0)):
        assert size(**kw) == 0


def tensors(dtype=torch.bfloat16, cache=torch.bfloat16, B=2, T=5, H=4, Hkv=2, D=64, pages=6, page=16, cols=3):
    t = dict(row_start=torch.tensor([0] + [T] * B, dtype=torch.int32), kv_len=torch.full((B,), 9, dtype=torch.int32),
             page_table=torch.zeros(B, cols, dtype=torch.int32), k_cache=torch.zeros(pages, page, Hkv, D).to(cache),
             v_cache=torch.zeros(pages, page, Hkv, D).to(cache), q=torch.zeros(T, H, D, dtype=dtype), o=torch.zeros(T, H, D, dtype=dtype),
             lse=torch.zeros(H, T), k=torch.zeros(T, Hkv, D, dtype=dtype), v=torch.zeros(T, Hkv, D, dtype=dtype))
    if cache == torch.float8_e4m3fn:
        t.update(k_exp=torch.zeros(pages, page, Hkv, dtype=torch.uint8), v_exp=torch.zeros(pages, page, Hkv, dtype=torch.uint8))
    return t


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn])
def test_binding_fills_the_block(cache):
    t = tensors(cache=cache)
    p = binding.make_paged_params(**t, window=7, sinks=2, max_kv=9, scale=0.25)
    assert (p.T, p.B, p.H, p.Hkv, p.D, p.pages, p.page_size, p.table_cols) == (5, 2, 4, 2, 64, 6, 16, 3)
    assert (p.window, p.sinks, p.max_kv, p.scale) == (7, 2, 9, 0.25)
    assert all(binding.check_paged_args(p, call) == 0 for call in (WRITE, READ, FWD))
    head_first = torch.zeros(6, 2, 16, 64).to(cache).transpose(1, 2)
    p = binding.make_paged_params(**{**t, "k_cache": head_first, "q": torch.zeros(5, 3, 4, 64, dtype=torch.bfloat16)[:, 1]})
    assert tuple(p.k_cache_strides) == (2 * 16 * 64, 64, 16 * 64) and tuple(p.q_strides) == (3 * 4 * 64, 64)
    assert all(binding.check_paged_args(p, call) == 0 for call in (WRITE, READ, FWD))
    empty = tensors(cache=cache, T=0)
    assert binding.check_paged_args(binding.make_paged_params(**empty), FWD) == 0
    with pytest.raises((ValueError, binding.S2AttnError)):
        binding.s2attn_paged_fwd(p)               # tensors of the CPU


@pytest.mark.parametrize("change", [
    dict(row_start=torch.zeros(3, dtype=torch.int64)), dict(row_start=torch.zeros(2, dtype=torch.int32)), dict(kv_len=torch.zeros(2, 1, dtype=torch.int32)),
    dict(page_table=torch.zeros(3, dtype=torch.int32).expand(2, 3)), dict(q=torch.zeros(1, 1, 64, dtype=torch.bfloat16).expand(5, 4, 64)),
    dict(page_table=torch.zeros(3, 3, dtype=torch.int32)), dict(page_table=torch.zeros(3, 2, dtype=torch.int32).t()),
    dict(v_cache=torch.zeros(6, 16, 2, 128, dtype=torch.bfloat16)), dict(v_cache=torch.zeros(6, 16, 2, 64)),
    dict(k_cache=torch.zeros(6, 16, 64, 2, dtype=torch.bfloat16).transpose(2, 3), v_cache=torch.zeros(6, 16, 64, 2, dtype=torch.bfloat16).transpose(2, 3)),
    dict(k_exp=torch.zeros(6, 16, 2, dtype=torch.uint8)), dict(q=None, o=None, k=None, v=None, lse=None), dict(o=None), dict(v=None),
    dict(o=torch.zeros(5, 4, 64)), dict(o=torch.zeros(5, 8, 64, dtype=torch.bfloat16)[:, ::2]), dict(q=torch.zeros(5, 4, 32, dtype=torch.bfloat16)),
    dict(lse=torch.zeros(5, 4)), dict(lse=torch.zeros(4, 5, dtype=torch.float64)), dict(k=torch.zeros(6, 2, 64, dtype=torch.bfloat16)),
    dict(k=torch.zeros(5, 2, 64)), dict(q=torch.zeros(5, 4, 64, dtype=torch.float16), o=torch.zeros(5, 4, 64, dtype=torch.float16)),
    dict(q=torch.zeros(5, 4, 64, device="meta")),
], ids=lambda c: "+".join(c))
def test_binding_refuses(change):
    with pytest.raises((ValueError, TypeError)):
        binding.make_paged_params(**{**tensors(), **change})


@pytest.mark.parametrize("missing", [dict(k_exp=None), dict(v_exp=torch.zeros(6, 16, 2)), dict(v_exp=torch.zeros(6, 16, 1, dtype=torch.uint8))], ids=str)
def test_binding_refuses_missing_exponents(missing):
    with pytest.raises(ValueError):
        binding.make_paged_params(**{**tensors(cache=torch.float8_e4m3fn), **missing})


def test_reference_quantisation():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(500, 64, generator=gen, dtype=torch.float64) * 2.0 ** torch.randint(-40, 40, (500, 1), generator=gen)
    y, e = ref.quantise(x)
    amax, scale = x.abs().amax(1), 2.0 ** (e.double() - 127)
    assert (amax <= 448 * scale).all() and (amax > 224 * scale).all()
    assert torch.equal(y, (x / scale[:, None]).float().to(torch.float8_e4m3fn).double())     # nothing of these is lost in float
    y, e = ref.quantise(torch.tensor([[0.0, 0.0], [448.0, 1.0], [449.0, 1.0], [float("inf"), 1.0], [float("nan"), 0.0]]))
    assert e.tolist() == [17, 127, 128, 119, 17] and torch.isnan(y[3, 0]) and torch.isnan(y[4, 0]) and y[3, 1] == 256
