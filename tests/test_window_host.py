"""Refusals of the window calls, and the reference of their tests against itself; no GPU."""
import pytest
import torch

import attention_reference as ref
from paper_2309_12307_amd import binding
from test_abi_host import params


def rc(window=100, sinks=4, backward=True, **kw):
    return binding.check_window_args(params(**kw), window, sinks, backward)


def test_accepts():
    assert rc() == 0
    assert rc(backward=False, workspace=None, workspace_bytes=0) == 0
    assert rc(H=5, Hkv=5) == 0 and rc(H=3, Hkv=1, N=7) == 0 and rc(N=1) == 0       # no groups, no even heads
    assert rc(G=0) == 0 and rc(G=7, shift_rule=9, wrap_variant=5, bwd_algo=7, head_offset=3, heads_total=1) == 0   # not read
    assert rc(window=1, sinks=0) == 0 and rc(window=2 ** 31 - 1, sinks=2 ** 31 - 1) == 0
    assert rc(N=1 << 20, H=32, Hkv=32) == 0


@pytest.mark.parametrize("code,kw", [
    (-16, dict(window=0)), (-16, dict(window=-5)), (-16, dict(sinks=-1)),
    (-1, dict(q=None)), (-1, dict(lse=None)), (-1, dict(dk=None)),
    (-3, dict(N=0)), (-3, dict(B=-1)), (-3, dict(H=0)),
    (-5, dict(H=6, Hkv=4)), (-6, dict(D=96)), (-9, dict(dtype=binding.E4M3)), (-9, dict(dtype=9)),
    (-2, dict(q=0x10008)), (-2, dict(o=0x10002)), (-2, dict(workspace=0x10010)),
    (-8, dict(workspace=None)), (-8, dict(workspace_bytes=100)),
    (-13, dict(q_strides=(1024 * 4 * 128, 4 * 128 + 4, 128))),
    (-13, dict(dk_strides=(1024 * 4 * 128, 0, 128))),              # an output that lies on itself
    (-12, dict(N=(1 << 30) + 1)), (-12, dict(B=40000)), (-12, dict(N=1 << 30, H=512, Hkv=512)),
])
def test_refuses(code, kw):
    assert rc(**kw) == code, (rc(**kw), binding.strerror(rc(**kw)))


def test_no_workspace_size_for_invalid_shapes():
    for kw in (dict(N=0), dict(H=3, Hkv=2), dict(Hkv=0)):
        assert binding.window_workspace_bytes(params(**kw), 100, 4) == 0
    assert binding.window_workspace_bytes(params(), 0, 4) == 0 == binding.window_workspace_bytes(params(), 4, -1)


@pytest.mark.parametrize("kw", [dict(), dict(H=16, Hkv=1, N=5000), dict(dtype=binding.F32, N=100), dict(D=64, H=32, Hkv=8, B=2),
                                dict(N=100000, H=8, Hkv=8)], ids=str)
@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 4), (1000, 300), (10 ** 9, 0)])
def test_wanted_workspace_is_enough(kw, window, sinks):
    p = params(**kw)
    p.workspace_bytes = binding.window_workspace_bytes(p, window, sinks)
    assert p.workspace_bytes > 0 and binding.check_window_args(p, window, sinks, True) == 0


def test_binding_refuses_before_the_library():
    x = torch.zeros(1, 8, 2, 64)
    p = binding.make_params(x, x, x, torch.zeros_like(x), torch.zeros(1, 2, 8), 0)
    assert binding.check_window_args(p, 4, 0, False) == 0
    with pytest.raises((ValueError, binding.S2AttnError)):
        binding.s2attn_window_fwd(p, 4, 0)        # tensors of the CPU


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (5, 3), (100, 0), (7, 100)])
def test_reference_gradients_are_autograds(window, sinks):
    gen = torch.Generator().manual_seed(1)
    q, k, v, do = (torch.randn(1, 23, h, 64, generator=gen, dtype=torch.float64) for h in (4, 2, 2, 4))
    r = ref.window_reference(q, k, v, do, window, sinks)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    Q, K, V = leaves[0].transpose(1, 2), *(x.repeat_interleave(2, 2).transpose(1, 2) for x in leaves[1:])
    i, j = torch.arange(23)[:, None], torch.arange(23)[None]
    hidden = (j > i) | ((i - j >= window) & (j >= sinks))
    s = (Q @ K.transpose(2, 3) / 8).masked_fill(hidden, -torch.inf)
    o = (torch.softmax(s, -1) @ V).transpose(1, 2)
    (o * do).sum().backward()
    for name, x in (("o", o.detach()), ("dq", leaves[0].grad), ("dk", leaves[1].grad), ("dv", leaves[2].grad)):
        assert (r[name] - x).abs().max() < 1e-12, name
    assert (r["lse"] - torch.logsumexp(s, -1)).abs().max() < 1e-12


@pytest.mark.parametrize("change", [
    dict(q=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)), dict(v=lambda x: x[:, :7]), dict(v=lambda x: x.float()),
    dict(o=lambda x: x[..., :32]), dict(lse=lambda x: x.transpose(1, 2).contiguous()), dict(lse=lambda x: x.double()), dict(dq=lambda x: x[:, :, :1]),
    dict(dk=lambda x: x[:, ::2]), dict(dout=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2), strided=True),
    dict(k=lambda x: x.as_strided(x.shape, (0, 0, 0, 1)), strided=True),
], ids=lambda c: "+".join(c))
def test_binding_refuses_tensors_that_do_not_fit(change):
    """A view that is not told of, a shape or a type that is off: said by the window calls before anything is launched."""
    x = lambda h: torch.zeros(1, 8, h, 64, dtype=torch.bfloat16)
    t = dict(q=x(4), k=x(2), v=x(2), o=x(4), lse=torch.zeros(1, 4, 8), dout=x(4), dq=x(4), dk=x(2), dv=x(2))
    strided = change.pop("strided", False)
    assert binding.make_params(**t, G=0, strided=strided).problem is None
    t.update({n: f(t[n]) for n, f in change.items()})
    p = binding.make_params(**t, G=0, strided=strided)
    for call in (binding.s2attn_window_fwd, binding.s2attn_window_bwd):
        with pytest.raises(ValueError, match=next(iter(change)) + " "):
            call(p, 4, 0)
