"""Attention with a window and sinks, forward and gradient, against the formulas in 64 bits: sizes from one token on, windows
and sinks at the edges of the kernels' tiles, strided and overlapping tensors, small workspaces, other streams and graphs."""
import pytest
import torch

import attention_reference as ref
from paper_2309_12307_amd import binding

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(dtype, B, N, H, Hkv, D, seed, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    return [(size * torch.randn(B, N, h, D, generator=gen)).to(dt) if i == 0 else torch.randn(B, N, h, D, generator=gen).to(dt)
            for i, h in enumerate((H, Hkv, Hkv, H))]


def least_workspace(p, window, sinks):
    lo, hi = 0, binding.window_workspace_bytes(p, window, sinks) // 256   # the check itself says what is too little
    p.workspace = 1 << 20
    while lo < hi:
        mid = (lo + hi) // 2
        p.workspace_bytes = mid * 256
        if binding.check_window_args(p, window, sinks, True) == 0:
            hi = mid
        else:
            lo = mid + 1
    return hi * 256


def run(q, k, v, do, window, sinks, ws_bytes=None, **kw):
    """On the GPU; outputs start as NaN.  Returns them, and what to keep alive."""
    B, N, H, D = q.shape
    o = torch.full((B, N, H, D), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((B, H, N), float("nan"), device="cuda")
    grads = {}
    if do is not None:
        grads = dict(dout=do, dq=torch.full_like(o, float("nan")), dk=torch.full(k.shape, float("nan"), dtype=k.dtype, device="cuda"),
                     dv=torch.full(v.shape, float("nan"), dtype=v.dtype, device="cuda"))
        grads.update({n: kw.pop(n) for n in ("dq", "dk", "dv") if n in kw})
    p = binding.make_params(q, k, v, o, lse, 0, **grads, **kw)
    binding.s2attn_window_fwd(p, window, sinks)
    out = dict(o=o.clone(), lse=lse.clone())
    if do is not None:
        n = binding.window_workspace_bytes(p, window, sinks) if ws_bytes is None else ws_bytes(p)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # NaN in all that is read before it is written
        binding.s2attn_window_bwd(binding.make_params(q, k, v, o, lse, 0, workspace=ws, **grads, **kw), window, sinks)
        torch.cuda.synchronize()
        out.update({n: grads[n] for n in ("dq", "dk", "dv")})
    torch.cuda.synchronize()
    return out


def check(dtype, shape, window, sinks, seed, backward=True, **kw):
    B, N, H, Hkv, D = shape
    q, k, v, do = make(dtype, B, N, H, Hkv, D, seed, kw.pop("size", 1.0))
    want = ref.window_reference(q, k, v, do if backward else None, window, sinks, kw.get("scale"))
    got = run(q.cuda(), k.cuda(), v.cuda(), do.cuda() if backward else None, window, sinks, **kw)
    for name in got:
        ref.hold(name, got[name], want)
    return got


# (B, N, H, Hkv, D), window, sinks
SMALL = [
    ((1, 1, 1, 1, 64), 1, 0),
    ((1, 1, 2, 1, 128), 5, 3),
    ((2, 2, 3, 3, 128), 1, 1),
    ((1, 17, 3, 1, 64), 1, 0),           # every token sees itself alone
    ((1, 33, 2, 2, 128), 16, 1),
    ((3, 65, 5, 5, 64), 64, 0),
    ((1, 127, 4, 2, 128), 200, 4),       # a window beyond the sequence
    ((2, 130, 6, 2, 64), 31, 200),       # sinks beyond it: plain causal
    ((1, 257, 8, 1, 128), 100, 7),
    ((1, 300, 7, 7, 64), 32, 33),        # odd heads
    ((1, 520, 4, 4, 128), 129, 128),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", SMALL, ids=str)
def test_small(dtype, case):
    shape, window, sinks = case
    check(dtype, shape, window, sinks, seed=sum(shape) + window)


# enough rows for the kernels of large tiles, with sequences cut into stretches, sinks cut into segments and left whole
LARGE = [
    ("f32", (1, 1300, 9, 9, 64), 257, 4),
    ("f32", (2, 1030, 6, 2, 128), 100, 70),
    ("f32", (1, 2600, 5, 5, 64), 64, 600),      # ten tiles of sinks
    ("f32", (1, 1100, 12, 3, 128), 1500, 0),
    ("bf16", (1, 1500, 9, 9, 128), 257, 4),
    ("bf16", (2, 1030, 8, 2, 128), 64, 130),
    ("bf16", (1, 2100, 6, 1, 128), 300, 1100),  # nine tiles of sinks
    ("bf16", (1, 1200, 12, 12, 128), 128, 0),
    ("bf16", (1, 1500, 3, 3, 64), 257, 4),
    ("bf16", (2, 1030, 8, 2, 64), 64, 130),
    ("bf16", (1, 2100, 6, 1, 64), 1, 1100),
    ("bf16", (1, 900, 16, 2, 64), 1000, 5),
]


@pytest.mark.parametrize("case", LARGE, ids=str)
def test_large(case):
    dtype, shape, window, sinks = case
    check(dtype, shape, window, sinks, seed=sum(shape) + window)


@pytest.mark.parametrize("sinks", [0, 70])
def test_long_window_forward(sinks):
    """Eight waves to a workgroup from a window of 4096 on."""
    N, H, window = 4500, 4, 4200
    q, k, v, _ = make("bf16", 1, N, H, 2, 128, seed=5)
    want = ref.window_reference(q, k, v, None, window, sinks, heads=(1, 3))
    got = run(q.cuda(), k.cuda(), v.cuda(), None, window, sinks)
    for h in (1, 3):
        ref.hold("o", got["o"], want, (0, slice(None), h))
        ref.hold("lse", got["lse"], want, (0, h))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_peaked_scores(dtype):
    check(dtype, (1, 400, 4, 2, 64), 90, 3, seed=3, size=6.0)
    check(dtype, (1, 200, 2, 2, 128), 50, 0, seed=4, scale=0.5)


@pytest.mark.parametrize("dtype,D,N", [("f32", 64, 200), ("f32", 128, 1100), ("bf16", 64, 500), ("bf16", 128, 300), ("bf16", 128, 1400)])
def test_packed_views(dtype, D, N):
    """q, k, v and their gradients as slices of packed projections."""
    B, H = 2, 8
    q, k, v, do = make(dtype, B, N, H, H, D, seed=11)
    want = ref.window_reference(q, k, v, do, 70, 5)
    x = torch.stack([q, k, v], 2).cuda()
    g = torch.full_like(x, float("nan"))
    run(x[:, :, 0], x[:, :, 1], x[:, :, 2], do.cuda(), 70, 5, strided=True, dq=g[:, :, 0], dk=g[:, :, 1], dv=g[:, :, 2])
    for i, name in enumerate(("dq", "dk", "dv")):
        ref.hold(name, g[:, :, i], want)


@pytest.mark.parametrize("over", ["q", "o", "do"])
@pytest.mark.parametrize("dtype,shape", [("f32", (1, 200, 4, 2, 64)), ("f32", (1, 1400, 10, 5, 128)), ("bf16", (1, 300, 4, 2, 128)),
                                         ("bf16", (1, 1500, 8, 4, 128)), ("bf16", (1, 700, 4, 2, 64))], ids=str)
def test_dq_over_an_input(dtype, shape, over):
    q, k, v, do = make(dtype, *shape, seed=21)
    want = ref.window_reference(q, k, v, do, 90, 3)
    B, N, H = shape[:3]
    t = dict(q=q.cuda(), k=k.cuda(), v=v.cuda(), do=do.cuda(), o=torch.empty_like(q, device="cuda"))
    lse = torch.empty(B, H, N, device="cuda")
    dk, dv = torch.empty_like(t["k"]), torch.empty_like(t["v"])
    kw = dict(dout=t["do"], dq=t[over], dk=dk, dv=dv)
    p = binding.make_params(t["q"], t["k"], t["v"], t["o"], lse, 0, **kw)
    binding.s2attn_window_fwd(p, 90, 3)
    ws = torch.empty(binding.window_workspace_bytes(p, 90, 3), dtype=torch.uint8, device="cuda")
    binding.s2attn_window_bwd(binding.make_params(t["q"], t["k"], t["v"], t["o"], lse, 0, workspace=ws, **kw), 90, 3)
    torch.cuda.synchronize()
    for name, x in (("dq", t[over]), ("dk", dk), ("dv", dv)):
        ref.hold(name, x, want)


@pytest.mark.parametrize("dtype,shape,window,sinks", [("f32", (1, 700, 16, 1, 64), 300, 4), ("bf16", (1, 2000, 16, 1, 128), 1000, 4),
                                                      ("bf16", (1, 2000, 16, 1, 64), 1000, 40)], ids=str)
def test_least_workspace(dtype, shape, window, sinks):
    """The parts of a kv head's query heads need workspace; without it they run in one."""
    check(dtype, shape, window, sinks, seed=31, ws_bytes=lambda p: least_workspace(p, window, sinks))
    check(dtype, shape, window, sinks, seed=31)


def test_gradient_against_differences():
    """Along a direction: sum(grad * direction) against differences of the 64-bit forward.  h = 2^-10: the third derivative's
    part, of the order of h^2 = 1e-6 of the value, goes in with 2^-16 of the sum of magnitudes."""
    shape, window, sinks = (1, 150, 4, 2, 64), 40, 3
    q, k, v, do = make("f32", *shape, seed=41)
    got = run(q.cuda(), k.cuda(), v.cuda(), do.cuda(), window, sinks)
    bounds = ref.window_reference(q, k, v, do, window, sinks)
    gen = torch.Generator().manual_seed(42)
    h = 2.0 ** -10
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        way = torch.randn(x.shape, generator=gen, dtype=torch.float64)

        def loss(step):
            y = {n: t.double() for n, t in (("dq", q), ("dk", k), ("dv", v))}
            y[name] = y[name] + step * way
            return (ref.window_reference(y["dq"], y["dk"], y["dv"], None, window, sinks)["o"] * do.double()).sum()

        want = (loss(h) - loss(-h)) / (2 * h)
        have = (got[name].double().cpu() * way).sum()
        room = (bounds["b_" + name] * way.abs()).sum() + 2.0 ** -16 * (bounds[name] * way).abs().sum()
        assert (have - want).abs() <= room, (name, float(have), float(want), float(room))


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("bf16", 64), ("bf16", 128)])
def test_padding_rows(dtype, D):
    """Rows behind a sequence's end with dout = 0 leave the gradients of the others alone, whatever finite k and v they have."""
    q, k, v, do = make(dtype, 1, 600, 4, 4, D, seed=51)
    n = 411
    do[:, n:] = 0
    want = ref.window_reference(q[:, :n], k[:, :n], v[:, :n], do[:, :n], 100, 4)
    q[:, n:], k[:, n:], v[:, n:] = 3.0, -7.0, 1e4
    got = run(q.cuda(), k.cuda(), v.cuda(), do.cuda(), 100, 4)
    for name in ("o", "dq", "dk", "dv"):
        ref.hold(name, got[name][:, :n], want)
    assert not got["dq"][:, n:].any()


@pytest.mark.parametrize("dtype,D,N", [("f32", 64, 500), ("bf16", 128, 500), ("bf16", 128, 1500), ("bf16", 64, 1100)])
def test_runs_repeat_and_capture(dtype, D, N):
    """Same bits every time: eager, on another stream, and on every replay of a graph between eager calls on other data."""
    window, sinks = 130, 6
    q, k, v, do = (x.cuda() for x in make(dtype, 1, N, 8, 2, D, seed=61))
    o, lse = torch.empty_like(q), torch.empty(1, 8, N, device="cuda")
    g = dict(dout=do, dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v))
    p = binding.make_params(q, k, v, o, lse, 0, **g)
    ws = torch.empty(binding.window_workspace_bytes(p, window, sinks), dtype=torch.uint8, device="cuda")
    p = binding.make_params(q, k, v, o, lse, 0, workspace=ws, **g)
    outs = (o, lse, g["dq"], g["dk"], g["dv"])

    def step():
        binding.s2attn_window_fwd(p, window, sinks)
        binding.s2attn_window_bwd(p, window, sinks)

    def clear():
        for x in outs:
            x.fill_(float("nan"))
        ws.fill_(255)

    def eager(seed):
        for x, y in zip((q, k, v, do), make(dtype, 1, N, 8, 2, D, seed)):
            x.copy_(y)
        clear()
        step()
        torch.cuda.synchronize()
        return [x.clone() for x in outs]

    first = eager(61)
    stream = torch.cuda.Stream()
    clear()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for seed in (62, 61, 63):
        want = eager(seed)
        clear()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), seed
    assert all(torch.equal(a, b) for a, b in zip(eager(61), first))
