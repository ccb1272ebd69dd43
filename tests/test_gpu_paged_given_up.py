"""Attention over a paged cache whose pages before the window have been given up: what no row sees may hold anything, up to
the sinks and to the first row's window, in every kind of workgroup."""
import pytest
import torch

import attention_reference as ref
from paged_cases import Batch

pytestmark = pytest.mark.gpu


def give_up(b, window, sinks):
    """NaN in every cached place that no row of its sequence sees; how many there are."""
    places = []
    for s, (n, kv) in enumerate(b.lens):
        lo = max(kv - n - window + 1, 0)
        places += [(int(b.table[s, j // b.page]), j % b.page) for j in range(min(sinks, lo), lo)]
    pages, at = (torch.tensor(x, device="cuda", dtype=torch.long) for x in zip(*places))
    for name in ("k", "v"):
        x = b.dev[name]
        if x.dtype == torch.float8_e4m3fn:
            x.view(torch.uint8)[pages, at] = 0x7F
            b.dev[name + "_exp"][pages, at] = 255
        else:
            x[pages, at] = float("nan")
    return len(places)


# lens, H, Hkv, D, page
CASES = [
    ([(1, 300), (1, 64), (1, 1300)], 8, 4, 64, 16),                  # single tokens
    ([(1, 300), (1, 64), (1, 1300)], 16, 1, 128, 24),
    ([(1, 200), (1, 1000)], 20, 1, 128, 16),                         # 20 heads to a kv head (e4m3: two blocks of rows)
    ([(1, 200), (1, 1000)], 24, 1, 64, 7),
    ([(1, 700), (20, 200), (130, 400), (16, 900)], 4, 2, 64, 16),    # few and many rows in one call
    ([(1, 700), (20, 200), (130, 400), (16, 900)], 4, 2, 128, 40),
    ([(300, 1000)], 2, 2, 128, 64),                                  # a chunk
]


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")])
@pytest.mark.parametrize("window,sinks", [(33, 0), (41, 5), (1, 70)])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_given_up(n, window, sinks, dtype, cache):
    lens, H, Hkv, D, page = CASES[n]
    b = Batch(lens, H, Hkv, D, page, dtype, cache, ("token", "head", "gaps")[n % 3], seed=n)
    want = b.reference(window, sinks)
    assert give_up(b, window, sinks) > 100
    b.check(*b.attend(window, sinks), want)
    b.check(*b.attend(window, sinks, workspace=0), want)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(100, 0), (333, 5), (1, 70)])
def test_given_up_before_a_long_chunk(window, sinks, cache):
    """Rows enough for eight waves to a workgroup: two kv heads out of many are compared."""
    b = Batch([(600, 1100), (520, 900)], 80, 80, 128, 16, "bf16", cache, seed=2)
    some = [0, 43]
    sub = {n: x[:, :, some] if x is not None else None for n, x in b.host.items()}
    want = ref.paged_reference(b.q[:, some], sub["k"], sub["v"], sub["k_exp"], sub["v_exp"], b.row_start, b.kv_len, b.table, window, sinks)
    assert give_up(b, window, sinks) > 100
    o, lse = b.attend(window, sinks)
    ref.hold("o", o[:, some], want)
    ref.hold("lse", lse[some], want)
