"""Workspace that the paged attention asks for: bounded by what fills the chip, not by the longest prompt; no GPU."""
import pytest

from paper_2309_12307_amd.binding import BF16, E4M3, F32, paged_workspace_bytes
from test_paged_host import block

MIB = 1 << 20


@pytest.mark.parametrize("kw,most", [
    (dict(T=4097, B=2, table_cols=512), 17),           # a chunk of 4096 rows beside one token at 32k
    (dict(T=16385, B=2, table_cols=2048), 17),         # 16 384 beside one at 128k
    (dict(T=8192, B=2, table_cols=128), 17),           # two prompts of 4096 over up to 8k
])
def test_short_sequences_beside_prompts(kw, most):
    """Pieces of sixteen rows of each sequence and kv head at most, 16 * 8 * 128 pieces * 2 sequences of 129 floats: 16.1 MiB."""
    assert 0 < paged_workspace_bytes(block(H=64, Hkv=8, page_size=64, **kw)) <= most * MIB


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F32, F32), (BF16, E4M3)])
@pytest.mark.parametrize("H,Hkv,D", [(64, 8, 128), (32, 32, 64), (8, 1, 128), (40, 1, 128), (4, 4, 64)])
def test_bounded(H, Hkv, D, dtype, cache):
    """At most 2048 workgroups of pieces of 64 rows (a few more where the last does not divide), whatever the batch is."""
    for B in (1, 2, 3, 16, 100, 1000, 5000):
        for T in (1, 2, 17, 100, 300, 1000, 4096, 20000):
            for cols in (10, 300, 6000):
                for window in (0, 4096):
                    n = paged_workspace_bytes(block(T=T, B=B, H=H, Hkv=Hkv, D=D, dtype=dtype, cache_dtype=cache, table_cols=cols, window=window))
                    assert n <= 300 * MIB, (B, T, cols, window, n / MIB)
