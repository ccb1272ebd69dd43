"""Parameter blocks of the binding: what they are made of, and what the calls check; no GPU."""
from paper_2309_12307_amd import binding


def test_blocks_without_tensors():
    """A block that only asks for a workspace's size has dimensions and a type, and addresses or nothing."""
    dims = (1, 1024, 4, 2, 128)
    for nothing in (None, 0x10000):
        p = binding.make_params(nothing, nothing, nothing, nothing, nothing, 256, dims=dims, dtype=binding.BF16)
        assert (p.B, p.N, p.H, p.Hkv, p.D, p.G, p.dtype) == (*dims, 256, binding.BF16) and p.q == nothing
        assert binding.bwd_workspace_bytes_ex(p) >= binding.bwd_workspace_bytes(*dims, 256)
        assert binding.window_workspace_bytes(p, 100, 4) > 0
