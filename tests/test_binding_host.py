"""Parameter blocks of the binding: what they are made of, and what the calls check; no GPU."""
import pytest
import torch

from paper_2309_12307_amd import binding


def test_blocks_without_tensors():
    """A block that only asks for a workspace's size has dimensions and a type, and addresses or nothing."""
    dims = (1, 1024, 4, 2, 128)
    for nothing in (None, 0x10000):
        p = binding.make_params(nothing, nothing, nothing, nothing, nothing, 256, dims=dims, dtype=binding.BF16)
        assert (p.B, p.N, p.H, p.Hkv, p.D, p.G, p.dtype) == (*dims, 256, binding.BF16) and p.q == nothing
        assert binding.bwd_workspace_bytes_ex(p) >= binding.bwd_workspace_bytes(*dims, 256)
        assert binding.window_workspace_bytes(p, 100, 4) > 0


def tensors():
    x = lambda h: torch.zeros(1, 8, h, 64, dtype=torch.bfloat16)
    return dict(q=x(4), k=x(2), v=x(2), o=x(4), lse=torch.zeros(1, 4, 8), dout=x(4), dq=x(4), dk=x(2), dv=x(2))


def test_s2attn_blocks_are_made_without_a_look_at_the_tensors(monkeypatch):
    """What only the window calls ask is not found out for the others: it took longer than the block itself."""
    asked = []
    monkeypatch.setattr(binding, "_problem_of", lambda *a: asked.append(a))
    monkeypatch.setattr(binding, "_device_of", lambda *a: asked.append(a) or -1)
    t = tensors()
    p = binding.make_params(**t, G=4)
    assert binding.check_args(p, False) == 0 and not asked
    with pytest.raises(ValueError, match="not on a GPU"):
        binding.s2attn_window_fwd(p, 4)
    assert len(asked) == 2


@pytest.mark.parametrize("G", [0, 4])
@pytest.mark.parametrize("change", [dict(v=lambda x: x[:, :7]), dict(lse=lambda x: x.double()), dict(dk=lambda x: x[:, ::2]), dict(k=lambda x: x.float())], ids=lambda c: "+".join(c))
def test_window_calls_look_at_any_block(change, G):
    t = tensors()
    t.update({n: f(t[n]) for n, f in change.items()})
    p = binding.make_params(**t, G=G)
    for call in (binding.s2attn_window_fwd, binding.s2attn_window_bwd):
        with pytest.raises(ValueError, match=next(iter(change)) + " "):
            call(p, 4, 0)


def test_tensors_beside_addresses_and_tensors_that_are_gone():
    t = tensors()
    p = binding.make_params(**{**t, "k": 0x10000, "v": 0x10000}, G=4, dims=(1, 8, 4, 2, 64))
    with pytest.raises(ValueError, match="not on a GPU"):
        binding.s2attn_window_fwd(p, 4)
    t["v"] = t["v"][:, :7]
    p = binding.make_params(**t, G=4)
    del t["v"]
    with pytest.raises(ValueError, match="not on a GPU"):
        binding.s2attn_window_fwd(p, 4)


@pytest.mark.parametrize("G", [0, 4])
@pytest.mark.parametrize("workspace", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 21, dtype=torch.uint8)[::2],
                                       torch.zeros(1 << 20, dtype=torch.uint8, device="meta")], ids=["expanded", "strided", "elsewhere"])
def test_workspaces_that_are_not_there(workspace, G):
    """Fewer bytes than elements, or bytes of another device: the kernels would write outside."""
    t = tensors()
    p = binding.make_params(**t, workspace=workspace, G=G)
    with pytest.raises(ValueError, match="workspace must be contiguous on q's device"):
        binding.s2attn_window_bwd(p, 4, 0)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    cache, q = torch.zeros(6, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="workspace must be contiguous|one device"):
        binding.make_paged_params(i32(2), i32(1), i32(1, 3), cache, cache, q=q, o=q, workspace=workspace)
