"""A workspace is memory that a kernel writes: it has to be contiguous, or its element count says more than there is."""
import pytest
import torch

from paper_2506_05413_b200 import binding


@pytest.mark.parametrize("t", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, 2)[:, 0], torch.zeros(4, 8).T])
def test_a_workspace_that_is_not_contiguous_is_refused(t):
    with pytest.raises(ValueError):
        binding._workspace(t)


def test_a_contiguous_workspace_reaches_the_device_check():
    assert binding._workspace(None) == (None, 0)
    with pytest.raises(TypeError):
        binding._workspace(torch.zeros(16))


@pytest.mark.gpu
def test_calls_refuse_it():
    from paper_2506_05413_b200 import build
    build.build()
    z = lambda *s, t=torch.float16: torch.zeros(*s, dtype=t, device="cuda:0")  # noqa: E731
    need = binding.attn_decode_workspace_bytes(1, 4, 2, 128)
    cache = z(1, 2, 16, 128)
    before = binding.launch_count()
    for ws in (z(1, t=torch.uint8).expand(need), z(need, 2, t=torch.uint8)[:, 0]):
        with pytest.raises(ValueError):
            binding.attn_decode(z(1, 512), cache, cache.clone(), z(1, 1, t=torch.int32), z(1, t=torch.int32), z(1, 512), workspace=ws)
        with pytest.raises(ValueError):
            binding.linear(z(4, 128, t=torch.uint8), z(4, t=torch.float32), z(128, 128, t=torch.uint8), z(128, t=torch.float32), z(4, 128), ws)
        with pytest.raises(ValueError):
            binding.fuse_weights_search(z(4, 256), None, 0.5, 4, z(4, 128, t=torch.uint8), z(4, t=torch.float32), workspace=ws)
    assert binding.launch_count() == before
    assert binding._workspace(z(3, 5, t=torch.float32))[1] == 60
