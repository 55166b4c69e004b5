"""A call that fails says so itself, and leaves nothing behind that a later call would report."""
import pytest
import torch

from gpu_util import DEV


@pytest.mark.gpu
def test_a_failed_allocation_is_not_the_next_calls_error(dp):
    import paper_2108_01624_amd as pkg

    x = torch.ones(8, device=DEV)
    with pytest.raises(pkg.DpError) as e:
        pkg.Context(workspace_bytes=1 << 60)   # (more than there is)
    assert e.value.status == -8
    dp.zero_f32(x)
    dp.sync()
    assert not x.any()
