"""CPU-only: arguments of the wrong kind are named, not left to fail somewhere inside."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_1412_2302_amd import binding
    return binding


@pytest.mark.parametrize("what", [None, [1.0], torch.zeros(4, 40, dtype=torch.int8)], ids=["none", "list", "tensor"])
def test_what_is_no_checkpoint(B, what):
    for call in (lambda: B.checkpoint_unpack(what), lambda: B.checkpoint_fc_backward_weight(what, torch.zeros(4, 3))):
        with pytest.raises(TypeError, match="expected a Checkpoint"):
            call()


@pytest.mark.gpu
def test_statistics_that_are_no_tensors(lib):
    x = torch.zeros((2, 4, 8), device="cuda")
    for mean, rstd in ((None, None), (x[:, 0, :2].contiguous(), None), (1.0, x[:, 0, :2].contiguous())):
        with pytest.raises(TypeError, match="mean"):
            lib.group_norm_backward(x, x, mean, rstd, None, None)
