"""What rollout.py refuses on its own account, on the CPU and over stand-ins for the library."""
import pytest
import torch


def test_log_probabilities_need_targets():
    """And say so at once, not in the backward pass."""
    from paper_2409_19256_amd import rollout
    x = torch.randn(3, 7).requires_grad_()
    with pytest.raises(ValueError, match="targets"):
        rollout.logprobs(x, None)
