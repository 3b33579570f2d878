"""Log probabilities at the ends of the temperatures: whatever 1 / temperature is in 32 bits, equal logits are equal, and others are nothing beside them or as good as equal."""
import numpy as np
import pytest
import torch

from tests.test_rollout_gpu import U, host, near, say


@pytest.mark.gpu
@pytest.mark.parametrize("temperature", [3.5e-39, 2.0 ** -126, 2.0 ** 126, 2e38])
@pytest.mark.parametrize("vocab", [1030, 131072 + 13])
def test_logprobs(vocab, temperature):
    from paper_2409_19256_amd import rollout
    say("[logprobs, temperatures]", vocab, temperature)
    x = torch.full((3, vocab), 0.25, device="cuda")
    x[1, 1::3] -= 1
    x[2] = -0.0
    t = float(np.float32(1 / temperature)) ** -1  # what the kernel is given is exact
    y = host(x) / t
    lp = y - y.max(1, keepdims=True)
    lp -= np.log(np.exp(lp).sum(1, keepdims=True))
    p = np.exp(lp)
    targets = torch.tensor([0, 3, vocab - 1], device="cuda")
    r = rollout.token_logprobs(x, targets, t, top=2)
    # terms of 1 or 0, or within 2^-100 of 1: vocab / 64 + 80 additions, and roundings of numbers up to ln vocab
    rel = (vocab / 64 + 80) * U + 4 * U * np.log(vocab)
    near(host(r.logprob), lp[np.arange(3), targets.cpu().numpy()], np.full(3, rel), "logprob")
    near(host(r.entropy), -(p * np.where(p > 0, lp, 0)).sum(1), np.full(3, 4 * rel), "entropy")
    near(host(r.top_logprobs), -np.sort(-lp, 1)[:, :2], np.full((3, 2), rel), "likeliest")
    grad = rollout.token_logprobs_back(x, targets, r.norm, r.entropy, torch.full((3,), min(1.0, t), device="cuda"), None, t)
    assert torch.isfinite(grad).all()
