"""The rollout operators beside torch's autograd: results that may be written to, writes that it has to know of, gradients that are not taken."""
import pytest
import torch

from tests.test_rollout_gpu import near, say


def log_softmax_pair(x, t, temperature=1.0):
    logp = torch.log_softmax(x.double() / temperature, 1)
    return logp.gather(1, t[:, None])[:, 0], -(logp.exp() * logp).sum(1)


def leaf(rows=6, vocab=77, dtype=torch.float32, seed=1):
    gen = torch.Generator("cuda").manual_seed(seed)
    x = (2 * torch.randn(rows, vocab, generator=gen, device="cuda")).to(dtype).requires_grad_()
    return x, torch.randint(0, vocab, (rows,), generator=gen, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("change", ["mul_", "masked_fill_", "detached logprob", "detached entropy"])
def test_results_may_be_written_to(change):
    """As masking a loss does: in place, each of the two by itself, with the gradient unharmed."""
    from paper_2409_19256_amd import rollout
    say("[in place]", change)
    x, t = leaf()
    keep = torch.tensor([1, 0, 1, 1, 0, 1], device="cuda").bool()
    y = x.detach().clone().requires_grad_()
    lp, ent = rollout.logprobs(x, t)
    want, want_ent = log_softmax_pair(y, t)
    if change == "mul_":
        lp.mul_(keep)
        ent.mul_(2)
        loss, want = lp.sum() + ent.sum(), (want * keep).sum() + 2 * want_ent.sum()
    elif change == "masked_fill_":
        lp.masked_fill_(~keep, 0.0)
        ent.masked_fill_(keep, 0.0)
        loss, want = lp.sum() + ent.sum(), want[keep].sum() + want_ent[~keep].sum()
    else:
        loss, want = 2 * lp.sum() + ent.sum(), 2 * want.sum() + want_ent.sum()
        (lp if "logprob" in change else ent).detach().zero_()
    loss.backward()
    want.backward()
    # every factor within 2^-18 of itself (logits below 2^4, sums of 77), gradients of order 1
    near(x.grad.double().cpu().numpy(), y.grad.double().cpu().numpy(), 2.0 ** -17, "gradient")
