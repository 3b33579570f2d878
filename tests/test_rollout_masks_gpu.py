"""Log probabilities and their gradient over rows with finite mask values, from 2^24 / T to the type's lowest, at several temperatures.

Tolerances: as in test_rollout_gpu.py, with every logit counted by its distance from the row's largest y, and not by its own size: a sum's terms are
off by their distance times 2 u log2 e, what is far away weighs nothing, and a log probability is off by its own distance's rounding and the sum's.
"""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as R
from tests.test_rollout_gpu import HALF_STEP, SMALLEST, TYPES, U, host, near, say

MASKS = {"bf16": (-1e8, -1e9, -1e10, -1e12, -1e20, -1e30, -1e38, "lowest"), "f16": (-60000, "lowest"),
         "f32": (-1e8, -1e9, -1e10, -1e12, -1e20, -1e30, -1e38, "lowest")}


def masked_rows(dtype, mask, vocab, temperature):
    """Rows under one mask value, their targets: everything masked; all but a few; the first half, the second half, every lane's first vectors;
    ruled-out tokens (-inf) beside masked ones; the lowest value beside masked ones; the mask and what is next above it."""
    gen = torch.Generator().manual_seed(vocab)
    low = torch.finfo(TYPES[dtype]).min
    mask = low if mask == "lowest" else mask
    few = torch.randperm(vocab, generator=gen)[:max(2, vocab // 300)]
    x = 2 * torch.randn(10, vocab, generator=gen)
    kept = x.clone()
    x[0] = mask
    x[1] = mask
    x[1, few] = kept[1, few]
    x[2, :vocab // 2] = mask
    x[3, vocab // 2:] = mask
    x[4, torch.arange(vocab) < min(vocab - 1, 16384)] = mask
    x[5] = mask
    x[5, ::3] = -np.inf
    x[5, few[:1]] = 1
    x[6] = mask
    x[6, 1::2] = low
    x[7] = low
    x[7, 1::2] = mask
    x[7, few] = kept[7, few]
    x[8] = -np.inf
    x[8, few] = mask
    x = x.to(TYPES[dtype])
    # neighbours of the mask value: a step away, which is a distance of its own
    x[9] = mask
    step = torch.nextafter(x[9, :1].clone(), torch.zeros(1, dtype=x.dtype))
    x[9, few] = step
    targets = torch.tensor([vocab - 1, int(few[0]), vocab - 1, 0, vocab - 1, int(few[0]), 0, int(few[1]), int(few[0]), int(few[1])])
    return x.cuda(), targets.cuda()


def check(x, targets, temperature):
    from paper_2409_19256_amd import rollout
    dtype = {v: k for k, v in TYPES.items()}[x.dtype]
    vocab, top = x.shape[1], min(20, x.shape[1])
    got = rollout.token_logprobs(x, targets, temperature, top)
    gen = torch.Generator("cuda").manual_seed(vocab)
    g, h = torch.randn(len(x), generator=gen, device="cuda"), torch.randn(len(x), generator=gen, device="cuda")
    dx = rollout.token_logprobs_back(x, targets, got.norm, got.entropy, g, h, temperature)
    torch.cuda.synchronize()
    xs, t = host(x), targets.cpu().numpy()
    lp, ent, lse, logp, live = R.logprobs(xs, t, temperature)
    rel = (vocab / 64 + 80) * U + 16 * U
    fin = lambda a: np.where(np.isfinite(a), np.abs(a), 0)  # noqa: E731
    near(host(got.logprob), lp, rel + 12 * U * fin(lp), "logprob")
    near(host(got.lse), lse, rel + 4 * U * fin(lse), "lse")
    near(host(got.entropy), ent, (2 * rel + 8 * U) * (1 + np.log(vocab) + fin(ent)) * 2, "entropy")
    want = R.top_ids(xs, top)
    assert np.array_equal(got.top_ids.cpu().numpy(), want)
    w = np.take_along_axis(logp, want, 1)
    near(host(got.top_logprobs), w, rel + 12 * U * fin(w), "top")
    dwant, p, logp = R.logprobs_back(xs, t, temperature, host(g), host(h))
    ln = fin(logp)
    d, e = rel + 4 * U * (3 * ln + 2), (4 * rel + 16 * U) * (1 + np.log(vocab) + np.abs(ent[:, None]))
    ag, ah = np.abs(host(g))[:, None], np.abs(host(h))[:, None]
    tol = (p * ((ag + ah * (ln + np.abs(ent[:, None]))) * (d + 8 * U) + ah * (d + e)) + 8 * U * ag) / temperature
    near(host(dx), dwant, tol * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(dwant) + SMALLEST[dtype] + 2.0 ** -126, "dx")


@pytest.mark.gpu
@pytest.mark.parametrize("temperature", [0.7, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("vocab", [40, 5004, 33000])
@pytest.mark.parametrize("dtype,mask", [(d, m) for d in MASKS for m in MASKS[d]], ids=str)
def test_mask_values(dtype, mask, vocab, temperature):
    say("[mask values]", dtype, mask, vocab, temperature)
    check(*masked_rows(dtype, mask, vocab, temperature), temperature)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,temperature", [("f16", 1e-3), ("f16", 2e-4), ("bf16", 1e-6), ("f32", 1e-30)])
def test_mask_values_at_low_temperatures(dtype, temperature):
    """Here ordinary logits too are past 2^24 once they are divided."""
    say("[mask values, low temperature]", dtype, temperature)
    check(*masked_rows(dtype, "lowest", 5004, temperature), temperature)


@pytest.mark.gpu
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("temperature", [0.7, 1.0])
def test_logits_about_where_the_base_changes(sign, temperature):
    """32-bit logits on both sides of 2^24 in base 2, a step or two apart: lanes of a row differ in how they hold their base, and are joined."""
    say("[about the limit]", sign, temperature)
    gen = torch.Generator().manual_seed(3)
    at = 2 ** 24 * np.log(2) * temperature
    x = sign * at + 3 * torch.randn(6, 20000, generator=gen, dtype=torch.float64)
    x[1] += 40 * sign
    x[2] -= 40 * sign
    x[3, :9000] = sign * at * 1.5
    x[4, 9000:] = sign * at / 1.5
    x[5] = torch.linspace(at * sign - 200, at * sign + 200, 20000, dtype=torch.float64)
    x = x.float().cuda()
    check(x, x.argmax(1), temperature)
