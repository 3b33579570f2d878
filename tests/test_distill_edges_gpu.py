"""Distillation where the forward pass takes a row apart: every place at which a lane, a batch, a window of the bitmap or the row begins or ends holds half of what is summed, so that an element
that is lost or counted twice moves the results by thousands of tolerances; bases past 2^24, where the sum is counted from an element itself; and the loads past the caches.

Tolerances.  u = 2^-24.  The sum over the unnamed tokens, relative to itself (`rel`):
 - a lane adds its terms one after another, u each; lanes and wavefronts another 10;
 - a term's exponent of base 2 is off by u |D| from the rounding of c = log2(e) / temperature and by u |d| from its own, where D is counted from the row's largest unnamed element and d from the
   lane's base, which is at most 8.5 below it: together (2 |D| + 9) u ln 2 of the term, and 2 u for the hardware's exponential; |D| is at most 22 (35 in the test of bases), and terms far below are small;
 - a sum moves to another base at most four times on the way and twice at the end, 2 u each.
That is 61 u (79 u) beside the additions: 64 (80) here.  norm[1], its logarithm, is off by rel and by half a step of its own.  A probability of the named tokens or of the rest is off by 2 rel of itself and its
logarithm by 2 rel, the loss by 2 rel of the sizes that the oracle gives and two roundings.  A slope is a product of two numbers that are off so, one of them a sum over all: 8 rel of the oracle's size; then six
roundings, the gradient's own exponential (its argument (x - m) / temperature - norm[1] goes through three roundings and holds that of norm[1], 4 u of its size) and one to the type.
"""
import numpy as np
import pytest
import torch

from oracle import steps_oracle as S
from tests.test_rollout_gpu import HALF_STEP, SMALLEST, TYPES, U, host, near, say
from tests.test_steps_gpu import bits_of, gen_of

QS = torch.tensor([0.3, 0.2, 0.1, 0.05, 0.05])  # a teacher's named tokens; 0.3 is left for the others


def lanes_of(dtype, vocab):
    """Lanes of a row, and elements of a vector."""
    kv = 4 if dtype == "f32" else 8
    return next(n for n, most in ((64, 512), (256, 2048), (512, 8192), (1024, 1 << 30)) if vocab // kv <= most), kv


def rel_of(dtype, vocab, others=64):
    lanes, kv = lanes_of(dtype, vocab)
    return ((-(-(vocab // kv) // lanes) + 1) * kv + others) * U


def by_logarithms(x, ids, lq, temperature, w, rest):
    """What the oracle gives, for rows whose tokens are named once each: every probability by its logarithm, from differences of logits alone.  (The oracle asks whether the others' sum is above 0 where
    e^-65504 is 0 in 64 bits, too, and adds a logarithm of order 1 to logits of 10^38.)"""
    rows, vocab = x.shape
    loss, grad, loss_size, grad_size = np.zeros(rows), np.zeros((rows, vocab)), np.zeros(rows), np.zeros((rows, vocab))
    y = x / temperature
    for r in range(rows):
        other = np.ones(vocab, bool)
        other[ids[r]] = False
        top, m = y[r].max(), y[r][other].max()
        s = np.log(np.exp(y[r][other] - m).sum())
        parts = np.append(y[r][ids[r]] - top, (m - top) + s)
        lp = parts - np.log(np.exp(parts).sum())
        q = np.append(np.exp(lq[r]), 1 - np.exp(lq[r]).sum())
        lq_all = np.append(lq[r], np.log(q[-1]))
        p, counts = np.exp(lp), np.append(np.ones(len(ids[r])), float(rest))
        back = np.where(p > 0, p * (lp - lq_all), 0)
        loss[r] = (counts * ((0 if w == 1 else (1 - w) * q * (lq_all - lp)) + w * back)).sum()
        loss_size[r] = (counts * ((1 - w) * q + w * (np.abs(back) + p))).sum()
        f = counts * (-(1 - w) * q + w * (back + p))  # p times dloss/dp
        slope, size = f - p * f.sum(), counts * ((1 - w) * (q + p) + w * (np.abs(back) + p * (2 + abs((counts * back).sum())))) + (1 - counts) * p * (1 + abs(f.sum()))
        share = np.exp(np.minimum(y[r] - m, 0) - s)
        grad[r], grad_size[r] = share * slope[-1] / temperature, share * size[-1] / temperature
        grad[r][ids[r]], grad_size[r][ids[r]] = slope[:-1] / temperature, size[:-1] / temperature
    return loss, grad, loss_size, grad_size, y.max(1, keepdims=True) - y, np.ones(rows, bool)


def test_by_logarithms_agrees_with_the_oracle():
    rng = np.random.default_rng(1)
    x, ids = 3 * rng.standard_normal((9, 40)), np.stack([rng.permutation(40)[:5] for _ in range(9)])
    lq = np.tile(np.log(QS.numpy().astype(np.float64)), (9, 1))
    for w in (0.0, 0.3, 1.0):
        for rest in (True, False):
            for a, b in zip(by_logarithms(x, ids, lq, 0.7, w, rest), S.distill(x, ids, lq, 0.7, w, rest)):
                assert np.allclose(a, b, rtol=1e-12, atol=1e-13)


def compared(x, ids, lq, temperature, reverse, rest, dtype, gen, rel, what, oracle=S.distill):
    """Loss, gradient and norm against the oracle."""
    from paper_2409_19256_amd import rollout
    r = rollout.top_distill(x, ids, lq, temperature, reverse, rest)
    g = 0.5 + torch.rand(len(x), generator=gen, device="cuda")
    grad = rollout.top_distill_back(x, ids, r.norm, r.slopes, g, temperature)
    loss, slope, loss_size, grad_size, spread, live = oracle(host(x), ids.cpu().numpy(), host(lq), temperature, reverse, rest)
    assert live.all()
    near(host(r.loss), loss, (2 * rel + 2 * U) * loss_size + 2 * U * np.abs(loss), what + " loss")
    others = torch.ones_like(x, dtype=torch.bool).scatter_(1, ids.long(), False)
    y = np.where(others.cpu().numpy(), host(x), -np.inf)
    m = y.max(1)
    sums = np.log(np.exp((y - m[:, None]) / temperature).sum(1))
    assert np.array_equal(host(r.norm)[:, 0], m), what
    near(host(r.norm)[:, 1], sums, rel + U * np.abs(sums), what + " norm")
    w = host(g)[:, None]
    d = 4 * (np.minimum(spread, 200.0) + sums[:, None]) * U
    near(host(grad), w * slope, w * (8 * rel + 12 * U + d) * grad_size + HALF_STEP[dtype] * np.abs(w * slope) + SMALLEST[dtype] + 2.0 ** -126, what + " gradient")
    return r, sums


EDGES = [(d, v) for d, sizes in (("f32", (1031, 2051, 2052, 8195, 32770, 32772, 50257, 131072, 131072 + 13, 300007)), ("bf16", (1031, 4103, 4104, 16391, 65543, 131072 + 13, 262144 + 9)),
                                 ("f16", (515, 16384, 32000, 65552, 140001))) for v in sizes]


@pytest.mark.gpu
@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("dtype,vocab", EDGES)
def test_edges(dtype, vocab, named):
    """A row to an edge.  Its element holds half of the sum; or it is named, and as large as the sum that it may not get into."""
    say("[distill, edges]", dtype, vocab, named)
    gen = gen_of(dtype, vocab, named)
    lanes, kv = lanes_of(dtype, vocab)
    window, batch = {64: 1 << 13, 256: 1 << 15}.get(lanes, 1 << 17), lanes * kv
    per = 4 if dtype == "f32" else 2
    at = {0, 1, kv - 1, kv, vocab - 1, vocab - 2, vocab // kv * kv - 1, vocab // kv * kv, vocab // kv * kv - kv}
    for step in (batch, per * batch, 2 * per * batch, vocab // (per * batch) * per * batch, vocab // batch * batch, window, 2 * window):
        at |= {step - 1, step, step + kv}
    edges = torch.tensor(sorted(e for e in at if 0 <= e < vocab), device="cuda")
    rows = len(edges)
    x = 0.5 * torch.randn(rows, vocab, generator=gen, device="cuda")
    x[torch.arange(rows), edges] = float(np.log(vocab)) + 0.1
    x = x.to(TYPES[dtype])
    free = torch.rand(rows, vocab, generator=gen, device="cuda")
    free[:, edges] = 0
    ids = free.topk(5, 1).indices.int()
    if named:
        ids[:, 2] = edges.int()
    lq = QS.log().cuda().expand(rows, 5).contiguous()
    rel = rel_of(dtype, vocab)
    for reverse, rest, temperature in ((0.0, True, 1.0), (1.0, True, 0.5), (0.5, False, 1.0)):
        r, sums = compared(x, ids, lq, temperature, reverse, rest, dtype, gen, rel, f"{reverse} {rest}")
        # what one element's loss, or a second count of it, would do to norm[1]: at the least this many tolerances
        share = np.exp((host(x)[np.arange(rows), edges.cpu().numpy()] - host(r.norm)[:, 0]) / temperature - sums)
        least = np.log1p(share) if named else np.minimum(np.log1p(share), -np.log1p(-np.minimum(share, 1 - 1e-12)))
        assert (least > 1000 * (rel + U * np.abs(sums))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("reverse", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("dtype,vocab,temperature", [("f32", 1030, 1.0), ("f32", 140001, 0.5), ("bf16", 1030, 1.0), ("bf16", 140001, 0.5), ("f16", 1030, 1.0), ("f16", 50257, 0.5)])
def test_lowest_values(dtype, vocab, temperature, reverse, rest):
    """Rows in which finite logits stand beside the type's lowest value: the others at it, half of all, the named ones, a part, all but one of the others, whole lanes' first elements, and all."""
    say("[distill, lowest values]", dtype, vocab, temperature, reverse, rest)
    gen = gen_of(dtype, vocab, temperature, reverse, rest)
    x = torch.randn(8, vocab, generator=gen, device="cuda").to(TYPES[dtype])
    low = torch.finfo(x.dtype).min
    ids = torch.rand(8, vocab, generator=gen, device="cuda").topk(5, 1).indices.int()
    others = torch.ones_like(x, dtype=torch.bool).scatter_(1, ids.long(), False)
    x[0] = torch.where(others[0], low, x[0])
    x[1, ::2] = low
    x[2, ids[2].long()] = low
    x[3] = torch.where(torch.rand(vocab, generator=gen, device="cuda") < 0.3, low, x[3])
    one = int(others[4].nonzero()[vocab // 2])
    x[4] = torch.where(others[4] & (torch.arange(vocab, device="cuda") != one), low, x[4])
    x[5, :vocab * 2 // 3] = low
    x[6, vocab // 3:] = low
    x[7] = low
    lq = QS.log().cuda().expand(8, 5).contiguous()
    # (a term at the lowest value is nothing or, among others like it, 1)
    compared(x, ids, lq, temperature, reverse, rest, dtype, gen, rel_of(dtype, vocab), "lowest", by_logarithms)


@pytest.mark.gpu
@pytest.mark.parametrize("reverse,rest", [(0.0, True), (0.5, True), (1.0, False)])
@pytest.mark.parametrize("vocab", [1030, 50257, 300007])
def test_bases_past_whole_numbers(vocab, reverse, rest):
    """Logits whose exponents are near and past 2^24 and a few apart: rows on either side of it, across it (so that lanes with both bases are joined), negative ones, and logits that a low temperature brings there."""
    say("[distill, far bases]", vocab, reverse, rest)
    gen = gen_of("far", vocab, reverse, rest)
    steps = torch.randint(0, 25, (8, vocab), generator=gen, device="cuda").float()
    place = torch.arange(vocab, device="cuda")
    x = steps.clone()
    x[0] += 11629080 - 12        # 2^24 ln 2 is 11629080: both bases in a row
    x[1] = -11629080 + 12 - steps[1]
    x[2] = 3e7 + 2 * (steps[2] // 2)
    x[3] = -3e7 - 2 * (steps[3] // 2)
    x[4] = torch.where(steps[4] < 12, 11629080 - steps[4], 1000 + steps[4])
    x[5] += 1e7                  # below it throughout
    x[6] = torch.where(place < vocab // 2, 11629076 - steps[6] // 8, 11629084 + steps[6] // 8)  # the far ones last
    lanes, kv = lanes_of("f32", vocab)
    x[7] = torch.where(place // kv % lanes % 64 < 40, 11629078 - steps[7] // 8, 11629081 + steps[7] // 8)  # lanes with one base beside lanes with the other
    ids = torch.rand(8, vocab, generator=gen, device="cuda").topk(5, 1).indices.int()
    lq = QS.log().cuda().expand(8, 5).contiguous()
    rel = rel_of("f32", vocab, 80)
    compared(x, ids, lq, 1.0, reverse, rest, "f32", gen, rel, "large logits")
    cold = 2.0 ** -24            # its reciprocal is exact
    y = 2 + (steps // 4) * 2.0 ** -22
    y[1] = 0.6931471 + (steps[1] - 12) * 2.0 ** -24  # across 2^24 again
    y[2] = -y[2]
    compared(y, ids, lq, cold, reverse, rest, "f32", gen, rel, "a low temperature")


@pytest.mark.gpu
@pytest.mark.parametrize("places", [7, 200])
@pytest.mark.parametrize("dtype,vocab", [("f32", 2048), ("f32", 8192), ("f32", 32003), ("f32", 128256), ("bf16", 4096), ("bf16", 16000), ("bf16", 65536), ("bf16", 100003), ("f16", 4103), ("f16", 16384),
                                         ("f16", 32000), ("f16", 131072 + 13)])
def test_past_the_caches(dtype, vocab, places):
    """Above 512 MiB the forward pass reads past the caches: the same bits as of the two halves, which it reads plainly; and three rows against the oracle."""
    from paper_2409_19256_amd import rollout
    say("[distill, past the caches]", dtype, vocab, places)
    gen = gen_of("once", dtype, vocab, places)
    size = 4 if dtype == "f32" else 2
    rows = (512 << 20) // (size * vocab) + 3
    x = torch.empty(rows, vocab, device="cuda", dtype=TYPES[dtype]).normal_(generator=gen)
    ids = torch.randint(-1, vocab + 1, (rows, places), generator=gen, device="cuda").int()
    lq = torch.log_softmax(torch.randn(rows, places + 1, generator=gen, device="cuda"), 1)[:, :places].contiguous()
    ids[5] = -1
    half = rows // 2
    assert rows * vocab * size > 512 << 20 >= (rows - half) * vocab * size
    whole = list(rollout.top_distill(x, ids, lq, 0.9, 0.5))
    parts = [list(rollout.top_distill(x[at], ids[at], lq[at], 0.9, 0.5)) for at in (slice(0, half), slice(half, rows))]
    for a, b in zip(whole, (torch.cat(p) for p in zip(*parts))):
        assert torch.equal(bits_of(a), bits_of(b))
    some = torch.tensor([0, half, rows - 1], device="cuda")
    loss, _, size_, *_ = S.distill(host(x[some]), ids[some].cpu().numpy(), host(lq[some]), 0.9, 0.5, True)
    rel = rel_of(dtype, vocab, 80)  # (a temperature that is rounded: u |D| more)
    near(host(whole[0][some]), loss, (2 * rel + 2 * U) * size_ + 2 * U * np.abs(loss), "loss")


@pytest.mark.gpu
@pytest.mark.parametrize("temperature", [3.5e-39, 2.0 ** -126, 2.0 ** 126, 2e38])
@pytest.mark.parametrize("vocab", [1030, 131072 + 13])
def test_the_ends_of_the_temperatures(vocab, temperature):
    """Whatever 1 / temperature is in 32 bits: equal logits are equal, and others are nothing beside them or as good as equal."""
    from paper_2409_19256_amd import rollout
    say("[distill, temperatures]", vocab, temperature)
    gen = gen_of("ends", vocab, temperature)
    x = torch.full((3, vocab), 0.25, device="cuda")
    x[1, 1::3] -= 1
    x[2] = 3e38
    ids = torch.arange(5, device="cuda", dtype=torch.int32).expand(3, 5) * 3  # among the largest
    lq = QS.log().cuda().expand(3, 5).contiguous()
    t = float(np.float32(1 / temperature)) ** -1  # what the kernel is given is exact
    for reverse in (0.0, 1.0):
        r = rollout.top_distill(x, ids.contiguous(), lq, t, reverse)
        loss, _, size, *_ = by_logarithms(host(x), ids.cpu().numpy(), host(lq), t, reverse, True)
        rel = rel_of("f32", vocab)
        near(host(r.loss), loss, (2 * rel + 2 * U) * size + 2 * U * np.abs(loss), "loss")
        grad = rollout.top_distill_back(x, ids.contiguous(), r.norm, r.slopes, torch.full((3,), min(1.0, t), device="cuda"), t)
        assert torch.isfinite(grad).all()
