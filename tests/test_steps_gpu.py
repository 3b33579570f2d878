"""What surrounds a rollout's steps, against the oracle in 64 bits, at the sizes, layouts and masks where it can go wrong.

Tolerances.  u = 2^-24 is half a unit in the last place of 1 in 32 bits; HALF_STEP is half a step of the output's type, relative to the value.
 - adjusted logits: at most six operations in 32 bits (quotient, product of frequency and count, two differences, sum), each off by u of what has gone into it so
   far: 6 u of the sum of the absolute values; then one rounding to the type.
 - distillation: a row's sum over the tokens that are not named has terms whose exponent d = (x - m) c is off by 3 u |d| of base e (c is rounded, so is the product; a
   term far below the largest is small by more than its error grows: |d| 2^-|d| < 1, so d counts as at most 64), by the hardware exponential's 2 u, and goes through vocab / 64 + 80 additions: `rel` together.  Every
   logarithm of a probability is off by rel, every probability by rel of itself; what is made of them is off by rel times the sizes that the oracle gives.  Then roundings to 32 bits
   (two on the way to a loss, six more on the way to a gradient, with another exponential of d) and one to the type.
 - tables, lengths, counts, slots and what is copied: the same bits.
"""
import zlib

import numpy as np
import pytest
import torch

from oracle import steps_oracle as S
from tests.test_rollout_gpu import HALF_STEP, SMALLEST, TYPES, U, host, near, new_cache, say


def gen_of(*key):
    return torch.Generator("cuda").manual_seed(zlib.crc32(repr(key).encode()))


def logits_of(gen, rows, vocab, dtype, pad=0, spread=2.0):
    """Rows of logits `pad` elements further apart than they are long."""
    return (spread * torch.randn(rows, vocab + pad, generator=gen, device="cuda")).to(TYPES[dtype])[:, :vocab]


def bits_of(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


# ---- adjust --------------------------------------------------------------------------------------------------------------

ADJUSTS = [
    # dtype, rows, vocab, pad, width, token type, biases, masks, order of tokens
    ("bf16", 1, 1, 0, 1, torch.int64, 1, 1),
    ("f32", 3, 7, 1, 5, torch.int32, 2, 2),
    ("f16", 5, 31, 0, 40, torch.int64, 3, 0),
    ("bf16", 4, 4096, 0, 300, torch.int64, 17, 3),
    ("bf16", 3, 4097, 1, 1000, torch.int32, 300, 2),
    ("f32", 2, 5004, 0, 2050, torch.int64, 0, 1),
    ("f16", 7, 12289, 3, 257, torch.int64, 5, 7),
    ("f32", 2, 32001, 2, 9, torch.int32, 1000, 0),
    ("bf16", 2, 50257, 0, 0, torch.int64, 0, 2),
    ("bf16", 2, 32000, 8, 0, torch.int64, 9, 0),
    ("f16", 66, 130, 0, 64, torch.int32, 4, 5),
    ("bf16", 3, 9001, 0, 9000, torch.int64, 20, 2),  # more tokens than the lanes hold
    ("f32", 17, 8192, 0, 5000, torch.int32, 70, 2),
    ("f16", 2, 16385, 1, 40000, torch.int32, 700, 0),  # counts of 32 bits
]


def adjustment(dtype, rows, vocab, pad, width, tokens, biases, masks, gen):
    """Arguments on the GPU; with tokens and biases that come often, more than once, or from outside the vocabulary."""
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    a = {}
    if width:
        wide = (rand(rows, width + 3) ** 2 * (vocab + 2)).to(tokens) - 1
        a["tokens"] = wide[:, :width]
        a["lens"] = (rand(rows) * (width + 3)).int() - 1  # below 0 and past the width, too
        a["prompt_lens"] = (rand(rows) * width).int()
        a["repetition"], a["frequency"], a["presence"] = 0.8 + rand(rows), rand(rows) - 0.3, rand(rows) - 0.3
    if biases:
        a["bias_ids"] = (rand(rows, biases) ** 2 * (vocab + 2)).int() - 1
        a["bias"] = 3 * torch.randn(rows, biases, generator=gen, device="cuda")
    if masks:
        words = (vocab + 31) // 32
        m = torch.randint(-2 ** 31, 2 ** 31, (masks, words + 1), generator=gen, device="cuda").int()
        m[0] = -1 if masks > 1 else 0  # all of a row, or none
        a["allowed"] = m[:, :words]
        a["allowed_rows"] = torch.randint(-1, masks + 1, (rows,), generator=gen, device="cuda").int()
    return a


def plain(v):
    return None if v is None else v.cpu().numpy()


def adjusted(x, a):
    p = {k: plain(v) for k, v in a.items()}
    if "allowed" in p:
        p["allowed"] = p["allowed"].view(np.uint32)
    return S.adjust(host(x), **p)


def check_adjusted(got, x, a, dtype, what):
    want, touched, size = adjusted(x, a)
    exact = np.where(np.isfinite(want), np.abs(want), 0)
    near(host(got), want, 6 * U * size + HALF_STEP[dtype] * exact + SMALLEST[dtype], what)
    same = (bits_of(got) == bits_of(x)).cpu().numpy()
    assert same[~touched].all(), what


@pytest.mark.gpu
@pytest.mark.parametrize("case", ADJUSTS, ids=str)
def test_adjust(case):
    from paper_2409_19256_amd import rollout
    say("[adjust]", case)
    dtype, rows, vocab, pad, width, tokens, biases, masks = case
    gen = gen_of(case)
    x = logits_of(gen, rows, vocab, dtype, pad)
    a = adjustment(*case, gen)
    before = x.clone()
    got = rollout.adjust_logits(x, **a)
    assert torch.equal(x, before) and got.shape == x.shape and got.dtype == x.dtype
    check_adjusted(got, x, a, dtype, "out of place")
    # into rows of another stride, and in place, with what lies between the rows left alone
    room = torch.full((rows, vocab + 5), 7.0, device="cuda", dtype=x.dtype)
    assert rollout.adjust_logits(x, **a, out=room[:, :vocab]).data_ptr() == room.data_ptr()
    assert torch.equal(bits_of(room[:, :vocab]), bits_of(got)) and (room[:, vocab:] == 7).all()
    store = torch.full((rows, vocab + 3), 7.0, device="cuda", dtype=x.dtype)
    mine = store[:, :vocab]
    mine.copy_(x)
    assert rollout.adjust_logits(mine, **a, out=mine) is mine
    assert torch.equal(bits_of(mine), bits_of(got)) and (store[:, vocab:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_adjust_one_thing_at_a_time(dtype):
    from paper_2409_19256_amd import rollout
    say("[adjust, parts]", dtype)
    gen = gen_of(dtype)
    x = logits_of(gen, 6, 4999, dtype)
    a = adjustment(dtype, 6, 4999, 0, 700, torch.int64, 8, 3, gen)
    text = {k: a[k] for k in ("tokens", "lens")}
    for part in (dict(), text, dict(text, prompt_lens=a["prompt_lens"], presence=a["presence"]), dict(text, repetition=a["repetition"]), dict(text, frequency=a["frequency"]),
                 {k: a[k] for k in ("bias_ids", "bias")}, {k: a[k] for k in ("allowed", "allowed_rows")},
                 dict(allowed=a["allowed"][:1].expand(6, -1)), dict(text, **{k: a[k] for k in ("allowed", "allowed_rows")})):
        got = rollout.adjust_logits(x, **part)
        check_adjusted(got, x, part, dtype, str(sorted(part)))
        mine = x.clone()
        rollout.adjust_logits(mine, **part, out=mine)
        assert torch.equal(bits_of(mine), bits_of(got)), sorted(part)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_adjust_infinities_and_nan(dtype):
    """What is not touched keeps its bits, a token that is ruled out is -inf whatever it was, and a row may be ruled out whole."""
    from paper_2409_19256_amd import rollout
    say("[adjust, infinities]", dtype)
    gen = gen_of(dtype, 1)
    x = logits_of(gen, 4, 515, dtype)
    low = torch.finfo(x.dtype).min
    x[0, ::5], x[1, ::7], x[2, ::3], x[3, ::2] = float("nan"), -float("inf"), low, float("inf")
    a = adjustment(dtype, 4, 515, 0, 90, torch.int32, 6, 2, gen)
    a["repetition"] = torch.full((4,), 0.75, device="cuda")  # what is at the type's end goes past it
    a["allowed"][1] &= 0x0F0F0F0F
    a["allowed"][0] = 0
    a["allowed_rows"][:] = torch.tensor([1, 1, 5, 0], device="cuda")
    got = rollout.adjust_logits(x, **a)
    want, touched, size = adjusted(x, a)
    # past the largest number: up to half a step (float16: 65504 and 32 / 2) it rounds to that number, then to infinity
    big, step = float(torch.finfo(x.dtype).max), float(torch.finfo(x.dtype).eps)
    over = np.abs(want) >= big * (1 + step / 2 / (2 - step))
    want = np.where(over, np.copysign(np.inf, want), np.where(np.isnan(want), want, np.clip(want, -big, big)))
    size = np.where(np.isfinite(size), size, 0)
    near(host(got), want, 6 * U * size + HALF_STEP[dtype] * np.where(np.isfinite(want), np.abs(want), 0) + SMALLEST[dtype], "values")
    assert (bits_of(got) == bits_of(x)).cpu().numpy()[~touched].all() and (got[3] == -float("inf")).all()
    mine = x.clone()
    rollout.adjust_logits(mine, **a, out=mine)
    assert torch.equal(bits_of(mine), bits_of(got)) or torch.equal(mine.isnan(), got.isnan()) and torch.equal(mine.nan_to_num(), got.nan_to_num())


@pytest.mark.gpu
@pytest.mark.parametrize("width", [900, 33000])
@pytest.mark.parametrize("biases", [0, 20, 100])
@pytest.mark.parametrize("dtype,tokens,vocab", [("bf16", torch.int64, 40001), ("f32", torch.int32, 40960), ("f16", torch.int64, 39999)])
def test_adjust_few_tokens_in_place(dtype, tokens, vocab, biases, width):
    """Rows of which little changes, beside one of which much does and one with a mask."""
    from paper_2409_19256_amd import rollout
    say("[adjust, in place]", dtype, biases, width)
    gen = gen_of(dtype, biases, width)
    x = logits_of(gen, 7, vocab, dtype, 1)
    a = adjustment(dtype, 7, vocab, 0, width, tokens, biases, 2, gen)
    a["lens"] = torch.tensor([0, 1, 63, 500, 880, width, 700], device="cuda", dtype=torch.int32)
    a["prompt_lens"] = torch.tensor([0, 0, 30, 499, 1000, width // 2, -1], device="cuda", dtype=torch.int32)
    a["allowed_rows"] = torch.tensor([-1, -1, 5, -1, 2, -1, 1], device="cuda", dtype=torch.int32)
    got = rollout.adjust_logits(x, **a)
    check_adjusted(got, x, a, dtype, "out of place")
    store = torch.full((7, vocab + 3), 7.0, device="cuda", dtype=x.dtype)
    mine = store[:, :vocab]
    mine.copy_(x)
    rollout.adjust_logits(mine, **a, out=mine)
    assert torch.equal(bits_of(mine), bits_of(got)) and (store[:, vocab:] == 7).all()


@pytest.mark.gpu
def test_adjust_many_times_the_same_token():
    from paper_2409_19256_amd import rollout
    say("[adjust, 70000 times one token]")
    x = torch.zeros(2, 9, device="cuda")
    tokens = torch.full((2, 70001), 4, device="cuda")
    lens = torch.tensor([70001, 70000], device="cuda", dtype=torch.int32)
    got = rollout.adjust_logits(x, tokens, lens, torch.tensor([1, 70000], device="cuda", dtype=torch.int32), frequency=torch.ones(2, device="cuda"))
    assert got[:, 4].tolist() == [-70000.0, 0.0] and (got != 0).sum() == 1


# ---- distill -------------------------------------------------------------------------------------------------------------

DISTILLS = [
    # dtype, rows, vocab, pad, places, temperature, reverse, rest
    ("f32", 3, 1, 0, 1, 1.0, 0.5, True),
    ("bf16", 2, 2, 1, 1, 1.0, 0.0, True),
    ("f16", 4, 9, 0, 9, 0.7, 1.0, True),      # the whole vocabulary is named
    ("f32", 5, 130, 3, 64, 1.3, 0.5, False),
    ("bf16", 6, 515, 0, 20, 1.0, 0.25, True),
    ("f16", 3, 4103, 1, 256, 1.0, 1.0, True),  # one wavefront, the longest list
    ("bf16", 3, 4104, 0, 5, 1.0, 0.0, False),
    ("f32", 2, 8195, 1, 65, 0.9, 1.0, False),
    ("bf16", 5, 16391, 0, 3, 1.0, 0.5, True),
    ("f16", 3, 32000, 8, 20, 1.0, 0.0, True),
    ("f32", 2, 50257, 0, 100, 1.0, 0.75, True),
    ("bf16", 2, 131072 + 13, 0, 64, 1.0, 0.5, True),  # more than the bitmap spans
    ("f32", 2, 300007, 1, 33, 1.0, 0.0, True),
]


def teacher(gen, x, places, temperature=1.0):
    """The likeliest tokens of a teacher near the student, in any order, as int32 and float32."""
    t = x.float() + 0.7 * torch.randn(x.shape, generator=gen, device="cuda")
    best = torch.log_softmax(t / temperature, 1).topk(places, 1)
    deal = torch.rand(best.indices.shape, generator=gen, device="cuda").argsort(1)
    return best.indices.gather(1, deal).int(), best.values.gather(1, deal).contiguous()


def tolerances(want, x, temperature, dtype, grad_loss):
    loss, grad, loss_size, grad_size, spread, _ = want
    rel = (x.shape[1] / 64 + 80 + 2 + 3 * 64) * U
    d = 4 * np.minimum(np.abs(spread), 200.0) * U  # the gradient's own exponential: below e^-200 nothing is left in 32 bits
    g = np.abs(grad_loss)[:, None]
    whole = np.where(np.isfinite(grad), np.abs(grad), 0)
    return ((2 * rel + 2 * U) * loss_size + 2 * U * np.where(np.isfinite(loss), np.abs(loss), 0),
            g * (4 * rel + 12 * U + d) * grad_size + HALF_STEP[dtype] * g * whole + SMALLEST[dtype] + 2.0 ** -126)


def check_distilled(x, ids, lq, temperature, reverse, rest, dtype, gen, what=""):
    from paper_2409_19256_amd import rollout
    r = rollout.top_distill(x, ids, lq, temperature, reverse, rest)
    g = torch.randn(len(x), generator=gen, device="cuda")
    grad = rollout.top_distill_back(x, ids, r.norm, r.slopes, g, temperature)
    want = S.distill(host(x), ids.cpu().numpy(), host(lq), temperature, reverse, rest)
    loss_tol, grad_tol = tolerances(want, x, temperature, dtype, host(g))
    near(host(r.loss), want[0], loss_tol, what + " loss")
    exact = np.where(want[5][:, None], host(g)[:, None] * want[1], 0.0)
    near(host(grad), exact, grad_tol, what + " gradient")
    mine = x.clone()
    assert rollout.top_distill_back(mine, ids, r.norm, r.slopes, g, temperature, out=mine) is mine
    assert torch.equal(bits_of(mine), bits_of(grad))
    return r, grad


@pytest.mark.gpu
@pytest.mark.parametrize("case", DISTILLS, ids=str)
def test_distill(case):
    say("[distill]", case)
    dtype, rows, vocab, pad, places, temperature, reverse, rest = case
    gen = gen_of(case)
    x = logits_of(gen, rows, vocab, dtype, pad)
    x[torch.arange(rows), torch.randint(0, vocab, (rows,))] += 12  # some rows are sure
    ids, lq = teacher(gen, x, places)
    check_distilled(x, ids, lq, temperature, reverse, rest, dtype, gen)


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("reverse", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("vocab,places", [(53, 30), (5004, 30), (5004, 200), (140001, 129)])
def test_distill_lists(vocab, places, reverse, rest):
    """Places that name nothing, tokens that come twice, rows without a name."""
    say("[distill, lists]", vocab, places, reverse, rest)
    gen = gen_of(vocab, places, reverse, rest)
    x = logits_of(gen, 9, vocab, "f32", 1)
    ids, lq = teacher(gen, x, places)
    ids[0, ::3] = -1
    ids[1, 1::2] = vocab + torch.arange(places // 2, device="cuda").int()
    lq[2, ::4] = -float("inf")
    ids[3, 5:9] = ids[3, 4]               # the first of five counts
    ids[4, 20], lq[4, 3] = ids[4, 3], -float("inf")  # a place without a log probability, and another with the same token
    ids[5] = ids[5, 0]
    ids[6] = -1                            # nobody: not read
    x[6] = float("nan")
    lq[7] = -float("inf")
    x[7, 3] = float("inf")
    ids[8, 10], ids[8, 11], lq[8, 10], lq[8, 11] = ids[8, 12], ids[8, 12], -float("inf"), -float("inf")
    r, grad = check_distilled(x, ids, lq, 1.0, reverse, rest, "f32", gen)
    assert r.loss[6] == 0 and r.loss[7] == 0 and (grad[6:8] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("reverse", [0.0, 0.5, 1.0])
def test_distill_masks(dtype, reverse):
    """Tokens ruled out with -inf or with the type's lowest value, named and not, up to whole rows; NaN and infinity."""
    say("[distill, masks]", dtype, reverse)
    gen = gen_of(dtype, reverse)
    x = logits_of(gen, 10, 1030, dtype)
    low = torch.finfo(x.dtype).min
    ids, lq = teacher(gen, x, 16)
    free = torch.ones_like(x, dtype=torch.bool).scatter_(1, ids.long(), False)
    x[0] = torch.where(free[0], -float("inf"), x[0])     # none but the named ones
    x[1] = torch.where(free[1], low, x[1])
    x[2, ids[2, :5].long()] = -float("inf")              # some of the named ones: the way ahead is infinite
    x[3] = -float("inf")
    x[4] = low
    x[5, ::2] = low
    x[6, 7] = float("nan")
    x[7, ids[7, 0].long()] = float("inf")
    x[8, ::3] = -float("inf")
    lq[8] = lq[8].clamp(min=-3.0)                        # more than 1 in sum
    lq[9, 2] = float("nan")
    from paper_2409_19256_amd import rollout
    for rest in (True, False):
        r = rollout.top_distill(x, ids, lq, 1.0, reverse, rest)
        g = torch.rand(10, generator=gen, device="cuda")
        grad = rollout.top_distill_back(x, ids, r.norm, r.slopes, g)
        want = S.distill(host(x), ids.cpu().numpy(), host(lq), 1.0, reverse, rest)
        loss_tol, grad_tol = tolerances(want, x, 1.0, dtype, host(g))
        keep = [i for i in range(10) if i not in (1, 4, 5)]  # (the oracle's differences of lowest values are past 32 bits: looked at below)
        near(host(r.loss)[keep], want[0][keep], np.where(np.isfinite(loss_tol), loss_tol, 0)[keep], "loss")
        near(host(grad)[keep], (host(g)[:, None] * want[1])[keep], np.nan_to_num(grad_tol, posinf=0)[keep], "gradient")
        # a row at its lowest value throughout is a row of equal logits, and one where the others are is as if they were ruled out
        even = torch.zeros_like(x)
        even[1], even[5] = x[1].float().masked_fill(x[1] == low, -1e4).to(x.dtype), x[5].float().masked_fill(x[5] == low, -1e4).to(x.dtype)
        s = rollout.top_distill(even, ids, lq, 1.0, reverse, rest)
        other = rollout.top_distill_back(even, ids, s.norm, s.slopes, g)
        assert torch.allclose(r.loss[4], s.loss[4], rtol=1e-5) and torch.allclose(grad[4].float(), other[4].float(), rtol=2.0 ** -7, atol=1e-6)
        assert torch.isfinite(grad[[1, 4, 5]].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0.0, 20.0, 60.0])
def test_distill_a_small_rest(shift):
    """A student that is sure of the named tokens: what is left for the others keeps its bits, down to e^-60 of the row."""
    say("[distill, small rest]", shift)
    gen = gen_of(shift)
    x = logits_of(gen, 7, 2000, "f32")
    ids, lq = teacher(gen, x, 8)
    x.scatter_add_(1, ids.long(), torch.full(ids.shape, shift, device="cuda"))
    for reverse in (0.0, 1.0):
        check_distilled(x, ids, lq, 1.0, reverse, True, "f32", gen)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,vocab,places,rest", [("f32", 700, 9, True), ("f32", 33, 33, True), ("f32", 5004, 20, False)])
def test_distill_gradient_by_differences(dtype, vocab, places, rest):
    """Along a random direction, by the oracle's loss at two points: the gradient's and the formula's sums agree with the slope."""
    from paper_2409_19256_amd import rollout
    say("[distill, differences]", vocab, places, rest)
    gen = gen_of(vocab)
    x = logits_of(gen, 4, vocab, dtype)
    ids, lq = teacher(gen, x, places)
    leaf = x.clone().requires_grad_()
    loss = rollout.distill(leaf, ids, lq, temperature=0.9, reverse=0.4, rest=rest)
    w = torch.rand(4, generator=gen, device="cuda")
    (loss * w).sum().backward()
    way = torch.randn(x.shape, generator=gen, device="cuda")
    f = lambda s: (S.distill(host(x) + s * host(way), ids.cpu().numpy(), host(lq), 0.9, 0.4, rest)[0] * host(w)).sum()  # noqa: E731
    slope = (f(1e-5) - f(-1e-5)) / 2e-5
    got = (host(leaf.grad) * host(way)).sum()
    # central differences: h^2 = 1e-10 of third derivatives of order |way|^3, and the loss's rounding over 2e-5
    assert abs(got - slope) < 1e-6 * (1 + abs(host(leaf.grad) * host(way)).sum())


# ---- pages ---------------------------------------------------------------------------------------------------------------

def new_pool(gen, layers, pages, heads, page, dim, dtype="bf16", by="heads", extra=0):
    from paper_2409_19256_amd.rollout import PagePool
    return PagePool([new_cache(gen, pages, heads, page, dim, dtype, by, extra) for _ in range(layers)])


def images(pool):
    return [t.clone() for t in pool._tensors]


def sequences(gen, rows, width, page, pages, full=0.3, share=0.3, bad=0.05, used=0.7):
    """Tables and lengths of rows that share pages, some of them full to the last page, empty, or with numbers that name no page; and the counts."""
    rng = np.random.default_rng(int(torch.randint(0, 1 << 30, (1,), generator=gen, device="cuda")))
    order = list(rng.permutation(pages)[:int(pages * used)])
    tables, lens = np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32)
    for r in range(rows):
        n = int(rng.integers(0, width * page + 1))
        if rng.random() < full:
            n -= n % page
        shared = 0
        if r and rng.random() < share:  # full pages of another row first
            s = int(rng.integers(0, r))
            shared = min(lens[s], n) // page
            tables[r, :shared] = tables[s, :shared]
        need = -(-n // page) - shared
        while need > len(order):
            n -= page - (0 if n % page == 0 else page - n % page)
            n = max(n, 0)
            need = max(0, -(-n // page) - shared)
        for i in range(need):
            tables[r, shared + i] = order.pop()
        lens[r] = n
        tables[r, -(-n // page):] = rng.integers(-3, pages + 3, width - -(-n // page))  # behind: anything
        if n and rng.random() < bad:
            tables[r, int(rng.integers(0, -(-n // page)))] = rng.choice([-1, pages, -7, 1 << 30])
    refs = np.zeros(pages, np.int32)
    for r in range(rows):
        row = tables[r, :-(-lens[r] // page)]
        np.add.at(refs, row[(row >= 0) & (row < pages)], 1)
    spare = [p for p in range(pages) if refs[p] == 0]
    for p in spare[::5]:
        refs[p] = 2  # held by somebody else
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return dev(tables), dev(lens), dev(refs)


def same(got, want, what):
    assert np.array_equal(got.cpu().numpy(), want), (what, np.argwhere(got.cpu().numpy() != want)[:5])


def check_data(pool, before, copies):
    """Every buffer: what was copied, and nothing else."""
    for t, old in zip(pool._tensors, before):
        for src, to, n in copies:
            old[to, :, :n] = old[src, :, :n]
        assert torch.equal(bits_of(t), bits_of(old))


POOLS = [
    # layers, pages, heads, page, dim, dtype, order, extra, rows, width
    (1, 7, 1, 4, 1, "bf16", "heads", 0, 3, 2),
    (2, 40, 4, 16, 64, "bf16", "heads", 0, 9, 5),
    (3, 50, 2, 8, 128, "f16", "tokens", 0, 12, 4),
    (1, 60, 3, 4, 65, "bf16", "heads", 0, 10, 6),
    (2, 33, 3, 8, 72, "bf16", "tokens", 3, 7, 4),
    (2, 30, 2, 64, 20, "f16", "heads", 4, 5, 3),
    (80, 24, 2, 4, 8, "bf16", "heads", 0, 4, 3),
    (128, 9, 1, 4, 2, "f16", "tokens", 0, 2, 2),
    (1, 5000, 1, 4, 4, "bf16", "heads", 0, 700, 9),
    (1, 300, 8, 256, 256, "bf16", "heads", 0, 20, 3),
    # more rows, entries or pages than one workgroup keeps the books of
    (2, 9000, 2, 4, 8, "f16", "heads", 0, 2500, 3),
    (2, 3000, 2, 4, 8, "bf16", "tokens", 0, 50, 350),
    (3, 17001, 1, 4, 4, "bf16", "heads", 0, 90, 150),
    (1, 16384, 1, 8, 2, "bf16", "heads", 0, 1000, 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("used", [0.5, 0.95])
@pytest.mark.parametrize("case", POOLS, ids=str)
def test_fork(case, used):
    say("[fork]", case, used)
    layers, pages, heads, page, dim, dtype, by, extra, rows, width = case
    gen = gen_of(case, used)
    pool = new_pool(gen, layers, pages, heads, page, dim, dtype, by, extra)
    tables, lens, refs = sequences(gen, rows, width, page, pages, used=used)
    parents = torch.randint(-1, rows + 1, (2 * rows + 1,), generator=gen, device="cuda").int()
    want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents.cpu().numpy(), refs.cpu().numpy(), page)
    for in_place in (False, True):
        before = images(pool)
        counts = refs.clone()
        t, n, r = pool.fork(tables, lens, parents, counts, refs_out=counts if in_place else None)
        same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
        assert (r is counts) == in_place
        check_data(pool, before, want[3])


@pytest.mark.gpu
@pytest.mark.parametrize("out", [2000, 2100])
@pytest.mark.parametrize("order", ["in order", "any"])
def test_fork_into_many(out, order):
    """So many copies that a workgroup takes several together: of one page, of pages that take turns, of one page to different lengths."""
    say("[fork into many]", out, order)
    gen = gen_of("many", out, order)
    layers, pages, page = 40, 4200, 8
    pool = new_pool(gen, layers, pages, 1, page, 8)
    tables, lens, refs = sequences(gen, 20, 4, page, pages, used=0.02, full=0.1)
    tables[3], lens[3] = tables[2], (lens[2] - 1).clamp(min=0)  # (against the rule: two that go on in one page)
    parents = torch.randint(0, 20, (out,), generator=gen, device="cuda").int()
    if order == "in order":
        parents = parents.sort().values
    want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents.cpu().numpy(), refs.cpu().numpy(), page)
    assert len(want[3]) * 2 * layers > 4 * 16384
    before = images(pool)
    t, n, r = pool.fork(tables, lens, parents, refs)
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
    src, to, tokens = (torch.tensor(x, device="cuda") for x in zip(*want[3]))
    moved = (torch.arange(page, device="cuda") < tokens[:, None])[:, None, :, None]
    for x, old in zip(pool._tensors, before):
        old[to] = torch.where(moved, old[src], old[to])
        assert torch.equal(bits_of(x), bits_of(old))


@pytest.mark.gpu
@pytest.mark.parametrize("parents", ["same", "none", "one", "turned"])
def test_fork_of_whole_batches(parents):
    say("[fork, all]", parents)
    gen = gen_of(parents)
    pool = new_pool(gen, 2, 90, 2, 16, 32)
    tables, lens, refs = sequences(gen, 11, 5, 16, 90)
    i = torch.arange(11, device="cuda", dtype=torch.int32)
    p = dict(same=i, none=i[:0], one=torch.full((30,), 3, device="cuda", dtype=torch.int32), turned=i.flip(0).contiguous())[parents]
    want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), p.cpu().numpy(), refs.cpu().numpy(), 16)
    before = images(pool)
    t, n, r = pool.fork(tables, lens, p, refs)
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
    check_data(pool, before, want[3])


@pytest.mark.gpu
@pytest.mark.parametrize("used", [0.5, 0.9])
@pytest.mark.parametrize("most", [0, 1, 7, 40])
@pytest.mark.parametrize("case", POOLS, ids=str)
def test_grow(case, most, used):
    say("[grow]", case, most, used)
    layers, pages, heads, page, dim, dtype, by, extra, rows, width = case
    gen = gen_of(case, most, used)
    pool = new_pool(gen, 1, pages, heads, page, dim, dtype, by, extra)
    tables, lens, refs = sequences(gen, rows, width, page, pages, used=used)
    lens = (lens * torch.rand(rows, generator=gen, device="cuda")).int()
    counts = torch.randint(-1, most + 2, (rows,), generator=gen, device="cuda").int()
    want = S.grow(tables.cpu().numpy(), lens.cpu().numpy(), counts.cpu().numpy(), refs.cpu().numpy(), most, page)
    t, n, s, r = pool.grow(tables, lens, counts, refs, most)
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(s, want[2], "slots"), same(r, want[3], "refs")
    mine = tables.clone(), lens.clone(), refs.clone()
    t, n, s, r = pool.grow(mine[0], mine[1], counts, mine[2], most, tables_out=mine[0], lens_out=mine[1], refs_out=mine[2])
    assert t is mine[0] and n is mine[1] and r is mine[2]
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(s, want[2], "slots"), same(r, want[3], "refs")


@pytest.mark.gpu
@pytest.mark.parametrize("live", [0.0, 0.1, 0.5, 0.9, 1.0])
@pytest.mark.parametrize("case", POOLS, ids=str)
def test_compact(case, live):
    say("[compact]", case, live)
    layers, pages, heads, page, dim, dtype, by, extra, rows, width = case
    gen = gen_of(case, live)
    pool = new_pool(gen, layers, pages, heads, page, dim, dtype, by, extra)
    refs = (torch.rand(pages, generator=gen, device="cuda") < live).int() * torch.randint(1, 9, (pages,), generator=gen, device="cuda").int()
    tables = [torch.randint(-3, pages + 3, s, generator=gen, device="cuda").int() for s in ((rows, width), (5,), (2, 3, 4))]
    new, r_want, places, n, moves = S.compact(refs.cpu().numpy(), [t.cpu().numpy() for t in tables])
    for in_place in (False, True):
        before = images(pool)
        counts, mine = refs.clone(), [t.clone() for t in tables]
        t, r, at, many = pool.compact(counts, mine, mine if in_place else None, counts if in_place else None)
        for a, b in zip(t, new):
            same(a, b, "tables")
        same(r, r_want, "refs"), same(at, places, "places")
        assert int(many) == n and many.dim() == 0 and (r is counts) == in_place and (t[1] is mine[1]) == in_place
        check_data(pool, before, [(src, to, page) for src, to in moves])


@pytest.mark.gpu
def test_more_pages_than_a_tile_of_each_workgroup():
    """Past 2^20 pages a workgroup's tile grows."""
    say("[2^20 pages and more]")
    gen = gen_of("many")
    pages, page = (1 << 20) + 5003, 4
    pool = new_pool(gen, 1, pages, 1, page, 1)
    tables, lens, refs = sequences(gen, 300, 600, page, 200000)
    refs = torch.cat((refs, (torch.rand(pages - 200000, generator=gen, device="cuda") < 0.5).int()))
    refs[:150000].clamp_(min=1)
    parents = torch.randint(0, 300, (500,), generator=gen, device="cuda").int()
    want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents.cpu().numpy(), refs.cpu().numpy(), page)
    t, n, r = pool.fork(tables, lens, parents, refs)
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
    counts = torch.full((500,), 30, device="cuda", dtype=torch.int32)
    want = S.grow(t.cpu().numpy(), n.cpu().numpy(), counts.cpu().numpy(), r.cpu().numpy(), 30, page)
    t, n, s, r = pool.grow(t, n, counts, r, 30)
    same(t, want[0], "tables"), same(n, want[1], "lens"), same(s, want[2], "slots"), same(r, want[3], "refs")
    before = images(pool)
    (new,), r_want, places, many, moves = S.compact(r.cpu().numpy(), [t.cpu().numpy()])
    (t,), r, at, live = pool.compact(r, [t])
    same(t, new, "tables"), same(r, r_want, "refs"), same(at, places, "places")
    src, to = (torch.tensor(x, device="cuda") for x in zip(*moves))
    for x, old in zip(pool._tensors, before):
        old[to] = old[src]
        assert torch.equal(bits_of(x), bits_of(old))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,pages", [(9, 4, 30), (300, 5, 900), (2100, 3, 9000), (40, 300, 2000)])
def test_whatever_the_arrays_hold(rows, width, pages):
    """Counts that fit no table, lengths below 0 and past the table, numbers that name no page: defined all the same, and nothing outside the caches is touched."""
    say("[pages, anything]", rows, width, pages)
    gen = gen_of("anything", rows, width, pages)
    pool = new_pool(gen, 2, pages, 2, 4, 8)
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda").int()  # noqa: E731
    for _ in range(3):
        tables, lens, refs = rand(-5, pages + 5, rows, width), rand(-9, 4 * width + 9, rows), rand(-2, 4, pages)
        parents, counts = rand(-2, rows + 2, rows + 7), rand(-4, 12, rows)
        want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents.cpu().numpy(), refs.cpu().numpy(), 4)
        before = images(pool)
        t, n, r = pool.fork(tables, lens, parents, refs)
        same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
        check_data(pool, before, want[3])
        want = S.grow(tables.cpu().numpy(), lens.cpu().numpy(), counts.cpu().numpy(), refs.cpu().numpy(), 9, 4)
        t, n, s, r = pool.grow(tables, lens, counts, refs, 9)
        same(t, want[0], "tables"), same(n, want[1], "lens"), same(s, want[2], "slots"), same(r, want[3], "refs")
        (new,), r_want, places, many, moves = S.compact(refs.cpu().numpy(), [tables.cpu().numpy()])
        before = images(pool)
        (t,), r, at, live = pool.compact(refs, [tables])
        same(t, new, "tables"), same(r, r_want, "refs"), same(at, places, "places")
        check_data(pool, before, [(a, b, 4) for a, b in moves])


@pytest.mark.gpu
def test_nothing_at_all():
    """No rows, no width, no tokens, no tables."""
    from paper_2409_19256_amd import rollout
    say("[nothing]")
    e = lambda *s, t=torch.int32: torch.empty(*s, device="cuda", dtype=t)  # noqa: E731
    x = e(0, 50, t=torch.bfloat16)
    assert rollout.adjust_logits(x, e(0, 9, t=torch.int64), e(0), repetition=e(0, t=torch.float32)).shape == (0, 50)
    d = rollout.top_distill(x, e(0, 5), e(0, 5, t=torch.float32))
    assert d.loss.shape == (0,) and d.norm.shape == (0, 2) and d.slopes.shape == (0, 6)
    assert rollout.top_distill_back(x, e(0, 5), d.norm, d.slopes, e(0, t=torch.float32)).shape == (0, 50)
    leaf = x.float().requires_grad_()
    rollout.distill(leaf, e(0, 5), e(0, 5, t=torch.float32)).sum().backward()
    assert leaf.grad.shape == (0, 50)
    y = torch.randn(3, 50, device="cuda")
    assert torch.equal(rollout.adjust_logits(y), y) and rollout.adjust_logits(y, out=y) is y
    assert torch.equal(rollout.adjust_logits(y, e(3, 0, t=torch.int64), torch.zeros(3, device="cuda", dtype=torch.int32)), y)
    assert torch.equal(rollout.adjust_logits(y, bias_ids=e(3, 0), bias=e(3, 0, t=torch.float32)), y)
    pool = new_pool(gen_of("nothing"), 1, 5, 1, 4, 4)
    before, refs = images(pool), torch.tensor([0, 2, 0, 1, 0], device="cuda", dtype=torch.int32)
    for rows, out, width in ((0, 0, 0), (0, 3, 2), (2, 0, 0), (2, 3, 0)):
        lens = torch.full((rows,), 7, device="cuda", dtype=torch.int32)
        t, n, r = pool.fork(e(rows, width), lens, torch.zeros(out, device="cuda", dtype=torch.int32), refs)
        assert t.shape == (out, width) and not n.any() and (t == -1).all() and torch.equal(r, refs)
        t, n, s, r = pool.grow(e(rows, 0), lens, torch.ones(rows, device="cuda", dtype=torch.int32), refs, 2)
        assert t.shape == (rows, 0) and not n.any() and s.shape == (rows, 2) and (s == -1).all() and torch.equal(r, refs)
    tables, r, places, live = pool.compact(refs)
    assert tables == () and r.tolist() == [1, 2, 0, 0, 0] and places.tolist() == [-1, 1, -1, 0, -1] and int(live) == 2
    check_data(pool, before, [(3, 0, 4)])
    (t,), r, _, _ = pool.compact(torch.zeros_like(refs), [e(0, 7)])
    assert t.shape == (0, 7) and not r.any()


@pytest.mark.gpu
def test_rows_that_share_a_page_that_is_not_full():
    """Against the rule, by hand or by a cut length: the first that goes on in it has it, whoever it came from."""
    say("[shared open page]")
    gen = gen_of("shared")
    pool = new_pool(gen, 2, 40, 2, 8, 16)
    tables = torch.tensor([[3, 7, -1], [9, 7, 1], [3, 7, 5], [7, 7, 7]], device="cuda", dtype=torch.int32)
    lens = torch.tensor([13, 15, 20, 4], device="cuda", dtype=torch.int32)
    refs = torch.zeros(40, device="cuda", dtype=torch.int32)
    for p, n in ((3, 2), (7, 4), (9, 1), (5, 1), (0, 5)):
        refs[p] = n
    for parents in ([0, 1, 2, 3], [3, 1, 0, 0, 2, 2], [1, 1, 1], [2, 0]):
        p = torch.tensor(parents, device="cuda", dtype=torch.int32)
        want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents, refs.cpu().numpy(), 8)
        before = images(pool)
        t, n, r = pool.fork(tables, lens, p, refs)
        same(t, want[0], "tables"), same(n, want[1], "lens"), same(r, want[2], "refs")
        check_data(pool, before, want[3])


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Pages and rows more than 2^32 elements from the first."""
    from paper_2409_19256_amd import rollout
    say("[offsets past 32 bits]")
    gen = gen_of("far")
    pages, page, dim = 280, 65536, 256  # 2^24 elements a page
    pool = rollout.PagePool([rollout.KvCache.empty(pages, 1, page, dim)])
    refs = torch.ones(pages, device="cuda", dtype=torch.int32)
    refs[270], refs[275] = 0, 0
    for t in pool._tensors:
        t[260].normal_(generator=gen), t[270].zero_(), t[275].zero_(), t[0].zero_(), t[4].zero_()
    tables, lens = torch.tensor([[260]], device="cuda", dtype=torch.int32), torch.tensor([40001], device="cuda", dtype=torch.int32)
    t, n, r = pool.fork(tables, lens, torch.zeros(3, device="cuda", dtype=torch.int32), refs)
    assert t.tolist() == [[260], [270], [275]] and n.tolist() == [40001] * 3
    for x in pool._tensors:
        for p in (270, 275):
            assert torch.equal(x[p, :, :40001], x[260, :, :40001]) and not x[p, :, 40001:].any()
        assert not x[4].any() and not x[0].any()  # 260 * 2^24 is 2^32 past page 4
    r[0] = r[4] = 0
    (t,), r, places, live = pool.compact(r, [t])
    assert int(live) == 278 and places[278:].tolist() == [0, 4] and t.tolist() == [[260], [270], [275]]
    del pool, x
    torch.cuda.empty_cache()
    far, vocab = (1 << 31) + 3, 5003
    for dtype in ("bf16", "f32"):
        store = torch.empty(2 * far + vocab, device="cuda", dtype=TYPES[dtype])
        x = store.as_strided((3, vocab), (far, 1))
        x.copy_(logits_of(gen, 3, vocab, dtype))
        a = adjustment(dtype, 3, vocab, 0, 50, torch.int64, 5, 3, gen)
        near_ = x.contiguous()
        want = rollout.adjust_logits(near_, **a)
        ids, lq = teacher(gen, near_, 9)
        d = rollout.top_distill(near_, ids, lq)
        g = torch.ones(3, device="cuda")
        grad = rollout.top_distill_back(near_, ids, d.norm, d.slopes, g)
        e = rollout.top_distill(x, ids, lq)
        assert torch.equal(d.loss, e.loss) and torch.equal(rollout.top_distill_back(x, ids, e.norm, e.slopes, g), grad)
        rollout.adjust_logits(x, **a, out=x)
        assert torch.equal(bits_of(x), bits_of(want))
        x.copy_(near_)
        rollout.top_distill_back(x, ids, e.norm, e.slopes, g, out=x)
        assert torch.equal(bits_of(x), bits_of(grad))
        del store, x
        torch.cuda.empty_cache()


@pytest.mark.gpu
def test_caches_between_one_anothers_pages():
    """All layers in one allocation, a page of all of them in one piece."""
    from paper_2409_19256_amd.rollout import KvCache, PagePool
    say("[layers inside pages]")
    gen = gen_of("inside")
    store = torch.randn(30, 5, 2, 2, 8, 16, generator=gen, device="cuda").bfloat16()
    pool = PagePool([KvCache(store[:, i, 0], store[:, i, 1]) for i in range(5)])
    tables, lens, refs = sequences(gen, 6, 4, 8, 30)
    parents = torch.randint(0, 6, (9,), generator=gen, device="cuda").int()
    want = S.fork(tables.cpu().numpy(), lens.cpu().numpy(), parents.cpu().numpy(), refs.cpu().numpy(), 8)
    before = images(pool)
    t, n, r = pool.fork(tables, lens, parents, refs)
    same(t, want[0], "tables"), same(r, want[2], "refs")
    check_data(pool, before, want[3])
    (new,), r_want, places, many, moves = S.compact(r.cpu().numpy(), [t.cpu().numpy()])
    before = images(pool)
    (t,), r, at, live = pool.compact(r, [t])
    same(t, new, "tables"), same(r, r_want, "refs")
    check_data(pool, before, [(a, b, 8) for a, b in moves])


# ---- graphs, streams, calls at once --------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_captured_and_replayed():
    """Every call in one graph, replayed on new inputs between eager calls of its own."""
    from paper_2409_19256_amd import rollout
    say("[graph]")
    gen = gen_of("graph")
    x = logits_of(gen, 9, 5004, "bf16")
    a = adjustment("bf16", 9, 5004, 0, 100, torch.int64, 5, 3, gen)
    ids, lq = teacher(gen, x, 12)
    g = torch.rand(9, generator=gen, device="cuda")
    pool = new_pool(gen, 3, 200, 2, 16, 32)
    tables, lens, refs = sequences(gen, 13, 6, 16, 200)
    parents, counts = torch.randint(0, 13, (13,), generator=gen, device="cuda").int(), torch.randint(0, 9, (13,), generator=gen, device="cuda").int()

    def work():
        y = rollout.adjust_logits(x, **a)
        d = rollout.top_distill(y, ids, lq, 0.9, 0.5)
        grad = rollout.top_distill_back(y, ids, d.norm, d.slopes, g, 0.9)
        t, n, r = pool.fork(tables, lens, parents, refs)
        t, n, s, r = pool.grow(t, n, counts, r, 8)
        (t,), r, at, live = pool.compact(r, [t])
        return [y, d.loss, grad, t, n, s, r, at, live, *pool._tensors]

    images_ = images(pool)
    back = lambda: [t.copy_(o) for t, o in zip(pool._tensors, images_)]  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    for i in range(5):
        x.copy_(logits_of(gen, 9, 5004, "bf16"))
        x[:, ::9] = -float("inf")
        parents.copy_(torch.randint(-1, 13, (13,), generator=gen, device="cuda"))
        counts.copy_(torch.randint(0, 9, (13,), generator=gen, device="cuda"))
        back()
        eager = [t.clone() for t in work()]
        torch.cuda.synchronize()
        back()
        graph.replay()
        torch.cuda.synchronize()
        for k, (p, q) in enumerate(zip(captured, eager)):
            assert torch.equal(p, q) or torch.equal(p.isnan(), q.isnan()) and torch.equal(p.nan_to_num(), q.nan_to_num()), (i, k)


@pytest.mark.gpu
def test_autograd_in_a_graph():
    """The loss and its gradient captured together, beside an eager graph over other leaves that lives on."""
    from paper_2409_19256_amd import rollout
    say("[graph, autograd]")
    gen = gen_of("autograd")
    x = logits_of(gen, 5, 999, "f32")
    ids, lq = teacher(gen, x, 7)
    w = torch.rand(5, generator=gen, device="cuda")
    alive = x.clone().requires_grad_()
    kept = rollout.distill(alive, ids, lq, 0.9, 0.2)

    def step():
        leaf = x.detach().requires_grad_()
        loss = rollout.distill(leaf, ids, lq, 0.9, 0.2)
        return loss.detach(), torch.autograd.grad((loss * w).sum(), leaf)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grad = step()
    for i in range(4):
        x.copy_(logits_of(gen, 5, 999, "f32"))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1]), i
    (kept * w).sum().backward()
    assert torch.isfinite(alive.grad).all()


@pytest.mark.gpu
def test_on_two_streams_at_once():
    from paper_2409_19256_amd import rollout
    say("[two streams]")
    gen = gen_of("streams")
    sets = []
    for k in range(2):
        x = logits_of(gen, 300, 32000, "bf16")
        ids, lq = teacher(gen, x, 20)
        pool = new_pool(gen, 2, 3000, 2, 16, 64)
        tables, lens, refs = sequences(gen, 200, 12, 16, 3000)
        parents = torch.randint(0, 200, (200,), generator=gen, device="cuda").int()
        sets.append((x, adjustment("bf16", 300, 32000, 0, 900, torch.int64, 5, 3, gen), ids, lq, pool, tables, lens, refs, parents, torch.ones(300, device="cuda")))

    def work(x, a, ids, lq, pool, tables, lens, refs, parents, g):
        y = rollout.adjust_logits(x, **{k: v for k, v in a.items() if k != "allowed" and k != "allowed_rows"})
        d = rollout.top_distill(y, ids, lq)
        return [y, d.loss, rollout.top_distill_back(y, ids, d.norm, d.slopes, g), *pool.fork(tables, lens, parents, refs)]

    want = [[t.clone() for t in work(*s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(4):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(work(*sets[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for again in got[k]:
            for a, b in zip(again, want[k]):
                assert torch.equal(a, b)
