"""Attention where the weights that make up the output are small: a first token far ahead of all others whose value is zero (an attention sink), scores
that fall from tile to tile.

Tolerances: as in test_rollout_gpu.py, of sum p |v|, to which the sink adds nothing.  P of the others is off by 2^-16 of the largest weight among its tile of 32
tokens; in the sink's own tile that is the sink's, of which float16 keeps steps of 2^-32 there: 2^-33 of 31 tokens, 2^-28 max |v| in all.
"""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as R
from tests.test_rollout_gpu import HALF_STEP, SMALLEST, TYPES, U, host, near, say


def check(dtype, keys, values, q, samples, page, in_prompt, scale):
    """keys, values [token, KV head, element]: one prompt's, or every response's; q [sequence, query head, element]."""
    from paper_2409_19256_amd.rollout import KvCache
    n, hk, d = keys.shape
    b = len(q)
    pages = -(-n // page)
    c = KvCache.empty(pages, hk, page, d, dtype=TYPES[dtype])
    for t, x in ((c.k, keys), (c.v, values)):
        t.fill_(float("nan"))
        for j in range(pages):
            m = min(page, n - j * page)
            t[j, :, :m] = x[j * page:j * page + m].transpose(0, 1)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    lens = torch.full((b,), n, dtype=torch.int32, device="cuda")
    none = torch.zeros(b, dtype=torch.int32, device="cuda")
    if in_prompt:
        args = (none, torch.zeros(b, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, b], dtype=torch.int32, device="cuda"), lens[:1], table)
    else:
        args = (lens, table.expand(b, -1).contiguous(), None, None, None)
    out, lse = c.attend(q, *args, scale=scale)
    torch.cuda.synchronize()
    picked = sorted({0, b - 1})  # the rows differ in q alone
    some = q[picked]
    if in_prompt:
        few = (none[picked], args[1][picked], torch.tensor([0, len(picked)]), lens[:1], table)
    else:
        few = (lens[picked], args[1][picked], None, None, None)
    want, want_lse, size, score = R.attend(host(some), host(c.k), host(c.v), *(None if a is None else a.cpu().numpy() for a in few), scale)
    rel = 2 * (d + 2) * U * score + 8 * U + 3 * U * score + 2.0 ** -16 + n * U
    near(host(out)[picked], want, HALF_STEP[dtype] * np.abs(want) + rel[..., None] * size * 1.1 + 2.0 ** -28 * np.abs(host(values)).max() + SMALLEST[dtype], "out")
    near(host(lse)[picked], want_lse, rel + 4 * U * np.abs(want_lse), "lse")


# sequences, query heads, KV heads, head dim, page, tokens, whether they are a prompt's: a prompt with many rows, with few, responses by parts, short ones, both in
# one launch, pieces and single elements
FORMS = [(61, 16, 2, 128, 16, 4000, True), (3, 8, 8, 128, 16, 4000, True), (7, 8, 2, 64, 16, 3001, False), (200, 32, 8, 64, 16, 100, False), (2, 4, 2, 64, 16, 500, True),
         (40, 8, 4, 80, 16, 1500, True), (9, 4, 2, 65, 16, 1000, False), (5, 4, 2, 256, 8, 900, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("ahead", [2, 8, 12, 15, 16, 17, 18, 21, 25, 30])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_a_sink_without_value(form, ahead, dtype):
    b, hq, hk, d, page, n, in_prompt = form
    say("[sink]", form, ahead, dtype)
    gen = torch.Generator("cuda").manual_seed(ahead)
    scale = d ** -0.5
    for spread, value in ((0.0, 1.0), (0.0, 900.0), (1.0, 30.0)):  # the others' scores: equal, or about as wide as in earnest
        keys = torch.randn(n, hk, d, generator=gen, device="cuda") * spread
        keys[:, :, 0] = 0
        keys[0] = 0
        keys[0, :, 0] = ahead / scale / 4
        values = value * (1 if spread == 0 else torch.randn(n, hk, d, generator=gen, device="cuda").abs())
        values = torch.zeros(n, hk, d, device="cuda") + values
        values[0] = 0
        q = torch.randn(b, hq, d, generator=gen, device="cuda")
        q[..., 0] = 4
        check(dtype, keys.to(TYPES[dtype]), values.to(TYPES[dtype]), q.to(TYPES[dtype]), b, page, in_prompt, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form", FORMS[:5], ids=str)
def test_scores_that_fall_and_rise(form, dtype):
    """Every tile some nats below the one before it and only the last ones with a value; the same from the other end; sinks that come back."""
    b, hq, hk, d, page, n, in_prompt = form
    say("[falling scores]", form, dtype)
    scale = d ** -0.5
    tile = torch.arange(n, device="cuda") // 32
    for fall, last in ((0.02, 40), (6.0, 3), (30.0, 2), (200.0, 2)):
        for backwards in (False, True):
            x = -fall * tile.float()
            x = x - x.min() if -float(x.min()) < 2000 else x.clamp(min=-2000) + 2000
            if fall == 0.02:
                x[::257] = 16
            values = torch.zeros(n, device="cuda")
            values[tile > tile.max() - last] = 3.0
            if fall == 0.02:
                values = 5 * (x < 15).float()
            if backwards:
                x, values = x.flip(0), values.flip(0)
            keys = torch.zeros(n, hk, d, device="cuda")
            keys[:, :, 0] = x[:, None] / scale / 4
            q = torch.zeros(b, hq, d, device="cuda")
            q[..., 0] = 4
            v = values[:, None, None].expand(n, hk, d).contiguous()
            check(dtype, keys.to(TYPES[dtype]), v.to(TYPES[dtype]), q.to(TYPES[dtype]), b, page, in_prompt, scale)
