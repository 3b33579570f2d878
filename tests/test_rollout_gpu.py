"""The rollout operators against the oracle in 64 bits, at the sizes, layouts and masks where they can go wrong.

Tolerances.  u = 2^-24 is half a unit in the last place of 1 in 32 bits; r = 2^-9 (bfloat16) or 2^-12 (float16) half a unit in the last place,
relative to the value, of the output's type, at most twice that at the lower end of a binade (R below), and float16 has steps of 2^-24 below its normal range.
 - rotation: two products and a sum in 32 bits, at most 3 u (|a| + |b|), then one rounding: R |exact| beside it.
 - attention: a score is a sum of head_dim products (error at most (head_dim + 2) u sum |q||k| scale, twice: the largest score has the same error),
   an exponential of base 2 of hardware precision (2 u, and its argument's rounding, |x| u log2 e, with |x| at most twice the scores' size), P in two halves of the type (2^-16
   relative at least), sums over the tokens (at most tokens u).  All are relative errors of p, so the result is off by that share of sum p |v|.
   lse is off by the score's error and by the sum's relative error.
 - log probabilities: the same without the products; the sum of a row goes through at most vocab / 64 + 80 additions.
"""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as R

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": U}  # of a value, at most
SMALLEST = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def say(*a):
    print(*a, flush=True)


def near(got, want, tol, what):
    got, want = np.asarray(got), np.asarray(want)
    assert got.shape == want.shape
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)  # past what 32 bits hold
    same = (got == want) | (np.isnan(got) & np.isnan(want))  # infinities and NaN have to be alike
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want) - tol)
    bad = ~(off <= 0)
    if bad.any():
        at = tuple(int(i[0]) for i in np.nonzero(bad))
        pytest.fail(f"{what}: {int(bad.sum())} of {bad.size} off, the first at {at}: {got[at]} and not {want[at]}, tolerance {np.broadcast_to(tol, got.shape)[at]}")


def made(shape, gen, dtype, order="last"):
    """Random values on the GPU, exactly those that their host copy holds."""
    return torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype])


def new_cache(gen, pages, heads, page, dim, dtype, by="heads", extra=0, fill=None):
    """A cache in either order of memory; extra: elements between tokens (strides that are no multiple of 8 where it is odd)."""
    from paper_2409_19256_amd.rollout import KvCache
    shape = (pages, heads, page, dim + extra) if by == "heads" else (pages, page, heads, dim + extra)
    k, v = (torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype]) if fill is None else torch.full(shape, fill, device="cuda", dtype=TYPES[dtype])
            for _ in range(2))
    if by == "tokens":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return KvCache(k[..., :dim], v[..., :dim])


def bits(t):
    return t.contiguous().view(torch.int16)


# ---- append --------------------------------------------------------------------------------------------------------------

APPENDS = [
    # dtype, query heads, KV heads, head dim, rotated, tokens, page, order, extra, interleaved, fused
    ("bf16", 32, 32, 128, 128, 1, 64, "heads", 0, False, False),
    ("bf16", 64, 8, 128, 128, 37, 16, "tokens", 0, False, True),
    ("f16", 16, 2, 128, 64, 130, 4, "heads", 0, True, False),
    ("bf16", 4, 4, 64, 64, 9, 128, "heads", 0, True, True),
    ("f16", 8, 4, 72, 72, 33, 32, "tokens", 0, False, False),   # halves of 36: four elements at a time
    ("bf16", 8, 4, 72, 36, 33, 32, "heads", 0, False, True),    # halves of 18: two
    ("bf16", 2, 1, 65, 64, 5, 8, "heads", 0, False, False),     # an odd head: one
    ("f16", 4, 2, 3, 2, 7, 4, "tokens", 0, True, False),
    ("bf16", 6, 3, 256, 250, 4, 16, "heads", 3, False, True),   # strides that no vector divides
    ("f16", 5, 5, 1, 0, 3, 4, "heads", 0, False, False),
    ("bf16", 1, 1, 255, 254, 2, 4, "tokens", 1, True, False),
    ("bf16", 80, 40, 80, 16, 21, 16, "heads", 8, False, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append(case):
    dtype, hq, hk, d, rot, n, page, by, extra, inter, fused = case
    say("[append]", case)
    gen = torch.Generator("cuda").manual_seed(n + d)
    pages = n // page + 3
    c = new_cache(gen, pages, hk, page, d, dtype, by, extra)
    if fused:
        x = made((n, hq + 2 * hk, d), gen, dtype)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    else:
        q, k, v = (made((n, h, d), gen, dtype) for h in (hq, hk, hk))
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:n]
    positions = torch.randint(0, 50, (n,), generator=gen, device="cuda", dtype=torch.int32)
    cos, sin = (torch.randn(50, rot // 2, generator=gen, device="cuda") for _ in range(2)) if rot else (None, None)
    if n > 3:
        slots[1], slots[2], positions[3] = -1, pages * page, 50        # padding, past the cache, past the table
        if not rot:
            slots[3] = -7
    before_k, before_v = bits(c.k).clone(), bits(c.v).clone()
    q_out = torch.full((n, hq, d), 7.0, device="cuda", dtype=TYPES[dtype])
    c.append(k, v, slots, positions if rot else None, cos, sin, q=q, q_out=q_out, interleaved=inter)
    torch.cuda.synchronize()
    live = [t for t in range(n) if not (n > 3 and t in (1, 2, 3))]
    at = slots.cpu().numpy()[live]
    table = (np.zeros((50, 0)),) * 2 if not rot else (cos.cpu().numpy(), sin.cpu().numpy())
    pos = positions.cpu().numpy()[live]
    for name, src, got in (("q", q, host(q_out)[live]), ("k", k, host(c.k)[at // page, :, at % page])):
        want, size = R.rotate(host(src)[live], pos, *table, inter)
        turned = np.abs(np.broadcast_to(np.max([np.abs(t).max(initial=0) for t in table]), size.shape))
        near(got, want, HALF_STEP[dtype] * np.abs(want) + 3 * U * size * turned * (1 + HALF_STEP[dtype]) + SMALLEST[dtype], name)
        if rot < d:
            assert np.array_equal(got[..., rot:], host(src)[live][..., rot:])
    assert torch.equal(bits(c.v[at // page, :, at % page]), bits(v[live]))
    # everything else is as it was
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[torch.from_numpy(at)] = False
    for now, old in ((bits(c.k), before_k), (bits(c.v), before_v)):
        assert torch.equal(now.transpose(1, 2).reshape(pages * page, -1)[rest.cuda()], old.transpose(1, 2).reshape(pages * page, -1)[rest.cuda()])
    assert (q_out[[t for t in range(n) if t not in live]] == 7).all()
    # without queries, and with the queries turned in place
    k2, v2 = c.k.clone(), c.v.clone()
    c.append(k, v, slots, positions if rot else None, cos, sin, interleaved=inter)
    assert torch.equal(bits(c.k), bits(k2)) and torch.equal(bits(c.v), bits(v2))
    if not fused:
        keep = q.clone()
        c.append(k, v, slots, positions if rot else None, cos, sin, q=q, q_out=q, interleaved=inter)
        assert torch.equal(bits(q[live]), bits(q_out[live]))
        dead = [t for t in range(n) if t not in live]
        assert torch.equal(bits(q[dead]), bits(keep[dead]))


# ---- attention -----------------------------------------------------------------------------------------------------------

def check_attention(c, dtype, q, args, got, n_tokens, **bounds):
    out, lse = got
    d = q.shape[2]
    want, want_lse, size, score = R.attend(host(q), host(c.k), host(c.v), *(None if a is None else a.cpu().numpy() for a in args), bounds.pop("scale", d ** -0.5), **bounds)
    rel = 2 * (d + 2) * U * score + 8 * U + 3 * U * score + 2.0 ** -16 + n_tokens * U
    assert (rel < 0.05).all()
    near(host(out), want, HALF_STEP[dtype] * np.abs(want) + rel[..., None] * size * 1.1 + SMALLEST[dtype], "out")
    near(host(lse), want_lse, rel + 4 * U * np.where(np.isfinite(want_lse), np.abs(want_lse), 0), "lse")


def tables(gen, lens, page, at, width=None):
    """Page numbers for rows of these lengths out of the list `at`, -1 past them."""
    need = [max(0, -(-n // page)) for n in lens]
    t = torch.full((len(lens), max([1] + need) if width is None else width), -1, dtype=torch.int32)
    for i, k in enumerate(need):
        t[i, :k] = torch.tensor([at.pop() for _ in range(k)], dtype=torch.int32)
    return t.cuda()


def attention_inputs(gen, dtype, hq, hk, d, page, by, extra, groups, prefix, suffix):
    """Caches that hold NaN wherever no token is visible."""
    n = sum(groups)
    lens = [prefix[g % len(prefix)] for g in range(len(groups))], [suffix[i % len(suffix)] for i in range(n)]
    pages = sum(-(-x // page) for x in lens[0] + lens[1]) + 2
    c = new_cache(gen, pages, hk, page, d, dtype, by, extra, fill=float("nan"))
    at = torch.randperm(pages, generator=gen, device="cuda").tolist()
    pt, st = tables(gen, lens[0], page, at), tables(gen, lens[1], page, at)
    for t, ls in ((pt, lens[0]), (st, lens[1])):
        for i, x in enumerate(ls):
            for j in range(-(-x // page)):
                m = min(page, x - j * page)
                for y in (c.k, c.v):
                    y[int(t[i, j]), :, :m] = torch.randn(hk, m, d, generator=gen, device="cuda").to(TYPES[dtype])
    q = 1.5 * made((n, hq, d), gen, dtype)
    off = torch.tensor([0] + list(np.cumsum(groups)), dtype=torch.int32, device="cuda")
    pl, sl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in lens)
    return c, q, (sl, st, off, pl, pt), max(lens[0] + [0]) + max(lens[1] + [0])


ATTENTIONS = [
    # dtype, query heads, KV heads, head dim, page, order, extra, samples per prompt, prompt lengths, response lengths
    ("bf16", 4, 4, 64, 16, "heads", 0, (4,), (100,), (1, 17, 64, 0)),
    ("bf16", 8, 8, 128, 64, "heads", 0, (3, 1, 5), (127, 128, 129), (1, 31, 32, 33, 127, 128, 129, 200, 257)),
    ("f16", 16, 2, 128, 16, "tokens", 0, (7, 2), (700, 3), (5, 260)),
    ("bf16", 64, 8, 128, 4, "heads", 0, (5, 0, 2), (65, 9, 1), (3, 40, 130)),
    ("f16", 12, 12, 64, 128, "tokens", 0, (2, 20), (31, 400), (1, 2, 3)),
    ("bf16", 16, 8, 32, 8, "heads", 0, (9,), (33,), (1, 65)),
    ("bf16", 8, 4, 72, 8, "heads", 0, (6, 3), (50, 140), (9, 0, 150)),
    ("f16", 8, 4, 80, 16, "tokens", 16, (40,), (333,), (4, 5)),
    ("bf16", 40, 2, 128, 32, "heads", 0, (3, 2), (90, 0), (33, 1)),        # 20 query heads to a KV head
    ("bf16", 6, 2, 256, 16, "heads", 0, (4, 1), (129, 20), (7, 131)),
    ("f16", 2, 1, 192, 16, "tokens", 8, (3,), (66,), (35,)),
    ("bf16", 4, 2, 65, 16, "heads", 0, (3, 2), (40, 130), (1, 60)),          # single elements from here on
    ("f16", 4, 4, 3, 4, "tokens", 0, (2, 2), (11, 0), (0, 9)),
    ("bf16", 2, 2, 128, 16, "heads", 1, (2,), (35,), (20, 40)),
    ("bf16", 3, 1, 200, 8, "heads", 5, (2,), (35,), (20, 40)),
    ("f16", 1, 1, 1, 4, "heads", 0, (1,), (5,), (2,)),
    ("bf16", 32, 1, 128, 64, "heads", 0, (17,), (257,), (0, 1, 2)),           # one KV head, 544 rows to the prompt
    ("f16", 24, 8, 64, 32, "heads", 0, (60, 55), (95, 130), (3, 150, 40, 40, 0, 97)),  # more workgroups than the chip holds: longest first
    ("bf16", 8, 8, 32, 8, "tokens", 0, (4,) * 25, (20, 33), (1, 70, 35)),
    ("bf16", 8, 8, 64, 16, "heads", 0, (130, 140), (7,), (11, 3)),            # more sequences than a workgroup orders
    ("f16", 8, 2, 128, 16, "heads", 0, (5, 2, 4), (300, 1, 129), (600, 0, 290)),  # 20 rows
    ("bf16", 16, 2, 64, 4, "heads", 0, (12, 3), (150, 400), (10, 300)),       # 96 rows
    ("bf16", 32, 8, 64, 16, "heads", 0, (70, 40), (33,), (0, 1, 31, 64, 33, 97, 128)),  # a wavefront to a short response
    ("f16", 20, 10, 72, 8, "tokens", 0, (1,) * 90, (40, 0), (5, 0, 128)),
    ("bf16", 40, 2, 48, 16, "heads", 0, (200,), (9,), (7, 33)),               # and 20 query heads to a KV head
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", ATTENTIONS, ids=str)
def test_attention(case):
    dtype, hq, hk, d, page, by, extra, groups, prefix, suffix = case
    say("[attend]", case)
    gen = torch.Generator("cuda").manual_seed(d)
    c, q, args, n = attention_inputs(gen, dtype, hq, hk, d, page, by, extra, groups, prefix, suffix)
    got = c.attend(q, *args)
    again = c.attend(q, *args)
    torch.cuda.synchronize()
    check_attention(c, dtype, q, args, got, n)
    assert torch.equal(bits(got[0]), bits(again[0])) and torch.equal(got[1], again[1])
    # tight bounds and strided queries and output
    sl, st, off, pl, pt = args
    wide = torch.zeros(q.shape[0], hq + 3, d + (8 if d % 8 == 0 else 0), device="cuda", dtype=q.dtype)
    wide[:, 1:hq + 1, :d] = q
    into = torch.full((q.shape[0], hq, d + 5), 9.0, device="cuda", dtype=q.dtype)
    got = c.attend(wide[:, 1:hq + 1, :d], *args, max_group=max(groups), max_prefix=int(pl.max()), max_suffix=int(sl.max()), scale=0.07, out=into[..., :d])
    torch.cuda.synchronize()
    check_attention(c, dtype, q, args, got, n, scale=0.07)
    assert (into[..., d:] == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("loose", ["prompts", "responses"])
@pytest.mark.parametrize("case", ATTENTIONS, ids=str)
def test_attention_within_loose_bounds(case, loose):
    """Tables with room for far more tokens than there are: work is cut into parts by the bounds, whatever the lengths."""
    dtype, hq, hk, d, page, by, extra, groups, prefix, suffix = case
    say("[attend, loose bounds]", loose, case)
    gen = torch.Generator("cuda").manual_seed(d + 1)
    c, q, (sl, st, off, pl, pt), n = attention_inputs(gen, dtype, hq, hk, d, page, by, extra, groups, prefix, suffix)
    room = max(1, 2500 // page)
    wide = torch.full(((pt if loose == "prompts" else st).shape[0], room), -1, dtype=torch.int32, device="cuda")
    if loose == "prompts":
        pt = torch.cat([pt, wide], 1)
    else:
        st = torch.cat([st, wide], 1)
    args = (sl, st, off, pl, pt)
    got, again = c.attend(q, *args), c.attend(q, *args)
    torch.cuda.synchronize()
    check_attention(c, dtype, q, args, got, n)
    assert torch.equal(bits(got[0]), bits(again[0])) and torch.equal(got[1], again[1])


# dtype, query heads, KV heads, head dim, page, samples per prompt, prompt lengths, response lengths: on both sides of where contexts are short and few
SHORT = [
    ("bf16", 4, 4, 64, 16, (1,) * 70 + (3,), (33, 0, 64, 95, 128), (0, 1, 31, 32, 33)),
    ("f16", 2, 1, 128, 16, (2, 2), (31, 32), (0, 96, 97)),
    ("bf16", 8, 2, 128, 64, (4,), (512,), (128, 127, 1, 0)),
    ("bf16", 8, 2, 128, 64, (4,), (513,), (128, 127, 1, 0)),
    ("f16", 16, 8, 128, 16, (16,), (768,), (256, 255)),
    ("bf16", 6, 2, 256, 8, (3, 2), (256, 255), (64, 0)),
    ("bf16", 34, 2, 128, 4, (2, 3), (90, 1), (0, 40, 300)),
    ("f16", 3, 1, 65, 16, (2, 1), (64, 63), (64, 0, 1)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", SHORT, ids=lambda c: str(c)[:60])
def test_attention_over_short_contexts(case):
    dtype, hq, hk, d, page, groups, prefix, suffix = case
    say("[attend, short contexts]", case)
    gen = torch.Generator("cuda").manual_seed(d + 2)
    c, q, args, n = attention_inputs(gen, dtype, hq, hk, d, page, "heads", 0, groups, prefix, suffix)
    sl, st, off, pl, pt = args
    for offsets, most in ((off, None), (off + 1, None), (off, 1), (torch.zeros_like(off), None)):  # the last three leave sequences without a prompt
        args = (sl, st, offsets, pl, pt)
        got = c.attend(q, *args, **({} if most is None else dict(max_group=most)))
        torch.cuda.synchronize()
        check_attention(c, dtype, q, args, got, n, **({} if most is None else dict(max_group=most)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,by", [("bf16", "heads"), ("f16", "tokens")])
def test_attention_without_prompts(dtype, by):
    gen = torch.Generator("cuda").manual_seed(3)
    for lens in ((0, 1, 5, 128), (129, 3, 500, 0), (1,), (0,), (100, 3, 0) * 150):
        say("[attend without prompts]", dtype, by, lens)
        c, q, (sl, st, *_), n = attention_inputs(gen, dtype, 8, 2, 128, 16, by, 0, [len(lens)], (0,), lens)
        got = c.attend(q, sl, st)
        torch.cuda.synchronize()
        check_attention(c, dtype, q, (sl, st, None, None, None), got, n)


@pytest.mark.gpu
def test_a_prompt_processed_token_by_token():
    """Every token of a prompt as a sequence of its own over the same pages: a causal mask by lengths."""
    say("[causal]")
    gen = torch.Generator("cuda").manual_seed(4)
    c, q, (sl, st, *_), n = attention_inputs(gen, "bf16", 8, 4, 64, 16, "heads", 0, [1], (0,), (150,))
    q = made((150, 8, 64), gen, "bf16")
    lens, rows = torch.arange(1, 151, dtype=torch.int32, device="cuda"), st.expand(150, -1).contiguous()
    got = c.attend(q, lens, rows)
    torch.cuda.synchronize()
    check_attention(c, "bf16", q, (lens, rows, None, None, None), got, 150)


@pytest.mark.gpu
def test_entries_out_of_range_are_not_visible():
    """Page numbers outside the cache, lengths beyond the tables and below zero, groups that leave sequences out or are longer than they may be."""
    say("[entries out of range]")
    gen = torch.Generator("cuda").manual_seed(5)
    c, q, (sl, st, off, pl, pt), n = attention_inputs(gen, "bf16", 8, 2, 128, 16, "heads", 0, [4, 3], (90, 300), (40, 70, 16))
    for t in (c.k, c.v):
        t.nan_to_num_(nan=0.25)  # lengths are wrong on purpose here: whatever they reach is a number
    pt[0, 1], pt[1, 3], st[2, 0], st[1, 2] = -5, c.k.shape[0], 1 << 30, -(1 << 31)
    st[0, -1] = -1
    sl[0], sl[3] = 1 << 30, -3
    pl[0] = 80
    for offsets, most in (([0, 4, 7], 7), ([1, 4, 6], 7), ([0, 4, 7], 2), ([0, 0, 7], 7), ([0, 4, 4], 7)):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        got = c.attend(q, sl, st, off, pl, pt, max_group=most, max_prefix=200, max_suffix=64)
        torch.cuda.synchronize()
        check_attention(c, "bf16", q, (sl, st, off, pl, pt), got, n, max_group=most, max_prefix=200, max_suffix=64)


@pytest.mark.gpu
def test_attention_with_infinite_and_large_scores():
    """One key far ahead (the others' weights vanish), scores of -inf, and NaN in a visible value."""
    say("[large scores]")
    gen = torch.Generator("cuda").manual_seed(6)
    c, q, args, n = attention_inputs(gen, "f16", 4, 2, 64, 16, "heads", 0, [3], (200,), (50, 1, 0))
    sl, st, off, pl, pt = args
    c.k[int(pt[0, 9]), 1, 3] = 60000 * q[0, 2].sign()
    got = c.attend(q, *args)
    torch.cuda.synchronize()
    head = R.attend(host(q), host(c.k), host(c.v), *(a.cpu().numpy() for a in args), 64 ** -0.5)
    # scores of about 6e5 in 32 bits: off by (64 + 5) u of that, a few per cent, so only the row whose winner is alone is compared
    assert np.abs(host(got[0])[0, 2] - head[0][0, 2]).max() < 2.0 ** -11 * 4 and host(got[1])[0, 2] > 1e5
    near(host(got[0])[:, :2], head[0][:, :2], 1e-3, "other head")
    c.v[int(pt[0, 2]), 0, 5, 7] = float("nan")
    got = c.attend(q, *args)
    torch.cuda.synchronize()
    assert torch.isnan(got[0][:, :2, 7]).all() and not torch.isnan(got[0][:, :2, :7]).any() and not torch.isnan(got[0][:, 2:]).any()


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements; its last pages are written and read."""
    say("[long cache]")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    from paper_2409_19256_amd.rollout import KvCache
    gen = torch.Generator("cuda").manual_seed(7)
    page, heads, dim = 64, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 9
    c = KvCache.empty(pages, heads, page, dim)
    assert c.k.numel() > 1 << 32
    n = 3 * page
    k, v = (made((n, heads, dim), gen, "bf16") for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 7, pages - 3]], dtype=torch.int32, device="cuda")
    slots = (table.long()[0, :, None] * page + torch.arange(page, device="cuda")).flatten()
    c.append(k, v, slots)
    q = made((2, 8, dim), gen, "bf16")
    one = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    lens, none = torch.tensor([n - 5], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse = c.attend(q, none, torch.zeros(2, 1, dtype=torch.int32, device="cuda"), one, lens, table)
    torch.cuda.synchronize()
    small = KvCache(*(x.view(3, page, heads, dim).transpose(1, 2).contiguous() for x in (k, v)))
    mine = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    check_attention(small, "bf16", q, (none, torch.zeros(2, 1, dtype=torch.int32), one, lens, mine), (out, lse), n)


# ---- log probabilities ---------------------------------------------------------------------------------------------------

def logit_tolerance(x, temperature, vocab):
    """(relative error of a sum of exponentials, largest finite |y - max y|)"""
    y, fin = x / temperature, np.isfinite(x)
    reach = np.maximum(np.where(fin, y, -np.inf).max(1) - np.where(fin, y, np.inf).min(1), 0)
    size = np.where(fin, np.abs(y), 0).max(1)
    # an exponential's argument is rounded twice (|y - max| u log2 e each, and as much of the inverse temperature); what weighs e^-t t is below 1
    return (vocab / 64 + 80) * U + 16 * U, reach, size


def check_logprobs(logits, targets, temperature, top, got):
    x = host(logits)
    t = None if targets is None else targets.cpu().numpy()
    vocab = x.shape[1]
    lp, ent, lse, logp, live = R.logprobs(x, t, temperature)
    rel, reach, size = logit_tolerance(x, temperature, vocab)
    fin = lambda a: np.where(np.isfinite(a), np.abs(a), 0)  # noqa: E731
    if t is not None:
        near(host(got.logprob), lp, rel + 4 * U * (fin(lp) + 2 * reach), "logprob")
    near(host(got.lse), lse, rel + 4 * U * (fin(lse) + size), "lse")
    near(host(got.entropy), ent, (2 * rel + 8 * U) * (1 + np.log(vocab) + fin(ent)) * 2, "entropy")
    if top:
        want = R.top_ids(x, top)
        ids = got.top_ids.cpu().numpy()
        assert np.array_equal(ids[live], want[live])
        assert (ids[~live] == -1).all() and (got.top_logprobs.cpu().numpy()[~live] == 0).all()
        w = np.take_along_axis(logp, want, 1)[live]
        near(host(got.top_logprobs)[live], w, rel + 4 * U * (fin(w) + 2 * reach[live][:, None]), "top")


SCORES = [
    # dtype, rows, vocab, pad, top, temperature
    ("bf16", 5, 32000, 0, 5, 1.0), ("f32", 3, 128256, 0, 20, 0.7), ("f16", 7, 5004, 1, 64, 1.3), ("bf16", 4, 1, 0, 1, 1.0), ("f32", 6, 2, 3, 2, 1.0),
    ("f16", 3, 7, 0, 7, 0.5), ("bf16", 9, 64, 0, 64, 1.0), ("bf16", 3, 511, 2, 64, 1.0), ("f32", 3, 513, 1, 33, 2.0), ("bf16", 2, 4095, 0, 0, 1.0),
    ("bf16", 2, 4096, 7, 1, 1.0), ("f16", 2, 4104, 0, 3, 1.0), ("f32", 2, 32771, 1, 10, 1.0), ("bf16", 2, 65543, 0, 8, 1.0), ("bf16", 1, 128256, 0, 64, 1.0),
    ("f16", 300, 1024, 0, 4, 1.0), ("f32", 2, 300001, 0, 6, 1.0), ("bf16", 700, 33, 0, 2, 0.9),
]


def scores_inputs(case):
    dtype, rows, vocab, pad, top, temperature = case
    gen = torch.Generator("cuda").manual_seed(vocab + rows)
    store = (3 * torch.randn(rows, vocab + pad, generator=gen, device="cuda")).to(TYPES[dtype])
    logits = store[:, pad // 2:pad // 2 + vocab]
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    return gen, logits, targets


@pytest.mark.gpu
@pytest.mark.parametrize("case", SCORES, ids=str)
def test_logprobs(case):
    from paper_2409_19256_amd import rollout
    dtype, rows, vocab, pad, top, temperature = case
    say("[logprobs]", case)
    gen, logits, targets = scores_inputs(case)
    if rows > 4:
        targets[1], targets[2], targets[4] = -100, vocab, vocab - 1
        logits[1], logits[2] = float("nan"), float("inf")   # rows without a target are not read
    got = rollout.token_logprobs(logits, targets, temperature, top)
    narrow = rollout.token_logprobs(logits, targets.to(torch.int32), temperature, top)
    torch.cuda.synchronize()
    check_logprobs(logits, targets, temperature, top, got)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, narrow))
    if rows <= 4:
        every = rollout.token_logprobs(logits, None, temperature, top)
        torch.cuda.synchronize()
        assert every.logprob is None
        check_logprobs(logits, None, temperature, top, every)


def special_rows(dtype, vocab):
    """Rows with ties, ruled-out tokens, nothing left, the type's lowest value, all equal, ascending, descending."""
    gen = torch.Generator().manual_seed(vocab)
    low = torch.finfo(TYPES[dtype]).min
    big = torch.finfo(TYPES[dtype]).max
    x = torch.randn(12, vocab, generator=gen)
    x[0] = torch.randint(-2, 3, (vocab,), generator=gen).float()          # ties everywhere
    x[1, torch.randperm(vocab, generator=gen)[: vocab * 9 // 10]] = -np.inf
    x[2] = -np.inf
    x[3] = low
    x[4] = 0
    x[4, ::2] = -0.0
    x[5] = torch.linspace(-5, 5, vocab)
    x[6] = torch.linspace(5, -5, vocab)
    x[7] = -np.inf
    x[7, vocab // 2] = -3
    x[8, : vocab // 2] = low
    x[9] = low
    x[9, vocab - 1] = big
    x[10] = torch.arange(vocab).remainder(64).float()                      # equal ones at one distance: one lane's
    x[11] = 20 * torch.randn(vocab, generator=gen)
    return x.to(TYPES[dtype]).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [40, 1000, 5004, 33000])
def test_special_rows(dtype, vocab):
    from paper_2409_19256_amd import rollout
    say("[special rows]", dtype, vocab)
    x = special_rows(dtype, vocab)
    targets = torch.tensor([3, 1, 2, 0, 9, 8, 7, vocab // 2, 0, vocab - 1, 11, 39], device="cuda")
    got = rollout.token_logprobs(x, targets, 1.0, 20)
    torch.cuda.synchronize()
    check_logprobs(x, targets, 1.0, 20, got)
    # the same vectors in one lane's hands: more elements reach the bound than there is room for
    tall = torch.zeros(3, vocab, device="cuda", dtype=TYPES[dtype])
    size = 4 if dtype == "f32" else 8
    lane = (torch.arange(vocab, device="cuda") // size) % 64 < 20
    tall[0, lane] = 1 + (torch.arange(vocab, device="cuda", dtype=torch.float32)[lane] / vocab).to(TYPES[dtype])
    tall[1, lane] = 1
    tall[1, 0::997] = 2
    tall[2, lane] = -np.inf
    got = rollout.token_logprobs(tall, None, 1.0, 20)
    torch.cuda.synchronize()
    check_logprobs(tall, None, 1.0, 20, got)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [50, 5000, 40000])
def test_rows_with_nan_and_infinity(vocab):
    from paper_2409_19256_amd import rollout
    say("[nan rows]", vocab)
    x = torch.randn(5, vocab, device="cuda").to(torch.bfloat16)
    x[0, vocab // 3] = float("nan")
    x[1, vocab - 1] = float("inf")
    x[2] = float("nan")
    x[3] = torch.full((vocab,), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)  # a NaN with its sign
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    got = rollout.token_logprobs(x, t, 1.0, 20)
    torch.cuda.synchronize()
    for name in ("logprob", "entropy", "lse"):
        y = getattr(got, name)
        assert torch.isnan(y[:4]).all() or name == "lse" and torch.isnan(y[[0, 2, 3]]).all() and not torch.isfinite(y[1]), name
        assert torch.isfinite(y[4]), name
    ids = got.top_ids.cpu().numpy()
    assert ((ids >= 0) & (ids < vocab)).all() and all(len(set(r)) == 20 for r in ids.tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [50, 5000, 40000])
def test_rows_with_signalling_nan(vocab):
    from paper_2409_19256_amd import rollout
    say("[signalling nan rows]", vocab)
    x = torch.randn(3, vocab, device="cuda").to(torch.bfloat16)
    x.view(torch.int16)[0, vocab // 2] = 0x7F81
    x.view(torch.int16)[1] = 0x7F81
    x.view(torch.int16)[2, 7::9] = -0x7F  # with its sign
    got = rollout.token_logprobs(x, torch.zeros(3, dtype=torch.int64, device="cuda"), 1.0, 20)
    torch.cuda.synchronize()
    assert all(torch.isnan(t).all() for t in (got.logprob, got.entropy, got.lse))
    ids = got.top_ids.cpu().numpy()
    assert ((ids >= 0) & (ids < vocab)).all() and all(len(set(r)) == 20 for r in ids.tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("case", SCORES, ids=str)
def test_gradient(case):
    from paper_2409_19256_amd import rollout
    dtype, rows, vocab, pad, top, temperature = case
    say("[gradient]", case)
    gen, logits, targets = scores_inputs(case)
    if rows > 4:
        targets[1], targets[2], targets[4] = -100, vocab, vocab - 1
        logits[1], logits[2] = float("nan"), float("inf")
    if vocab > 2:
        logits[0, (int(targets[0]) + 1) % vocab] = -np.inf
    g, h = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    r = rollout.token_logprobs(logits, targets, temperature)
    t = targets.cpu().numpy()
    x = host(logits)
    lp, ent, lse, *_ = R.logprobs(x, t, temperature)
    rel, reach, size = logit_tolerance(x, temperature, vocab)

    def check(dx, g, h):
        want, p, logp = R.logprobs_back(x, t, temperature, host(g), host(h))
        live = ((t >= 0) & (t < vocab))[:, None]
        ln = np.where(np.isfinite(logp), np.abs(logp), 0)
        fl = np.where(np.isfinite(lse), np.abs(lse), 0)[:, None]
        # ln p = y - lse is off by the roundings of y and lse, and p by as much of itself; the entropy by its own tolerance
        d = rel + 4 * U * (size[:, None] + fl + ln + 2)
        e = (4 * rel + 16 * U) * (1 + np.log(vocab) + np.abs(ent[:, None]))
        ag, ah = np.abs(host(g))[:, None], np.abs(host(h))[:, None]
        tol = (np.where(np.isfinite(p), p, 0) * ((ag + ah * (ln + np.abs(ent[:, None]))) * (d + 8 * U) + ah * (d + e)) + 8 * U * ag) / temperature
        near(host(dx), want, np.where(live, tol * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(want) + SMALLEST[dtype] + 2.0 ** -126, 0), "dx")

    dx = rollout.token_logprobs_back(logits, targets, r.norm, r.entropy, g, h, temperature)
    torch.cuda.synchronize()
    check(dx, g, h)
    zero = torch.zeros_like(g)
    check(rollout.token_logprobs_back(logits, targets, r.norm, None, g, None, temperature), g, zero)
    check(rollout.token_logprobs_back(logits, targets, r.norm, r.entropy, None, h, temperature), zero, h)
    # in the logits' own place, and with room between the rows
    wide = torch.full((rows, vocab + 5), 9.0, device="cuda", dtype=logits.dtype)
    rollout.token_logprobs_back(logits, targets, r.norm, r.entropy, g, h, temperature, out=wide[:, 2:vocab + 2])
    assert torch.equal(wide[:, 2:vocab + 2], dx) and (wide[:, :2] == 9).all() and (wide[:, vocab + 2:] == 9).all()
    rollout.token_logprobs_back(logits, targets, r.norm, r.entropy, g, h, temperature, out=logits)
    assert torch.equal(logits, dx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradient_of_special_rows(dtype):
    from paper_2409_19256_amd import rollout
    say("[gradient of special rows]", dtype)
    x = special_rows(dtype, 1000)
    targets = torch.tensor([3, 1, 2, 0, 9, 8, 7, 500, 0, 999, 11, 39], device="cuda")
    g = torch.ones(12, device="cuda")
    r = rollout.token_logprobs(x, targets)
    dx = host(rollout.token_logprobs_back(x, targets, r.norm, r.entropy, g, g))
    want, p, logp = R.logprobs_back(host(x), targets.cpu().numpy(), 1.0, np.ones(12), np.ones(12))
    assert dx[2].sum() == 1 and dx[2, 2] == 1 and np.isfinite(dx).all()
    # as in test_gradient; logits of up to 80 and log p of up to -160 here, or all alike
    near(dx, want, HALF_STEP[dtype] * np.abs(want) + p * 2.0 ** -12 + 2.0 ** -20, "dx")


@pytest.mark.gpu
def test_gradient_through_autograd():
    from paper_2409_19256_amd import rollout
    say("[autograd]")
    gen = torch.Generator("cuda").manual_seed(8)
    x = (2 * torch.randn(6, 77, generator=gen, device="cuda")).requires_grad_()
    t = torch.tensor([3, 76, -100, 0, 5, 9], device="cuda")
    lp, ent = rollout.logprobs(x, t, 0.8)
    (lp.sum() + 0.5 * (ent ** 2).sum()).backward()      # the first gradient is a broadcast 1
    y = x.detach().double().cpu().requires_grad_()
    logp = torch.log_softmax(y / 0.8, 1)
    live = (t >= 0).cpu()
    want = logp[torch.arange(6), t.clamp(min=0).cpu()][live].sum() + 0.5 * ((-(logp.exp() * logp).sum(1))[live] ** 2).sum()
    want.backward()
    # every factor within 2^-18 of itself (logits below 2^4, sums of 77), gradients of order 1
    near(x.grad.cpu().numpy(), y.grad.numpy(), 2.0 ** -17, "autograd")


# ---- streams and graphs --------------------------------------------------------------------------------------------------

def rollout_step(gen):
    """A step with everything in it, on buffers that stay: returns (function, its inputs that may change, its outputs)."""
    from paper_2409_19256_amd import rollout
    c, q, (sl, st, off, pl, pt), n = attention_inputs(gen, "bf16", 8, 4, 64, 16, "heads", 0, [3, 2], (90, 200), (40, 7, 33))
    k, v = (made((5, 4, 64), gen, "bf16") for _ in range(2))
    slots = st[torch.arange(5, device="cuda"), ((sl - 1) // 16).long()].long() * 16 + (sl - 1) % 16
    positions = (sl - 1).contiguous()
    cos, sin = (torch.randn(300, 32, generator=gen, device="cuda") for _ in range(2))
    head = (0.1 * torch.randn(512, 203, generator=gen, device="cuda")).to(torch.bfloat16)
    targets = torch.tensor([1, 202, -1, 0, 7], device="cuda")
    adv = torch.randn(5, generator=gen, device="cuda")

    def step():
        turned = c.append(k, v, slots, positions, cos, sin, q=q)
        out, lse = c.attend(turned, sl, st, off, pl, pt)
        logits = out.view(5, 512) @ head
        r = rollout.token_logprobs(logits, targets, 0.9, 6)
        return (out, lse, logits) + tuple(r) + (rollout.token_logprobs_back(logits, targets, r.norm, r.entropy, adv, adv, 0.9),)

    return step, (q, k, v, adv)


@pytest.mark.gpu
def test_another_stream():
    say("[stream]")
    step, inputs = rollout_step(torch.Generator("cuda").manual_seed(9))
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(other):
            got = step()
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_graph():
    """Captured once, replayed with other inputs; every replay against the eager step, with eager work between."""
    say("[graph]")
    gen = torch.Generator("cuda").manual_seed(10)
    step, inputs = rollout_step(gen)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        step()
    torch.cuda.current_stream().wait_stream(other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outputs = step()
    for _ in range(4):
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
