"""Performance cases of what surrounds a rollout's steps: adjusting logits before a token is chosen, the pages of a cache whose sequences
are forked, grown and compacted, and the distillation loss over a teacher's top tokens with its gradient.

Heads, layers, widths and vocabularies are those of the benchmark's models and of their generation TP slices (the 70B shape over
four ranks has 2 KV heads), of the tiny decoder, or the tests' odd ones.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _named(c, name):
    return dict(c, name=name) if name else c


def _adjust(name, dtype, rows, vocab, prompt, answer, biases, grammars, pad=0):
    return _named(dict(op="adjust", dtype=dtype, rows=rows, vocab=vocab, prompt=prompt, answer=answer, biases=biases, grammars=grammars, pad=pad), name)


def _distill(name, dtype, rows, vocab, top, without=0.0, temperature=1.0, reverse=0.0, rest=True, pad=0):
    return _named(dict(op="distill", dtype=dtype, rows=rows, vocab=vocab, top=top, without=without, temperature=temperature, reverse=reverse, rest=rest,
                       pad=pad), name)


def _fork(name, dtype, heads, layers, page, rows, kept, each, tokens, spare, by="heads"):
    return _named(dict(op="fork", dtype=dtype, kv_heads=heads[0], head_dim=heads[1], layers=layers, page=page, rows=rows, kept=kept, each=each, tokens=tokens,
                       spare=spare, by=by), name)


def _grow(name, page, pages, rows, tokens, most):
    return _named(dict(op="grow", page=page, pages=pages, rows=rows, tokens=tokens, most=most), name)


def _compact(name, dtype, heads, layers, page, pages, live, rows, by="heads"):
    return _named(dict(op="compact", dtype=dtype, kv_heads=heads[0], head_dim=heads[1], layers=layers, page=page, pages=pages, live=live, rows=rows, by=by), name)


def listed():
    return [
        # one step of 64 sequences at the 7B shape's vocabulary, penalties and a few biases
        _adjust("adjust_step", "bf16", 64, 32000, 512, 512, 16, 0),
        # one step of 1024 sequences, half of them held to one of eight grammars
        _adjust("adjust_batch", "bf16", 1024, 32000, 512, 1024, 0, 8),
        # the 70B shape's vocabulary in 32 bits, long answers
        _adjust("adjust_large", "f32", 1024, 128256, 1024, 4096, 64, 4),
        # an odd batch over the tests' odd vocabulary, rows one element apart from their alignment, the student's divergence from the teacher
        _distill("distill_odd", "f16", 1361, 5004, 5, 0.2, 0.9, 1.0, pad=1),
        # a micro-batch at the 7B shape, a third of it prompt tokens without a teacher
        _distill("distill_7b", "bf16", 4096, 32000, 20, 0.33),
        # the 70B shape's vocabulary in 32 bits, both divergences in equal parts, the longest list that token_logprobs gives
        _distill("distill_large", "f32", 2048, 128256, 64, reverse=0.5),
        # the tiny decoder: three prompts become four samples each
        _fork("fork_tiny", "bf16", (4, 64), 2, 16, 3, 3, 4, 37, 20),
        # all layers of one of four ranks of the 70B shape: the best 32 of 128 answers go on four times each
        _fork("fork_70b", "bf16", (2, 128), 80, 64, 128, 32, 4, 448, 64),
        # one more token for every sequence of a step
        _grow("grow_step", 64, 4096, 256, 509, 1),
        # a batch of prompts comes in
        _grow("grow_prompts", 16, 300000, 4096, 0, 1024),
        # the tiny decoder's cache after half of its sequences have ended
        _compact("compact_tiny", "bf16", (4, 64), 2, 16, 256, 0.5, 12),
        # two layers of the 7B shape: most answers have ended, and the upper part of the memory is wanted back
        _compact("compact_7b", "bf16", (32, 128), 2, 64, 1024, 0.4, 64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adjust", "adjust", "distill", "distill", "fork", "grow", "compact"])
    if op in ("adjust", "distill"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        vocab = rng.choice([1024, 5004, 32000, 32000, 50257, 128256, _log_uniform(rng, 100, 130000)])
        size, pad = 4 if dtype == "f32" else 2, rng.choice([0, 0, 1, 8])
        rows = min(_log_uniform(rng, 1, 8192), (1 << 28) // (size * vocab) + 1)
        if op == "adjust":
            prompt, answer = _log_uniform(rng, 1, 2048), _log_uniform(rng, 1, 4096)
            return _adjust("", dtype, rows, vocab, prompt, answer, rng.choice([0, 1, 16, 300]), rng.choice([0, 0, 1, 8]), pad)
        top = rng.choice([1, 5, 20, 64, _log_uniform(rng, 1, 100)])
        return _distill("", dtype, rows, vocab, top, rng.choice([0.0, 0.33, 0.5]), rng.choice([1.0, 1.0, 0.7, 1.3]), rng.choice([0.0, 0.0, 0.5, 1.0]),
                        rng.random() < 0.7, pad)
    if op == "grow":
        page, rows = rng.choice([4, 16, 32, 64, 128]), _log_uniform(rng, 1, 4096)
        tokens, most = _log_uniform(rng, 1, 2048), rng.choice([1, 1, _log_uniform(rng, 1, 1024)])
        pages = rows * (-(-tokens // page) + -(-most // page)) + _log_uniform(rng, 1, 10000)
        return _grow("", page, pages, rows, tokens, most)
    heads = rng.choice([(32, 128), (20, 128), (8, 128), (2, 128), (12, 64), (4, 64), (8, 32), (4, 72), (3, 65)])
    dtype, by, page = rng.choice(["bf16", "bf16", "f16"]), rng.choice(["heads", "heads", "tokens"]), rng.choice([8, 16, 32, 64, 128])
    layers = _log_uniform(rng, 1, 80)
    most = (3 << 29) // (4 * heads[0] * heads[1] * page * layers)  # pages in 1.5 GiB
    if op == "fork":
        kept, each = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 8)
        rows, tokens = kept + rng.choice([0, _log_uniform(rng, 1, 64)]), _log_uniform(rng, 1, 2048)
        while rows * (tokens // page + 1) + kept * each + 1 > most:
            rows, kept, tokens = max(1, rows // 2), max(1, kept // 2), max(1, tokens // 2)
            if rows == kept == tokens == 1:
                layers, most = max(1, layers // 2), most * 2
        return _fork("", dtype, heads, layers, page, rows, kept, each, tokens, kept * each + 1, by)
    pages = max(4, min(most, _log_uniform(rng, 16, 20000)))
    return _compact("", dtype, heads, layers, page, pages, rng.choice([0.1, 0.4, 0.5, 0.9]), _log_uniform(rng, 1, 256), by)


# ---- what sizes a case has: by the case alone, the seed only deals them out ----------------------------------------------

def _without(c):
    return int(c["rows"] * c["without"])


def _history(c):
    """(prompt tokens, tokens in all) of every row: prompts from half the longest up to it, answers evenly from none to the longest."""
    prompt = [c["prompt"] - (i * 77) % (c["prompt"] // 2 + 1) for i in range(c["rows"])]
    return prompt, [p + c["answer"] * i // max(1, c["rows"] - 1) for i, p in enumerate(prompt)]


def _lens(c):
    """Tokens of every sequence, evenly from one to the longest (grow may begin with none); those that a fork keeps come from the whole range."""
    n = c["rows"]
    lens = [min(c["tokens"], 1 + ((c["tokens"] - 1) * (i + 1)) // n) for i in range(n)]
    step = next(s for s in (7, 11, 13, 17, 1) if s == 1 or n % s)
    return [lens[i * step % n] for i in range(n)]


def _new(c):
    """New tokens of every sequence: the most, or evenly from one to the most."""
    return [1 + ((c["most"] - 1) * (i + 1)) // c["rows"] for i in range(c["rows"])]


def _pages_of(lens, page):
    return [-(-n // page) for n in lens]


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _logits(c, gen, dtype):
    """Logits with the spread of a language model's."""
    r, width = c["rows"], c["vocab"] + c["pad"]
    store = torch.empty(r, width, device="cuda", dtype=dtype)
    for i in range(0, r, 512):
        n = min(512, r - i)
        store[i:i + n] = 2.2 * torch.randn(n, width, generator=gen, device="cuda")
    return store[:, :c["vocab"]]


def _prepare_adjust(c, gen, dtype):
    r, v = c["rows"], c["vocab"]
    s = dict(logits=_logits(c, gen, dtype))
    prompt, total = _history(c)
    deal = torch.randperm(r, generator=gen, device="cuda")
    s["prompt_lens"], s["lens"] = (torch.tensor(x, dtype=torch.int32, device="cuda")[deal].contiguous() for x in (prompt, total))
    # tokens repeat as words do: a few make up most of a text
    width = c["prompt"] + c["answer"]
    s["tokens"] = (v * torch.rand(r, width, generator=gen, device="cuda", dtype=torch.float64) ** 3).long().clamp(max=v - 1)
    s["repetition"] = 1 + 0.3 * torch.rand(r, generator=gen, device="cuda")
    s["frequency"], s["presence"] = (0.5 * torch.rand(r, generator=gen, device="cuda") for _ in range(2))
    s["bias_ids"] = s["bias"] = s["allowed"] = s["allowed_rows"] = None
    if c["biases"]:
        s["bias_ids"] = torch.randint(0, v, (r, c["biases"]), generator=gen, device="cuda", dtype=torch.int32)
        s["bias_ids"][torch.rand(r, c["biases"], generator=gen, device="cuda") < 0.2] = -1  # rows with fewer
        s["bias"] = 4 * torch.randn(r, c["biases"], generator=gen, device="cuda")
    if c["grammars"]:
        words = -(-v // 32)
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (c["grammars"], words), generator=gen, device="cuda", dtype=torch.int64)
        s["allowed"] &= torch.randint(-2 ** 31, 2 ** 31, (c["grammars"], words), generator=gen, device="cuda", dtype=torch.int64)
        s["allowed"] = s["allowed"].to(torch.int32)
        s["allowed_rows"] = torch.randint(0, c["grammars"], (r,), generator=gen, device="cuda", dtype=torch.int32)
        s["allowed_rows"][torch.randperm(r, generator=gen, device="cuda")[:r // 2]] = -1
    return s


def _prepare_distill(c, gen, dtype):
    """A teacher that mostly agrees; its list of the likeliest tokens in falling order."""
    r, v = c["rows"], c["vocab"]
    s = dict(logits=_logits(c, gen, dtype), temperature=c["temperature"], reverse=c["reverse"], rest=c["rest"])
    top = min(c["top"], v)
    s["top_ids"] = torch.empty(r, top, device="cuda", dtype=torch.int32)
    s["top_logprobs"] = torch.empty(r, top, device="cuda")
    sure = torch.randint(0, v, (r,), generator=gen, device="cuda")
    for i in range(0, r, 512):
        rows = torch.arange(i, min(r, i + 512), device="cuda")
        at = torch.arange(len(rows), device="cuda")
        s["logits"][rows, sure[rows]] += (9 * torch.rand(len(rows), generator=gen, device="cuda")).to(dtype)
        t = s["logits"][rows].float() + 0.7 * torch.randn(len(rows), v, generator=gen, device="cuda")
        t[at, sure[rows]] += 2 * torch.rand(len(rows), generator=gen, device="cuda")
        best = (t - t.logsumexp(1, keepdim=True)).topk(top, dim=1)
        s["top_logprobs"][rows], s["top_ids"][rows] = best.values, best.indices.to(torch.int32)
    left = torch.randperm(r, generator=gen, device="cuda")[:_without(c)]
    s["top_ids"][left], s["top_logprobs"][left] = -1, 0.0
    s["grad_loss"] = torch.rand(r, generator=gen, device="cuda")  # weights of the rows; a mean's 1 / rows is made up for, as losses in 16 bits are scaled
    return s


def _caches(c, pages, gen, dtype):
    """All layers' keys and values in one allocation [layer, 2, page, KV head, token, element], in either order of memory."""
    h, p, d = c["kv_heads"], c["page"], c["head_dim"]
    shape = (c["layers"], 2, pages, h, p, d) if c["by"] == "heads" else (c["layers"], 2, pages, p, h, d)
    store = torch.empty(shape, device="cuda", dtype=dtype)
    for layer in store:
        layer.normal_(generator=gen)
    return store, store if c["by"] == "heads" else store.transpose(3, 4)


def _table(lens, page, at, width):
    """Page tables: every row its own pages, dealt out of `at` (a permutation); unused entries -1."""
    need = torch.tensor(_pages_of(lens, page))
    begin = torch.cumsum(need, 0) - need
    i = torch.arange(width)[None, :]
    where = (begin[:, None] + i).clamp(max=at.numel() - 1).cuda()
    return torch.where((i < need[:, None]).cuda(), at[where], -1).to(torch.int32).contiguous()


def _refs(table, pages):
    named = table[table >= 0].long()
    return torch.zeros(pages, device="cuda", dtype=torch.int32).index_add_(0, named, torch.ones_like(named, dtype=torch.int32))


def _prepare_fork(c, gen, dtype):
    rows, lens = c["rows"], _lens(c)
    pages = sum(_pages_of(lens, c["page"])) + c["spare"]
    s = {"page": c["page"]}
    s["store"], s["caches"] = _caches(c, pages, gen, dtype)
    deal = torch.randperm(rows, generator=gen, device="cuda")  # where row i of the case lies
    width = max(_pages_of(lens, c["page"])) + 1
    table = _table(lens, c["page"], torch.randperm(pages, generator=gen, device="cuda"), width)
    s["tables"], s["lens"] = torch.empty_like(table), torch.empty(rows, device="cuda", dtype=torch.int32)
    s["tables"][deal], s["lens"][deal] = table, torch.tensor(lens, dtype=torch.int32, device="cuda")
    parents = deal[:c["kept"]].repeat_interleave(c["each"])
    s["parents"] = parents[torch.randperm(len(parents), generator=gen, device="cuda")].to(torch.int32)
    s["refs"] = _refs(s["tables"], pages)
    return s


def _prepare_grow(c, gen, dtype):
    rows, lens, new = c["rows"], _lens(c), _new(c)
    deal = torch.randperm(rows, generator=gen, device="cuda")
    width = max(_pages_of([a + b for a, b in zip(lens, new)], c["page"]))
    table = _table(lens, c["page"], torch.randperm(c["pages"], generator=gen, device="cuda"), width)
    s = {"page": c["page"], "most": c["most"], "tables": table[deal].contiguous()}
    s["lens"], s["counts"] = (torch.tensor(x, dtype=torch.int32, device="cuda")[deal].contiguous() for x in (lens, new))
    s["refs"] = _refs(s["tables"], c["pages"])
    # the smallest cache that has such pages: nothing is read or written in it
    s["store"] = torch.zeros(1, 2, c["pages"], 1, c["page"], 1, device="cuda", dtype=torch.bfloat16)
    s["caches"] = s["store"]
    return s


def _prepare_compact(c, gen, dtype):
    s = {"page": c["page"]}
    s["store"], s["caches"] = _caches(c, c["pages"], gen, dtype)
    live, rows = int(c["pages"] * c["live"]), c["rows"]
    # pages that lie anywhere: as many stand past the live ones' number as that leaves room for below it
    room = live * (c["pages"] - live) // c["pages"]
    low, high = (torch.randperm(n, generator=gen, device="cuda") for n in (live, c["pages"] - live))
    at = torch.cat((low[:live - room], live + high[:room]))[torch.randperm(live, generator=gen, device="cuda")]
    # every live page in one row or another, the first of them (a shared beginning) in every row
    width = 1 + -(-live // rows)
    table = torch.full((rows, width), -1, device="cuda", dtype=torch.int32)
    if live:
        table[:, 0] = at[0]
        i = torch.arange(1, live, device="cuda")
        table[(i - 1) % rows, 1 + (i - 1) // rows] = at[1:live].to(torch.int32)
    s["tables"], s["refs"] = table, _refs(table, c["pages"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"adjust": _prepare_adjust, "distill": _prepare_distill, "fork": _prepare_fork, "grow": _prepare_grow, "compact": _prepare_compact}[case["op"]]
    s = make(case, gen, DTYPES[case.get("dtype", "bf16")])
    s["op"] = case["op"]
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _adjust_plain(s):
    x = s["logits"].float()
    r, v = x.shape
    at = torch.arange(s["tokens"].shape[1], device=x.device)[None, :]
    inside = (at < s["lens"][:, None]) & (s["tokens"] >= 0) & (s["tokens"] < v)
    answer = inside & (at >= s["prompt_lens"][:, None])
    place = s["tokens"].clamp(0, v - 1)
    seen = torch.zeros(r, v, device=x.device).scatter_add_(1, place, inside.float()) > 0
    count = torch.zeros(r, v, device=x.device).scatter_add_(1, place, answer.float())
    rep = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(count > 0, x - s["frequency"][:, None] * count - s["presence"][:, None], x)
    if s["bias"] is not None:
        # of several biases of a token the last one holds
        n = s["bias"].shape[1]
        given = (s["bias_ids"] >= 0) & (s["bias_ids"] < v)
        last = torch.zeros(r, v, device=x.device, dtype=torch.int32)
        last.scatter_reduce_(1, s["bias_ids"].clamp(0, v - 1).long(), torch.where(given, torch.arange(1, n + 1, device=x.device, dtype=torch.int32), 0), "amax")
        x = torch.where(last > 0, x + s["bias"].gather(1, (last - 1).clamp(min=0).long()), x)
    if s["allowed"] is not None:
        held = (s["allowed_rows"] >= 0) & (s["allowed_rows"] < s["allowed"].shape[0])
        bits = (s["allowed"][:, :, None] >> torch.arange(32, device=x.device, dtype=torch.int32)) & 1
        open_ = bits.flatten(1)[:, :v].bool()[s["allowed_rows"].clamp(min=0).long()]
        x = x.masked_fill(held[:, None] & ~open_, -math.inf)
    return {"logits": x.to(s["logits"].dtype)}


def _distill_plain(s):
    """Both directions at once: the gradient of sum grad_loss * loss."""
    t, w = s["temperature"], s["reverse"]
    x = s["logits"].float() / t
    v = x.shape[1]
    named = (s["top_ids"] >= 0) & (s["top_ids"] < v) & (s["top_logprobs"] > -math.inf)
    live = named.any(1)
    # a place without a name writes to a column behind the last
    at = torch.where(named, s["top_ids"], v).long()
    inside = torch.zeros(x.shape[0], v + 1, device=x.device, dtype=torch.bool).scatter_(1, at, True)[:, :v]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    others = torch.where(inside, 0.0, e).sum(1, keepdim=True).double()
    mine = torch.where(named, x.gather(1, at.clamp(max=v - 1)) - m, -math.inf).double()
    z = mine.exp().sum(1, keepdim=True) + others
    # what the lists say, in 64 bits: one minus a sum of probabilities
    lq = torch.where(named, s["top_logprobs"].double(), 0.0)
    q = torch.where(named, lq.exp(), 0.0)
    lp = torch.where(named, mine - z.log(), 0.0)
    p = torch.where(named, lp.exp(), 0.0)
    rest = (others > 0) & s["rest"]
    q_rest = torch.where(rest, (1 - q.sum(1, keepdim=True)).clamp(min=0), 0.0)
    p_rest = torch.where(rest, others / z, 0.0)
    lq_rest = torch.where(rest, (1 - q.sum(1, keepdim=True)).clamp(min=2.0 ** -24).log(), 0.0)
    lp_rest = torch.where(rest, p_rest.log(), 0.0)
    ahead = (q * (lq - lp)).sum(1, keepdim=True) + torch.where(q_rest > 0, q_rest * (q_rest.log() - lp_rest), 0.0)
    back = (p * (lp - lq)).sum(1, keepdim=True) + p_rest * (lp_rest - lq_rest)
    loss = (1 - w) * ahead + w * back
    # what an unnamed token's probability is multiplied by, and the named ones' gradients
    mass, share = q.sum(1, keepdim=True) + q_rest, p.sum(1, keepdim=True) + p_rest
    factor = (1 - w) * (mass - torch.where(rest, q_rest / p_rest, 0.0)) + w * (torch.where(rest, lp_rest - lq_rest + 1, 0.0) - back - share)
    slopes = (1 - w) * (p * mass - q) + w * p * (lp - lq + 1 - back - share)
    scale = s["grad_loss"][:, None] / t
    grad = (e / z.float()) * (factor.float() * scale)
    grad = torch.cat((grad, grad[:, :1]), 1).scatter_(1, at, slopes.float() * scale)[:, :v]
    grad = torch.where(live[:, None], grad, 0.0).to(s["logits"].dtype)
    return {"loss": torch.where(live, loss[:, 0], 0.0).float(), "grad": grad}


def _count(refs, entries, by):
    named = (entries >= 0).to(torch.int32) * by
    return refs.index_add_(0, entries.clamp(min=0).flatten().long(), named.flatten())


def _free_list(refs):
    """The free pages in rising order, behind them anything; and how many there are."""
    free = refs == 0
    n = free.sum()
    order = torch.where(free, 0, 1).to(torch.int32).argsort(stable=True)
    return order, n


def _fork_plain(s):
    page, tables, refs = s["page"], s["tables"], s["refs"].clone()
    rows, width = tables.shape
    pages = refs.numel()
    slot = torch.arange(width, device=tables.device)[None, :]
    there = lambda t, n: torch.where((slot < (n[:, None] + page - 1) // page) & (t >= 0) & (t < pages), t, -1)  # noqa: E731
    lens = s["lens"].clamp(0, width * page)
    old = there(tables, lens)
    given = (s["parents"] >= 0) & (s["parents"] < rows)
    src = torch.where(given, s["parents"], 0).long()
    n = torch.where(given, lens[src], 0)
    new = there(tables[src], n)
    # the first sequence that goes on in a page that is not full keeps it; the others take copies
    out = torch.arange(len(src), device=tables.device)
    last_at = ((n + page - 1) // page - 1).clamp(min=0).long()[:, None]
    last = new.gather(1, last_at)[:, 0]
    part = (n % page > 0) & (last >= 0)
    first = torch.full((pages + 1,), len(src), device=tables.device).scatter_reduce_(0, torch.where(part, last, pages).long(), out, "amin")
    copies = part & (first[last.clamp(min=0).long()] != out)
    new = new.scatter(1, last_at, torch.where(copies, -1, last)[:, None])
    _count(_count(refs, old, -1), new, 1)
    order, free = _free_list(refs)
    place = torch.cumsum(copies, 0) - 1
    got = copies & (place < free)
    to = order[place.clamp(0, pages - 1)].to(torch.int32)
    # a sequence for which no page is left comes out empty
    lost = copies & ~got
    _count(refs, torch.where(lost[:, None], new, -1), -1)
    refs.index_add_(0, to.long(), got.to(torch.int32))
    new = torch.where(lost[:, None], -1, new.scatter(1, last_at, torch.where(got, to, new.gather(1, last_at)[:, 0])[:, None]))
    n = torch.where(lost, 0, n)
    at = got.nonzero()[:, 0]
    begun = (torch.arange(page, device=tables.device) < (n[at] % page)[:, None])[:, None, :, None]
    src, to = last[at].long(), to[at].long()
    s["caches"][:, :, to] = torch.where(begun, s["caches"][:, :, src], s["caches"][:, :, to])
    return {"tables": new, "lens": n, "refs": refs, "caches": s["store"]}


def _grow_plain(s):
    page, tables, refs = s["page"], s["tables"], s["refs"].clone()
    rows, width = tables.shape
    lens = s["lens"].clamp(0, width * page)
    count = s["counts"].clamp(0, s["most"])
    have, want = (lens + page - 1) // page, (lens + count + page - 1) // page
    fits = want <= width
    need = torch.where(fits, want - have, 0)
    before = torch.cumsum(need, 0) - need
    order, free = _free_list(refs)
    ok = fits & ((need == 0) | (before + need <= free))
    slot = torch.arange(width, device=tables.device)[None, :]
    fresh = ok[:, None] & (slot >= have[:, None]) & (slot < want[:, None])
    to = order[(before[:, None] + slot - have[:, None]).clamp(0, refs.numel() - 1)].to(torch.int32)
    new = torch.where(fresh, to, torch.where((slot < have[:, None]) & (tables >= 0) & (tables < refs.numel()), tables, -1))
    _count(refs, torch.where(fresh, to, -1), 1)
    i = torch.arange(s["most"], device=tables.device)[None, :]
    at = lens[:, None] + i
    named = new.gather(1, (at // page).clamp(max=width - 1).long()).long()
    slots = torch.where((ok[:, None] & (i < count[:, None])) & (named >= 0), named * page + at % page, -1)
    return {"tables": new, "lens": torch.where(ok, lens + count, lens), "slots": slots, "refs": refs}


def _compact_plain(s):
    refs, tables = s["refs"], s["tables"]
    pages = refs.numel()
    number = torch.arange(pages, device=refs.device)
    live = refs != 0
    n = live.sum()
    src = (live & (number >= n)).nonzero()[:, 0]
    to = (~live & (number < n)).nonzero()[:, 0]
    places = torch.where(live, number, -1)
    places[src] = to
    places = places.to(torch.int32)
    moved = torch.zeros_like(refs)
    moved.index_add_(0, places.clamp(min=0).long(), torch.where(live, refs, 0))
    inside = (tables >= 0) & (tables < pages)
    new = torch.where(inside, places[tables.clamp(0, pages - 1).long()], tables)
    s["caches"][:, :, to] = s["caches"][:, :, src]
    return {"tables": new, "refs": moved, "places": places, "live": n.to(torch.int32), "caches": s["store"]}


# ---- the framework's operators -------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2409_19256_amd import rollout
    if s["op"] == "adjust":
        return {"logits": rollout.adjust_logits(s["logits"], s["tokens"], s["lens"], s["prompt_lens"], repetition=s["repetition"], frequency=s["frequency"],
                                                presence=s["presence"], bias_ids=s["bias_ids"], bias=s["bias"], allowed=s["allowed"],
                                                allowed_rows=s["allowed_rows"])}
    if s["op"] == "distill":
        r = rollout.top_distill(s["logits"], s["top_ids"], s["top_logprobs"], temperature=s["temperature"], reverse=s["reverse"], rest=s["rest"])
        grad = rollout.top_distill_back(s["logits"], s["top_ids"], r.norm, r.slopes, s["grad_loss"], temperature=s["temperature"])
        return {"loss": r.loss, "grad": grad}
    if "pool" not in s:  # the handle that a program keeps beside its caches
        s["pool"] = rollout.PagePool([rollout.KvCache(k, v) for k, v in s["caches"]])
    pool = s["pool"]
    if s["op"] == "fork":
        tables, lens, refs = pool.fork(s["tables"], s["lens"], s["parents"], s["refs"])
        return {"tables": tables, "lens": lens, "refs": refs, "caches": s["store"]}
    if s["op"] == "grow":
        tables, lens, slots, refs = pool.grow(s["tables"], s["lens"], s["counts"], s["refs"], most=s["most"])
        return {"tables": tables, "lens": lens, "slots": slots, "refs": refs}
    (tables,), refs, places, live = pool.compact(s["refs"], [s["tables"]])
    return {"tables": tables, "refs": refs, "places": places, "live": live, "caches": s["store"]}


def run(state):
    if own:
        return _run_own(state)
    return {"adjust": _adjust_plain, "distill": _distill_plain, "fork": _fork_plain, "grow": _grow_plain, "compact": _compact_plain}[state["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    c = case
    size = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "adjust":
        n = c["rows"] * c["vocab"]
        read = n * size + 8 * sum(_history(c)[1]) + c["rows"] * (20 + 8 * c["biases"]) + c["grammars"] * 4 * -(-c["vocab"] // 32)
        return {"bytes": read + n * size, "flops": 2 * n}
    if c["op"] == "distill":
        live = c["rows"] - _without(c)
        n, lists = live * c["vocab"], 8 * c["rows"] * min(c["top"], c["vocab"])
        # the softmax has to be whole before the first gradient: read, then written
        return {"bytes": n * size + c["rows"] * c["vocab"] * size + lists + 12 * c["rows"], "flops": 8 * n}
    if c["op"] == "grow":
        have, new = _pages_of(_lens(c), c["page"]), _new(c)
        fresh = sum(_pages_of([a + b for a, b in zip(_lens(c), new)], c["page"])) - sum(have)
        return {"bytes": 8 * sum(have) + 4 * fresh + 16 * c["rows"] + 8 * c["rows"] * c["most"] + 8 * c["pages"], "flops": c["pages"]}
    token = 2 * size * c["kv_heads"] * c["head_dim"] * c["layers"]
    if c["op"] == "fork":
        lens = _lens(c)
        pages, kept = _pages_of(lens, c["page"]), range(c["kept"])
        moved = sum(lens[i] % c["page"] * ((c["each"] > 1) + c["each"] - 1) for i in kept)  # read once, written for each further sequence
        entries = sum(pages) + c["each"] * sum(pages[i] for i in kept)
        return {"bytes": moved * token + 4 * entries + 8 * (sum(pages) + c["spare"]) + 8 * c["kept"] * c["each"], "flops": entries}
    live = int(c["pages"] * c["live"])
    moved = live * (c["pages"] - live) // c["pages"]
    return {"bytes": 2 * moved * c["page"] * token + 8 * live + 16 * c["pages"], "flops": c["pages"]}


# ---- 64 bits -------------------------------------------------------------------------------------------------------------

def _exact_adjust(s):
    r, v = s["logits"].shape
    out = torch.empty(r, v, device="cuda", dtype=torch.float64)
    total, prompt, held = (s[n].tolist() if s[n] is not None else None for n in ("lens", "prompt_lens", "allowed_rows"))
    shift = torch.arange(32, device="cuda")
    for i in range(r):
        x = s["logits"][i].double()
        text, answer = s["tokens"][i, :total[i]], s["tokens"][i, prompt[i]:total[i]]
        there = torch.bincount(text, minlength=v) != 0
        times = torch.bincount(answer, minlength=v).double()
        rep = s["repetition"][i].double()
        x[there] = torch.maximum(x[there], torch.zeros_like(x[there])) / rep + torch.minimum(x[there], torch.zeros_like(x[there])) * rep
        x -= times * s["frequency"][i].double() + times.clamp(max=1) * s["presence"][i].double()
        if s["bias"] is not None:
            given = {j: b for j, b in zip(s["bias_ids"][i].tolist(), s["bias"][i].tolist()) if j >= 0}
            x[torch.tensor(list(given), device="cuda", dtype=torch.int64)] += torch.tensor(list(given.values()), device="cuda", dtype=torch.float64)
        if held is not None and held[i] >= 0:
            x[((s["allowed"][held[i]].long()[:, None] >> shift) % 2 == 0).flatten()[:v]] = -math.inf
        out[i] = x
    return {"logits": out}


def _exact_distill(s):
    """By autograd over the definition: log probabilities of the named tokens and of all others together."""
    r, v = s["logits"].shape
    loss = torch.zeros(r, device="cuda", dtype=torch.float64)
    grad = torch.zeros(r, v, device="cuda", dtype=torch.float64)
    w = s["reverse"]
    for rows in (s["top_ids"][:, 0] >= 0).nonzero()[:, 0].split(256):
        x = s["logits"][rows].double().requires_grad_()
        ids, lq = s["top_ids"][rows].long(), s["top_logprobs"][rows].double()
        logp = torch.log_softmax(x / s["temperature"], 1)
        lp = logp.gather(1, ids)
        if s["rest"] and ids.shape[1] < v:
            lp = torch.cat((lp, logp.scatter(1, ids, -math.inf).logsumexp(1, keepdim=True)), 1)
            over = 1 - lq.exp().sum(1, keepdim=True)
            lq = torch.cat((lq, over.clamp(min=2.0 ** -24).log()), 1)
            q = torch.cat((lq[:, :-1].exp(), over.clamp(min=0)), 1)
        else:
            q = lq.exp()
        one = (1 - w) * (torch.special.xlogy(q, q) - q * lp).sum(1) + w * (lp.exp() * (lp - lq)).sum(1)
        one.backward(s["grad_loss"][rows].double())
        loss[rows], grad[rows] = one.detach(), x.grad
    return {"loss": loss, "grad": grad}


def _moved(s, pairs):
    """The caches after pages (from, to, tokens) were copied."""
    store = s["store"].double()
    if pairs:
        token = torch.arange(s["page"], device="cuda")
        src, to, n = (torch.tensor(x, device="cuda") for x in zip(*pairs))
        whole = (token < n[:, None])[None, None, :, None, :, None]
        caches = store if s["caches"].stride() == s["store"].stride() else store.transpose(3, 4)
        caches[:, :, to] = torch.where(whole, caches[:, :, src], caches[:, :, to])
    return store


def _exact_fork(s):
    """Sequence after sequence, as a program on the host keeps its books."""
    page, width = s["page"], s["tables"].shape[1]
    tables, lens, parents, refs = (s[n].tolist() for n in ("tables", "lens", "parents", "refs"))
    rows = [t[:-(-n // page)] for t, n in zip(tables, lens)]
    for row in rows:
        for p in row:
            refs[p] -= 1
    taken, new, ends, wanted = set(), [], [], []
    for i, parent in enumerate(parents):
        row = list(rows[parent]) if parent >= 0 else []
        n = lens[parent] if parent >= 0 else 0
        if n % page and row[-1] in taken:
            wanted.append((i, row[-1], n % page))
            row[-1] = -1
        elif n % page:
            taken.add(row[-1])
        for p in row:
            if p >= 0:
                refs[p] += 1
        new.append(row)
        ends.append(n)
    free = [p for p, n in enumerate(refs) if n == 0]
    pairs = []
    for (i, src, n), p in zip(wanted, free):
        new[i][-1], refs[p] = p, 1
        pairs.append((src, p, n))
    new = [row + [-1] * (width - len(row)) for row in new]
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return {"tables": i32(new), "lens": i32(ends), "refs": i32(refs), "caches": _moved(s, pairs)}


def _exact_grow(s):
    page = s["page"]
    tables, lens, counts, refs = (s[n].tolist() for n in ("tables", "lens", "counts", "refs"))
    free = iter([p for p, n in enumerate(refs) if n == 0])
    slots = []
    for i, row in enumerate(tables):
        places = []
        for t in range(lens[i], lens[i] + counts[i]):
            if t % page == 0:
                row[t // page] = next(free)
                refs[row[t // page]] = 1
            places.append(row[t // page] * page + t % page)
        lens[i] += counts[i]
        slots.append(places + [-1] * (s["most"] - len(places)))
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return {"tables": i32(tables), "lens": i32(lens), "slots": torch.tensor(slots, device="cuda"), "refs": i32(refs)}


def _exact_compact(s):
    tables, refs = s["tables"].tolist(), s["refs"].tolist()
    live = [p for p, n in enumerate(refs) if n]
    room = iter([p for p in range(len(live)) if not refs[p]])
    place = {p: p if p < len(live) else next(room) for p in live}
    moved = [0] * len(refs)
    for p, to in place.items():
        moved[to] = refs[p]
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return {"tables": i32([[place.get(p, -1) for p in row] for row in tables]), "refs": i32(moved), "places": i32([place.get(p, -1) for p in range(len(refs))]),
            "live": i32(len(live)), "caches": _moved(s, [(p, to, s["page"]) for p, to in place.items() if p != to])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"adjust": _exact_adjust, "distill": _exact_distill, "fork": _exact_fork, "grow": _exact_grow, "compact": _exact_compact}[case["op"]](s)
