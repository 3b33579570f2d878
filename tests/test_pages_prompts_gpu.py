"""Pages beside the framework's way to sample: prompts whose pages are shared by their samples (attend's groups), samples with pages of their own that grow by a token a step, are dropped and
continued within their prompt, and moved together with the prompts'.  Beside it every sequence's keys and values as plain arrays, from which attention is computed again in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_rollout_gpu import HALF_STEP, U, host, near

LAYERS, HEADS, KV, DIM, PAGE, PAGES, WIDTH, SAMPLES = 2, 4, 2, 64, 8, 70, 6, 4
PROMPTS = [21, 16, 0, 3]  # pages in part, whole pages, no tokens, less than a page


@pytest.mark.gpu
def test_samples_of_shared_prompts():
    from paper_2409_19256_amd import rollout
    gen = torch.Generator("cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    ints = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    empty = lambda rows: (torch.full((rows, WIDTH), -1, device="cuda", dtype=torch.int32), ints([0] * rows))  # noqa: E731
    pool = rollout.PagePool([rollout.KvCache.empty(PAGES, KV, PAGE, DIM) for _ in range(LAYERS)])
    groups, rows = len(PROMPTS), len(PROMPTS) * SAMPLES
    # the prompts come in at once
    p_tables, p_lens = empty(groups)
    p_tables, p_lens, slots, refs = pool.grow(p_tables, p_lens, ints(PROMPTS), pool.refs(), max(PROMPTS))
    assert p_lens.tolist() == PROMPTS and int(refs.sum()) == sum(-(-n // PAGE) for n in PROMPTS)
    k, v = rand(LAYERS, groups, max(PROMPTS), KV, DIM), rand(LAYERS, groups, max(PROMPTS), KV, DIM)
    for i, cache in enumerate(pool.caches):
        cache.append(k[i].flatten(0, 1), v[i].flatten(0, 1), slots.flatten())
    prompts = [(host(k[:, g, :n]), host(v[:, g, :n])) for g, n in enumerate(PROMPTS)]  # [layer, token, KV head, element]
    tables, lens = empty(rows)
    offsets = ints([SAMPLES * g for g in range(groups + 1)])
    shadow = [[] for _ in range(rows)]
    for step in range(26):
        print("[prompts] step", step, flush=True)
        if step in (6, 11, 17):  # within every prompt: one ends, one goes on twice
            parents = [SAMPLES * (r // SAMPLES) + ((0, 1, 1, 3), (2, 0, 2, 2), (3, 2, 1, 0))[step % 3][r % SAMPLES] for r in range(rows)]
            tables, lens, refs = pool.fork(tables, lens, ints(parents), refs, refs_out=refs)
            shadow = [list(shadow[p]) for p in parents]
        if step in (8, 19):
            (p_tables, tables), refs, _, live = pool.compact(refs, [p_tables, tables], [p_tables, None], refs)
            assert int(live) == int((refs > 0).sum()) and not refs[int(live):].any()
        used = torch.zeros(PAGES, dtype=torch.int32)
        for table, n in [(t, n) for t, n in zip(p_tables.tolist(), PROMPTS)] + [(t, len(s)) for t, s in zip(tables.tolist(), shadow)]:
            for p in table[:-(-n // PAGE)]:
                used[p] += 1
        assert torch.equal(used, refs.cpu())
        tables, lens, slots, refs = pool.grow(tables, lens, ints([1] * rows), refs, refs_out=refs)
        q, k, v = rand(rows, HEADS, DIM), rand(LAYERS, rows, KV, DIM), rand(LAYERS, rows, KV, DIM)
        for r in range(rows):
            shadow[r].append((host(k[:, r]), host(v[:, r])))
        for i, cache in enumerate(pool.caches):
            cache.append(k[i], v[i], slots[:, 0].contiguous())
            got, _ = cache.attend(q, lens, tables, offsets, p_lens, p_tables, max_group=SAMPLES)
            for r in range(rows if step % 5 == 0 or step in (6, 8, 11, 17, 19) else 0):
                keys, values = (np.concatenate([prompts[r // SAMPLES][n][i], np.stack([t[n][i] for t in shadow[r]])]).transpose(1, 0, 2) for n in (0, 1))
                x = np.einsum("gqd,gtd->gqt", host(q[r]).reshape(KV, HEADS // KV, DIM), keys) / DIM ** 0.5
                p = np.exp(x - x.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                want, size = np.einsum("gqt,gtd->gqd", p, values), np.einsum("gqt,gtd->gqd", p, np.abs(values))
                # as tests/test_rollout_gpu.py has it: scores of 64 products of numbers up to the largest, twice; weights in two halves of bfloat16; sums over at most 47 tokens
                scores = np.einsum("gqd,gtd->gqt", np.abs(host(q[r])).reshape(KV, HEADS // KV, DIM), np.abs(keys)).max() / DIM ** 0.5
                rel = 2 * 66 * U * scores + 4 * np.abs(x).max() * U + 2.0 ** -16 + 60 * U
                near(host(got[r]).reshape(want.shape), want, rel * size + HALF_STEP["bf16"] * np.abs(want), f"attention of step {step}, row {r}, layer {i}")
    assert lens.tolist() == [len(s) for s in shadow] == [26] * rows
    tables, lens, refs = pool.fork(tables, lens, ints([-1] * rows), refs)
    assert int(refs.sum()) == sum(-(-n // PAGE) for n in PROMPTS)  # the prompts' own are left
    p_tables, p_lens, refs = pool.fork(p_tables, p_lens, ints([]), refs)  # nobody goes on
    assert not refs.any()
