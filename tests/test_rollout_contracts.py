"""What the header promises of calls that do not fit a grid and of tensors that overlap: refused on the host, before anything is enqueued."""
import ctypes as C

import pytest

from paper_2409_19256_amd import binding as B
from tests.test_rollout_refusals import AT, append, attention, cache, logits, run_append, run_attend, run_back, run_score  # noqa: F401

FAR = 1 << 50


def wide_cache(**kw):
    """Heads of 128 in pages of 64, eight KV heads."""
    a = dict(k=FAR, v=2 * FAR, n_kv_heads=8, head_dim=128, page_tokens=64, n_pages=1 << 10, page_stride=65536, head_stride=8192, token_stride=128)
    return cache(**{**a, **kw})


def wide(**kw):
    a = dict(q=3 * FAR, out=4 * FAR, lse=5 * FAR, n_q_heads=64, q_stride=8192, q_head_stride=128, out_stride=8192, out_head_stride=128,
             workspace=6 * FAR, workspace_bytes=1 << 62)
    return attention(**{**a, **kw})


# n_seqs, n_groups, max_group, prefix pages, suffix pages
GRIDS = [
    (1 << 18, 1 << 20, 4, 64, 0),  # prompts with many rows: 2^23 workgroups of 512 lanes
    (1 << 20, 1, 1, 1 << 14, 0),   # the merge alone: a workgroup to a row, because a prompt may have many parts
    (1 << 22, 0, 0, 0, 1024),      # responses
]


@pytest.mark.parametrize("case", GRIDS, ids=str)
def test_grids(case):
    n, groups, most, prefix, suffix = case
    a = wide(n_seqs=n, n_groups=groups, max_group=most, prefix_width=prefix, suffix_width=suffix, max_prefix=prefix * 64, max_suffix=suffix * 64)
    assert run_attend(wide_cache(), a) == B.HF_ERANGE and b"launch" in B.hf_last_error()


@pytest.mark.gpu
def test_more_short_responses_than_workgroups_fit():
    """Four of them share a workgroup: 2^24 fit where a workgroup to each would not."""
    import torch
    from paper_2409_19256_amd.rollout import KvCache
    n, heads = (1 << 21) + 3, 8
    print("[2^24 short responses]", flush=True)
    gen = torch.Generator("cuda").manual_seed(1)
    c = KvCache(*(torch.randn(64, heads, 4, 8, generator=gen, device="cuda").bfloat16() for _ in range(2)))
    q = torch.randn(n, heads, 8, generator=gen, device="cuda").bfloat16()
    page = torch.arange(n, device="cuda") * 7 % 64
    out, lse = c.attend(q, torch.ones(n, dtype=torch.int32, device="cuda"), page.int()[:, None])
    torch.cuda.synchronize()
    assert torch.equal(out, c.v[page, :, 0])  # one token each: its value
    want = (q.float() * c.k[page, :, 0].float()).sum(2) * 8 ** -0.5
    assert (lse - want).abs().max() < 1e-4


@pytest.mark.parametrize("bad", [
    dict(q_out=5 * AT), dict(q_out=5 * AT + 16), dict(q_out=6 * AT - 128), dict(q_out=7 * AT), dict(q_out=8 * AT + 4), dict(q_out=9 * AT - 8), dict(q_out=10 * AT),
    dict(q_out=AT), dict(q_out=2 * AT + 64), dict(k=AT), dict(v=AT + 64), dict(k=2 * AT), dict(q=AT, q_out=AT), dict(q=2 * AT + 8), dict(slots=AT), dict(cos=2 * AT),
    dict(q=3 * AT, q_out=3 * AT, k=3 * AT + 32)], ids=str)
def test_appends_over_their_own_inputs(bad):
    assert run_append(cache(), append(**{**dict(n_tokens=4), **bad})) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(v=AT + 64), dict(v=AT + 8), dict(v=AT + 128 * 3 - 2), dict(v=AT - 2 * 64 * 2), dict(token_stride=16, v=AT + 8, page_stride=128, head_stride=64),
                                 dict(token_stride=16, v=AT + 16 + 64 * 4 + 8, page_stride=128, head_stride=64)], ids=str)
def test_keys_over_values(bad):
    assert run_append(cache(**bad), append(n_tokens=4)) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [
    dict(out=AT), dict(out=2 * AT + 32), dict(out=6 * AT - 16), dict(out=7 * AT), dict(out=8 * AT), dict(out=9 * AT), dict(out=10 * AT), dict(lse=3 * AT), dict(lse=4 * AT),
    dict(lse=AT), dict(lse=6 * AT + 20), dict(workspace=3 * AT), dict(workspace=4 * AT), dict(workspace=AT), dict(workspace=5 * AT + 16), dict(workspace=10 * AT)], ids=str)
def test_attentions_over_their_own_inputs(bad):
    big = dict(prefix_width=700, max_prefix=2800)  # enough for parts, which take a workspace
    assert run_attend(cache(), attention(**{**dict(workspace=20 * AT, workspace_bytes=1 << 30), **big, **bad})) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(logprob=AT), dict(entropy=AT + 296), dict(lse=2 * AT + 8), dict(norm=2 * AT), dict(top_ids=AT + 4, top_n=5), dict(top_logprobs=2 * AT, top_n=5),
                                 dict(logprob=3 * AT, entropy=3 * AT), dict(lse=3 * AT, norm=3 * AT + 8), dict(top_ids=3 * AT, top_logprobs=3 * AT + 56, top_n=5)], ids=str)
def test_scores_over_their_own_inputs(bad):
    assert run_score(logits(rows=3), **bad) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(dlogits=2 * AT), dict(dlogits=3 * AT - 200), dict(dlogits=3 * AT + 20), dict(dlogits=4 * AT), dict(dlogits=5 * AT), dict(dlogits=6 * AT),
                                 dict(dlogits=AT + 50, dlogits_stride=50), dict(dlogits=AT + 150, dlogits_stride=75)], ids=str)
def test_gradients_over_their_own_inputs(bad):
    assert run_back(logits(rows=3), **bad) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


# ---- and what only looks like it: tensors that lie between one another's rows ------------------------------------------------

@pytest.mark.gpu
def test_slices_of_one_tensor():
    import torch
    from paper_2409_19256_amd import rollout
    print("[slices of one tensor]", flush=True)
    gen = torch.Generator("cuda").manual_seed(2)
    n, hq, hk, d, page = 37, 8, 2, 64, 16
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    cos, sin = (torch.randn(50, d // 2, generator=gen, device="cuda") for _ in range(2))
    positions = torch.randint(0, 50, (n,), generator=gen, device="cuda", dtype=torch.int32)
    slots = torch.randperm(5 * page, generator=gen, device="cuda")[:n]
    x = rand(n, 2 * hq + 2 * hk, d)
    q, k, v, room = x.split([hq, hk, hk, hq], 1)
    plain = rollout.KvCache.empty(5, hk, page, d)
    want = plain.append(k.contiguous(), v.contiguous(), slots, positions, cos, sin, q=q.contiguous())
    # keys and values side by side: by page, by head, by token
    for shape, at in (((5, 2, hk, page, d), 1), ((5, hk, 2, page, d), 2), ((5, hk, page, 2, d), 3)):
        pool = torch.zeros(shape, device="cuda", dtype=torch.bfloat16)
        c = rollout.KvCache(pool.select(at, 0), pool.select(at, 1))
        c.append(k, v, slots, positions, cos, sin, q=q, q_out=room)
        assert torch.equal(room, want)
        live = slots // page, slice(None), slots % page
        assert torch.equal(c.k[live], plain.k[live]) and torch.equal(c.v[live], v)
    # queries turned in place, inside the projection
    turned = x.clone()
    tq, tk, tv, _ = turned.split([hq, hk, hk, hq], 1)
    c.append(tk, tv, slots, positions, cos, sin, q=tq, q_out=tq)
    assert torch.equal(tq, want) and torch.equal(tk, k) and torch.equal(tv, v)
    # the output of attention beside its queries
    lens, pages = torch.full((n,), 3, dtype=torch.int32, device="cuda"), torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    c.k.normal_(generator=gen), c.v.normal_(generator=gen)
    alone, _ = c.attend(want, lens, pages)
    beside, _ = c.attend(tq, lens, pages, out=turned[:, hq + 2 * hk:])
    assert torch.equal(alone, beside) and torch.equal(tq, want)
    # the gradient beside the logits
    both = rand(5, 2, 203)
    logits, room, targets = both[:, 0], both[:, 1], torch.arange(5, device="cuda")
    r = rollout.token_logprobs(logits, targets)
    one = torch.ones(5, device="cuda")
    alone = rollout.token_logprobs_back(logits.contiguous(), targets, r.norm, None, one)
    rollout.token_logprobs_back(logits, targets, r.norm, None, one, out=room)
    assert torch.equal(room, alone)
