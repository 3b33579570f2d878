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
