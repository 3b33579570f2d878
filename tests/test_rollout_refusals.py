"""What the rollout operators refuse, on the host before anything is enqueued; and calls with nothing to do."""
import ctypes as C

import pytest

from paper_2409_19256_amd import binding as B

AT = 1 << 20  # a pointer that is never followed: every call here ends in the checks


def cache(**kw):
    a = dict(k=AT, v=2 * AT, dtype=B.HF_BF16, n_kv_heads=2, head_dim=8, page_tokens=4, n_pages=3, page_stride=64, head_stride=32, token_stride=8)
    a.update(kw)
    return B.hf_kv_cache(**a)


def append(**kw):
    a = dict(q=3 * AT, q_out=4 * AT, k=5 * AT, v=6 * AT, cos=7 * AT, sin=8 * AT, positions=9 * AT, slots=10 * AT, q_stride=32, q_head_stride=8,
             q_out_stride=32, q_out_head_stride=8, k_stride=16, k_head_stride=8, v_stride=16, v_head_stride=8, n_tokens=0, n_q_heads=4, rot_dim=8,
             n_positions=5, flags=0)
    a.update(kw)
    return B.hf_append(**a)


def attention(**kw):
    a = dict(q=3 * AT, out=4 * AT, lse=5 * AT, suffix_lens=6 * AT, suffix_pages=7 * AT, group_offsets=8 * AT, prefix_lens=9 * AT, prefix_pages=10 * AT,
             workspace=None, workspace_bytes=0, q_stride=32, q_head_stride=8, out_stride=32, out_head_stride=8, n_seqs=6, n_q_heads=4, n_groups=2,
             max_group=3, prefix_width=2, suffix_width=1, max_prefix=8, max_suffix=4, scale=0.5)
    a.update(kw)
    return B.hf_attention(**a)


def logits(**kw):
    a = dict(logits=AT, targets=2 * AT, rows=0, row_stride=50, dtype=B.HF_BF16, vocab=50, target_bytes=8, inv_temperature=1.0)
    a.update(kw)
    return B.hf_logits(**a)


def run_append(c, a):
    return B.hf_append_kv(C.byref(c), C.byref(a), None)


def run_attend(c, a):
    return B.hf_attend(C.byref(c), C.byref(a), None)


def run_score(i, **kw):
    return B.hf_token_logprobs(C.byref(i), C.byref(B.hf_logprobs(**kw)), None)


def run_back(i, **kw):
    a = dict(norm=3 * AT, entropy=4 * AT, grad_logprob=5 * AT, grad_entropy=6 * AT, dlogits=16 * AT, dlogits_stride=50)
    a.update(kw)
    return B.hf_token_logprobs_back(C.byref(i), C.byref(B.hf_logprobs_grad(**a)), None)


def test_sizes_of_the_structs():
    assert [C.sizeof(t) for t in (B.hf_kv_cache, B.hf_append, B.hf_attention, B.hf_logits, B.hf_logprobs, B.hf_logprobs_grad)] == [64, 152, 152, 48, 56, 48]


BAD_CACHES = [dict(k=None), dict(v=None), dict(v=AT), dict(k=AT + 1), dict(dtype=B.HF_F32), dict(dtype=7), dict(n_kv_heads=0), dict(head_dim=0),
              dict(head_dim=257), dict(page_tokens=2), dict(page_tokens=24), dict(page_tokens=131072), dict(n_pages=0), dict(n_pages=1 << 31),
              dict(page_stride=-64), dict(page_stride=63), dict(head_stride=31), dict(token_stride=7), dict(token_stride=0),
              dict(page_stride=1 << 62)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_caches(bad):
    c = cache(**bad)
    assert run_append(c, append()) == B.HF_EINVAL and B.hf_last_error()
    assert run_attend(c, attention()) == B.HF_EINVAL
    assert B.hf_attend_workspace_bytes(C.byref(c), C.byref(attention())) == C.c_size_t(-1).value


def test_a_call_with_nothing_to_do():
    assert run_append(cache(), append()) == B.HF_OK
    assert run_append(cache(token_stride=16, head_stride=8), append(k=None, v=None)) == B.HF_OK  # tokens outside heads
    assert run_attend(cache(), attention(n_seqs=0)) == B.HF_OK
    assert run_score(logits(), logprob=3 * AT, top_n=5, top_ids=4 * AT) == B.HF_OK
    assert run_back(logits()) == B.HF_OK


@pytest.mark.parametrize("bad", [
    dict(n_tokens=-1), dict(flags=2), dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=10), dict(q=None), dict(q_out=None), dict(n_q_heads=0),
    dict(k=None), dict(v=None), dict(slots=None), dict(cos=None), dict(sin=None), dict(positions=None), dict(n_positions=0), dict(slots=AT + 4),
    dict(k=5 * AT + 1), dict(cos=AT + 2), dict(q_stride=-1), dict(k_stride=-8), dict(v_head_stride=-8), dict(q_out_stride=16), dict(q_out_head_stride=4),
    dict(q_out=3 * AT + 32), dict(q_out=3 * AT, q_out_stride=64), dict(k_stride=1 << 61)], ids=str)
def test_appends(bad):
    assert run_append(cache(), append(**{**dict(n_tokens=4), **bad})) == B.HF_EINVAL and B.hf_last_error()


def test_null_arguments():
    null = C.POINTER(B.hf_append)()
    assert B.hf_append_kv(C.byref(cache()), null, None) == B.HF_EINVAL
    assert B.hf_append_kv(None, C.byref(append()), None) == B.HF_EINVAL
    assert B.hf_attend(C.byref(cache()), None, None) == B.HF_EINVAL
    assert B.hf_attend(None, C.byref(attention()), None) == B.HF_EINVAL
    assert B.hf_token_logprobs(None, C.byref(B.hf_logprobs()), None) == B.HF_EINVAL
    assert B.hf_token_logprobs(C.byref(logits()), None, None) == B.HF_EINVAL
    assert B.hf_token_logprobs_back(C.byref(logits()), None, None) == B.HF_EINVAL


@pytest.mark.parametrize("bad", [
    dict(n_seqs=-1), dict(n_groups=-1), dict(max_group=-1), dict(prefix_width=-1), dict(suffix_width=-1), dict(max_prefix=-1), dict(max_suffix=-1),
    dict(n_q_heads=3), dict(n_q_heads=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None), dict(suffix_lens=None),
    dict(suffix_pages=None), dict(group_offsets=None), dict(prefix_lens=None), dict(prefix_pages=None), dict(lse=AT + 2), dict(prefix_lens=AT + 1),
    dict(out_stride=31), dict(out_head_stride=0), dict(q_stride=-1), dict(out=3 * AT), dict(out=3 * AT + 64), dict(workspace=None),
    dict(workspace=AT + 8, workspace_bytes=1 << 40), dict(workspace=AT, workspace_bytes=8)], ids=str)
def test_attentions(bad):
    assert run_attend(cache(), attention(**{**dict(workspace=20 * AT, workspace_bytes=1 << 30), **bad})) == B.HF_EINVAL and B.hf_last_error()


def test_too_many_queries():
    assert run_attend(cache(), attention(n_seqs=1 << 29, workspace=20 * AT, workspace_bytes=1 << 62)) == B.HF_ERANGE


def test_workspace_of_attention():
    need = lambda **kw: B.hf_attend_workspace_bytes(C.byref(cache()), C.byref(attention(**kw)))  # noqa: E731
    assert need(n_groups=0) == 0 and need(n_groups=0, max_suffix=0, suffix_width=0) == 0   # one part a row: no merge
    assert need(max_prefix=0) == 0 and need(max_group=0) == 0 and need(n_seqs=0, n_groups=0) == 0
    assert need() >= 6 * 4 * 2 * (8 + 2) * 4                                                # a row's two parts
    # the pointers are not looked at
    assert need(q=None, out=None, suffix_lens=None) == need()
    assert need(n_groups=0, suffix_width=1 << 20, max_suffix=1 << 22) > 0


@pytest.mark.parametrize("bad", [dict(logits=None), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dtype=3), dict(dtype=-1),
                                 dict(inv_temperature=0.0), dict(inv_temperature=-1.0), dict(inv_temperature=float("nan")),
                                 dict(inv_temperature=float("inf")), dict(row_stride=-1), dict(logits=AT + 1), dict(logits=AT + 2, dtype=B.HF_F32),
                                 dict(target_bytes=2), dict(targets=AT + 4), dict(row_stride=1 << 62)], ids=str)
def test_logits(bad):
    i = logits(**{**dict(rows=3), **bad})
    assert run_score(i, logprob=3 * AT) == B.HF_EINVAL and B.hf_last_error()
    assert run_back(i) == B.HF_EINVAL


def test_scores():
    i = logits(rows=3)
    for bad in (dict(top_n=-1), dict(top_n=51), dict(logprob=AT + 2), dict(top_ids=AT + 1, top_n=2), dict(lse=AT + 1), dict(norm=AT + 2)):
        assert run_score(i, **bad) == B.HF_EINVAL, bad
    assert run_score(logits(rows=3, vocab=1000, row_stride=1000), top_n=65) == B.HF_EINVAL
    assert run_score(logits(rows=3, targets=None), logprob=3 * AT) == B.HF_EINVAL
    assert run_score(logits(rows=1 << 23)) == B.HF_ERANGE


def test_gradients():
    i = logits(rows=3)
    for bad in (dict(norm=None), dict(dlogits=None), dict(entropy=None), dict(norm=AT + 2), dict(dlogits=AT + 1), dict(dlogits_stride=49),
                dict(dlogits_stride=-50), dict(dlogits=AT + 100), dict(dlogits=AT, dlogits_stride=51)):
        assert run_back(i, **bad) == B.HF_EINVAL, bad
    assert run_back(logits(rows=3, targets=None)) == B.HF_EINVAL
    assert run_back(logits(rows=1 << 25), dlogits=1 << 45) == B.HF_ERANGE
