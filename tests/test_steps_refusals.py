"""What the operators around a rollout's steps refuse, on the host before anything is enqueued; and calls with nothing to do."""
import ctypes as C

import pytest

from paper_2409_19256_amd import binding as B
from tests.test_rollout_refusals import AT, cache, logits  # AT: a pointer that is never followed, every call here ends in the checks

FAR = 1 << 44


def adjustment(**kw):
    a = dict(logits=AT, out=2 * AT, tokens=3 * AT, lens=4 * AT, prompt_lens=5 * AT, repetition=6 * AT, frequency=7 * AT, presence=8 * AT, bias_ids=9 * AT, bias=10 * AT,
             allowed=11 * AT, allowed_rows=12 * AT, rows=3, row_stride=50, out_stride=50, tokens_stride=20, allowed_stride=2, dtype=B.HF_BF16, vocab=50, token_bytes=8,
             width=20, n_bias=4, n_allowed=2)
    return B.hf_adjustment(**{**a, **kw})


def run_adjust(a):
    return B.hf_adjust_logits(C.byref(a), None)


def run_distill(i, **kw):
    a = dict(ids=3 * AT, logprobs=4 * AT, loss=5 * AT, norm=6 * AT, slopes=7 * AT, n=5, reverse=0.5, flags=B.HF_DISTILL_REST)
    return B.hf_top_distill(C.byref(i), C.byref(B.hf_distillation(**{**a, **kw})), None)


def run_distill_back(i, **kw):
    a = dict(ids=3 * AT, norm=6 * AT, slopes=7 * AT, grad_loss=8 * AT, dlogits=16 * AT, dlogits_stride=50, n=5)
    return B.hf_top_distill_back(C.byref(i), C.byref(B.hf_distillation_grad(**{**a, **kw})), None)


def pool(*caches):
    """The pool and what it points to."""
    many = (B.hf_kv_cache * max(1, len(caches)))(*caches)
    return B.hf_page_pool(C.cast(many, C.POINTER(B.hf_kv_cache)), len(caches)), many


def two():
    return pool(cache(), cache(k=30 * AT, v=31 * AT))


def fork(**kw):
    a = dict(tables=3 * AT, lens=4 * AT, parents=5 * AT, refs=6 * AT, tables_out=7 * AT, lens_out=8 * AT, refs_out=9 * AT, workspace=20 * AT, workspace_bytes=1 << 19, rows=2,
             rows_out=3, width=4)
    return B.hf_page_fork(**{**a, **kw})


def grow(**kw):
    a = dict(tables=3 * AT, lens=4 * AT, counts=5 * AT, refs=6 * AT, tables_out=7 * AT, lens_out=8 * AT, slots=10 * AT, refs_out=9 * AT, workspace=20 * AT, workspace_bytes=1 << 19,
             rows=2, width=4, most=3)
    return B.hf_page_grow(**{**a, **kw})


def compact(entries=(3 * AT,), entries_out=(4 * AT,), n_entries=(10,), **kw):
    a = dict(refs=6 * AT, refs_out=9 * AT, places=10 * AT, live=11 * AT, workspace=20 * AT, workspace_bytes=1 << 19)
    return B.hf_page_compact(entries=(C.c_void_p * 4)(*entries), entries_out=(C.c_void_p * 4)(*entries_out), n_entries=(C.c_int64 * 4)(*n_entries), **{**a, **kw})


def run_fork(a, p=None):
    p = p or two()
    return B.hf_fork_pages(C.byref(p[0]), C.byref(a), None)


def run_grow(a, p=None):
    p = p or two()
    return B.hf_grow_pages(C.byref(p[0]), C.byref(a), None)


def run_compact(a, p=None):
    p = p or two()
    return B.hf_compact_pages(C.byref(p[0]), C.byref(a), None)


def test_sizes_of_the_structs():
    assert [C.sizeof(t) for t in (B.hf_adjustment, B.hf_distillation, B.hf_distillation_grad, B.hf_page_pool, B.hf_page_fork, B.hf_page_grow, B.hf_page_compact)] == [
        160, 56, 56, 16, 88, 96, 144]


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(out=None), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dtype=3), dict(dtype=-1), dict(width=-1), dict(n_bias=-1), dict(n_allowed=-1),
    dict(tokens=None), dict(lens=None), dict(token_bytes=2), dict(bias=None), dict(bias_ids=None), dict(logits=AT + 1), dict(out=2 * AT + 1), dict(tokens=3 * AT + 4),
    dict(lens=4 * AT + 2), dict(repetition=AT + 1), dict(allowed=11 * AT + 2), dict(allowed_rows=12 * AT + 1), dict(logits=AT + 2, dtype=B.HF_F32), dict(row_stride=-1),
    dict(row_stride=1 << 62), dict(out_stride=49), dict(out_stride=-50), dict(tokens_stride=-1), dict(tokens_stride=1 << 62), dict(allowed_stride=-2)], ids=str)
def test_adjustments(bad):
    assert run_adjust(adjustment(**bad)) == B.HF_EINVAL and B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(out=AT + 50), dict(out=AT, out_stride=60), dict(out=3 * AT), dict(out=4 * AT - 8), dict(out=5 * AT), dict(out=6 * AT), dict(out=7 * AT), dict(out=8 * AT),
                                 dict(out=9 * AT), dict(out=10 * AT), dict(out=11 * AT), dict(out=12 * AT)], ids=str)
def test_adjustments_over_their_own_inputs(bad):
    assert run_adjust(adjustment(**bad)) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


def test_adjustments_that_fit_no_grid():
    assert run_adjust(adjustment(rows=1 << 40, row_stride=50, out_stride=50, tokens=None, lens=None, allowed=None, out=FAR * 16)) == B.HF_ERANGE
    assert run_adjust(adjustment(rows=1 << 20, vocab=1 << 20, row_stride=1 << 20, out_stride=1 << 20, out=FAR, tokens=None, lens=None, allowed=None)) == B.HF_ERANGE


@pytest.mark.parametrize("bad", [dict(n=0), dict(n=257), dict(n=-1), dict(reverse=-0.1), dict(reverse=1.1), dict(reverse=float("nan")), dict(flags=2), dict(norm=None), dict(slopes=None),
                                 dict(ids=None), dict(logprobs=None), dict(ids=AT + 2), dict(loss=AT + 1), dict(slopes=AT + 2)], ids=str)
def test_distillations(bad):
    assert run_distill(logits(rows=3, targets=None), **bad) == B.HF_EINVAL and B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(loss=AT), dict(norm=3 * AT), dict(slopes=4 * AT + 56), dict(loss=6 * AT), dict(norm=7 * AT + 68), dict(slopes=AT + 296)], ids=str)
def test_distillations_over_their_own_inputs(bad):
    assert run_distill(logits(rows=3, targets=None), **bad) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(n=0), dict(n=300), dict(ids=None), dict(norm=None), dict(slopes=None), dict(grad_loss=None), dict(dlogits=None), dict(dlogits=16 * AT + 1),
                                 dict(dlogits_stride=49), dict(dlogits_stride=-1), dict(grad_loss=AT + 1), dict(dlogits=3 * AT), dict(dlogits=6 * AT), dict(dlogits=7 * AT), dict(dlogits=8 * AT),
                                 dict(dlogits=AT + 50), dict(dlogits=AT, dlogits_stride=51)], ids=str)
def test_gradients(bad):
    assert run_distill_back(logits(rows=3, targets=None), **bad) == B.HF_EINVAL and B.hf_last_error()


def test_distillation_has_no_targets():
    assert run_distill(logits(rows=3)) == B.HF_EINVAL and run_distill_back(logits(rows=3)) == B.HF_EINVAL
    assert run_distill(logits(rows=3, targets=None, vocab=0)) == B.HF_EINVAL and run_distill_back(logits(rows=3, targets=None, inv_temperature=0.0)) == B.HF_EINVAL
    many = logits(rows=1 << 40, targets=None)
    assert run_distill(many, ids=FAR * 64, logprobs=FAR * 128, loss=None, norm=None, slopes=None) == B.HF_ERANGE


@pytest.mark.parametrize("bad", [dict(k=None), dict(dtype=B.HF_F32), dict(page_tokens=24), dict(head_stride=31), dict(n_pages=0)], ids=str)
def test_pools(bad):
    for p in (pool(cache(**bad)), pool(cache(), cache(**{**dict(k=30 * AT, v=31 * AT), **bad}))):
        assert run_fork(fork(), p) == B.HF_EINVAL and run_grow(grow(), p) == B.HF_EINVAL and run_compact(compact(), p) == B.HF_EINVAL
        assert B.hf_fork_pages_workspace_bytes(C.byref(p[0]), C.byref(fork())) == C.c_size_t(-1).value


def test_pools_that_are_none():
    none = pool()
    many = pool(*(cache(k=(100 + i) * AT, v=(400 + i) * AT) for i in range(129)))
    for p in (none, many):
        assert run_fork(fork(), p) == B.HF_EINVAL and run_grow(grow(), p) == B.HF_EINVAL and run_compact(compact(), p) == B.HF_EINVAL
    assert B.hf_fork_pages(None, C.byref(fork()), None) == B.HF_EINVAL and B.hf_grow_pages(C.byref(two()[0]), None, None) == B.HF_EINVAL
    assert B.hf_fork_pages(C.byref(B.hf_page_pool()), C.byref(fork()), None) == B.HF_EINVAL
    assert B.hf_compact_pages(C.byref(two()[0]), None, None) == B.HF_EINVAL and B.hf_adjust_logits(None, None) == B.HF_EINVAL
    assert B.hf_top_distill(None, None, None) == B.HF_EINVAL and B.hf_top_distill_back(C.byref(logits(targets=None)), None, None) == B.HF_EINVAL


@pytest.mark.parametrize("other", [dict(page_stride=72), dict(n_pages=4), dict(head_dim=7), dict(n_kv_heads=1), dict(dtype=B.HF_F16), dict(page_tokens=8, page_stride=128, head_stride=64)], ids=str)
def test_caches_that_differ(other):
    assert run_fork(fork(), pool(cache(), cache(**{**dict(k=30 * AT, v=31 * AT), **other}))) == B.HF_EINVAL and b"alike" in B.hf_last_error()


@pytest.mark.parametrize("second", [dict(k=AT, v=31 * AT), dict(k=30 * AT, v=2 * AT + 128), dict(k=AT + 64, v=31 * AT), dict(k=30 * AT, v=30 * AT + 16)], ids=str)
def test_caches_that_overlap(second):
    p = pool(cache(), cache(**second))
    assert run_fork(fork(), p) == B.HF_EINVAL and b"overlap" in B.hf_last_error()
    assert run_compact(compact(), p) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


def between(n, **kw):
    """Caches whose pages lie between one another's: page p of all of them in one piece."""
    return [cache(k=FAR + 256 * i, v=FAR + 256 * i + 128, page_stride=128 * n, n_pages=50, **kw) for i in range(n)]


def test_caches_between_one_anothers_pages():
    """Those that only look like it pass: the last check finds the workspace missing, so that nothing runs."""
    ok = lambda caches: run_fork(fork(workspace=None), pool(*caches)) == B.HF_EINVAL and b"workspace" in B.hf_last_error()  # noqa: E731
    assert ok(between(5))
    caches = between(100)
    for moved, meets in ((0, False), (16, True), (-16, True), (128 * 100 * 2 * 49 + 8, True), (128 * 100 * 2 * 50, False)):
        caches[37].k = FAR + 256 * 37 + moved
        assert run_fork(fork(workspace=None), pool(*caches[:37], *caches[38:], caches[37])) == B.HF_EINVAL
        assert (b"overlap" if meets else b"workspace") in B.hf_last_error(), moved


@pytest.mark.parametrize("inside", ["heads", "tokens"])
def test_caches_between_one_anothers_heads(inside):
    """Four buffers whose heads, or tokens, take turns."""
    stride = dict(heads=dict(head_stride=128, token_stride=8, page_stride=256), tokens=dict(head_stride=128, token_stride=32, page_stride=256))[inside]
    step = 64 if inside == "heads" else 16  # bytes from one buffer's first to the next one's
    at = [FAR + step * i for i in range(4)]
    for moved, meets in ((0, False), (2, True), (-2, True)):
        p = pool(cache(k=at[0], v=at[1], n_pages=50, **stride), cache(k=at[2] + moved, v=at[3], n_pages=50, **stride))
        assert run_fork(fork(workspace=None), p) == B.HF_EINVAL and (b"overlap" if meets else b"workspace") in B.hf_last_error(), moved


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows_out=-1), dict(width=-1), dict(tables=None), dict(lens=None), dict(parents=None), dict(refs=None), dict(tables_out=None), dict(lens_out=None), dict(refs_out=None),
    dict(workspace=None), dict(workspace=20 * AT + 8), dict(workspace_bytes=8), dict(tables=AT + 2), dict(refs_out=9 * AT + 1)], ids=str)
def test_forks(bad):
    assert run_fork(fork(**bad)) == B.HF_EINVAL and B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(tables_out=3 * AT), dict(lens_out=4 * AT), dict(lens_out=5 * AT + 8), dict(refs_out=6 * AT + 4), dict(refs_out=7 * AT + 44), dict(tables_out=6 * AT),
                                 dict(refs=7 * AT, refs_out=7 * AT), dict(workspace=7 * AT), dict(workspace=6 * AT), dict(tables_out=AT), dict(tables=2 * AT + 16), dict(refs_out=30 * AT),
                                 dict(workspace=31 * AT)], ids=str)
def test_forks_over_their_own_inputs(bad):
    assert run_fork(fork(**bad)) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(width=-1), dict(most=-1), dict(tables=None), dict(lens=None), dict(counts=None), dict(refs=None), dict(tables_out=None), dict(lens_out=None), dict(refs_out=None),
    dict(slots=None), dict(slots=10 * AT + 4), dict(workspace=None), dict(workspace_bytes=8), dict(counts=AT + 1)], ids=str)
def test_growths(bad):
    assert run_grow(grow(**bad)) == B.HF_EINVAL and B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(tables_out=3 * AT + 4), dict(tables_out=4 * AT), dict(lens_out=5 * AT), dict(slots=7 * AT + 8), dict(slots=6 * AT), dict(refs_out=6 * AT + 4),
                                 dict(lens_out=3 * AT, tables_out=3 * AT), dict(workspace=10 * AT), dict(refs=10 * AT, refs_out=10 * AT)], ids=str)
def test_growths_over_their_own_inputs(bad):
    assert run_grow(grow(**bad)) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(refs=None), dict(refs_out=None), dict(places=None), dict(live=None), dict(workspace=None), dict(workspace_bytes=8), dict(entries=()), dict(entries_out=()),
                                 dict(n_entries=(-1,)), dict(n_entries=(1 << 41,)), dict(entries=(3 * AT + 2,)), dict(places=10 * AT + 2)], ids=str)
def test_compactions(bad):
    assert run_compact(compact(**bad)) == B.HF_EINVAL and B.hf_last_error()


@pytest.mark.parametrize("bad", [dict(places=6 * AT), dict(live=10 * AT + 8), dict(refs_out=6 * AT + 4), dict(entries_out=(3 * AT + 4,)), dict(entries_out=(6 * AT,)), dict(places=3 * AT),
                                 dict(entries=(3 * AT, 5 * AT), entries_out=(5 * AT, 4 * AT), n_entries=(5, 5)), dict(entries=(3 * AT, 3 * AT), entries_out=(3 * AT, 3 * AT), n_entries=(5, 5)),
                                 dict(entries_out=(AT,)), dict(workspace=4 * AT), dict(refs=2 * AT)], ids=str)
def test_compactions_over_their_own_inputs(bad):
    assert run_compact(compact(**bad)) == B.HF_EINVAL and b"overlap" in B.hf_last_error()


def test_ranges():
    assert run_fork(fork(rows=1 << 30, rows_out=1 << 30)) == B.HF_ERANGE and run_grow(grow(rows=(1 << 30) + 5)) == B.HF_ERANGE
    big = dict(n_kv_heads=1 << 10, head_dim=256, page_tokens=65536, token_stride=256, head_stride=256 * 65536, page_stride=256 * 65536 << 10, n_pages=1)
    p = pool(cache(k=FAR, v=4 * FAR, **big))
    assert run_fork(fork(), p) == B.HF_ERANGE and run_compact(compact(), p) == B.HF_ERANGE


def test_workspaces():
    p = two()
    need = lambda f, a: f(C.byref(p[0]), C.byref(a))  # noqa: E731
    # the pointers are not looked at
    assert 0 < need(B.hf_fork_pages_workspace_bytes, fork(tables=None, workspace=None)) < 1 << 12
    assert 0 < need(B.hf_grow_pages_workspace_bytes, grow(tables=None)) < 1 << 12 and 0 < need(B.hf_compact_pages_workspace_bytes, compact(refs=None)) < 1 << 12


def test_nothing_to_do():
    assert run_adjust(adjustment(rows=0)) == B.HF_OK and run_adjust(adjustment(rows=0, logits=None, out=None)) == B.HF_OK
    assert run_distill(logits(targets=None)) == B.HF_OK and run_distill_back(logits(targets=None)) == B.HF_OK
