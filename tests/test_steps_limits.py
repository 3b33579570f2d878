"""Where the operators around a rollout's steps begin to refuse sizes, on both sides of every limit.  What is within one has to come to a later check, so that
no call here runs: the operands overlap, or a pointer of the next check is missing."""
import ctypes as C

import pytest

from paper_2409_19256_amd import binding as B
from tests.test_rollout_refusals import AT, cache
from tests.test_steps_refusals import FAR, adjustment, grow, pool, run_adjust, run_grow

LANES = 1 << 32  # a grid holds fewer


@pytest.mark.parametrize("vocab,pieces", [(32, 1), (8192, 1), (8193, 2), (128256, 16)])
def test_adjustments_up_to_a_grid(vocab, pieces):
    """Workgroups of 512 lanes, one to 8192 logits of a row."""
    most = (LANES - 1) // 512 // pieces
    bare = dict(vocab=vocab, row_stride=vocab, out_stride=vocab, tokens=None, lens=None, allowed=None, n_bias=0, repetition=None, frequency=None, presence=None, prompt_lens=None)
    for rows, code in ((most, B.HF_EINVAL), (most + 1, B.HF_ERANGE), (2 * most, B.HF_ERANGE), (2 * most + 2, B.HF_ERANGE)):
        a = adjustment(**bare, rows=rows, logits=FAR, out=FAR + 2)
        assert run_adjust(a) == code, rows
        assert (b"overlaps" if code == B.HF_EINVAL else b"too many rows") in B.hf_last_error(), rows


@pytest.mark.parametrize("what", ["width", "n_bias"])
def test_adjustments_of_long_lists(what):
    """Lanes go through lists in steps of 512, in numbers of 32 bits."""
    most = (1 << 31) - 512
    for n in (most - 1, most, most + 1, (1 << 31) - 1):
        a = adjustment(**{what: n}, rows=1, tokens=FAR * 4, bias_ids=FAR * 8, bias=FAR * 16, out=AT + 2)
        assert run_adjust(a) == (B.HF_ERANGE if n > most else B.HF_EINVAL), n
        assert (b"2^31 - 512" if n > most else b"overlaps") in B.hf_last_error(), n


@pytest.mark.parametrize("at", [AT, AT + 368, 2 * AT + 128, 30 * AT + 208, 31 * AT - 4, 31 * AT + 368])
@pytest.mark.parametrize("what", ["tables_out", "lens_out", "slots", "refs_out", "workspace"])
def test_growths_over_a_cache(what, at):
    """Caches of 384 bytes at AT, 2 AT, 30 AT and 31 AT: grow does not write to them, and its outputs may not lie there."""
    at -= at % {"workspace": 16, "slots": 8}.get(what, 4)
    p = pool(cache(), cache(k=30 * AT, v=31 * AT))
    # (the workspace is missing or too small besides, so that nothing can run)
    short = dict(workspace_bytes=8) if what == "workspace" else dict(workspace=None)
    assert run_grow(grow(**{**short, what: at}), p) == B.HF_EINVAL
    assert b"cache overlaps an output" in B.hf_last_error()


def test_growths_between_the_pages_of_a_cache():
    """Inputs may lie in a cache, outputs beside it and in the room between its pages."""
    wide = dict(page_stride=192)  # 128 bytes of a page, 256 to the next one
    p = pool(cache(**wide), cache(k=30 * AT, v=31 * AT, **wide))
    for a in (dict(tables_out=AT + 128), dict(slots=AT + 384 + 128 + 208), dict(lens_out=31 * AT - 8), dict(refs_out=31 * AT + 2 * 384 + 128), dict(tables=AT, lens=2 * AT, counts=30 * AT, refs=31 * AT)):
        assert run_grow(grow(workspace=None, **a), p) == B.HF_EINVAL and b"workspace" in B.hf_last_error(), a
