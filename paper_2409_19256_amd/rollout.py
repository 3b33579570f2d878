"""The rollout operators for callers that use PyTorch: a paged cache of keys and values that is appended to and attended
over, its pages (forked, grown, compacted), log probabilities of given tokens with their gradient, logits adjusted before a token is chosen, and
distillation from a teacher's top tokens.  torch allocates and hands out pointers and streams; two
native modules (_rollout, _steps) check types and shapes and call the library, which checks sizes and strides; all work runs in its HIP kernels
on torch's current stream of the tensors' GPU, whichever is current; all tensors of a call are on one.  There is no CPU path.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as B

try:
    from . import _rollout as _native, _steps
except ImportError as e:
    raise ImportError(f"{e}: build it with `python -m paper_2409_19256_amd.build` (there is no fallback path)") from e

_native.set_error(B.HfError)
_steps.set_error(B.HfError)
_TYPES = {torch.bfloat16: B.HF_BF16, torch.float16: B.HF_F16}
_stream_of = torch._C._cuda_getCurrentRawStream


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _device_of(t) -> int:
    _need(isinstance(t, torch.Tensor) and t.is_cuda, "tensors on the GPU are wanted: the operators have no CPU path")
    return t.get_device()


class KvCache:
    """Keys and values, each [page, KV head, token of the page, element] in any order of memory with the last contiguous
    (`KvCache.empty` makes one), for hf_append_kv and hf_attend.  Both are for generation and scoring: they take no gradient, and refuse
    tensors that require one where torch would take it (call them under torch.no_grad()), and dual tensors of forward mode."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _need(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.is_cuda and k.device == v.device,
              "keys and values: two tensors [pages, KV heads, page tokens, head dim] of one type on one GPU are wanted")
        _need(k.dtype in (torch.bfloat16, torch.float16), "a cache is bfloat16 or float16")
        _need(k.stride() == v.stride() and (k.stride(3) == 1 or k.shape[3] == 1), "keys and values need the same strides, the last dimension contiguous")
        self.k, self.v = k, v
        pages, heads, tokens, dim = k.shape
        self._c = bytes(B.hf_kv_cache(k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], heads, dim, tokens, pages, *k.stride()[:3]))

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_tokens: int, head_dim: int, dtype=torch.bfloat16, device="cuda:0") -> "KvCache":
        return cls(*(torch.empty(pages, kv_heads, page_tokens, head_dim, dtype=dtype, device=device) for _ in range(2)))

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
               cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, interleaved: bool = False) -> Optional[torch.Tensor]:
        """Writes keys and values [token, KV head, element] to slots[token] = page * page tokens + token of the page (int64;
        negative: left out), the keys turned by cos and sin [position, pairs] at positions[token] (int32); without a table
        they are copied.  q [token, query head, element] is turned the same way into q_out (may be q; made if not given),
        which is returned."""
        return _native.append(self._c, self.k, self.v, _stream_of(_device_of(k)), k, v, slots, positions, cos, sin, q, q_out, interleaved)

    def attend(self, q: torch.Tensor, suffix_lens: torch.Tensor, suffix_pages: torch.Tensor, group_offsets: Optional[torch.Tensor] = None,
               prefix_lens: Optional[torch.Tensor] = None, prefix_pages: Optional[torch.Tensor] = None, max_group: Optional[int] = None,
               max_prefix: Optional[int] = None, max_suffix: Optional[int] = None, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """One query token per sequence, q [sequence, query head, element], over its own pages (lengths int32 [sequence], page
        numbers int32 [sequence, width]) and, where sequences are grouped by prompt, over their prompt's (group_offsets int32
        [prompts + 1], lengths [prompts], page numbers [prompts, width]).  max_*: upper bounds of the samples per
        prompt and of the lengths; by default all sequences and what the tables can name.  Returns (out, lse)."""
        return _native.attend(self._c, self.k, self.v, _stream_of(_device_of(q)), q, suffix_lens, suffix_pages, group_offsets, prefix_lens, prefix_pages,
                              max_group, max_prefix, max_suffix, scale, out, lse, workspace)


class Logprobs:
    """What token_logprobs gives for every row: logprob (None without targets), entropy, lse, norm [rows, 2] (for token_logprobs_back), and
    top_ids, top_logprobs [rows, top] (None without).  The first four are views of one tensor, made when they are asked for."""
    __slots__ = ("_all", "_rows", "_given", "top_ids", "top_logprobs")

    def __init__(self, all_, rows, given, top_ids, top_logprobs):
        self._all, self._rows, self._given, self.top_ids, self.top_logprobs = all_, rows, given, top_ids, top_logprobs

    @property
    def logprob(self):
        return self._all[:self._rows] if self._given else None

    @property
    def entropy(self):
        return self._all[self._rows:2 * self._rows]

    @property
    def lse(self):
        return self._all[2 * self._rows:3 * self._rows]

    @property
    def norm(self):
        return self._all[3 * self._rows:].view(self._rows, 2)

    def __iter__(self):
        return iter((self.logprob, self.entropy, self.lse, self.norm, self.top_ids, self.top_logprobs))


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], temperature: float = 1.0, top: int = 0) -> Logprobs:
    """Log probability of targets[row] (int64 or int32; outside the vocabulary: the row is left out), entropy, log sum of exponentials
    (lse, and in two parts for token_logprobs_back: norm) and the `top` likeliest tokens of every row of logits [rows, vocab] over the
    temperature.  Not differentiable by itself: see logprobs."""
    stats, ids, values, _ = _native.token_logprobs(_stream_of(_device_of(logits)), logits, targets, temperature, top, False)
    return Logprobs(stats, len(logits), targets is not None, ids, values)


def token_logprobs_back(logits: torch.Tensor, targets: torch.Tensor, norm: torch.Tensor, entropy: Optional[torch.Tensor],
                        grad_logprob: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) with respect to the logits; out may be the logits."""
    return _native.token_logprobs_back(_stream_of(_device_of(logits)), logits, targets, norm, entropy, grad_logprob, grad_entropy, temperature, out)


class _Logprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, temperature):
        stats, _, _, logprob = _native.token_logprobs(_stream_of(_device_of(logits)), logits, targets, temperature, 0, True)
        r = Logprobs(stats, len(logits), True, None, None)
        ctx.save_for_backward(logits, targets, r.norm, r.entropy)
        ctx.temperature = temperature
        return logprob, r.entropy.clone()  # the caller's own, both: a loss may mask them in place

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logprob, grad_entropy):
        logits, targets, norm, entropy = ctx.saved_tensors
        # a gradient that was broadcast from a sum has stride 0
        return token_logprobs_back(logits, targets, norm, entropy, grad_logprob.contiguous(), grad_entropy.contiguous(), ctx.temperature), None, None


def logprobs(logits: torch.Tensor, targets: torch.Tensor, temperature: float = 1.0):
    """(log probability of targets, entropy) of every row, differentiable with respect to the logits."""
    _need(targets is not None, "targets: a tensor is wanted (entropy alone: token_logprobs)")
    return _Logprobs.apply(logits, targets, temperature)


def adjust_logits(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None,
                  prompt_lens: Optional[torch.Tensor] = None, *, repetition: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                  presence: Optional[torch.Tensor] = None, bias_ids: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                  allowed: Optional[torch.Tensor] = None, allowed_rows: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Logits [rows, vocab] on their way to a choice of token.  tokens [rows, width] (int32 or int64) are what a row has so far, lens[row] of them (int32), the first
    prompt_lens[row] its prompt.  A token that is there: x / repetition[row] where x > 0, else x * repetition[row]; n times behind the prompt: less
    frequency[row] * n + presence[row] (all float32 [rows]); without tokens these have nothing to apply to.  bias_ids, bias [rows, places] (int32, float32): added to their tokens, of several the last; ids outside the vocabulary
    are left out.  allowed (int32 [masks, ceil(vocab / 32)], bit j % 32 of word j / 32): tokens whose bit is not set become -inf, by the mask
    allowed_rows[row] (int32; outside the masks: none) or by the row's own.  out may be the logits; rows without a mask and with few tokens are then not moved.  For
    generation: it takes no gradient, and refuses tensors that require one where torch would take it, and dual tensors of forward mode."""
    return _steps.adjust(_stream_of(_device_of(logits)), logits, tokens, lens, prompt_lens, repetition, frequency, presence, bias_ids, bias, allowed, allowed_rows, out)


class Distilled:
    """What top_distill gives: loss [rows], and norm [rows, 2] and slopes [rows, places + 1] for top_distill_back.  The last two lie in one allocation, which either
    holds; where all three are 4 KiB or less, the loss lies there too."""
    __slots__ = ("loss", "norm", "slopes")

    def __init__(self, loss, norm, slopes):
        self.loss, self.norm, self.slopes = loss, norm, slopes

    def __iter__(self):
        return iter((self.loss, self.norm, self.slopes))


def top_distill(logits: torch.Tensor, top_ids: torch.Tensor, top_logprobs: torch.Tensor, temperature: float = 1.0, reverse: float = 0.0,
                rest: bool = True) -> Distilled:
    """How far every row of logits [rows, vocab] over the temperature is from a teacher known by log probabilities of some tokens, top_ids and top_logprobs
    [rows, places] (int32, float32; what token_logprobs(top=...) gives): (1 - reverse) KL(teacher || student) + reverse KL(student || teacher) over these
    tokens and, with rest, all others as one more.  Ids outside the vocabulary and log probabilities of -inf name nothing; rows without
    a name have loss 0 and no gradient.  Not differentiable by itself: see distill."""
    return Distilled(*_steps.distill(_stream_of(_device_of(logits)), logits, top_ids, top_logprobs, temperature, reverse, rest))


def top_distill_back(logits: torch.Tensor, top_ids: torch.Tensor, norm: torch.Tensor, slopes: torch.Tensor, grad_loss: torch.Tensor, temperature: float = 1.0,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(grad_loss * loss) with respect to the logits; out may be the logits."""
    return _steps.distill_back(_stream_of(_device_of(logits)), logits, top_ids, norm, slopes, grad_loss, temperature, out)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_ids, top_logprobs, temperature, reverse, rest):
        loss, norm, slopes = _steps.distill(_stream_of(_device_of(logits)), logits, top_ids, top_logprobs, temperature, reverse, rest)
        ctx.save_for_backward(logits, top_ids, norm, slopes)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        logits, top_ids, norm, slopes = ctx.saved_tensors
        # a gradient that was broadcast from a sum has stride 0
        return top_distill_back(logits, top_ids, norm, slopes, grad_loss.contiguous(), ctx.temperature), None, None, None, None, None


def distill(logits: torch.Tensor, top_ids: torch.Tensor, top_logprobs: torch.Tensor, temperature: float = 1.0, reverse: float = 0.0,
            rest: bool = True) -> torch.Tensor:
    """top_distill's loss of every row, differentiable with respect to the logits.  The teacher takes no gradient.  A backward pass is captured into a graph as torch's own
    are: while no eager autograd graph of the same leaves is alive (torch would wait for its stream in the middle of the capture)."""
    _need(not (torch.is_grad_enabled() and isinstance(top_logprobs, torch.Tensor) and top_logprobs.requires_grad),
          "top_logprobs: no gradient is taken to the teacher: detach them")
    return _Distill.apply(logits, top_ids, top_logprobs, temperature, reverse, rest)


class PagePool:
    """The pages of a model's caches (KvCache, one per layer, all alike): sequences are tables of page numbers (int32 [rows, width], as KvCache.attend takes
    them) with lengths in tokens (int32 [rows]), and refs (int32 [pages]) counts the rows that name a page; one with 0 is free.  Full pages may be shared, one that is not full
    belongs to one row.  All calls run on the GPU without a trip to the host; what they return is new unless given (refs_out may be refs).
    What one call returns anew lies in one allocation, with the call's workspace if that is small: each of these tensors holds all of it, torch.save writes all of it, and resize_ may
    grow one over the next.  A tensor that is to outlive the others (compact's n, say) is cloned."""

    def __init__(self, caches: Sequence[KvCache]):
        _need(len(caches) > 0 and all(isinstance(c, KvCache) for c in caches), "at least one KvCache is wanted")
        first = caches[0].k
        _need(all(c.k.shape == first.shape and c.k.stride() == first.stride() and c.k.dtype == first.dtype and c.k.device == first.device for c in caches),
              "the caches of a pool have to be alike")
        self.caches = list(caches)
        self._c, self._tensors = b"".join(c._c for c in caches), tuple(t for c in caches for t in (c.k, c.v))

    def refs(self) -> torch.Tensor:
        """The reference counts of a pool that nothing is in."""
        k = self.caches[0].k
        return torch.zeros(k.shape[0], dtype=torch.int32, device=k.device)

    def fork(self, tables: torch.Tensor, lens: torch.Tensor, parents: torch.Tensor, refs: torch.Tensor, tables_out: Optional[torch.Tensor] = None,
             lens_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """Row r goes on where row parents[r] (int32; outside the rows: empty) stands; rows that nobody continues give their pages back.  Full pages are
        shared; of a page that is not full the first row that continues it has it and the others take copies.  A row for which no page is left comes out empty.  Returns (tables, lens, refs)."""
        return _steps.fork(self._c, self._tensors, _stream_of(_device_of(tables)), tables, lens, parents, refs, tables_out, lens_out, refs_out, workspace)

    def grow(self, tables: torch.Tensor, lens: torch.Tensor, counts: torch.Tensor, refs: torch.Tensor, most: int = 1, tables_out: Optional[torch.Tensor] = None,
             lens_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None):
        """Room for counts[row] more tokens (int32, cut to 0 .. most) in every row.  slots [rows, most] (int64) are their places for KvCache.append, -1 where
        there is none.  A row that does not fit the table or for which no pages are left stays as it is.  tables_out may be tables, lens_out lens.  Returns
        (tables, lens, slots, refs)."""
        return _steps.grow(self._c, self._tensors, _stream_of(_device_of(tables)), tables, lens, counts, refs, most, tables_out, lens_out, slots, refs_out, workspace)

    def compact(self, refs: torch.Tensor, tables: Sequence[torch.Tensor] = (), tables_out: Optional[Sequence[Optional[torch.Tensor]]] = None,
                refs_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """Moves pages so that the n in use are the first n.  Up to four tables (any shape) have their entries replaced.  Returns (tables, refs, places, n): where
        every page is now (int32, -1: free), and n (int32, no dimension).  tables_out may be tables."""
        _need(not isinstance(tables, torch.Tensor) and not isinstance(tables_out, torch.Tensor), "tables: a list of tensors is wanted")
        tables = tuple(tables)
        return _steps.compact(self._c, self._tensors, _stream_of(_device_of(refs)), refs, tables, tuple(tables_out) if tables_out is not None else (None,) * len(tables),
                              refs_out, workspace)
