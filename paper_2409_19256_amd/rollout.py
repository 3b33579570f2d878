"""The rollout operators for callers that use PyTorch: a paged cache of keys and values that is appended to and attended
over, and log probabilities of given tokens with their gradient.  torch allocates and hands out pointers and streams; a
native module (_rollout) checks types and shapes and calls the library, which checks sizes and strides; all work runs in its HIP kernels
on torch's current stream of the tensors' GPU, whichever is current; all tensors of a call are on one.  There is no CPU path.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B

try:
    from . import _rollout as _native
except ImportError as e:
    raise ImportError(f"{e}: build it with `python -m paper_2409_19256_amd.build` (there is no fallback path)") from e

_native.set_error(B.HfError)
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
    tensors that require one where torch would take it (call them under torch.no_grad())."""

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
