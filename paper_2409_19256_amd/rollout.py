"""The rollout operators for callers that use PyTorch: a paged cache of keys and values that is appended to and attended
over, and log probabilities of given tokens with their gradient.  torch allocates and hands out pointers and streams;
shapes and types are checked here, sizes and strides in the library, and all work runs in its HIP kernels on
torch's current stream.  There is no CPU path.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple
from typing import Optional

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.HF_BF16, torch.float16: B.HF_F16, torch.float32: B.HF_F32}


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _whole(t: Optional[torch.Tensor], name: str, dtype, shape) -> Optional[int]:
    """Address of a contiguous tensor of that type and shape; None for none."""
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on the GPU is wanted")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, dtype, shape):
    """(address, first stride, second stride) of a tensor of three dimensions whose last one is contiguous."""
    s = t.stride()
    if not (t.is_cuda and t.dtype == dtype and t.shape == shape and (s[2] == 1 or shape[2] == 1)):
        raise ValueError(f"{name}: a {dtype} tensor of shape {tuple(shape)} on the GPU is wanted, its last dimension contiguous")
    return t.data_ptr(), s[0], s[1]


class KvCache:
    """Keys and values, each [page, KV head, token of the page, element] in any order of memory with the last contiguous
    (`KvCache.empty` makes one), for hf_append_kv and hf_attend."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _need(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.is_cuda and k.device == v.device,
              "keys and values: two tensors [pages, KV heads, page tokens, head dim] of one type on one GPU are wanted")
        _need(k.dtype in (torch.bfloat16, torch.float16), "a cache is bfloat16 or float16")
        _need(k.stride() == v.stride() and (k.stride(3) == 1 or k.shape[3] == 1), "keys and values need the same strides, the last dimension contiguous")
        self.k, self.v = k, v
        pages, heads, tokens, dim = k.shape
        self._c = B.hf_kv_cache(k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], heads, dim, tokens, pages, *k.stride()[:3])
        self._ref = C.byref(self._c)

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
        dtype, (n, heads, dim) = self.k.dtype, k.shape
        _need(heads == self._c.n_kv_heads and dim == self._c.head_dim, "keys do not fit the cache")
        kp, k0, k1 = _rows(k, "k", dtype, (n, heads, dim))
        vp, v0, v1 = _rows(v, "v", dtype, (n, heads, dim))
        qp = op = None
        q0 = q1 = o0 = o1 = n_q = 0
        if q is not None:
            n_q = q.shape[1]
            qp, q0, q1 = _rows(q, "q", dtype, (n, n_q, dim))
            if q_out is None:
                q_out = torch.empty(n, n_q, dim, dtype=dtype, device=q.device)
            op, o0, o1 = _rows(q_out, "q_out", dtype, (n, n_q, dim))
        cp = sp = pp = None
        rot = table = 0
        if cos is not None:
            table, pairs = cos.shape
            rot = 2 * pairs
            cp, sp = _whole(cos, "cos", torch.float32, (table, pairs)), _whole(sin, "sin", torch.float32, (table, pairs))
            pp = _whole(positions, "positions", torch.int32, (n,))
        a = B.hf_append(qp, op, kp, vp, cp, sp, pp, _whole(slots, "slots", torch.int64, (n,)), q0, q1, o0, o1, k0, k1, v0, v1,
                        n, n_q, rot, table, B.HF_ROT_INTERLEAVED if interleaved else 0)
        code = B.hf_append_kv(self._ref, C.byref(a), _stream(k))
        if code:
            B.check(code, "hf_append_kv")
        return q_out

    def attend(self, q: torch.Tensor, suffix_lens: torch.Tensor, suffix_pages: torch.Tensor, group_offsets: Optional[torch.Tensor] = None,
               prefix_lens: Optional[torch.Tensor] = None, prefix_pages: Optional[torch.Tensor] = None, max_group: Optional[int] = None,
               max_prefix: Optional[int] = None, max_suffix: Optional[int] = None, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """One query token per sequence, q [sequence, query head, element], over its own pages (lengths int32 [sequence], page
        numbers int32 [sequence, width]) and, where sequences are grouped by prompt, over their prompt's (group_offsets int32
        [prompts + 1], lengths [prompts], page numbers [prompts, width]).  max_*: upper bounds of the samples per
        prompt and of the lengths; by default all sequences and what the tables can name.  Returns (out, lse)."""
        n, heads, dim = q.shape
        dtype, dev = self.k.dtype, q.device
        qp, q0, q1 = _rows(q, "q", dtype, (n, heads, self._c.head_dim))
        if out is None:
            out = torch.empty(n, heads, dim, dtype=dtype, device=dev)
        op, o0, o1 = _rows(out, "out", dtype, (n, heads, dim))
        if lse is None:
            lse = torch.empty(n, heads, dtype=torch.float32, device=dev)
        page = self._c.page_tokens
        groups = width = 0
        gp = lp = pp = None
        if group_offsets is not None:
            groups, width = prefix_pages.shape
            gp = _whole(group_offsets, "group_offsets", torch.int32, (groups + 1,))
            lp = _whole(prefix_lens, "prefix_lens", torch.int32, (groups,))
            pp = _whole(prefix_pages, "prefix_pages", torch.int32, (groups, width))
        own = suffix_pages.shape[1]
        a = B.hf_attention(qp, op, _whole(lse, "lse", torch.float32, (n, heads)), _whole(suffix_lens, "suffix_lens", torch.int32, (n,)),
                           _whole(suffix_pages, "suffix_pages", torch.int32, (n, own)), gp, lp, pp, None, 0, q0, q1, o0, o1, n, heads, groups,
                           n if max_group is None else max_group, width, own,
                           width * page if max_prefix is None else max_prefix, own * page if max_suffix is None else max_suffix,
                           dim ** -0.5 if scale is None else scale)
        ref = C.byref(a)
        if workspace is None:
            need = B.hf_attend_workspace_bytes(self._ref, ref)
            if need == C.c_size_t(-1).value:
                raise B.HfError(B.HF_EINVAL, "hf_attend_workspace_bytes")
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        if workspace is not None:
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        code = B.hf_attend(self._ref, ref, _stream(q))
        if code:
            B.check(code, "hf_attend")
        return out, lse


Logprobs = namedtuple("Logprobs", "logprob entropy lse norm top_ids top_logprobs")


def _logits(logits: torch.Tensor, targets: Optional[torch.Tensor], temperature: float) -> B.hf_logits:
    _need(logits.dim() == 2 and logits.is_cuda and logits.dtype in _TYPES and (logits.stride(1) == 1 or logits.shape[1] == 1),
          "logits: [rows, vocab] of bfloat16, float16 or float32 on the GPU, the last dimension contiguous, is wanted")
    rows, vocab = logits.shape
    tp, size = None, 8
    if targets is not None:
        _need(targets.dtype in (torch.int64, torch.int32), "targets: int64 or int32 is wanted")
        tp, size = _whole(targets, "targets", targets.dtype, (rows,)), targets.element_size()
    _need(temperature > 0, "the temperature must be positive")
    return B.hf_logits(logits.data_ptr(), tp, rows, logits.stride(0), _TYPES[logits.dtype], vocab, size, 1.0 / temperature)


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], temperature: float = 1.0, top: int = 0) -> Logprobs:
    """Log probability of targets[row] (int64 or int32; outside the vocabulary: the row is left out), entropy, log sum of exponentials
    (lse, and in two parts for token_logprobs_back: norm) and the `top` likeliest tokens of every row of logits [rows, vocab] over the
    temperature.  Not differentiable by itself: see logprobs."""
    a = _logits(logits, targets, temperature)
    stats = torch.empty(5 * a.rows, dtype=torch.float32, device=logits.device)
    at, row = stats.data_ptr(), 4 * a.rows
    ids = values = None
    if top:
        ids = torch.empty(a.rows, top, dtype=torch.int32, device=logits.device)
        values = torch.empty(a.rows, top, dtype=torch.float32, device=logits.device)
    o = B.hf_logprobs(at if targets is not None else None, at + row, at + 2 * row, at + 3 * row, ids.data_ptr() if top else None, values.data_ptr() if top else None, top)
    code = B.hf_token_logprobs(C.byref(a), C.byref(o), _stream(logits))
    if code:
        B.check(code, "hf_token_logprobs")
    logprob, entropy, lse, norm = stats.split([a.rows, a.rows, a.rows, 2 * a.rows])
    return Logprobs(logprob if targets is not None else None, entropy, lse, norm.view(a.rows, 2), ids, values)


def token_logprobs_back(logits: torch.Tensor, targets: torch.Tensor, norm: torch.Tensor, entropy: Optional[torch.Tensor],
                        grad_logprob: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) with respect to the logits; out may be the logits."""
    a = _logits(logits, targets, temperature)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _need(out.is_cuda and out.shape == logits.shape and out.dtype == logits.dtype and (out.stride(1) == 1 or out.shape[1] == 1),
          "out: a tensor like the logits is wanted")
    row = (a.rows,)
    _need(norm is not None, "norm is wanted")
    g = B.hf_logprobs_grad(_whole(norm, "norm", torch.float32, (a.rows, 2)), _whole(entropy, "entropy", torch.float32, row),
                           _whole(grad_logprob, "grad_logprob", torch.float32, row), _whole(grad_entropy, "grad_entropy", torch.float32, row),
                           out.data_ptr(), out.stride(0))
    code = B.hf_token_logprobs_back(C.byref(a), C.byref(g), _stream(logits))
    if code:
        B.check(code, "hf_token_logprobs_back")
    return out


class _Logprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, temperature):
        r = token_logprobs(logits, targets, temperature)
        ctx.save_for_backward(logits, targets, r.norm, r.entropy)
        ctx.temperature = temperature
        return r.logprob, r.entropy

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logprob, grad_entropy):
        logits, targets, norm, entropy = ctx.saved_tensors
        # a gradient that was broadcast from a sum has stride 0
        return token_logprobs_back(logits, targets, norm, entropy, grad_logprob.contiguous(), grad_entropy.contiguous(), ctx.temperature), None, None


def logprobs(logits: torch.Tensor, targets: torch.Tensor, temperature: float = 1.0):
    """(log probability of targets, entropy) of every row, differentiable with respect to the logits."""
    return _Logprobs.apply(logits, targets, temperature)
