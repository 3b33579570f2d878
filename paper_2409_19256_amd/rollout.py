"""The rollout operators for callers that use PyTorch: a paged cache of keys and values that is appended to and attended
over, and log probabilities of given tokens with their gradient.  torch allocates and hands out pointers and streams;
shapes and types are checked here, sizes and strides in the library, and all work runs in its HIP kernels on
torch's current stream.  There is no CPU path.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.HF_BF16, torch.float16: B.HF_F16, torch.float32: B.HF_F32}

# A step of generation makes these calls for every layer, and the smallest of them wait for the host: the argument structs are packed (a third
# of the time that it takes to fill a ctypes structure) and handed over as bytes, and the stream is asked for by its number.
_APPEND, _ATTENTION = struct.Struct("8P8q4iIi"), struct.Struct("9PN4q8ifi")
_LOGITS, _LOGPROBS, _GRAD = struct.Struct("2P2q3if"), struct.Struct("6Pii"), struct.Struct("5Pq")
assert [s.size for s in (_APPEND, _ATTENTION, _LOGITS, _LOGPROBS, _GRAD)] == [
    C.sizeof(t) for t in (B.hf_append, B.hf_attention, B.hf_logits, B.hf_logprobs, B.hf_logprobs_grad)]
_stream_of = torch._C._cuda_getCurrentRawStream


def _packed(name, *args, result=C.c_int):
    f = B._lib[name]  # a function of its own: the binding's keeps its types
    f.argtypes, f.restype = args, result
    return f


_hf_append_kv = _packed("hf_append_kv", C.c_char_p, C.c_char_p, C.c_void_p)
_hf_attend = _packed("hf_attend", C.c_char_p, C.c_char_p, C.c_void_p)
_hf_attend_workspace_bytes = _packed("hf_attend_workspace_bytes", C.c_char_p, C.c_char_p, result=C.c_size_t)
_hf_token_logprobs = _packed("hf_token_logprobs", C.c_char_p, C.c_char_p, C.c_void_p)
_hf_token_logprobs_back = _packed("hf_token_logprobs_back", C.c_char_p, C.c_char_p, C.c_void_p)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _whole(t: Optional[torch.Tensor], name: str, dtype, shape) -> int:
    """Address of a contiguous tensor of that type and shape; 0 for none."""
    if t is None:
        return 0
    if not (t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on the GPU is wanted")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, dtype, shape):
    """(address, first stride, second stride) of a tensor of three dimensions whose last one is contiguous."""
    if not (t.is_cuda and t.dtype == dtype and t.shape == shape):
        raise ValueError(f"{name}: a {dtype} tensor of shape {tuple(shape)} on the GPU is wanted")
    a, b, c = t.stride()
    if c != 1 and shape[2] != 1:
        raise ValueError(f"{name}: the last dimension has to be contiguous")
    return t.data_ptr(), a, b


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
        self._dtype, self._heads, self._dim, self._page = k.dtype, heads, dim, tokens
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
        dtype, dim, n = self._dtype, self._dim, len(k)
        shape = (n, self._heads, dim)
        kp, k0, k1 = _rows(k, "k", dtype, shape)
        vp, v0, v1 = _rows(v, "v", dtype, shape)
        qp = op = q0 = q1 = o0 = o1 = n_q = 0
        if q is not None:
            n_q = q.shape[1]
            shape = (n, n_q, dim)
            qp, q0, q1 = _rows(q, "q", dtype, shape)
            if q_out is None:
                q_out = torch.empty(shape, dtype=dtype, device=q.device)
                op, o0, o1 = q_out.data_ptr(), n_q * dim, dim
            else:
                op, o0, o1 = _rows(q_out, "q_out", dtype, shape)
        cp = sp = pp = rot = table = 0
        if cos is not None:
            table, pairs = cos.shape
            rot = 2 * pairs
            cp, sp = _whole(cos, "cos", torch.float32, (table, pairs)), _whole(sin, "sin", torch.float32, (table, pairs))
            pp = _whole(positions, "positions", torch.int32, (n,))
        a = _APPEND.pack(qp, op, kp, vp, cp, sp, pp, _whole(slots, "slots", torch.int64, (n,)), q0, q1, o0, o1, k0, k1, v0, v1,
                         n, n_q, rot, table, B.HF_ROT_INTERLEAVED if interleaved else 0, 0)
        code = _hf_append_kv(self._c, a, _stream_of(k.get_device()))
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
        shape = n, heads, dim = tuple(q.shape)
        dtype, dev, page = self._dtype, q.device, self._page
        _need(dim == self._dim, "queries do not fit the cache")
        qp, q0, q1 = _rows(q, "q", dtype, shape)
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
            op, o0, o1 = out.data_ptr(), heads * dim, dim
        else:
            op, o0, o1 = _rows(out, "out", dtype, shape)
        if lse is None:
            lse = torch.empty((n, heads), dtype=torch.float32, device=dev)
            sp = lse.data_ptr()
        else:
            sp = _whole(lse, "lse", torch.float32, (n, heads))
        groups = width = gp = lp = pp = 0
        if group_offsets is not None:
            groups, width = prefix_pages.shape
            gp = _whole(group_offsets, "group_offsets", torch.int32, (groups + 1,))
            lp = _whole(prefix_lens, "prefix_lens", torch.int32, (groups,))
            pp = _whole(prefix_pages, "prefix_pages", torch.int32, (groups, width))
        own = suffix_pages.shape[1]
        pointers = (qp, op, sp, _whole(suffix_lens, "suffix_lens", torch.int32, (n,)),
                    _whole(suffix_pages, "suffix_pages", torch.int32, (n, own)), gp, lp, pp)
        rest = (q0, q1, o0, o1, n, heads, groups, n if max_group is None else max_group, width, own,
                width * page if max_prefix is None else max_prefix, own * page if max_suffix is None else max_suffix,
                dim ** -0.5 if scale is None else scale, 0)
        at = size = 0
        if workspace is None:
            size = _hf_attend_workspace_bytes(self._c, _ATTENTION.pack(*pointers, 0, 0, *rest))
            if size == C.c_size_t(-1).value:
                raise B.HfError(B.HF_EINVAL, "hf_attend_workspace_bytes")
            if size:
                workspace = torch.empty(size, dtype=torch.uint8, device=dev)
                at = workspace.data_ptr()
        else:
            at, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        code = _hf_attend(self._c, _ATTENTION.pack(*pointers, at, size, *rest), _stream_of(q.get_device()))
        if code:
            B.check(code, "hf_attend")
        return out, lse


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


def _logits(logits: torch.Tensor, targets: Optional[torch.Tensor], temperature: float) -> bytes:
    _need(logits.is_cuda and logits.dim() == 2 and logits.dtype in _TYPES, "logits: [rows, vocab] of bfloat16, float16 or float32 on the GPU is wanted")
    rows, vocab = logits.shape
    stride, one = logits.stride()
    _need(one == 1 or vocab == 1, "logits: the last dimension has to be contiguous")
    tp, size = 0, 8
    if targets is not None:
        size = targets.element_size()
        tp = _whole(targets, "targets", torch.int32 if size == 4 else torch.int64, (rows,))
    _need(temperature > 0, "the temperature must be positive")
    return _LOGITS.pack(logits.data_ptr(), tp, rows, stride, _TYPES[logits.dtype], vocab, size, 1.0 / temperature)


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], temperature: float = 1.0, top: int = 0) -> Logprobs:
    """Log probability of targets[row] (int64 or int32; outside the vocabulary: the row is left out), entropy, log sum of exponentials
    (lse, and in two parts for token_logprobs_back: norm) and the `top` likeliest tokens of every row of logits [rows, vocab] over the
    temperature.  Not differentiable by itself: see logprobs."""
    a = _logits(logits, targets, temperature)
    rows, dev = len(logits), logits.device
    stats = torch.empty(5 * rows, dtype=torch.float32, device=dev)
    at, row = stats.data_ptr(), 4 * rows
    ids = values = None
    ip = vp = 0
    if top:
        ids = torch.empty((rows, top), dtype=torch.int32, device=dev)
        values = torch.empty((rows, top), dtype=torch.float32, device=dev)
        ip, vp = ids.data_ptr(), values.data_ptr()
    o = _LOGPROBS.pack(at if targets is not None else 0, at + row, at + 2 * row, at + 3 * row, ip, vp, top, 0)
    code = _hf_token_logprobs(a, o, _stream_of(logits.get_device()))
    if code:
        B.check(code, "hf_token_logprobs")
    return Logprobs(stats, rows, targets is not None, ids, values)


def token_logprobs_back(logits: torch.Tensor, targets: torch.Tensor, norm: torch.Tensor, entropy: Optional[torch.Tensor],
                        grad_logprob: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) with respect to the logits; out may be the logits."""
    a = _logits(logits, targets, temperature)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    else:
        _need(out.is_cuda and out.shape == logits.shape and out.dtype == logits.dtype, "out: a tensor like the logits is wanted")
    stride, one = out.stride()
    _need(one == 1 or out.shape[1] == 1, "out: the last dimension has to be contiguous")
    rows = len(logits)
    row = (rows,)
    g = _GRAD.pack(_whole(norm, "norm", torch.float32, (rows, 2)), _whole(entropy, "entropy", torch.float32, row),
                   _whole(grad_logprob, "grad_logprob", torch.float32, row), _whole(grad_entropy, "grad_entropy", torch.float32, row),
                   out.data_ptr(), stride)
    code = _hf_token_logprobs_back(a, g, _stream_of(logits.get_device()))
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
