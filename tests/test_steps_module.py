"""What rollout.py and its native module do with devices, gradients and versions around a rollout's steps: without a GPU, over stand-ins."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HEAD = """
import sys
import torch
from tests.steps_module import Stand
s = Stand(sys.argv[1])
R, i32, i64, f32 = s.rollout, torch.int32, torch.int64, torch.float32
T = s.tensor


def pool(device=0, make=T):
    return R.PagePool([R.KvCache(make(5, 2, 4, 8, device=device), make(5, 2, 4, 8, device=device)) for _ in range(3)])


def refused(f, say=""):
    try:
        f()
    except ValueError as e:
        assert s.calls() == [], "called all the same"
        assert say in str(e), e
        return
    raise AssertionError("accepted: %s" % s.calls())
"""

DEVICES = HEAD + """
def all_of(d, lists=None, p=None):
    e = d if lists is None else lists
    p = p or pool(d)
    one = lambda n, dtype=i32: T(n, dtype=dtype, device=e)
    yield lambda: R.adjust_logits(T(3, 50, device=d), T(3, 9, dtype=i64, device=e), one(3), one(3), repetition=one(3, f32))
    yield lambda: R.adjust_logits(T(3, 50, device=d), bias_ids=T(3, 2, dtype=i32, device=e), bias=T(3, 2, dtype=f32, device=e))
    yield lambda: R.adjust_logits(T(3, 50, device=d), allowed=T(4, 2, dtype=i32, device=e), allowed_rows=one(3))
    yield lambda: R.top_distill(T(3, 50, device=d), T(3, 5, dtype=i32, device=e), T(3, 5, dtype=f32, device=e))
    yield lambda: R.top_distill_back(T(3, 50, device=d), T(3, 5, dtype=i32, device=e), T(3, 2, dtype=f32, device=e), T(3, 6, dtype=f32, device=e), one(3, f32))
    yield lambda: p.fork(T(3, 4, dtype=i32, device=d), one(3), one(6), one(5))
    yield lambda: p.grow(T(3, 4, dtype=i32, device=d), one(3), one(3), one(5), 2)
    yield lambda: p.compact(T(5, dtype=i32, device=d), [T(3, 4, dtype=i32, device=e), one(7)])


names = ["hf_adjust_logits"] * 3 + ["hf_top_distill", "hf_top_distill_back", "hf_fork_pages", "hf_grow_pages", "hf_compact_pages"]
for d in (0, 1, 3):
    for run in all_of(d):
        run()
    got = s.calls()
    assert got == [(n, d, 1000 + d) for n in names], got
    assert s.current_device() == 0
for d, e in ((0, 1), (1, 0), (2, 3)):
    for run in all_of(d, e):
        refused(run)
    for run in list(all_of(d, p=pool(e)))[5:]:
        refused(run)
x = T(3, 50, device=1)
refused(lambda: R.adjust_logits(x, out=T(3, 50)))
refused(lambda: pool(1).fork(T(3, 4, dtype=i32, device=1), T(3, dtype=i32, device=1), T(6, dtype=i32, device=1), T(5, dtype=i32, device=1), refs_out=T(5, dtype=i32)))
refused(lambda: R.PagePool([R.KvCache(T(5, 2, 4, 8), T(5, 2, 4, 8)), R.KvCache(T(5, 2, 4, 8, device=1), T(5, 2, 4, 8, device=1))]))
refused(lambda: R.PagePool([]))
refused(lambda: R.PagePool([R.KvCache(T(5, 2, 4, 8), T(5, 2, 4, 8)), R.KvCache(T(6, 2, 4, 8), T(6, 2, 4, 8))]))
assert s.current_device() == 0
print("ok")
"""

SHAPES = HEAD + """
x, one, p = T(3, 50), T(3, dtype=i32), pool()
tok = T(3, 9, dtype=i64)
refused(lambda: R.adjust_logits(torch.zeros(3, 50)), "GPU")
refused(lambda: R.adjust_logits(x, tok, T(2, dtype=i32)))
refused(lambda: R.adjust_logits(x, T(2, 9, dtype=i64), one))
refused(lambda: R.adjust_logits(x, T(3, 9, dtype=f32), one), "int32 or int64")
refused(lambda: R.adjust_logits(x, tok), "lens")
refused(lambda: R.adjust_logits(x, lens=one), "without tokens")
refused(lambda: R.adjust_logits(x, tok, one, repetition=T(4, dtype=f32)))
refused(lambda: R.adjust_logits(x, bias=T(3, 2, dtype=f32)), "go together")
refused(lambda: R.adjust_logits(x, bias=T(3, 2, dtype=f32), bias_ids=T(3, 3, dtype=i32)))
refused(lambda: R.adjust_logits(x, allowed=T(3, 1, dtype=i32)))
refused(lambda: R.adjust_logits(x, allowed=T(4, 2, dtype=i32)), "allowed_rows")
refused(lambda: R.adjust_logits(x, allowed_rows=one), "allowed")
refused(lambda: R.adjust_logits(x, out=T(3, 51)))
refused(lambda: R.adjust_logits(x, out=T(3, 50, dtype=f32)))
refused(lambda: R.adjust_logits(T(3, 50, dtype=i32)))
refused(lambda: R.top_distill(x, T(3, 5, dtype=i64), T(3, 5, dtype=f32)))
refused(lambda: R.top_distill(x, T(3, 5, dtype=i32), T(3, 4, dtype=f32)))
refused(lambda: R.top_distill(x, T(3, 5, dtype=i32), T(3, 5, dtype=f32), temperature=0.0), "positive")
refused(lambda: R.top_distill_back(x, T(3, 5, dtype=i32), T(3, 2, dtype=f32), T(3, 5, dtype=f32), T(3, dtype=f32)))
t = T(3, 4, dtype=i32)
refused(lambda: p.fork(t, one, T(2, 3, dtype=i32), T(5, dtype=i32)))
refused(lambda: p.fork(t, one, one, T(6, dtype=i32)), "refs")
refused(lambda: p.fork(T(3, 4, dtype=i64), one, one, T(5, dtype=i32)))
refused(lambda: p.fork(t, one, one, T(5, dtype=i32), tables_out=T(4, 4, dtype=i32)))
refused(lambda: p.grow(t, one, T(2, dtype=i32), T(5, dtype=i32)))
refused(lambda: p.grow(t, one, one, T(5, dtype=i32), -1))
refused(lambda: p.grow(t, one, one, T(5, dtype=i32), 2, slots=T(3, 3, dtype=i64)))
refused(lambda: p.compact(T(5, dtype=i32), [t] * 5))
refused(lambda: p.compact(T(5, dtype=i32), [t], [t, t]))
refused(lambda: p.compact(T(5, dtype=i32), t), "list")
refused(lambda: p.compact(T(5, dtype=i32), [t], t), "list")
refused(lambda: p.compact(T(5, dtype=i32), [T(3, 4, dtype=i64)]))
print("ok")
"""

GRADIENTS = HEAD + """
def calls(need):
    t = lambda name, *shape, dtype=torch.bfloat16: T(*shape, dtype=dtype).requires_grad_(name == need)
    yield lambda: R.adjust_logits(t("logits", 3, 50), T(3, 9, dtype=i64), T(3, dtype=i32), repetition=t("repetition", 3, dtype=f32), frequency=t("frequency", 3, dtype=f32),
                                  presence=t("presence", 3, dtype=f32), bias_ids=T(3, 2, dtype=i32), bias=t("bias", 3, 2, dtype=f32), out=t("out", 3, 50))
    p = pool(make=lambda *shape, device: t("cache", *shape))
    yield lambda: p.fork(T(3, 4, dtype=i32), T(3, dtype=i32), T(6, dtype=i32), T(5, dtype=i32))
    yield lambda: p.compact(T(5, dtype=i32))


for need, at in [(n, 0) for n in ("logits", "repetition", "frequency", "presence", "bias", "out")] + [("cache", 1), ("cache", 2)]:
    for k, run in enumerate(calls(need)):
        if k != at and not (need == "cache" and k):
            run()
            s.calls()
            continue
        refused(run, "no_grad")
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                run()
        s.calls()
lq = T(3, 5, dtype=f32).requires_grad_()
refused(lambda: R.distill(T(3, 50), T(3, 5, dtype=i32), lq), "detach")
with torch.no_grad():
    R.distill(T(3, 50), T(3, 5, dtype=i32), lq)
print("ok")
"""

VERSIONS = HEAD + """
def written(tensors, run):
    before = {n: t._version for n, t in tensors.items()}
    run()
    return sorted(n for n, t in tensors.items() if t._version != before[n])


t = dict(logits=T(3, 50), out=T(3, 50), bias=T(3, 2, dtype=f32), ids=T(3, 2, dtype=i32))
adjust = lambda **kw: R.adjust_logits(t["logits"], bias_ids=t["ids"], bias=t["bias"], **kw)
assert written(t, adjust) == [] and written(t, lambda: adjust(out=t["out"])) == ["out"] and written(t, lambda: adjust(out=t["logits"])) == ["logits"]
t = dict(logits=T(3, 50), out=T(3, 50), ids=T(3, 5, dtype=i32), norm=T(3, 2, dtype=f32), slopes=T(3, 6, dtype=f32), g=T(3, dtype=f32))
back = lambda **kw: R.top_distill_back(t["logits"], t["ids"], t["norm"], t["slopes"], t["g"], **kw)
assert written(t, back) == [] and written(t, lambda: back(out=t["out"])) == ["out"]
p = pool()
t = dict(tables=T(3, 4, dtype=i32), lens=T(3, dtype=i32), more=T(3, dtype=i32), refs=T(5, dtype=i32), tables_out=T(3, 4, dtype=i32), lens_out=T(3, dtype=i32),
         refs_out=T(5, dtype=i32), slots=T(3, 2, dtype=i64), workspace=T(4096, dtype=f32), k=p.caches[1].k, v=p.caches[2].v)
some = lambda *names: {n: t[n] for n in names}
assert written(t, lambda: p.fork(t["tables"], t["lens"], t["more"], t["refs"])) == ["k", "v"]
assert written(t, lambda: p.fork(t["tables"], t["lens"], t["more"], t["refs"], **some("tables_out", "lens_out", "refs_out", "workspace"))) == ["k", "lens_out", "refs_out", "tables_out", "v", "workspace"]
assert written(t, lambda: p.grow(t["tables"], t["lens"], t["more"], t["refs"], 2, refs_out=t["refs"], **some("slots"))) == ["refs", "slots"]
assert written(t, lambda: p.compact(t["refs"], [t["tables"]], [t["tables_out"]], **some("refs_out"))) == ["k", "refs_out", "tables_out", "v"]
with torch.inference_mode():
    R.adjust_logits(T(3, 50).view(3, 50), out=T(3, 50).view(3, 50))
print("ok")
"""


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    from tests.steps_module import build
    return build(str(tmp_path_factory.mktemp("steps")))


@pytest.mark.parametrize("script", [DEVICES, SHAPES, GRADIENTS, VERSIONS], ids=["devices", "shapes", "gradients", "versions"])
def test_module(module, script):
    p = subprocess.run([sys.executable, "-c", script, module], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip().endswith("ok"), p.stdout + p.stderr


@pytest.mark.gpu
def test_distill_under_autograd():
    """A loss masked in place, a broadcast gradient, a second use of the logits; and an overwritten operand is noticed."""
    from paper_2409_19256_amd import rollout
    print("[distill, autograd]", flush=True)
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(7, 301, generator=gen, device="cuda").requires_grad_()
    top = rollout.token_logprobs(torch.randn(7, 301, generator=gen, device="cuda"), None, top=9)
    keep = torch.rand(7, generator=gen, device="cuda") < 0.6

    def whole(y):  # the same in torch's own operations, in 64 bits
        logp, ids = torch.log_softmax(y / 0.8, 1), top.top_ids.long()
        lp = torch.cat((logp.gather(1, ids), logp.scatter(1, ids, -float("inf")).logsumexp(1, keepdim=True)), 1)
        lq = top.top_logprobs.double()
        lq = torch.cat((lq, (1 - lq.exp().sum(1, keepdim=True)).log()), 1)
        return 0.7 * (lq.exp() * (lq - lp)).sum(1) + 0.3 * (lp.exp() * (lp - lq)).sum(1)

    loss = rollout.distill(x, top.top_ids, top.top_logprobs, 0.8, reverse=0.3)
    loss.masked_fill_(~keep, 0)
    (loss.sum() + 0.01 * x.square().sum()).backward()
    y = x.detach().double().requires_grad_()
    (whole(y).masked_fill(~keep, 0).sum() + 0.01 * y.square().sum()).backward()
    # some tens of roundings of numbers of order 1 in 32 bits on either side
    assert torch.allclose(x.grad.double(), y.grad, rtol=1e-5, atol=1e-6)
    z = torch.randn(7, 301, generator=gen, device="cuda").requires_grad_()
    w = z * 1.0
    loss = rollout.distill(w, top.top_ids, top.top_logprobs)
    rollout.top_distill_back(w.detach(), top.top_ids, *list(rollout.top_distill(w.detach(), top.top_ids, top.top_logprobs))[1:], torch.ones(7, device="cuda"), out=w.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
