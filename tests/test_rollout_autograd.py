"""What rollout.py refuses on its own account, on the CPU and over stand-ins for the library."""
import subprocess
import sys

import pytest
import torch

from tests.test_rollout_devices import ROOT, module  # noqa: F401


def test_log_probabilities_need_targets():
    """And say so at once, not in the backward pass."""
    from paper_2409_19256_amd import rollout
    x = torch.randn(3, 7).requires_grad_()
    with pytest.raises(ValueError, match="targets"):
        rollout.logprobs(x, None)


GRADIENTS = """
import sys
import torch
from tests.rollout_module import Stand
s = Stand(sys.argv[1])
R, i32, f32 = s.rollout, torch.int32, torch.float32


def calls(need=()):
    t = lambda name, *shape, dtype=torch.bfloat16: s.tensor(*shape, dtype=dtype).requires_grad_(name in need)
    c = R.KvCache(t("cache_k", 3, 2, 4, 8), t("cache_v", 3, 2, 4, 8))
    yield "append", lambda: c.append(t("k", 5, 2, 8), t("v", 5, 2, 8), s.tensor(5, dtype=torch.int64), q=t("q", 5, 4, 8), q_out=t("q_out", 5, 4, 8))
    yield "attend", lambda: c.attend(t("q", 6, 4, 8), s.tensor(6, dtype=i32), s.tensor(6, 2, dtype=i32), out=t("out", 6, 4, 8), lse=t("lse", 6, 4, dtype=f32))


reads = dict(append=("cache_k", "cache_v", "k", "v", "q", "q_out"), attend=("cache_k", "cache_v", "q", "out", "lse"))
for name in sorted(set(reads["append"] + reads["attend"])):
    for call, run in calls((name,)):
        if name not in reads[call]:
            run()
            s.calls()
            continue
        try:
            run()
        except ValueError as e:
            assert "no_grad" in str(e), e
        else:
            raise AssertionError("%s takes %s that requires a gradient" % (call, name))
        assert s.calls() == [], "called all the same"
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                run()
        s.calls()
print("gradients ok")
"""


def run(script, module, last):
    p = subprocess.run([sys.executable, "-c", script, module], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and last in p.stdout, p.stdout + p.stderr


def test_a_gradient_is_not_lost_in_silence(module):  # noqa: F811
    """The cache's operators have no backward: asked for one, they refuse."""
    run(GRADIENTS, module, "gradients ok")


VERSIONS = """
import sys
import torch
from tests.rollout_module import Stand
s = Stand(sys.argv[1])
R, i32, f32 = s.rollout, torch.int32, torch.float32


def written(tensors, run):
    before = {n: t._version for n, t in tensors.items()}
    run()
    return sorted(n for n, t in tensors.items() if t._version != before[n])


c = R.KvCache(s.tensor(3, 2, 4, 8), s.tensor(3, 2, 4, 8))
slots, lens, pages = s.tensor(5, dtype=torch.int64), s.tensor(6, dtype=i32), s.tensor(6, 2, dtype=i32)
t = dict(cache_k=c.k, cache_v=c.v, k=s.tensor(5, 2, 8), v=s.tensor(5, 2, 8), q=s.tensor(5, 4, 8), q_out=s.tensor(5, 4, 8))
append = lambda k=t["k"], v=t["v"], **kw: c.append(k, v, slots, **kw)
assert written(t, append) == ["cache_k", "cache_v"]
assert written(t, lambda: append(q=t["q"])) == ["cache_k", "cache_v"]
assert written(t, lambda: append(q=t["q"], q_out=t["q_out"])) == ["cache_k", "cache_v", "q_out"]
assert written(t, lambda: append(q=t["q"], q_out=t["q"])) == ["cache_k", "cache_v", "q"]
t = dict(cache_k=c.k, cache_v=c.v, q=s.tensor(6, 4, 8), out=s.tensor(6, 4, 8), lse=s.tensor(6, 4, dtype=f32), workspace=s.tensor(4096, dtype=f32))
assert written(t, lambda: c.attend(t["q"], lens, pages)) == []
assert written(t, lambda: c.attend(t["q"], lens, pages, out=t["out"], lse=t["lse"], workspace=t["workspace"])) == ["lse", "out", "workspace"]
t = dict(logits=s.tensor(3, 50), out=s.tensor(3, 50), targets=s.tensor(3, dtype=torch.int64), norm=s.tensor(3, 2, dtype=f32), g=s.tensor(3, dtype=f32))
back = lambda **kw: R.token_logprobs_back(t["logits"], t["targets"], t["norm"], t["g"], t["g"], t["g"], **kw)
assert written(t, back) == []
assert written(t, lambda: back(out=t["out"])) == ["out"]
assert written(t, lambda: back(out=t["logits"])) == ["logits"]
with torch.inference_mode():  # tensors made here have no version
    c = R.KvCache(s.tensor(3, 2, 4, 8).view(3, 2, 4, 8), s.tensor(3, 2, 4, 8).view(3, 2, 4, 8))
    append()
append()
print("versions ok")
"""


def test_torch_knows_what_is_written_to(module):  # noqa: F811
    """A later backward over an overwritten tensor is caught by its version."""
    run(VERSIONS, module, "versions ok")
