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
