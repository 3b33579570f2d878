"""What rollout.py's native modules do with the tangents of forward-mode differentiation: they are refused where they would be lost.  Without a GPU, over stand-ins."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HEAD = """
import sys
import torch
import torch.autograd.forward_ad as forward

i32, i64, f32, bf16 = torch.int32, torch.int64, torch.float32, torch.bfloat16


def check(s, calls, names):
    for need in names:
        def t(name, *shape, dtype=bf16):
            x = s.tensor(*shape, dtype=dtype)
            return forward.make_dual(x, s.tensor(*shape, dtype=dtype)) if name == need else x

        with forward.dual_level():
            runs = list(calls(t))  # (what it takes, call)
            assert any(need in takes for takes, _ in runs)
            for mode in (torch.enable_grad, torch.no_grad):  # (no_grad does not end forward mode)
                for takes, run in runs:
                    try:
                        with mode():
                            run()
                        assert need not in takes, (need, "accepted", s.calls())
                    except ValueError as e:
                        assert need in takes and need in str(e) and "gradient" in str(e), e
                        assert s.calls() == [], "called all the same"
                    s.calls()
            with torch.inference_mode():
                for _, run in runs:
                    run()
        for _, run in runs:  # the level has ended, and the tangents with it
            run()
        s.calls()
    print("ok")
"""

STEPS = HEAD + """
from tests.steps_module import Stand
s = Stand(sys.argv[1])
R, T = s.rollout, s.tensor


def calls(t):
    a = {n: t(n, *shape, dtype=d) for n, shape, d in (("logits", (3, 50), bf16), ("repetition", (3,), f32), ("frequency", (3,), f32), ("presence", (3,), f32), ("bias", (3, 2), f32),
                                                      ("out", (3, 50), bf16))}
    yield tuple(a), lambda: R.adjust_logits(tokens=T(3, 9, dtype=i64), lens=T(3, dtype=i32), bias_ids=T(3, 2, dtype=i32), **a)
    p = R.PagePool([R.KvCache(T(5, 2, 4, 8), t("pool", 5, 2, 4, 8))])
    yield ("pool",), lambda: p.fork(T(3, 4, dtype=i32), T(3, dtype=i32), T(6, dtype=i32), T(5, dtype=i32))
    yield ("pool",), lambda: p.compact(T(5, dtype=i32))
    yield (), lambda: p.grow(T(3, 4, dtype=i32), T(3, dtype=i32), T(3, dtype=i32), T(5, dtype=i32))


check(s, calls, ["logits", "repetition", "frequency", "presence", "bias", "out", "pool"])
"""

ROLLOUT = HEAD + """
from tests.rollout_module import Stand
s = Stand(sys.argv[1])
R, T = s.rollout, s.tensor


def calls(t):
    c = R.KvCache(T(5, 2, 4, 8), t("cache", 5, 2, 4, 8))
    a = dict(k=t("k", 3, 2, 8), v=t("v", 3, 2, 8), q=t("q", 3, 4, 8), q_out=t("q_out", 3, 4, 8))
    yield ("cache", *a), lambda: c.append(slots=T(3, dtype=i64), **a)
    b = dict(q=a["q"], out=t("out", 3, 4, 8), lse=t("lse", 3, 4, dtype=f32))
    yield ("cache", *b), lambda: c.attend(suffix_lens=T(3, dtype=i32), suffix_pages=T(3, 2, dtype=i32), **b)


check(s, calls, ["cache", "k", "v", "q", "q_out", "out", "lse"])
"""


@pytest.mark.parametrize("which", ["steps", "rollout"])
def test_tangents(which, tmp_path):
    from tests import rollout_module, steps_module
    build, script = dict(steps=(steps_module.build, STEPS), rollout=(rollout_module.build, ROLLOUT))[which]
    p = subprocess.run([sys.executable, "-c", script, build(str(tmp_path))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip().endswith("ok"), p.stdout + p.stderr
