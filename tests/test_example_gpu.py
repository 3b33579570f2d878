"""The example runs the operators together: what generation sampled, token by token over shared pages, has the log probabilities that
one pass over prompt and answer recomputes, the update raises what it is meant to raise, and it reaches the training shards."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("length,steps", [(37, 21), (1, 1), (16, 17)])
def test_one_iteration(length, steps):
    print("[example]", length, steps, flush=True)
    spec = importlib.util.spec_from_file_location("rlhf_step", os.path.join(ROOT, "examples", "rlhf_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(length, steps)
    assert r["samples"] == 4 * 4 * 12
    # logits of order 1 out of two layers of bfloat16, whose roundings (2^-8 each, some tens of them on the way) fall differently in the two orders of summation
    assert r["worst"] < 0.1
    assert r["after"] > r["before"] and r["changed"] > 0
