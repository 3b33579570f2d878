"""The rollout operators on a GPU that is not the current one: the call is made with the tensors' GPU current, on its stream, and tensors of two GPUs are
refused.  Without a GPU, over stand-ins; on a machine with two, for real."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import sys
import torch
from tests.rollout_module import Stand
s = Stand(sys.argv[1])
R, i32, f32 = s.rollout, torch.int32, torch.float32


def cache(device):
    return R.KvCache(s.tensor(3, 2, 4, 8, device=device), s.tensor(3, 2, 4, 8, device=device))


def append(c, device, **kw):
    k, v, slots = (s.tensor(5, 2, 8, device=device), s.tensor(5, 2, 8, device=device), s.tensor(5, dtype=torch.int64, device=device))
    return c.append(k, v, slots, q=s.tensor(5, 4, 8, device=device), **kw)


def attend(c, device, **kw):
    return c.attend(s.tensor(6, 4, 8, device=device), s.tensor(6, dtype=i32, device=device), s.tensor(6, 2, dtype=i32, device=device), **kw)


def score(device, **kw):
    return R.token_logprobs(s.tensor(3, 50, device=device), s.tensor(3, dtype=torch.int64, device=device), top=4)


def back(device, **kw):
    one = lambda: s.tensor(3, dtype=f32, device=device)
    return R.token_logprobs_back(s.tensor(3, 50, device=device), s.tensor(3, dtype=torch.int64, device=device), s.tensor(3, 2, dtype=f32, device=device), one(), one(), one(), **kw)


def refused(f, *a, **kw):
    try:
        f(*a, **kw)
    except ValueError as e:
        assert s.calls() == [], "called all the same"
        return str(e)
    raise AssertionError("accepted: %s" % s.calls())


for device in (0, 1, 3):
    append(cache(device), device)
    attend(cache(device), device)
    score(device)
    back(device)
    want = [(n, device, 1000 + device) for n in ("hf_append_kv", "hf_attend", "hf_token_logprobs", "hf_token_logprobs_back")]
    got = s.calls()
    assert got == want, got
    assert s.current_device() == 0
for c, t in ((0, 1), (1, 0), (2, 3)):
    refused(append, cache(c), t)
    refused(attend, cache(c), t)
refused(attend, cache(1), 1, lse=s.tensor(6, 4, dtype=f32, device=0))
refused(back, 1, out=s.tensor(3, 50, device=0))
assert s.current_device() == 0
print("devices ok")
"""


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    from tests.rollout_module import build
    return build(str(tmp_path_factory.mktemp("rollout")))


def test_the_tensors_gpu_is_made_current(module):
    p = subprocess.run([sys.executable, "-c", SCRIPT, module], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "devices ok" in p.stdout, p.stdout + p.stderr


@pytest.mark.gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_on_the_second_gpu():
    from paper_2409_19256_amd import rollout
    torch.cuda.set_device(0)
    x = torch.randn(7, 501, device="cuda:1")
    t = torch.arange(7, device="cuda:1")
    r = rollout.token_logprobs(x, t)
    assert torch.allclose(r.logprob, torch.log_softmax(x, 1)[t, t], atol=1e-5) and torch.cuda.current_device() == 0
    c = rollout.KvCache.empty(4, 2, 16, 64, device="cuda:1")
    k, v = (torch.randn(5, 2, 64, device="cuda:1").bfloat16() for _ in range(2))
    c.append(k, v, torch.arange(5, device="cuda:1"))
    assert torch.equal(c.k[0, :, :5].transpose(0, 1), k) and torch.equal(c.v[0, :, :5].transpose(0, 1), v)
    with pytest.raises(ValueError):
        c.append(k.to("cuda:0"), v.to("cuda:0"), torch.arange(5, device="cuda:0"))
