"""What the outputs of the operators around a rollout's steps hold on to: without a GPU, over stand-ins."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import sys
import torch
from tests.steps_module import Stand
s = Stand(sys.argv[1])
R, T, i32, f32 = s.rollout, s.tensor, torch.int32, torch.float32
held = lambda t: t.untyped_storage().nbytes()

# a loss, which outlives its step, holds its own numbers and no more
lists = T(40, 64, dtype=i32), T(40, 64, dtype=f32)
d = R.top_distill(T(40, 500), *lists)
assert held(d.loss) == 160 and d.loss.storage_offset() == 0, held(d.loss)
assert d.norm.untyped_storage().data_ptr() == d.slopes.untyped_storage().data_ptr()
x = T(40, 500).requires_grad_()
loss = R.distill(x, *lists)
assert loss.requires_grad and held(loss) == held(loss.detach()) == 160
few = R.top_distill(T(3, 500), T(3, 64, dtype=i32), T(3, 64, dtype=f32)).loss  # (or a few numbers more)
assert held(few) <= 4096 and R.top_distill(T(0, 500), T(0, 64, dtype=i32), T(0, 64, dtype=f32)).loss.shape == (0,)

# tables, lengths and counts lie together, apart from one another
p = R.PagePool([R.KvCache(T(5, 2, 4, 8), T(5, 2, 4, 8))])
for out in (p.fork(T(3, 4, dtype=i32), T(3, dtype=i32), T(7, dtype=i32), T(5, dtype=i32)), p.grow(T(3, 4, dtype=i32), T(3, dtype=i32), T(3, dtype=i32), T(5, dtype=i32), 9)):
    assert len({t.untyped_storage().data_ptr() for t in out}) == 1
    places = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in out)
    assert all(a[1] <= b[0] for a, b in zip(places, places[1:])) and places[-1][1] <= out[0].untyped_storage().data_ptr() + held(out[0])
print("ok")
"""


def test_what_outputs_hold(tmp_path):
    from tests.steps_module import build
    p = subprocess.run([sys.executable, "-c", SCRIPT, build(str(tmp_path))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip().endswith("ok"), p.stdout + p.stderr
