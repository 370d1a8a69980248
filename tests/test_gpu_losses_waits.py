"""A bounded wait that runs out (checked build): the kernel ends by itself, the other waits of its block end with it, the
status word says IWP_ERR_TIMEOUT, and the context stays usable."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import ctypes as C, time
import torch
from paper_1901_01544_b200 import binding, losses
assert binding.LIB_PATH.endswith("libiwp_debug.so")
plan = losses.HeadLoss(40, 300, 64)
h, w = torch.randn(40, 64, device="cuda").bfloat16(), torch.randn(300, 64, device="cuda").bfloat16()
y = torch.randint(0, 300, (40,), device="cuda")
before = plan.cross_entropy_grad(h, w, y)
assert plan.status() == 0
gave_up = torch.zeros(1, dtype=torch.int32, device="cuda")
L = losses.lib()
L.iwp_loss_wait_probe.argtypes = [C.c_void_p] * 3
torch.cuda.synchronize()
start = time.monotonic()
assert L.iwp_loss_wait_probe(plan._state.data_ptr(), gave_up.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
torch.cuda.synchronize()
took = time.monotonic() - start
assert took < 2.0, took
assert gave_up.item() == 2  # one ran out, the other saw that it had
assert plan.status() == binding.IWP_ERR_TIMEOUT, plan.status()
try:
    plan.check()
    raise SystemExit("check() passed")
except losses.IwpError:
    pass
plan.reset()
after = plan.cross_entropy_grad(h, w, y)
assert plan.status() == 0 and torch.equal(before.dweight, after.dweight) and torch.equal(before.loss, after.loss)
print("waits ok")
"""


def test_a_wait_that_runs_out():
    sys.path.insert(0, ROOT)
    from paper_1901_01544_b200 import build as lib_build

    lib_build.build(debug=True)
    env = dict(os.environ, IWP_LIB_VARIANT="debug")
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "waits ok" in r.stdout, r.stdout + r.stderr
