"""The order of a traced backward's kernels, from a profile that has to have its records: in a process of its own, whose first profile it is.  And that a session of
tests takes the profiles first, where their records arrive."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = r"""
import sys
sys.path.insert(0, %r)
sys.path.insert(0, %r)
import torch
import paper_2408_08015_b200 as P
import stage_inputs as si
from harness import kernels
L, c, B, h, w = si.Layer, 64, 4, 14, 14
net = []
for _ in range(3):
    net += [L("conv", c, c, 1, 1, 0, len(net) - 1, -1), L("bn", c, c, 0, 1, 0, len(net), -1), L("relu", c, c, 0, 1, 0, len(net) + 1, -1)]
hdl = P.asteroid_stage_create(net, 0, len(net) - 1, h, w, B, 1, dtype=P.AST_BF16)
P.asteroid_stage_import_state(hdl, si.init_params(net, 0, len(net) - 1, 0))
x = torch.randn(B, h, w, c, device="cuda").to(torch.bfloat16)
y, dy, dx = torch.empty_like(x), torch.randn_like(x), torch.empty_like(x)
sp = torch.cuda.current_stream().cuda_stream
P.asteroid_stage_forward(hdl, 0, x.data_ptr(), y.data_ptr(), sp)
torch.cuda.synchronize()
P.asteroid_trace_start()
with kernels() as found:
    P.asteroid_stage_backward(hdl, 0, dy.data_ptr(), dx.data_ptr(), sp)
P.asteroid_trace_stop()
P.asteroid_stage_destroy(hdl)
print("ORDER", "".join("w" if "wgrad" in k["name"] else "d" for k in found if "wgrad" in k["name"] or "pw_mma" in k["name"]))
"""


@pytest.mark.gpu
def test_order_of_a_traced_backward_in_a_process_of_its_own():
    r = subprocess.run([sys.executable, "-c", CODE % (ROOT, os.path.join(ROOT, "tests"))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert re.search("^ORDER wdwdwd$", r.stdout, re.M), r.stdout[-500:]


def test_a_session_takes_the_profiles_first():
    def collected():
        r = subprocess.run([sys.executable, "-m", "pytest", "--collect-only", "-q", "-m", "gpu", "tests"], capture_output=True, text=True, timeout=300, cwd=ROOT,
                           env={k: v for k, v in os.environ.items() if k != "PYTEST_ADDOPTS"})
        assert r.returncode == 0, r.stdout[-2000:]
        return [l for l in r.stdout.splitlines() if "::" in l]
    ids = collected()
    assert ids[0] == "tests/test_gpu_traced_order.py::test_order_of_a_traced_backward"
    files = list(dict.fromkeys(i.split("::")[0] for i in ids))
    assert files[:2] == ["tests/test_gpu_traced_order.py", "tests/test_gpu_deep_requests.py"] and files[2:] == sorted(files[2:])
