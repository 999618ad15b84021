"""The checkpoint and embedding calls whose first use in a process is inside a capture: the header allows it, and the first use is where attributes are set and code is loaded."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = r"""
import sys
sys.path.insert(0, %r)
import torch as T
import paper_2408_08015_b200 as P
gen = T.Generator(device="cuda").manual_seed(1)
def whole(top, *shape, dt=T.float32):
    return T.randint(-top, top + 1, shape, device="cuda", generator=gen).to(dt)
def captured(call):
    g = T.cuda.CUDAGraph()
    with T.cuda.graph(g):
        call(T.cuda.current_stream().cuda_stream)
    g.replay()
    T.cuda.synchronize()
for bf16 in (0, 1):
    dt = T.bfloat16 if bf16 else T.float32
    for rows, ci, co in ((900, 512, 1024), (300, 77, 51)):
        x, dy = whole(127, rows, ci, dt=dt), whole(8, rows, co, dt=dt)
        ckpt = T.zeros(P.asteroid_ckpt8_bytes(rows, ci), device="cuda", dtype=T.uint8)
        y, back = T.zeros_like(x), T.zeros_like(x)
        need = P.asteroid_ckpt8_linear_wgrad_workspace(rows, ci, co, bf16)
        ws, dw, db = T.zeros(need + 16, device="cuda", dtype=T.uint8), T.zeros(co, ci, device="cuda"), T.zeros(co, device="cuda")
        captured(lambda st: P.asteroid_ckpt8_pack(x.data_ptr(), ci, rows, ci, bf16, ckpt.data_ptr(), st))
        captured(lambda st: P.asteroid_ckpt8_unpack(ckpt.data_ptr(), rows, ci, bf16, back.data_ptr(), ci, st))
        assert T.equal(back, x)
        captured(lambda st: P.asteroid_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, ci, co, bf16, dw.data_ptr(), db.data_ptr(), 0, ws.data_ptr(), need, st))
        assert T.equal(dw.double(), dy.double().T @ x.double()) and T.equal(db.double(), dy.double().sum(0))
        ckpt.zero_()
        captured(lambda st: P.asteroid_ckpt8_act_forward(P.AST_RELU, x.data_ptr(), ci, rows, ci, bf16, y.data_ptr(), ci, ckpt.data_ptr(), st))
        assert T.equal(y, x.clamp(min=0))
        captured(lambda st: P.asteroid_ckpt8_act_backward(P.AST_RELU, ckpt.data_ptr(), x.data_ptr(), ci, rows, ci, bf16, back.data_ptr(), ci, st))
        assert T.equal(back, x.clamp(min=0))
    for rows, vocab, dim in ((50, 30, 64), (20000, 700, 33), (70000, 900, 8)):
        table, ids, dy = whole(50, vocab, dim), T.randint(-1, vocab, (rows,), device="cuda", generator=gen, dtype=T.int32), whole(8, rows, dim, dt=dt)
        y, grad = T.zeros(rows, dim, device="cuda", dtype=dt), T.zeros(vocab, dim, device="cuda")
        captured(lambda st: P.asteroid_embedding_forward(table.data_ptr(), 0, ids.data_ptr(), rows, vocab, dim, 2.0, y.data_ptr(), dim, bf16, st))
        ok = (ids >= 0).double()[:, None]
        assert T.equal(y.double(), 2 * table.double()[ids.clamp(min=0).long()] * ok)
        need = P.asteroid_embedding_workspace(rows, dim)
        ws = T.zeros(need, device="cuda", dtype=T.uint8)
        captured(lambda st: P.asteroid_embedding_backward(ids.data_ptr(), dy.data_ptr(), dim, rows, vocab, dim, 2.0, bf16, grad.data_ptr(), 0, ws.data_ptr(), need, st))
        want = T.zeros(vocab, dim, device="cuda", dtype=T.float64).index_add_(0, ids.clamp(min=0).long(), 2 * dy.double() * ok)
        assert T.equal(grad.double(), want)
print("CAPTURED")
"""


def test_first_use_of_every_call_inside_a_capture():
    r = subprocess.run([sys.executable, "-c", CODE % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "CAPTURED" in r.stdout, r.stderr[-2000:]
