"""A linear layer of a stage with 8-bit slots whose weight gradient needs more scratch than other layers: from the checkpoint all the same."""
import numpy as np
import pytest

import stage_inputs as si

pytestmark = pytest.mark.gpu


def test_a_linear_layer_of_many_rows_takes_its_gradient_from_the_checkpoint(monkeypatch):
    """float32, 512 -> 2048 over 16704 rows, in whole numbers that a checkpoint keeps and whose sums are exact."""
    import torch as T
    import paper_2408_08015_b200 as P
    monkeypatch.setenv("ASTEROID_CHECK_GUARDS", "1")
    B, ci, co = 16704, 512, 2048
    assert P.asteroid_ckpt8_linear_wgrad_workspace(B, ci, co, P.AST_F32) > 4 * (8 << 20)
    gen = T.Generator(device="cuda").manual_seed(2)
    x = T.randint(-127, 128, (B, ci), device="cuda", generator=gen).float()
    dy = T.randint(-4, 5, (B, co), device="cuda", generator=gen).float()               # sums of at most 16704 * 127 * 4 < 2^24
    want_w, want_b = dy.double().T @ x.double(), dy.double().sum(0)
    net = [si.Layer("linear", ci, co, 1, 1, 0, -1, -1)]
    hdl = P.asteroid_stage_create_ckpt8(net, 0, 0, 1, 1, B, 1, dtype=P.AST_F32, need_input_grad=0)
    try:
        P.asteroid_stage_import_state(hdl, np.zeros(P.asteroid_stage_param_count(hdl), np.float32), None)
        y = T.empty(B, co, device="cuda")
        for trace in (True, False):
            P.asteroid_stage_forward(hdl, 0, x.data_ptr(), y.data_ptr(), 0)
            if trace:
                P.asteroid_trace_start()
            P.asteroid_stage_backward(hdl, 0, dy.data_ptr(), None, 0)
            kinds = {k["name"]: k["launches"] for k in P.asteroid_trace_stop()} if trace else kinds
            g = np.empty(P.asteroid_stage_param_count(hdl), np.float32)
            P.asteroid_stage_export_state(hdl, micro_grad=g)
            np.testing.assert_array_equal(g[:co * ci].reshape(co, ci), want_w.cpu().numpy())
            np.testing.assert_array_equal(g[co * ci:], want_b.cpu().numpy())
            P.asteroid_stage_accumulate(hdl, 0, 0)
            P.asteroid_stage_step(hdl, 0.0, 0.0, 0)
        assert kinds.get("ckpt8_wgrad") == 1, kinds
    finally:
        P.asteroid_stage_destroy(hdl)
