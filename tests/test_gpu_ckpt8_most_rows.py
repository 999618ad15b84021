"""The 8-bit checkpoint calls at 2^31 - 1 rows, the most that they take: the last step of 64 rows ends where a signed 32-bit number does."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_most_rows():
    import torch as T
    import paper_2408_08015_b200 as P
    T.cuda.empty_cache()
    rows = (1 << 31) - 1
    at = [0, 63, 64, (1 << 30) - 1, 1 << 30, rows - 129, rows - 64, rows - 63, rows - 62, rows - 1]
    vals = [3.0, -5.0, 7.0, 11.0, -13.0, 17.0, 19.0, 23.0, -29.0, 31.0]
    x = T.zeros(rows, device="cuda", dtype=T.bfloat16)
    x[at] = T.tensor(vals, device="cuda", dtype=T.bfloat16)
    ckpt = T.empty(P.asteroid_ckpt8_bytes(rows, 1), device="cuda", dtype=T.uint8)
    P.asteroid_ckpt8_pack(x.data_ptr(), 1, rows, 1, P.AST_BF16, ckpt.data_ptr(), 0)
    out = T.full_like(x, 4.0)
    P.asteroid_ckpt8_unpack(ckpt.data_ptr(), rows, 1, P.AST_BF16, out.data_ptr(), 1, 0)
    assert T.equal(out, x)
    del out, x
    # dy by tensor copies, by single values, and in float32; column c of dy has the row at[c] of x alone, the first column the remaining ones as well
    for bf16, co in ((True, 8), (True, 1), (False, 1)):
        dy = T.zeros(rows, co, device="cuda", dtype=T.bfloat16 if bf16 else T.float32)
        want = np.zeros(co)
        for k, (r, v) in enumerate(zip(at, vals)):
            c = k if k < co else 0
            dy[r, c] = float(k + 1)
            want[c] += (k + 1) * v
        need = P.asteroid_ckpt8_linear_wgrad_workspace(rows, 1, co, int(bf16))
        ws, dw, db = T.empty(need + 16, device="cuda", dtype=T.uint8), T.empty(co, device="cuda"), T.empty(co, device="cuda")
        P.asteroid_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, 1, co, int(bf16), dw.data_ptr(), db.data_ptr(), 0, ws.data_ptr(), need, 0)
        np.testing.assert_array_equal(dw.cpu().numpy(), want)
        np.testing.assert_array_equal(db.cpu().numpy(), dy[at].double().sum(0).cpu().numpy())
        del dy
        T.cuda.empty_cache()
