"""A workspace that suffices for some rows suffices for fewer: a ragged last micro-batch runs on that of the others."""
import random

import numpy as np
import pytest

import paper_2408_08015_b200 as P


@pytest.fixture(scope="module", autouse=True)
def library():
    P.build()


def never_shrinks(workspace, most):
    """Over all row counts up to 4096, and larger ones with their neighbours, a few at every doubling."""
    rng = random.Random(1)
    rows = set(range(0, 4097))
    at = 4096.0
    while at < most:
        r = int(at * rng.uniform(1.0, 1.02))
        rows.update(k for k in (r - 1, r, r + 1) if k <= most)
        at *= 1.02
    rows.add(most)
    last = 0
    for r in sorted(rows):
        need = workspace(r)
        assert need >= last, r
        last = need


@pytest.mark.parametrize("dim", [1, 16, 256, 257, 512, 1000, 4096, 300000, 605952, 606208, 1 << 20])
def test_embedding_workspace_never_shrinks(dim):
    most = min((1 << 31) - 1, (1 << 40) // dim)
    never_shrinks(lambda rows: P.asteroid_embedding_workspace(rows, dim), most)
    # ... where the stretches of a warp double, too
    for r in (4, 8, 16):
        for k in range(-3, 4):
            edge = 2 * r * (2367 // (-(-dim // 256))) + k
            if 0 < edge < most:
                assert P.asteroid_embedding_workspace(edge, dim) <= P.asteroid_embedding_workspace(edge + 1, dim)


def test_embedding_workspace_of_a_large_micro_batch_holds_a_smaller_one():
    assert P.asteroid_embedding_workspace(16384, 512) <= P.asteroid_embedding_workspace(37888, 512)


# c_in and c_out whose tiles leave 1 to 73 over for 74 pairs of multiprocessors, of 128 and of 256 input channels
@pytest.mark.parametrize("dt", [P.AST_F32, P.AST_BF16])
@pytest.mark.parametrize("ci,co", [(1, 1), (40, 24), (128, 1000), (100, 7 * 256), (512, 2048), (1024, 2800), (256, 36 * 256), (256, 37 * 256), (256, 55 * 256), (256, 71 * 256),
                                   (2560, 4096), (4096, 4096), (65536, 65536)])
def test_weight_gradient_workspace_never_shrinks(ci, co, dt):
    never_shrinks(lambda rows: P.asteroid_ckpt8_linear_wgrad_workspace(rows, ci, co, dt), (1 << 31) - 1)


def test_no_rows_need_no_workspace():
    assert P.asteroid_embedding_workspace(0, 64) == 0 and P.asteroid_ckpt8_linear_wgrad_workspace(0, 512, 2048, P.AST_BF16) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [8832, 8705, 4000, 100, 1])
def test_weight_gradient_on_a_larger_calls_workspace(rows, bf16):
    import torch as T
    most, ci, co = 8896, 1024, 2800
    dt = T.bfloat16 if bf16 else T.float32
    gen = T.Generator(device="cuda").manual_seed(rows)
    x = T.randint(-127, 128, (rows, ci), device="cuda", generator=gen).to(dt)
    dy = T.randint(-4, 5, (rows, co), device="cuda", generator=gen).to(dt)             # sums of at most 8832 * 127 * 4 < 2^24
    ckpt = T.empty(P.asteroid_ckpt8_bytes(rows, ci), device="cuda", dtype=T.uint8)
    P.asteroid_ckpt8_pack(x.data_ptr(), ci, rows, ci, int(bf16), ckpt.data_ptr(), 0)
    nbytes = P.asteroid_ckpt8_linear_wgrad_workspace(most, ci, co, int(bf16))
    ws = T.full((nbytes + 64,), 0xA5, device="cuda", dtype=T.uint8)
    dw, db = T.empty(co, ci, device="cuda"), T.empty(co, device="cuda")
    P.asteroid_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, ci, co, int(bf16), dw.data_ptr(), db.data_ptr(), 0, ws.data_ptr(), nbytes, 0)
    T.cuda.synchronize()
    assert (ws[nbytes:] == 0xA5).all()
    assert T.equal(dw.double(), dy.double().T @ x.double()) and T.equal(db.double(), dy.double().sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [16384, 18943, 18944, 18945, 9471, 5000, 1])
def test_embedding_gradient_on_a_larger_calls_workspace(rows):
    import torch as T
    most, vocab, dim = 37888, 700, 512
    gen = T.Generator(device="cuda").manual_seed(rows)
    ids = T.randint(0, vocab, (rows,), device="cuda", generator=gen, dtype=T.int32)
    dy = T.randint(-20, 21, (rows, dim), device="cuda", generator=gen).float()
    nbytes = P.asteroid_embedding_workspace(most, dim)
    ws = T.full((nbytes + 64,), 0xA5, device="cuda", dtype=T.uint8)
    grad = T.empty(vocab, dim, device="cuda")
    P.asteroid_embedding_backward(ids.data_ptr(), dy.data_ptr(), dim, rows, vocab, dim, 1.0, P.AST_F32, grad.data_ptr(), 0, ws.data_ptr(), nbytes, 0)
    T.cuda.synchronize()
    assert (ws[nbytes:] == 0xA5).all()
    want = np.zeros((vocab, dim))
    np.add.at(want, ids.cpu().numpy(), dy.cpu().double().numpy())
    np.testing.assert_array_equal(grad.cpu().double().numpy(), want)
