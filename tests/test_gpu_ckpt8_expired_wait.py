"""The weight gradient from 8-bit checkpoints when a wait of its kernel runs out: what the pair of multiprocessors concerned had yet to give is NaN, all of it, and everything
else as ever.  The self-test stops the pair that has the first tile after some steps; its waits are short there."""
import numpy as np
import pytest

import paper_2408_08015_b200 as P

STEP, TILE = 64, 256


def tiles_of_the_first_pair(T, ci, co):
    """Tiles [256 output x 256 input channels] of pair 0 in its order, as (first output, first input) channel: whole ones while there is one for every pair, then its first
    part of those left over."""
    tm, tn = -(-co // TILE), -(-ci // TILE)
    pairs = T.cuda.get_device_properties(0).multi_processor_count // 2
    whole = tm * tn // pairs * pairs

    def at(t):                     # tiles in blocks of 8 rows of tiles, column by column
        b, q = divmod(t, 8 * tn)
        h = min(8, tm - 8 * b)
        return (8 * b + q % h) * TILE, q // h * TILE
    assert whole >= 2 * pairs and whole < tm * tn
    return [at(t) for t in list(range(0, whole, pairs)) + [whole]]


@pytest.mark.gpu
@pytest.mark.parametrize("add", [0, 1])
@pytest.mark.parametrize("silent_after", [0, 1, 2, 3, 4, 7, 8])
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_nothing_finite_is_left_of_a_pair_that_gave_up(bf16, silent_after, add):
    """Units of one span, several a pair: 4 steps each (the last one is a part of a tile, of 2 or more).  Whole numbers, whose sums are exact."""
    import torch as T
    rows, ci, co = 4 * STEP - 5, 2560, 4096
    dt = T.bfloat16 if bf16 else T.float32
    gen = T.Generator(device="cuda").manual_seed(3)
    x = T.randint(-127, 128, (rows, ci), device="cuda", generator=gen).to(dt)
    dy = T.randint(-8, 9, (rows, co), device="cuda", generator=gen).to(dt)
    ckpt = T.empty(P.asteroid_ckpt8_bytes(rows, ci), device="cuda", dtype=T.uint8)
    P.asteroid_ckpt8_pack(x.data_ptr(), ci, rows, ci, int(bf16), ckpt.data_ptr(), 0)
    need = P.asteroid_ckpt8_linear_wgrad_workspace(rows, ci, co, int(bf16))
    ws = T.zeros(need + 16, device="cuda", dtype=T.uint8)
    dw, db = T.full((co, ci), 3.0, device="cuda"), T.full((co,), 3.0, device="cuda")
    rc = P.asteroid_selftest_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, ci, co, int(bf16), dw.data_ptr(), db.data_ptr(), add, ws.data_ptr(), need,
                                                silent_after)
    assert rc == P.AST_ERR_TIMEOUT
    want_w, want_b = (dy.double().T @ x.double() + 3 * add).float(), (dy.double().sum(0) + 3 * add).float()
    for o, i in tiles_of_the_first_pair(T, ci, co)[silent_after // 4:]:
        want_w[o:o + TILE, i:i + TILE] = float("nan")
        if i == 0:
            want_b[o:o + TILE] = float("nan")
    assert T.equal(T.isnan(dw), T.isnan(want_w)) and T.equal(T.isnan(db), T.isnan(want_b))
    assert T.equal(dw.nan_to_num(7e30), want_w.nan_to_num(7e30)) and T.equal(db.nan_to_num(7e30), want_b.nan_to_num(7e30))
    # the context stays usable, and the call itself gives all of it
    P.asteroid_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, ci, co, int(bf16), dw.data_ptr(), db.data_ptr(), 0, ws.data_ptr(), need, 0)
    assert T.equal(dw.double(), dy.double().T @ x.double()) and T.equal(db.double(), dy.double().sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_no_further_step(bf16):
    import torch as T
    rows, ci, co = 100, 64, 32
    dt = T.bfloat16 if bf16 else T.float32
    x, dy = T.ones(rows, ci, device="cuda", dtype=dt), T.ones(rows, co, device="cuda", dtype=dt)
    ckpt = T.empty(P.asteroid_ckpt8_bytes(rows, ci), device="cuda", dtype=T.uint8)
    P.asteroid_ckpt8_pack(x.data_ptr(), ci, rows, ci, int(bf16), ckpt.data_ptr(), 0)
    need = P.asteroid_ckpt8_linear_wgrad_workspace(rows, ci, co, int(bf16))
    ws, dw = T.zeros(need + 16, device="cuda", dtype=T.uint8), T.empty(co, ci, device="cuda")
    rc = P.asteroid_selftest_ckpt8_linear_wgrad(ckpt.data_ptr(), dy.data_ptr(), co, rows, ci, co, int(bf16), dw.data_ptr(), None, 0, ws.data_ptr(), need, 2)
    assert rc == P.AST_OK and (dw == rows).all()


def test_refusals():
    P.build()
    A = 1 << 20
    good = [A, A, 24, 900, 40, 24, P.AST_F32, A, A, 0, A, 1 << 40, 1]
    for at, v in ((0, 0), (1, 0), (1, A + 4), (2, 25), (3, 0), (5, 23), (7, 0), (12, -1)):
        args = list(good)
        args[at] = v
        assert P.asteroid_selftest_ckpt8_linear_wgrad(*args) == P.AST_ERR_ARG
