"""SiLU where its sigmoid is no normal number any more but its value still is one: x * exp(x) from -80 to where it vanishes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_silu_far_left(bf16):
    """The sigmoid is a multiple of 2^-149, of which its exponential (2 units in the last place) and its product make up to three, times |x| <= 108.  float32: an exponential, a sum, a
    quotient and products, all within 2^-19 beside that.  bfloat16: the exponent of 2, up to 32 + 1.45 * 108 < 192 and so rounded to 2^-17, and its factor's rounding, 2^-25 of it,
    move the exponential by less than 2^-15; the result rounds to 2^-8 of itself or half of 2^-133."""
    import torch as T
    import paper_2408_08015_b200 as P
    dt = T.bfloat16 if bf16 else T.float32
    x = T.linspace(-108.0, -80.0, 64 * 32, device="cuda").to(dt).view(64, 32)
    y, dx, kept, dy = T.empty_like(x), T.empty_like(x), T.empty_like(x), T.full_like(x, 1.5)
    ckpt = T.empty(P.asteroid_ckpt8_bytes(64, 32), device="cuda", dtype=T.uint8)
    P.asteroid_ckpt8_act_forward(P.AST_SILU, x.data_ptr(), 32, 64, 32, int(bf16), y.data_ptr(), 32, ckpt.data_ptr(), 0)
    P.asteroid_ckpt8_act_backward(P.AST_SILU, ckpt.data_ptr(), dy.data_ptr(), 32, 64, 32, int(bf16), dx.data_ptr(), 32, 0)
    P.asteroid_ckpt8_unpack(ckpt.data_ptr(), 64, 32, int(bf16), kept.data_ptr(), 32, 0)
    xh, kh = x.double().cpu().numpy(), kept.double().cpu().numpy()
    rel = 2.0 ** -8 + 2.0 ** -15 if bf16 else 2.0 ** -19
    step = 3 * 108 * 2.0 ** -149 + (2.0 ** -134 if bf16 else 2.0 ** -149)
    ref = xh / (1 + np.exp(-xh))
    assert (np.abs(ref) > 32 * step).sum() > 500
    assert (np.abs(y.double().cpu().numpy() - ref) <= rel * np.abs(ref) + step).all()
    ref = 1.5 * (1 + kh / (1 + np.exp(kh))) / (1 + np.exp(-kh))
    assert (np.abs(dx.double().cpu().numpy() - ref) <= rel * np.abs(ref) + 3 * step).all()
