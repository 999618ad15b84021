"""Stages with 8-bit slots: the layers whose backward reads copies kept beside the tensors (columns of a first layer, the positions that a strided layer reads), pooled features,
SiLU and squeeze-excite behind a BatchNorm; a round in a caller's own graph; replicas of a device group."""
import numpy as np
import pytest

import oracle as O
import oracle.layers as OL
import paper_2408_08015_b200 as P
import stage_inputs as si
from test_gpu_stage_ckpt8 import kept64, layer, run_round, sparse_conv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    import torch
    return torch


def bn(rng, c):
    return np.concatenate([rng.uniform(0.5, 1.5, c), rng.uniform(-0.5, 0.5, c)]).astype(np.float32)


def dense(rng, *shape):
    return (0.1 * rng.standard_normal(int(np.prod(shape)))).astype(np.float32)


def whole_number_nets(rng):
    """name: layers, parameters, h, w.  Every stored value that a backward reads is a whole number up to 127."""
    out = {}
    for name, stride in (("columns", 1), ("columns_strided", 2)):
        n = [layer("conv", 3, 16, -1, 3, stride, 1), layer("bn", 16, 16, 0), layer("relu6", 16, 16, 1), layer("conv", 16, 24, 2)]
        out[name] = (n, np.concatenate([sparse_conv(rng, 16, 3, 3), bn(rng, 16), dense(rng, 24, 16)]), 9, 7)
    n = [layer("conv", 64, 64, -1, 1, 2), layer("bn", 64, 64, 0), layer("relu", 64, 64, 1), layer("conv", 64, 32, 2)]
    out["positions"] = (n, np.concatenate([sparse_conv(rng, 64, 1, 64), bn(rng, 64), dense(rng, 32, 64)]), 9, 6)
    n = [layer("conv", 64, 64, -1, 3, 2, 1), layer("relu", 64, 64, 0), layer("conv", 64, 64, 1, 3, 1, 1), layer("conv", 64, 128, 2, 1, 2)]
    out["strided_dense"] = (n, np.concatenate([sparse_conv(rng, 64, 3, 64), sparse_conv(rng, 64, 3, 64), dense(rng, 128, 64)]), 12, 10)
    # a projection shortcut: both branches strided, a sum whose ReLU is stored
    n = [layer("conv", 64, 64, -1, 3, 2, 1), layer("conv", 64, 64, -1, 1, 2), layer("add", 64, 64, 0, add_from=1), layer("relu", 64, 64, 2), layer("conv", 64, 40, 3)]
    out["projection"] = (n, np.concatenate([sparse_conv(rng, 64, 3, 64), sparse_conv(rng, 64, 1, 64), dense(rng, 40, 64)]), 8, 8)
    n = [layer("dwconv", 40, 40, -1, 5, 2, 2), layer("relu6", 40, 40, 0), layer("dwconv", 40, 40, 1, 7, 1, 3), layer("conv", 40, 16, 2)]
    dw5, dw7 = np.zeros((40, 5, 5), np.float32), np.zeros((40, 7, 7), np.float32)
    dw5[np.arange(40), rng.integers(0, 5, 40), rng.integers(0, 5, 40)] = 1.0
    dw7[np.arange(40), rng.integers(0, 7, 40), rng.integers(0, 7, 40)] = -1.0
    out["depthwise_wide"] = (n, np.concatenate([dw5.ravel(), dw7.ravel(), dense(rng, 16, 40)]), 11, 9)
    n = [layer("conv", 32, 96, -1), layer("relu", 96, 96, 0), layer("gap", 96, 96, 1), layer("linear", 96, 40, 2)]
    out["pooled"] = (n, np.concatenate([sparse_conv(rng, 96, 1, 32), dense(rng, 40, 96), dense(rng, 40)]), 4, 4)
    return out


NAMES = ["columns", "columns_strided", "positions", "strided_dense", "projection", "depthwise_wide", "pooled"]


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", NAMES)
def test_values_that_are_kept_as_they_are_give_the_ordinary_stage_to_the_bit(T, name, bf16, monkeypatch):
    monkeypatch.setenv("ASTEROID_CHECK_GUARDS", "1")
    rng = np.random.default_rng(31)
    net, params, h, w = whole_number_nets(rng)[name]
    B, M = 6, 5
    dt = T.bfloat16 if bf16 else T.float32
    shape = si.out_shape(net, 0, len(net) - 1, h, w)[len(net) - 1]
    # the pooled net's inputs are the same at every position, so that the mean of 16 is a whole number
    xs = [T.from_numpy(rng.integers(-60, 61, (B, 1, 1, net[0].c_in) if name == "pooled" else (B, h, w, net[0].c_in)).astype(np.float32)).cuda().to(dt)
          .expand(B, h, w, net[0].c_in).contiguous() for _ in range(M)]
    dys = [T.from_numpy(rng.integers(-8, 9, (B,) + shape).astype(np.float32)).cuda().to(dt) for _ in range(M)]
    for slots in (1, 3):
        plain = run_round(P, T, P.asteroid_stage_create, net, params, h, w, B, M, slots, bf16, xs, dys, rounds=4)
        kept = run_round(P, T, P.asteroid_stage_create_ckpt8, net, params, h, w, B, M, slots, bf16, xs, dys, rounds=4)
        for r, ((y, dx, g), (py, pdx, pg)) in enumerate(zip(kept, plain)):
            for m in range(M):
                assert bool(T.equal(y[m], py[m])) and bool(T.equal(dx[m], pdx[m])), (name, slots, r, m)
                np.testing.assert_array_equal(g[m], pg[m])


class KeptStage(O.Stage):
    """The stage in 64 bits whose backward reads stored tensors as a checkpoint keeps them (BatchNorm statistics and a squeeze-excite layer's vectors as they are), and the least
    distance of a stored value from a rounding border, in steps."""
    margin = 1.0

    def keep(self, mb):
        val, cache = self.saved[mb]
        fresh = {}
        for i in range(self.first - 1, self.last + 1):
            ly = self.net[i] if i >= self.first else None
            # what the stage stores: its input, outputs of convolutions in front of their BatchNorm, of SiLU, squeeze-excite and pooling
            if ly is None or ly.op in ("conv", "dwconv", "linear", "silu", "se", "gap"):
                v = val[i]
                flat = np.zeros(-(-v.size // 32) * 32)
                flat[:v.size] = v.ravel()
                k, margin = kept64(flat)
                if i != self.last:
                    self.margin = min(self.margin, margin)
                fresh[i] = k[:v.size].reshape(v.shape)
            elif ly.op == "bn":
                mu, var, _ = cache[i]
                xhat = (fresh[ly.src] - mu) / np.sqrt(var + self.eps)
                cache[i] = (mu, var, xhat)
                fresh[i] = self.p[(i, "gamma")] * xhat + self.p[(i, "beta")]
            else:
                fresh[i] = OL.act_forward(ly.op, fresh[ly.src])
        self.saved[mb] = (fresh, cache)


def smooth_net():
    return [layer("conv", 8, 32, -1), layer("bn", 32, 32, 0), layer("silu", 32, 32, 1), layer("se", 32, 32, 2, k=4), layer("conv", 32, 16, 3), layer("bn", 16, 16, 4),
            layer("silu", 16, 16, 5)]


def smooth_case(seed):
    rng = np.random.default_rng(seed)
    net, B = smooth_net(), 3
    params = np.concatenate([dense(rng, 32, 8) * 4, bn(rng, 32), dense(rng, 4, 32) * 2, dense(rng, 4), dense(rng, 32, 4) * 5, dense(rng, 32), dense(rng, 16, 32) * 2, bn(rng, 16)])
    x = rng.standard_normal((B, 2, 2, 8)).astype(np.float32)
    dy = rng.standard_normal((B, 2, 2, 16)).astype(np.float32)
    st = KeptStage(net, 0, len(net) - 1, B, 1, params)
    y = st.forward(0, x)
    st.keep(0)
    return net, params, x, dy, st, y


def test_silu_and_squeeze_excite_behind_a_batchnorm_against_64_bits(T):
    """float32, of inputs whose kept values lie off every rounding border by more than float32 arithmetic moves them: a convolution's sum of up to 32 products by 34 * 2^-24 of its sum of
    magnitudes, some 3 times the largest value, 127 * 3 * 34 * 2^-24 = 0.8e-3 steps; a SiLU or gated value by a BatchNorm more, whose sums of 12 values and division add some
    tens of roundings: twice that.  Gradients pass five such products and two BatchNorms' backwards, whose differences of sums may lose a digit: 5 * 34 * 2^-24 * 10 = 1e-4 of
    their largest entry.  Values read as they were before they were kept would be off by 4e-3."""
    net, params, x, dy, st, y = next(c for c in (smooth_case(s) for s in range(4000)) if c[4].margin > 1.6e-3)
    dx = st.backward(0, dy.astype(np.float64))
    xs, dys = [T.from_numpy(x).cuda()], [T.from_numpy(dy).cuda()]
    got = run_round(P, T, P.asteroid_stage_create_ckpt8, net, params, 2, 2, 3, 1, 1, False, xs, dys)[0]
    assert np.abs(got[0][0].cpu().numpy() - y).max() <= 1e-4 * np.abs(y).max()
    assert np.abs(got[1][0].cpu().numpy() - dx).max() <= 1e-4 * np.abs(dx).max()
    at = 0
    for i, ly in enumerate(net):
        for key in [k for k in st.p if k[0] == i]:
            want = st.g[key].ravel()
            assert np.abs(got[2][0][at:at + want.size] - want).max() <= 1e-4 * np.abs(want).max(), key
            at += want.size
    assert at == params.size


def test_silu_and_squeeze_excite_in_bfloat16_stay_near_the_ordinary_stage(T):
    """A value is kept to half a step of its group, whose largest has 64 or more: some 1 % of an ordinary value.  Gradients that a few kept tensors go into stay within a tenth, in norm."""
    rng = np.random.default_rng(3)
    net, B, M = smooth_net(), 8, 3
    params = smooth_case(3)[1]
    xs = [T.from_numpy(rng.standard_normal((B, 9, 7, 8)).astype(np.float32)).cuda().bfloat16() for _ in range(M)]
    dys = [T.from_numpy(rng.standard_normal((B, 9, 7, 16)).astype(np.float32)).cuda().bfloat16() for _ in range(M)]
    plain = run_round(P, T, P.asteroid_stage_create, net, params, 9, 7, B, M, 2, True, xs, dys)[0]
    kept = run_round(P, T, P.asteroid_stage_create_ckpt8, net, params, 9, 7, B, M, 2, True, xs, dys)[0]
    for m in range(M):
        assert T.equal(plain[0][m], kept[0][m])
        for a, b in ((plain[1][m].double().cpu().numpy().ravel(), kept[1][m].double().cpu().numpy().ravel()), (plain[2][m], kept[2][m])):
            assert np.linalg.norm(a - b) <= 0.1 * np.linalg.norm(a)
            assert not np.array_equal(a, b)


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", ["positions", "pooled"])
def test_a_round_in_a_callers_graph(T, name, bf16):
    """Rounds of 4 micro-batches on 2 slots, call by call and replayed from one capture: the same state to the bit."""
    rng = np.random.default_rng(7)
    net, params, h, w = whole_number_nets(rng)[name]
    B, M, K, dt = 4, 4, 2, T.bfloat16 if bf16 else T.float32
    shape = si.out_shape(net, 0, len(net) - 1, h, w)[len(net) - 1]
    xs = [T.from_numpy(rng.standard_normal((B, h, w, net[0].c_in)).astype(np.float32)).cuda().to(dt) for _ in range(M)]
    dys = [T.from_numpy(rng.standard_normal((B,) + shape).astype(np.float32)).cuda().to(dt) for _ in range(M)]
    ys, dxs = [T.empty((B,) + shape, device="cuda", dtype=dt) for _ in range(M)], [T.empty_like(x) for x in xs]

    def a_round(hdl, stream):
        for m in range(M + K - 1):
            if m < M:
                P.asteroid_stage_forward(hdl, m, xs[m].data_ptr(), ys[m].data_ptr(), stream)
            if m >= K - 1:
                P.asteroid_stage_backward(hdl, m - K + 1, dys[m - K + 1].data_ptr(), dxs[m - K + 1].data_ptr(), stream)
                P.asteroid_stage_accumulate(hdl, m - K + 1, stream)
        P.asteroid_stage_step(hdl, 0.05, 0.9, stream)

    results = []
    for graphed in (False, True):
        hdl = P.asteroid_stage_create_ckpt8(net, 0, len(net) - 1, h, w, B, M, dtype=int(bf16), slots=K, need_input_grad=1)
        try:
            P.asteroid_stage_import_state(hdl, np.ascontiguousarray(params, np.float32), None)
            T.cuda.synchronize()
            if graphed:
                g = T.cuda.CUDAGraph()
                with T.cuda.graph(g):             # the stage's first use
                    a_round(hdl, T.cuda.current_stream().cuda_stream)
                for _ in range(3):
                    g.replay()
            else:
                for _ in range(3):
                    a_round(hdl, 0)
            T.cuda.synchronize()
            w1, v1 = np.empty(params.size, np.float32), np.empty(params.size, np.float32)
            P.asteroid_stage_export_state(hdl, params=w1, momentum=v1)
            results.append((w1, v1, [d.clone() for d in dxs], [y.clone() for y in ys]))
        finally:
            P.asteroid_stage_destroy(hdl)
    a, b = results
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[1], b[1])
    assert not np.array_equal(a[0], params)
    assert all(T.equal(p, q) for p, q in zip(a[2] + a[3], b[2] + b[3]))


def test_replicas_of_a_device_group(T):
    """Shares of 5 and 3 of each micro-batch on two replicas, one after the other, their gradient arenas summed by share: the ordinary group's update to the bit."""
    from paper_2408_08015_b200 import dp
    rng = np.random.default_rng(9)
    net, params, h, w = whole_number_nets(rng)["pooled"]
    shares, M, x0 = (5, 3), 2, 0
    xs = [T.from_numpy(rng.integers(-60, 61, (8, 1, 1, 32)).astype(np.float32)).cuda().expand(8, h, w, 32).contiguous() for _ in range(M)]
    dys = [T.from_numpy(rng.integers(-8, 9, (8, 1, 1, 40)).astype(np.float32)).cuda() for _ in range(M)]
    states = []
    for create in (P.asteroid_stage_create, P.asteroid_stage_create_ckpt8):
        hs, lo, hold = [], 0, []
        try:
            for n in shares:
                hdl = create(net, 0, 3, h, w, n, M, dtype=P.AST_F32, slots=M, need_input_grad=1)
                hs.append(hdl)
                P.asteroid_stage_import_state(hdl, np.ascontiguousarray(params, np.float32), None)
                for m in range(M):
                    x, dy = xs[m][lo:lo + n].contiguous(), dys[m][lo:lo + n].contiguous()
                    y, dx = T.empty_like(dy), T.empty_like(x)
                    hold += [x, dy, y, dx]
                    P.asteroid_stage_forward(hdl, m, x.data_ptr(), y.data_ptr(), 0)
                    P.asteroid_stage_backward(hdl, m, dy.data_ptr(), dx.data_ptr(), 0)
                    P.asteroid_stage_accumulate(hdl, m, 0)
                lo += n
            T.cuda.synchronize()
            arenas = [dp.grad_tensor(hdl) for hdl in hs]
            total = sum(t * (n / 8) for t, n in zip(arenas, shares))
            for t in arenas:
                t.copy_(total)
            T.cuda.synchronize()
            got = []
            for hdl in hs:
                P.asteroid_stage_step(hdl, 0.05, 0.9, 0)
                w1 = np.empty(params.size, np.float32)
                P.asteroid_stage_export_state(hdl, params=w1)
                got.append(w1)
            np.testing.assert_array_equal(got[0], got[1])
            states.append(got[0])
        finally:
            for hdl in hs:
                P.asteroid_stage_destroy(hdl)
    np.testing.assert_array_equal(states[0], states[1])
    assert not np.array_equal(states[0], params)
