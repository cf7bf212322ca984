"""Pins of the float64 oracle of the operators over sequences: central differences on every gradient, a convolution and a
scan written out by other means, and masks that leave nothing."""
import numpy as np
import pytest

from oracle import sequence_ops as O


def _differences(f, x, d, h=1e-5):
    """Derivative of the scalar f at x along d, by a fourth-order central difference."""
    return (8 * (f(x + h * d) - f(x - h * d)) - (f(x + 2 * h * d) - f(x - 2 * h * d))) / (12 * h)


def _conv_problem(seed=0, t=7, N=3, D=4, W=4):
    r = np.random.default_rng(seed)
    return dict(x=r.standard_normal((t, N, D)), w=r.standard_normal((D, W)), bias=r.standard_normal(D), s_in=r.standard_normal((N, W - 1, D)),
                lengths=np.array([t, 2, 0]), dy=r.standard_normal((t, N, D)), ds_out=r.standard_normal((N, W - 1, D))), r


@pytest.mark.parametrize("silu", [True, False])
def test_conv_gradients_are_the_differences(silu):
    p, r = _conv_problem()
    out = O.conv(**p, silu=silu)

    def total(**kw):
        q = {**p, **kw}
        o = O.conv(q["x"], q["w"], q["bias"], q["s_in"], q["lengths"], silu)
        return (o["y"] * p["dy"]).sum() + (o["s_out"] * p["ds_out"]).sum()

    for name, grad in (("x", "dx"), ("w", "dw"), ("bias", "dbias"), ("s_in", "ds_in")):
        d = r.standard_normal(p[name].shape)
        got = _differences(lambda v: total(**{name: v}), p[name], d)
        assert abs(got - (out[grad] * d).sum()) < 1e-8 * (1 + abs(got)), name


def test_conv_is_a_convolution_and_rows_without_steps_hand_their_state_on():
    p, _ = _conv_problem()
    out = O.conv(**p, silu=False)
    ext = np.concatenate([p["s_in"][0], p["x"][:, 0]])
    for d in range(4):
        assert np.allclose(out["y"][:, 0, d], np.convolve(ext[:, d], p["w"][d, ::-1], mode="valid") + p["bias"][d])
    assert np.array_equal(out["s_out"][2], p["s_in"][2]) and np.array_equal(out["ds_in"][2], p["ds_out"][2])
    assert not out["y"][2:, 1].any() and not out["y"][:, 2].any()


def _scan_problem(seed=0, t=6, N=3, D=4, S=3, G=2, gate=True):
    r = np.random.default_rng(seed)
    return dict(u=r.standard_normal((t, N, D)), delta=r.standard_normal((t, N, D)) - 1, A=-np.exp(r.standard_normal((D, S))),
                Bm=r.standard_normal((t, N, G * S)), Cm=r.standard_normal((t, N, G * S)), skip=r.standard_normal(D),
                z=r.standard_normal((t, N, D)) if gate else None, bias=r.standard_normal(D), s_in=r.standard_normal((N, D, S)),
                lengths=np.array([t, 1, 0]), dy=r.standard_normal((t, N, D)), ds_out=r.standard_normal((N, D, S)), groups=G), r


@pytest.mark.parametrize("gate,soft", [(True, True), (False, True), (True, False)])
def test_scan_gradients_are_the_differences(gate, soft):
    p, r = _scan_problem(gate=gate)
    if not soft:
        p["delta"] = np.abs(p["delta"])
        p["bias"] = np.abs(p["bias"])
    out = O.scan(**p, soft=soft)

    def total(**kw):
        q = {**p, **kw}
        o = O.scan(**{**q, "dy": None, "ds_out": None}, soft=soft)
        return (o["y"] * p["dy"]).sum() + (o["s_out"] * p["ds_out"]).sum()

    for name, grad in (("u", "du"), ("delta", "ddelta"), ("A", "dA"), ("Bm", "dB"), ("Cm", "dC"), ("skip", "dskip"), ("z", "dz"),
                       ("bias", "ddelta_bias"), ("s_in", "ds_in")):
        if p[name] is None:
            continue
        d = r.standard_normal(p[name].shape)
        got = _differences(lambda v: total(**{name: v}), p[name], d, 1e-4)
        assert abs(got - (out[grad] * d).sum()) < 1e-7 * (1 + abs(got)), name


def test_scan_is_the_sum_over_earlier_inputs():
    p, _ = _scan_problem(gate=False, G=1)
    out = O.scan(**p)
    dt = np.log1p(np.exp(p["delta"] + p["bias"]))[:, 0]
    for k in range(6):
        y = p["skip"] * p["u"][k, 0]
        for j in range(-1, k + 1):
            fed = p["s_in"][0] if j < 0 else (dt[j] * p["u"][j, 0])[:, None] * p["Bm"][j, 0]
            y = y + (p["Cm"][k, 0] * np.exp(p["A"] * dt[j + 1:k + 1].sum(0)[:, None]) * fed).sum(1)
        assert np.allclose(out["y"][k, 0], y)
    assert np.array_equal(out["s_out"][2], p["s_in"][2]) and not out["dB"][1:, 1].any()


def test_distill_gradient_is_the_differences_and_repeated_tokens_add_up():
    r = np.random.default_rng(0)
    R, V, K = 5, 11, 4
    x, v, w = r.standard_normal((R, V)), r.standard_normal((R, K)), r.random(R)
    i = r.integers(0, V, (R, K))
    i[0] = 3                              # one token four times
    i[1, 2:] = -1
    i[2] = -1                             # no entry
    w[3] = 0
    v[4, 1] = -np.inf
    out = O.distill(x, i, v, w, 1.7, 0.3)
    d = r.standard_normal((R, V))
    got = _differences(lambda y: O.distill(y, i, v, w, 1.7, 0.3)["loss"], x, d)
    # the loss has a factor T^2 and the logits one of 1 / T
    assert abs(got - (out["dlogits"] * d).sum()) < 1e-8
    assert out["row_loss"][2] == out["row_loss"][3] == 0 and not out["dlogits"][2:4].any()
    # all of the teacher's weight on one token: cross entropy of that token
    assert np.isclose(out["dlogits"][0, 3], 0.3 * w[0] * 1.7 * (np.exp(x[0, 3] / 1.7) / np.exp(x[0] / 1.7).sum() - 1))
