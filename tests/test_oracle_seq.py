"""Pins of the sequence operators' oracle: cases worked out by hand, and every gradient against differences of the function."""
import numpy as np
import pytest

from oracle import seq as os_


def test_norm_by_hand():
    x = np.array([[[1.0, 3.0, 10.0, 10.0]]])
    y, mean, rstd = os_.norm_fwd(x, np.array([1.0, 2.0, 1.0, 1.0]), np.array([0.0, 0.5, 0.0, -1.0]), 2, 1e-30, False)
    assert np.allclose(mean, [[2.0, 10.0]]) and np.isclose(rstd[0, 0], 1.0)
    assert np.allclose(y[0, 0], [-1.0, 2.5, 0.0, -1.0])


def test_conv_by_hand():
    x = np.array([[[1.0], [2.0], [4.0]]])
    w = np.array([[10.0, 1.0]])
    y, state = os_.conv_fwd(x, w, np.array([0.5]), False)
    assert np.allclose(y[0, :, 0], [1.5, 12.5, 24.5]) and np.allclose(state, [[[4.0]]])
    y, state = os_.conv_fwd(x, w, None, False, lengths=[1], state=np.array([[[3.0]]]))
    assert np.allclose(y[0, :, 0], [31.0, 0.0, 0.0]) and np.allclose(state, [[[1.0]]])


def test_scan_by_hand():
    u, dt = np.array([[[1.0], [3.0]]]), np.array([[[1.0], [2.0]]])
    A, Bm, Cm = np.array([[-np.log(2.0)]]), np.ones((1, 2, 1, 1)), np.array([[[[1.0]], [[10.0]]]])
    y, state = os_.scan_fwd(u, dt, A, Bm, Cm, skip=np.array([100.0]), softplus=False, state=np.array([[[4.0]]]))
    # h = 4/2 + 1 = 3, then 3/4 + 6 = 6.75
    assert np.allclose(y[0, :, 0], [103.0, 367.5]) and np.allclose(state, 6.75)


def differences(f, x, g, eps=1e-6):
    """The gradient of sum(f(x) * g) by central differences."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + eps
        hi = sum((a * b).sum() for a, b in zip(f(), g))
        x[i] = keep - eps
        lo = sum((a * b).sum() for a, b in zip(f(), g))
        x[i] = keep
        out[i] = (hi - lo) / (2 * eps)
    return out


def close(a, b):
    assert np.allclose(a, b, rtol=1e-6, atol=1e-7 * max(1.0, np.abs(b).max(initial=0))), np.abs(a - b).max()


@pytest.mark.parametrize("silu", [False, True])
def test_norm_gradients(silu):
    rng = np.random.default_rng(1)
    x, gamma, beta, dy = (rng.standard_normal(s) for s in ((2, 3, 6), 6, 6, (2, 3, 6)))
    got = os_.norm_bwd(x, gamma, beta, 2, 1e-3, silu, dy)
    for a, grad in zip((x, gamma, beta), got):
        close(grad, differences(lambda: [os_.norm_fwd(x, gamma, beta, 2, 1e-3, silu)[0]], a, [dy]))


@pytest.mark.parametrize("silu, K", [(False, 3), (True, 4), (True, 1)])
def test_conv_gradients(silu, K):
    rng = np.random.default_rng(2)
    B, L, D = 3, 5, 2
    x, w, bias, state, dy, ds = (rng.standard_normal(s) for s in ((B, L, D), (D, K), D, (B, K - 1, D), (B, L, D), (B, K - 1, D)))
    lengths = [5, 0, 2]
    got = os_.conv_bwd(x, w, bias, silu, dy, lengths, state, ds)
    for a, grad in zip((x, w, bias, state), got):
        close(grad, differences(lambda: os_.conv_fwd(x, w, bias, silu, lengths, state), a, [dy, ds]))


@pytest.mark.parametrize("gate, softplus, G", [(True, True, 1), (False, False, 2), (True, False, 2)])
def test_scan_gradients(gate, softplus, G):
    rng = np.random.default_rng(3)
    B, L, D, N = 3, 4, 4, 3
    v = {"u": (B, L, D), "dt": (B, L, D), "A": (D, N), "Bm": (B, L, G, N), "Cm": (B, L, G, N), "skip": (D,), "z": (B, L, D),
         "dt_bias": (D,), "state": (B, D, N)}
    v = {k: rng.standard_normal(s) * 0.7 for k, s in v.items()}
    v["A"] = -np.abs(v["A"])
    if not gate:
        v["z"] = None
    dy, ds = rng.standard_normal((B, L, D)), rng.standard_normal((B, D, N))
    got = os_.scan_bwd(dy=dy, softplus=softplus, lengths=[4, 1, 0], dstate_out=ds, **v)
    for name, a in v.items():
        if a is not None:
            close(got[name], differences(lambda: os_.scan_fwd(softplus=softplus, lengths=[4, 1, 0], **v), a, [dy, ds]))
