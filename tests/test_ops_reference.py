"""The 64-bit forms that the operators are tested against, pinned on the CPU:
gradients against central differences, forms against torch's own layers,
closed cases, and planted mistakes that must show."""

import numpy as np
import pytest
import torch

import ops_reference as R

H = 1e-6


def differences(fn, x, weights):
    """d(sum(weights * fn(x))) / dx by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        for sign in (1, -1):
            x[i] += sign * H
            g[i] += sign * sum((w * v).sum() for w, v in zip(weights, fn(x)))
            x[i] -= sign * H
    return g / (2 * H)


# a central difference of values near one: H^2 of curvature and 2^-53 / H of
# rounding, times the handful of terms that an input reaches
TOL = dict(rtol=1e-6, atol=2e-8)


@pytest.mark.parametrize("a", [R.NONE, R.RELU, R.SILU])
def test_group_norm(a):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(2, 3, 2, 6)) + 0.5
    gamma, beta = rng.normal(size=6), rng.normal(size=6)
    r = R.group_norm(x, 3, gamma, beta, a, 1e-5)
    t = torch.nn.functional.group_norm(
        torch.from_numpy(x).movedim(-1, 1), 3, torch.from_numpy(gamma),
        torch.from_numpy(beta), 1e-5).movedim(1, -1)
    t = {R.NONE: t, R.RELU: t.relu(),
         R.SILU: torch.nn.functional.silu(t)}[a]
    np.testing.assert_allclose(r["y"][0], t.numpy(), rtol=1e-12, atol=1e-12)
    dy = rng.normal(size=x.shape)
    b = R.group_norm_backward(dy, x, 3, r["mean"][0], r["rstd"][0], gamma,
                              beta, a)
    for name, v, fn in (
            ("dx", x, lambda q: (R.group_norm(q, 3, gamma, beta, a,
                                              1e-5)["y"][0],)),
            ("dgamma", gamma, lambda q: (R.group_norm(x, 3, q, beta, a,
                                                      1e-5)["y"][0],)),
            ("dbeta", beta, lambda q: (R.group_norm(x, 3, gamma, q, a,
                                                    1e-5)["y"][0],))):
        np.testing.assert_allclose(b[name][0], differences(fn, v, (dy,)),
                                   err_msg=name, rtol=1e-5, atol=1e-7)


SEQ = [dict(), dict(reverse=True),
       dict(lengths=np.array([5, 0, 3]), reverse=True),
       dict(lengths=np.array([1, 5, 9])),
       dict(reset=np.array([[0, 1, 0], [0, 0, 0], [1, 0, 1], [0, 1, 0],
                            [0, 0, 1]], np.uint8)),
       dict(reset=np.array([[0, 1, 0], [0, 0, 0], [1, 0, 1], [0, 1, 0],
                            [0, 0, 1]], np.uint8), reverse=True,
            lengths=np.array([4, 5, 3]))]


@pytest.mark.parametrize("kw", SEQ)
@pytest.mark.parametrize("k", [1, 3, 4])
def test_time_conv(kw, k):
    rng = np.random.default_rng(2)
    t, b, c = 5, 3, 2
    x, w, bias = (rng.normal(size=(t, b, c)), rng.normal(size=(k, c)),
                  rng.normal(size=c))
    win = rng.normal(size=(k - 1, b, c))
    dy, dwo = rng.normal(size=x.shape), rng.normal(size=win.shape)

    def fwd(x_=x, w_=w, b_=bias, win_=win):
        r = R.time_conv(x_, w_, b_, R.SILU, win_, **kw)
        return r["y"][0], r["window"][0]

    r = R.time_conv_backward(dy, x, w, bias, R.SILU, win, dwindow_out=dwo,
                             **kw)
    for name, v, fn in (("dx", x, lambda q: fwd(x_=q)),
                        ("dweight", w, lambda q: fwd(w_=q)),
                        ("dbias", bias, lambda q: fwd(b_=q)),
                        ("dwindow", win, lambda q: fwd(win_=q))):
        np.testing.assert_allclose(r[name][0], differences(fn, v, (dy, dwo)),
                                   err_msg=name, **TOL)


def test_time_conv_is_conv1d():
    rng = np.random.default_rng(3)
    x, w = rng.normal(size=(9, 2, 4)), rng.normal(size=(3, 4))
    y = R.time_conv(x, w, None, R.NONE)["y"][0]
    t = torch.nn.functional.conv1d(
        torch.from_numpy(x).permute(1, 2, 0), torch.from_numpy(w.T[:, None]),
        padding=2, groups=4)[..., :9].permute(2, 0, 1)
    np.testing.assert_allclose(y, t.numpy(), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("kw", SEQ)
@pytest.mark.parametrize("gate", [True, False])
def test_gated_scan(kw, gate):
    rng = np.random.default_rng(4)
    t, b, c = 5, 3, 2
    v, f = rng.normal(size=(t, b, c)), rng.normal(size=(t, b, c))
    o = rng.normal(size=(t, b, c)) if gate else None
    h, dh = rng.normal(size=(b, c)), rng.normal(size=(b, c))
    dy = rng.normal(size=(t, b, c))

    def fwd(v_=v, f_=f, o_=o, h_=h):
        r = R.gated_scan(v_, f_, o_, h_, **kw)
        return r["y"][0], r["h"][0]

    r = R.gated_scan_backward(dy, v, f, o, h, dh=dh, **kw)
    for name, x, fn in (("dv", v, lambda q: fwd(v_=q)),
                        ("df", f, lambda q: fwd(f_=q)),
                        ("do", o, lambda q: fwd(o_=q)),
                        ("dh", h, lambda q: fwd(h_=q))):
        if x is not None:
            np.testing.assert_allclose(
                r[name][0], differences(fn, x, (dy, dh)), err_msg=name,
                **TOL)


def test_gated_scan_closed_form():
    """A constant gate a and input u: h_s = a^s h + (1 - a^s) u."""
    a = 0.75
    f = np.full((20, 1, 1), np.log(a / (1 - a)))
    r = R.gated_scan(np.full((20, 1, 1), 3.0), f, None, np.full((1, 1), -1.0))
    s = np.arange(1, 21)
    np.testing.assert_allclose(r["y"][0][:, 0, 0], 3 - 4 * a ** s,
                               rtol=1e-12)


def test_planted_mistakes_show():
    """Steps one off, a reset that cuts one step late and a window read in
    the wrong order are all outside the bounds."""
    rng = np.random.default_rng(5)
    x, w = rng.normal(size=(6, 2, 3)), rng.normal(size=(3, 3))
    win = rng.normal(size=(2, 2, 3))
    good, bound = R.time_conv(x, w, None, R.NONE, win)["y"]
    wrong = R.time_conv(x, w, None, R.NONE, win[::-1])["y"][0]
    assert (np.abs(good - wrong) > bound + 2e-3 * np.abs(good)).any()
    f = rng.normal(size=(6, 2, 3))
    reset = np.zeros((6, 2), np.uint8)
    reset[2] = 1
    late = np.roll(reset, 1, 0)
    good, bound = R.gated_scan(x, f, None, reset=reset)["y"]
    for wrong in (R.gated_scan(x, f, None, reset=late)["y"][0],
                  R.gated_scan(x, np.roll(f, 1, 0), None,
                               reset=reset)["y"][0]):
        assert (np.abs(good - wrong) > bound + 2e-2 * np.abs(good)).any()
