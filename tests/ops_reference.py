"""Plain 64-bit forms of the operators behind the encoder, step by step as
their definitions read, each with a bound on what 32-bit arithmetic may add.

Every function returns {name: (value, bound)}: `bound` is the absolute error
that rounded 32-bit steps can reach, without the final rounding to the output
type (half a step, added by `check`).  U = 2^-24 is half a step of a 32-bit
value of magnitude one.  A forget gate is taken to be within SIG = 8 U of
itself, relative (exponential 2 U, sum and quotient 2 U each, the rest spare).
A sigmoid that scales a value once (SiLU, the output gate) is within
SIG + 1.25 U |x| of itself: its exponent x log2 e is rounded to half a step of
itself, U |x| of the exponential, and so is log2 e, U |x| / 4.  The derivative
of SiLU, p (1 + x n), is within SIG of a true one in absolute terms: where such
a factor is off by more, x e^-|x| has made the term small."""

import numpy as np
import torch

U = 2.0 ** -24
SIG = 8 * U
NONE, RELU, SILU = 0, 1, 2
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11,
             torch.bfloat16: 2.0 ** -8}
# below these a type's steps no longer shrink with the value
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -14,
        torch.bfloat16: 2.0 ** -126}


def f64(x):
    return None if x is None else x.detach().double().cpu().numpy()


def check(got, want, bound, what):
    """|got - want| <= half a step of the output's type at the value, plus
    the bound; NaN and infinities agree."""
    assert tuple(got.shape) == tuple(want.shape), (what, got.shape, want.shape)
    g = f64(got)
    h = HALF_STEP[got.dtype]
    bad = np.isnan(want) | np.isinf(want)
    np.testing.assert_array_equal(g[bad], want[bad], err_msg=what)
    g, w = g[~bad], want[~bad]
    b = np.broadcast_to(bound, want.shape)[~bad]
    # the value that is rounded lies within b of the exact one
    tol = b + h * np.maximum(np.abs(w) + b, TINY[got.dtype])
    err = np.abs(g - w)
    assert np.isfinite(g).all(), f"{what}: not finite"
    worst = int(np.argmax(err - tol)) if err.size else 0
    assert not err.size or (err <= tol).all(), (
        f"{what}: off by {err.flat[worst]:.3e}, allowed "
        f"{tol.flat[worst]:.3e}, value {w.flat[worst]:.6e} "
        f"({int((err > tol).sum())} of {err.size})")


def sig(x):
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def once(z, a=SILU):
    """Relative bound of what a sigmoid of z scaled."""
    return SIG + 1.25 * U * np.abs(z) if a == SILU else SIG


def act(z, a):
    if a == RELU:
        return np.maximum(z, 0)
    return z * sig(z) if a == SILU else z


def dact(z, a):
    if a == RELU:
        return (z > 0).astype(z.dtype)
    if a == SILU:
        return sig(z) * (1 + z * sig(-z))
    return np.ones_like(z)


# -------------------------------------------------------------- group norm

def _groups(x, groups):
    """[n, ..., c] -> [n, sites, groups, c / groups]."""
    return x.reshape(x.shape[0], -1, groups, x.shape[-1] // groups)


def group_norm(x, groups, gamma, beta, a, eps):
    v = _groups(x, groups)
    mean = v.mean((1, 3))
    m4 = mean[:, None, :, None]
    var = ((v - m4) ** 2).mean((1, 3))
    rstd = 1 / np.sqrt(var + eps)
    r4 = rstd[:, None, :, None]
    # Values are taken relative to one of the group, which lies within twice
    # the largest deviation `far` of them all.  Sums join in trees of batches:
    # 16 roundings of `far` stand for a mean.  A batch mean off by 8 U far
    # shifts its squared distance from the whole mean by twice that times the
    # distance, whose mean over the batches is a deviation at most: 16 U far
    # rstd of the variance, relative, half of it in rstd; 16 U for the sums.
    far = np.abs(v - m4).max((1, 3))
    e_mean = 16 * U * far
    e_rstd = rstd * (16 * U + 16 * U * far * rstd)
    e_used = e_mean + U * np.abs(mean)   # rounded where it is subtracted
    g = np.ones(x.shape[-1]) if gamma is None else gamma
    b = np.zeros(x.shape[-1]) if beta is None else beta
    xh = ((v - m4) * r4).reshape(x.shape)
    z = xh * g + b
    e_xh = ((e_used[:, None, :, None] + 2 * U * np.abs(v - m4)) * r4 +
            np.abs(v - m4) * e_rstd[:, None, :, None]).reshape(x.shape)
    e_z = np.abs(g) * e_xh + 4 * U * (np.abs(xh * g) + np.abs(b))
    y = act(z, a)
    return {"y": (y, 1.1 * e_z + once(z, a) * np.abs(y)), "mean": (mean, e_mean),
            "rstd": (rstd, e_rstd)}


def group_norm_backward(dy, x, groups, mean, rstd, gamma, beta, a):
    c = x.shape[-1]
    g = np.ones(c) if gamma is None else gamma
    b = np.zeros(c) if beta is None else beta
    v = _groups(x, groups)
    m4, r4 = mean[:, None, :, None], rstd[:, None, :, None]
    xh4 = (v - m4) * r4
    xh = xh4.reshape(x.shape)
    z = xh * g + b
    dz = dy * dact(z, a)
    e_xh = 4 * U * np.abs(xh)
    e_z = np.abs(g) * e_xh + 2 * U * (np.abs(xh * g) + np.abs(b))
    # SiLU's second derivative stays below 1/2
    e_dz = np.abs(dy) * (0.5 * e_z + SIG) if a == SILU else 0 * dz
    d4 = _groups(dz * g, groups)
    e4 = _groups(np.abs(g) * e_dz + 2 * U * np.abs(dz * g), groups)
    m = d4.shape[1] * d4.shape[3]
    s1, s2 = d4.sum((1, 3)) / m, (d4 * xh4).sum((1, 3)) / m
    # a thread adds at most a few hundred values in a row: 256 roundings of
    # the sum of magnitudes bound any order of addition here
    e_s1 = (e4 + 256 * U * np.abs(d4)).sum((1, 3)) / m
    e_s2 = ((e4 + 256 * U * np.abs(d4)) * np.abs(xh4) +
            np.abs(d4) * 4 * U * np.abs(xh4)).sum((1, 3)) / m
    s14, s24 = s1[:, None, :, None], s2[:, None, :, None]
    dx = r4 * (d4 - s14 - xh4 * s24)
    e_dx = r4 * (e4 + e_s1[:, None, :, None] +
                 np.abs(xh4) * e_s2[:, None, :, None] +
                 8 * U * (np.abs(d4) + np.abs(s14) + np.abs(xh4 * s24)))
    ax = tuple(range(x.ndim - 1))
    return {
        "dx": (dx.reshape(x.shape), e_dx.reshape(x.shape)),
        "dgamma": ((dz * xh).sum(ax), ((e_dz + 256 * U * np.abs(dz)) *
                                       np.abs(xh) + np.abs(dz) * e_xh).sum(ax)),
        "dbeta": (dz.sum(ax), (e_dz + 256 * U * np.abs(dz)).sum(ax))}


# --------------------------------------------------------------- sequences

def walk(t, b, lengths, reset, reverse):
    """Per running step: (time of every row, rows that have it, rows that a
    reset cuts before it)."""
    n = np.full(b, t) if lengths is None else np.clip(lengths, 0, t)
    for s in range(t):
        live = s < n
        time = np.where(live, n - 1 - s, s) if reverse else np.full(b, s)
        cut = np.zeros(b, bool)
        if reset is not None:
            cut = live & (reset[time, np.arange(b)] != 0)
        yield time, live, cut


def time_conv(x, w, bias, a, window=None, lengths=None, reset=None,
              reverse=False):
    t, b, c = x.shape
    k = w.shape[0]
    rows = np.arange(b)
    bias = np.zeros(c) if bias is None else bias
    win = (np.zeros((k - 1, b, c)) if window is None else window.copy())
    y, e = np.zeros((t, b, c)), np.zeros((t, b, c))
    for time, live, cut in walk(t, b, lengths, reset, reverse):
        old = np.where(cut[None, :, None], 0, win)
        taps = np.concatenate([old, x[time, rows][None]])
        z = bias + (w[:, None, :] * taps).sum(0)
        e_z = (k + 1) * U * (np.abs(w[:, None, :] * taps).sum(0) +
                             np.abs(bias))
        out = act(z, a)
        y[time[live], rows[live]] = out[live]
        e[time[live], rows[live]] = (1.1 * e_z + once(z, a) * np.abs(out))[live]
        win = np.where(live[None, :, None], taps[1:], win)
    return {"y": (y, e), "window": (win, 0.0)}


def time_conv_backward(dy, x, w, bias, a, window=None, lengths=None,
                       reset=None, reverse=False, dwindow_out=None):
    t, b, c = x.shape
    k = w.shape[0]
    rows = np.arange(b)
    bias = np.zeros(c) if bias is None else bias
    win = np.zeros((k - 1, b, c)) if window is None else window.copy()
    steps, taps_at = list(walk(t, b, lengths, reset, reverse)), []
    for time, live, cut in steps:
        old = np.where(cut[None, :, None], 0, win)
        taps = np.concatenate([old, x[time, rows][None]])
        taps_at.append(taps)
        win = np.where(live[None, :, None], taps[1:], win)
    dwin = (np.zeros((k - 1, b, c)) if dwindow_out is None
            else dwindow_out.copy())
    e_win = np.zeros_like(dwin)
    dx, e_dx = np.zeros((t, b, c)), np.zeros((t, b, c))
    dw, e_dw = np.zeros_like(w), np.zeros_like(w)
    db, e_db = np.zeros(c), np.zeros(c)
    aw = np.abs(w)[:, None, :]
    for (time, live, cut), taps in zip(reversed(steps), reversed(taps_at)):
        l3 = live[None, :, None]
        z = bias + (w[:, None, :] * taps).sum(0)
        e_z = (k + 1) * U * (np.abs(w[:, None, :] * taps).sum(0) +
                             np.abs(bias))
        g = np.where(live[:, None], dy[time, rows], 0)
        dz = g * dact(z, a)
        e_dz = np.abs(g) * (0.5 * e_z + SIG) if a == SILU else 0 * dz
        dtaps = w[:, None, :] * dz
        e_taps = aw * e_dz + (k + 2) * U * np.abs(dtaps)
        dtaps[1:] += np.where(l3, dwin, 0)
        # the sum so far is rounded once more per tap that joins it
        e_taps[1:] += np.where(l3, e_win + 2 * U * np.abs(dwin), 0)
        dx[time[live], rows[live]] = dtaps[k - 1][live]
        e_dx[time[live], rows[live]] = e_taps[k - 1][live]
        dw += (taps * dz).sum(1)
        # any order of at most a few hundred additions in a row
        e_dw += (np.abs(taps) * (e_dz + 256 * U * np.abs(dz))).sum(1)
        db += dz.sum(0)
        e_db += (e_dz + 256 * U * np.abs(dz)).sum(0)
        keep = l3 & ~cut[None, :, None]
        dwin = np.where(keep, dtaps[:-1], np.where(l3, 0, dwin))
        e_win = np.where(keep, e_taps[:-1], np.where(l3, 0, e_win))
    return {"dx": (dx, e_dx), "dweight": (dw, e_dw), "dbias": (db, e_db),
            "dwindow": (dwin, e_win)}


def gated_scan(v, f, o, h=None, lengths=None, reset=None, reverse=False):
    """The bound follows the recurrence: each step adds its own roundings to
    what the decay leaves of the earlier ones, in whatever way steps are
    joined (a product of n gates is off by n such errors, relative)."""
    t, b, c = v.shape
    rows = np.arange(b)
    h = np.zeros((b, c)) if h is None else h.copy()
    mag, e = np.abs(h), np.zeros((b, c))
    y, e_y = np.zeros((t, b, c)), np.zeros((t, b, c))
    states, e_states = [], []
    for s, (time, live, cut) in enumerate(walk(t, b, lengths, reset,
                                               reverse)):
        if s % 16 == 0:
            states.append(np.where(live[:, None], h, np.nan))
            e_states.append(e)
        x, q = v[time, rows], f[time, rows]
        c2, l2 = cut[:, None], live[:, None]
        keep = np.where(c2, 0, sig(q))
        new = keep * h + sig(-q) * x
        add = np.abs(sig(-q) * x)
        e = np.where(l2, keep * e + 2 * SIG * (keep * mag + add), e)
        mag = np.where(l2, keep * mag + add, mag)
        h = np.where(l2, new, h)
        g, e_g = np.ones((b, c)), SIG
        if o is not None:
            g, e_g = sig(o[time, rows]), once(o[time, rows])
        y[time[live], rows[live]] = (h * g)[live]
        e_y[time[live], rows[live]] = (g * (e + 2 * e_g * np.abs(h)))[live]
    if not states:
        states, e_states = np.zeros((0, b, c)), np.zeros((0, b, c))
    return {"y": (y, e_y), "h": (h, e),
            "states": (np.array(states), np.array(e_states))}


def gated_scan_backward(dy, v, f, o, h=None, lengths=None, reset=None,
                        reverse=False, dh=None):
    t, b, c = v.shape
    rows = np.arange(b)
    h = np.zeros((b, c)) if h is None else h.copy()
    mag, e = np.abs(h), np.zeros((b, c))
    steps, at = list(walk(t, b, lengths, reset, reverse)), []
    for time, live, cut in steps:
        x, q = v[time, rows], f[time, rows]
        c2, l2 = cut[:, None], live[:, None]
        was, e_was = np.where(c2, 0, h), np.where(c2, 0, e)
        m_was = np.where(c2, 0, mag)
        keep, write = sig(q), sig(-q)
        e_new = keep * e_was + 2 * SIG * (keep * m_was + np.abs(write * x))
        new = keep * was + write * x
        at.append((was, e_was, new, e_new))
        h, e = np.where(l2, new, h), np.where(l2, e_new, e)
        mag = np.where(l2, keep * m_was + np.abs(write * x), mag)
    d = np.zeros((b, c)) if dh is None else dh.copy()
    m_d, e_d = np.abs(d), np.zeros((b, c))
    out = {n: (np.zeros((t, b, c)), np.zeros((t, b, c)))
           for n in ("dv", "df", "do")}
    for (time, live, cut), (was, e_was, new, e_new) in zip(reversed(steps),
                                                           reversed(at)):
        x, q = v[time, rows], f[time, rows]
        c2, l2 = cut[:, None], live[:, None]
        keep, write = sig(q), sig(-q)
        g = dy[time, rows]
        if o is not None:
            p, n = sig(o[time, rows]), sig(-o[time, rows])
            go, e_go = g * new * p * n, np.abs(g) * p * n * (
                e_new + 3 * SIG * np.abs(new))
            out["do"][0][time[live], rows[live]] = go[live]
            out["do"][1][time[live], rows[live]] = e_go[live]
            g = g * p
        s, e_s = d + g, e_d + 2 * SIG * (m_d + np.abs(g))
        m_s = m_d + np.abs(g)
        gv, e_gv = s * write, write * (e_s + 2 * SIG * np.abs(s))
        span = np.abs(was) + np.abs(x)
        gf = s * (was - x) * keep * write
        e_gf = keep * write * (e_s * np.abs(was - x) + np.abs(s) *
                               (e_was + 2 * SIG * span) +
                               4 * SIG * np.abs(s) * np.abs(was - x))
        for name, val, err in (("dv", gv, e_gv), ("df", gf, e_gf)):
            out[name][0][time[live], rows[live]] = val[live]
            out[name][1][time[live], rows[live]] = err[live]
        pass_on = np.where(c2, 0, keep)
        d = np.where(l2, s * pass_on, d)
        e_d = np.where(l2, pass_on * (e_s + 2 * SIG * m_s), e_d)
        m_d = np.where(l2, m_s * pass_on, m_d)
    out["dh"] = (d, e_d)
    return out
