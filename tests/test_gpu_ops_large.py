"""The operators behind the encoder at sizes that take other ways through them:
images by the batch, inputs that the caches cannot hold, and gradients of more
rows than the blocks of a launch."""

import pytest
import torch

import ops_reference as R
from ops_reference import f64
from paper_2410_20790_amd import ops
from parity_util import say
from test_gpu_ops import axes, compare, dev, rnd

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def big(seed, *shape, dtype=F32, shift=0.0):
    """Drawn on the device: these are too many for the host."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) + shift).to(dtype)


@pytest.mark.parametrize("t,b,c,k,dtype", [
    (9, 2100, 512, 4, F32), (9, 700, 515, 4, BF16), (40, 1100, 260, 5, F16),
    (17, 2500, 300, 2, F32)])
@pytest.mark.parametrize("kind", ["", "lr", "b", "lrb"])
def test_conv_gradients_of_many_rows(t, b, c, k, dtype, kind):
    """More rows and tiles than a launch has blocks: every thread takes several
    in turn, and their parameters' sums go on."""
    say(f"[gpu] time conv, gradients of {b} rows {t} {c} {k} {dtype} {kind!r}")
    ln, rs, rev = axes(kind, t, b)
    kw = dict(lengths=dev(ln), reset=dev(rs), reverse=rev)
    ref = dict(lengths=ln, reset=rs, reverse=rev)
    x, w, bias = rnd(211, t, b, c, dtype=dtype), rnd(212, k, c), rnd(213, c)
    wi, dy = (rnd(214 + i, n, b, c, dtype=dtype)
              for i, n in enumerate((k - 1, t)))
    dwo = rnd(216, k - 1, b, c, dtype=dtype)
    got = ops.time_conv_backward(dy, x, w, bias, act=2, window=wi,
                                 dwindow_out=dwo, **kw)
    compare(dict(zip(("dx", "dweight", "dbias", "dwindow"), got)),
            R.time_conv_backward(f64(dy), f64(x), f64(w), f64(bias), R.SILU,
                                 f64(wi), dwindow_out=f64(dwo), **ref), kind)


@pytest.mark.parametrize("shape,groups,pair", [
    ((5, 256, 256, 512), 32, (BF16, BF16)),
    ((5, 250, 260, 256), 1, (F32, F32)),
    ((3, 300, 290, 257), 257, (F32, F16))])
def test_norm_of_batches(shape, groups, pair):
    """Images that are summed up and finished by the batch, the last batch a
    part of one: the same bits as one by one, also in place; one of them, and
    the parameters' gradients, against 64 bits."""
    say(f"[gpu] group norm of batches {shape} / {groups} {pair}")
    n, c = shape[0], shape[-1]
    x, dy = big(221, *shape, dtype=pair[0], shift=0.5), big(222, *shape,
                                                            dtype=pair[1])
    gm, bt = rnd(223, c, shift=1.0), rnd(224, c)
    y, mean, rstd = ops.group_norm(x, groups, gm, bt, act=2,
                                   out_dtype=pair[1])
    dx, dg, db = ops.group_norm_backward(dy, x, groups, mean, rstd, gm, bt,
                                         act=2)
    for i in range(n):
        s = slice(i, i + 1)
        one = ops.group_norm(x[s], groups, gm, bt, act=2, out_dtype=pair[1])
        for p, q in zip(one, (y, mean, rstd)):
            assert torch.equal(p, q[s]), i
        assert torch.equal(ops.group_norm_backward(
            dy[s], x[s], groups, mean[s], rstd[s], gm, bt, act=2)[0],
            dx[s]), i
    sums = torch.zeros(4, c, dtype=torch.float64, device="cuda")
    for i in range(n):
        v = x[i].double().reshape(-1, groups, c // groups)
        m = v.mean((0, 2), keepdim=True)
        r = ((v - m) ** 2).mean((0, 2), keepdim=True).add(1e-5).rsqrt()
        if i == n // 2:
            # rounded at the end, after sums of thousands: far inside 2^-20
            torch.testing.assert_close(mean[i], m.flatten().float(),
                                       rtol=2 ** -20, atol=2 ** -20)
            torch.testing.assert_close(rstd[i], r.flatten().float(),
                                       rtol=2 ** -20, atol=0)
        # from the statistics that the backward call is given
        m, r = (q[i].double()[None, :, None] for q in (mean, rstd))
        xh = ((v - m) * r).reshape(-1, c)
        z = xh * gm.double() + bt.double()
        p = torch.sigmoid(z)
        dz = dy[i].double().reshape(-1, c) * p * (1 + z * (1 - p))
        sums[0] += (dz * xh).sum(0)
        sums[1] += dz.sum(0)
        sums[2] += (dz * xh).abs().sum(0)
        sums[3] += dz.abs().sum(0)
        if i == n // 2:
            # mean and rstd off by 2^-20 of a deviation each move z by gamma
            # (below 4) times 2^-20 (1 + |z|), y by 1.1 of that
            half = R.HALF_STEP[pair[1]]
            err = (y[i].double().reshape(-1, c) - z * p).abs()
            assert (err <= half * (z * p).abs() + 2.0 ** -18 *
                    (1 + z.abs()) + 2.0 ** -25).all()
    # any order of at most a few hundred additions in a row, and the
    # derivative's own error
    u = 300 * R.U
    assert ((dg.double() - sums[0]).abs() <= u * sums[2]).all()
    assert ((db.double() - sums[1]).abs() <= u * sums[3]).all()
    if pair[0] == pair[1]:
        z = x.clone()
        ops.group_norm(z, groups, gm, bt, act=2, out=z)
        assert torch.equal(z, y)
        z = x.clone()
        got = ops.group_norm_backward(dy, z, groups, mean, rstd, gm, bt,
                                      act=2, out=z)
        for p, q in zip(got, (dx, dg, db)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("t,b,c,dtype", [
    (9, 1300, 2048, F32),        # walked
    (1000, 64, 1024, BF16),      # split along time
    (33, 2200, 1024, F16)])      # walked, more than 32 steps
@pytest.mark.parametrize("kind", ["", "lrb"])
def test_scan_beyond_the_caches(t, b, c, dtype, kind):
    """Inputs larger than the caches, whose loads go past them: the same bits
    as a part of their rows or channels alone; some against 64 bits."""
    say(f"[gpu] gated scan beyond the caches {t} {b} {c} {dtype} {kind!r}")
    ln, rs, rev = axes(kind, t, b)
    v, o, dy = (big(231 + i, t, b, c, dtype=dtype) for i in range(3))
    f = big(234, t, b, c, dtype=dtype, shift=3.0)
    h, dh = big(235, b, c), big(236, b, c)
    kw = dict(lengths=dev(ln), reset=dev(rs), reverse=rev)
    y, ho, st = ops.gated_scan(v, f, o, h=h, save=True, **kw)
    back = ops.gated_scan_backward(dy, v, f, o, states=st, dh=dh, **kw)
    # walked rows keep their bits in any part; split ones in rows
    part = slice(0, 40), slice(64, 128)
    if t > 32:
        part = slice(0, 40 if t > 500 else b), slice(0, c)
    r, q = part
    k2 = dict(lengths=None if ln is None else dev(ln[r].copy()),
              reset=None if rs is None else dev(rs[:, r].copy()), reverse=rev)
    if (r.stop - r.start, q.stop - q.start) != (b, c):
        ins = [a[:, r, q] for a in (v, f, o)]
        hp, dp = h[r, q].contiguous(), dh[r, q].contiguous()
        y2, h2, s2 = ops.gated_scan(*ins, h=hp, save=True, **k2)
        assert torch.equal(y2, y[:, r, q]) and torch.equal(h2, ho[r, q])
        got = ops.gated_scan_backward(
            dy[:, r, q], *ins, states=st[:, r, q].contiguous(), dh=dp, **k2)
        for a, w in zip(got, back):
            assert torch.equal(a, w[..., r, q])
    # rows of every length, channels at both ends
    for cs in (slice(0, 8), slice(c - 8, c)):
        rows = slice(0, 12)
        sub = [f64(a[:, rows, cs]) for a in (v, f, o)]
        k3 = dict(lengths=None if ln is None else ln[rows],
                  reset=None if rs is None else rs[:, rows], reverse=rev)
        want = R.gated_scan(*sub, f64(h[rows, cs]), **k3)
        want.pop("states")
        compare(dict(y=y[:, rows, cs], h=ho[rows, cs]), want, "beyond")
        want = R.gated_scan_backward(f64(dy[:, rows, cs]), *sub,
                                     f64(h[rows, cs]),
                                     dh=f64(dh[rows, cs]), **k3)
        compare({n: a[..., rows, cs] for n, a in
                 zip(("dv", "df", "do", "dh"), back)}, want, "beyond, back")


def test_norm_of_more_images_than_a_grid():
    """Tiny images, more than one launch has blocks for."""
    say("[gpu] group norm of more images than a grid")
    n, c, groups = (1 << 20) + 70001, 8, 2
    x, dy = big(241, n, 1, 2, c), big(242, n, 1, 2, c)
    gm, bt = rnd(243, c, shift=1.0), rnd(244, c)
    y, mean, rstd = ops.group_norm(x, groups, gm, bt, act=2)
    dx, dg, db = ops.group_norm_backward(dy, x, groups, mean, rstd, gm, bt,
                                         act=2)
    for s in (slice(0, 500), slice((1 << 20) - 300, (1 << 20) + 300),
              slice(n - 500, n)):
        want = R.group_norm(f64(x[s]), groups, f64(gm), f64(bt), R.SILU, 1e-5)
        compare(dict(y=y[s], mean=mean[s], rstd=rstd[s]), want, "images")
        want = R.group_norm_backward(
            f64(dy[s]), f64(x[s]), groups, f64(mean[s]), f64(rstd[s]),
            f64(gm), f64(bt), R.SILU)
        compare(dict(dx=dx[s]), want, "images, back")
    # the parameters' gradients, in f64 on the device
    m, r = (q.double().repeat_interleave(c // groups, 1)[:, None, None]
            for q in (mean, rstd))
    xh = (x.double() - m) * r
    z = xh * gm.double() + bt.double()
    p = torch.sigmoid(z)
    dz = dy.double() * p * (1 + z * (1 - p))
    for got, v in ((dg, dz * xh), (db, dz)):
        err = (got.double() - v.sum((0, 1, 2))).abs()
        assert (err <= 16 * R.U * v.abs().sum((0, 1, 2))).all()
