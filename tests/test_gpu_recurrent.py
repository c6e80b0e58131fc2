"""The recurrent video model: encoder, time convolution, gated recurrence and
group norm run together, over frames, chunks and both, and the gradients of the
whole head."""

import numpy as np
import pytest
import torch

import ops_reference as R
from ops_reference import f64
from paper_2410_20790_amd import RecurrentHead, RecurrentNet, SparseTemNet
from parity_util import say, to_dev
from workloads import LayerSpec, toy_net, toy_video

pytestmark = pytest.mark.gpu


def make_net(c, dtype="f32", H=24, W=20, max_frames=5):
    net = toy_net(H=H, W=W, dtype=dtype)
    rng = np.random.default_rng(4)
    last = LayerSpec(src=0, c_in=16, c_out=3 * c, k=(1, 1), s=(1, 1),
                     p=(0, 0), act=0, name="vfo",
                     weight=rng.normal(0, 0.3, (3 * c, 16, 1, 1)).astype(
                         np.float32),
                     bias=np.zeros(3 * c, np.float32))
    return SparseTemNet([net.layers[0], last], 1, H, W, 16, dtype,
                        max_frames=max_frames)


def make_head(c, seed=5, **kw):
    head = RecurrentHead(c, **kw)
    g = torch.Generator().manual_seed(seed)
    for p, scale, shift in ((head.weight, 0.5, 0.0), (head.bias, 0.1, 0.0),
                            (head.gamma, 0.2, 1.0), (head.beta, 0.1, 0.0)):
        p.copy_(torch.randn(p.shape, generator=g) * scale + shift)
    return head


@pytest.mark.parametrize("c,taps", [(12, 4), (7, 1), (16, 8)])
def test_frames_and_chunks(c, taps):
    """A reference frame and nine diff frames one by one, and in two chunks
    with a single frame between: the same outputs (the maps agree to 1e-5,
    chunked or not, and a norm of them to 1e-4), and the same memory."""
    say(f"[gpu] recurrent net {c} channels, {taps} taps")
    frames = [to_dev(f, "f32") for f in toy_video(seed=6, n_frames=10, H=24,
                                                  W=20)]
    thr = [0.05, 0.0, 0.0]
    outs, mems = [], []
    for cut in ([1] * 9, [4, 1, 4], [5, 4]):
        m = RecurrentNet(make_net(c), make_head(c, taps=taps))
        ys, at = [m.encode_reference(frames[0])], 1
        for k in cut:
            if k == 1:
                ys.append(m.encode_diff(frames[at], thr))
            else:
                ys.extend(m.encode_chunk(torch.stack(frames[at:at + k]), thr))
            at += k
        outs.append(torch.stack(ys))
        mems.append(type(m.state)(*(q.clone() for q in m.state)))
        if cut == [5, 4]:
            before = m.state.h.clone()
            again = m.encode_reference(frames[0])    # the memory runs on
            assert not torch.equal(again, ys[0])
            assert not torch.equal(before, m.state.h)
            m.reset()
            torch.testing.assert_close(m.encode_reference(frames[0]), ys[0],
                                       rtol=0, atol=0)
        m.close()
    for o, s in zip(outs[1:], mems[1:]):
        torch.testing.assert_close(o, outs[0], rtol=1e-4, atol=1e-4)
        torch.testing.assert_close(s.h, mems[0].h, rtol=1e-4, atol=1e-5)


def chain(head, feats, window, h, reset):
    """The head in 64 bits: (y, backward)."""
    t, n, hh, w, c3 = feats.shape
    c, rows = c3 // 3, n * hh * w
    seq = feats.reshape(t, rows, c3)
    v, f, o = seq[..., :c], seq[..., c:2 * c], seq[..., 2 * c:]
    p = {k: f64(getattr(head, k)) for k in ("weight", "bias", "gamma",
                                            "beta")}
    cv = R.time_conv(v, p["weight"], p["bias"], R.SILU, window, reset=reset)
    u = cv["y"][0]
    sc = R.gated_scan(u, f, o, h, reset=reset)
    z = sc["y"][0].reshape(t * n, hh, w, c)
    nm = R.group_norm(z, head.groups, p["gamma"], p["beta"], head.act,
                      head.eps)

    def back(dy, dwin, dh):
        g = R.group_norm_backward(
            dy.reshape(t * n, hh, w, c), z, head.groups, nm["mean"][0],
            nm["rstd"][0], p["gamma"], p["beta"], head.act)
        s = R.gated_scan_backward(g["dx"][0].reshape(t, rows, c), u, f, o, h,
                                  reset=reset, dh=dh)
        k = R.time_conv_backward(s["dv"][0], v, p["weight"], p["bias"],
                                 R.SILU, window, reset=reset,
                                 dwindow_out=dwin)
        d = np.concatenate([k["dx"][0], s["df"][0], s["do"][0]], -1)
        return d.reshape(feats.shape), dict(
            weight=k["dweight"][0], bias=k["dbias"][0],
            gamma=g["dgamma"][0], beta=g["dbeta"][0]), (k["dwindow"][0],
                                                        s["dh"][0])
    return nm["y"][0].reshape(t, n, hh, w, c), cv["window"][0], \
        sc["h"][0], back


@pytest.mark.parametrize("cuts", [False, True])
def test_gradients_of_the_head(cuts):
    """The whole head, forward and backward, against its 64-bit form: within
    1e-5 of each tensor's largest value (some forty steps of three operators,
    each within a few 2^-24 of values that the norm scales by less than ten),
    and against differences of that form along a random direction."""
    say(f"[gpu] gradients of the head, cuts {cuts}")
    g = torch.Generator().manual_seed(8)
    t, n, hh, w, c = 7, 2, 5, 6, 12
    head = make_head(c, taps=3, groups=3)
    feats = torch.randn(t, n, hh, w, 3 * c, generator=g).cuda()
    rows = n * hh * w
    reset = None
    if cuts:
        reset = (torch.rand(t, rows, generator=g) < 0.2).to(
            torch.uint8).cuda()
    st = head.new_state(rows)
    st.window.copy_(torch.randn(st.window.shape, generator=g))
    st.h.copy_(torch.randn(st.h.shape, generator=g))
    win0, h0 = f64(st.window), f64(st.h)
    y, saved = head.forward(feats, st, reset=reset, save=True)
    rs = None if reset is None else reset.cpu().numpy()
    wy, ww, wh, back = chain(head, f64(feats), win0, h0, rs)

    def near(got, want):
        assert np.abs(f64(got) - want).max() <= 1e-5 * np.abs(want).max()
    near(y, wy)
    near(st.h, wh)
    near(st.window, ww)
    dy = torch.randn(y.shape, generator=g).cuda()
    dst = type(st)(torch.randn(st.window.shape, generator=g).cuda(),
                   torch.randn(st.h.shape, generator=g).cuda())
    df, grads, ds = head.backward(dy, saved, dst)
    wdf, wg, wds = back(f64(dy), f64(dst.window), f64(dst.h))
    near(df, wdf)
    near(ds.window, wds[0])
    near(ds.h, wds[1])
    for k in wg:
        near(grads[k], wg[k])
    # along a direction, differences of the forward form
    d = np.random.default_rng(9).normal(size=feats.shape)
    e = 1e-5
    tot = []
    for s in (e, -e):
        a, b, cc, _ = chain(head, f64(feats) + s * d, win0, h0, rs)
        tot.append((a * f64(dy)).sum() + (b * f64(dst.window)).sum() +
                   (cc * f64(dst.h)).sum())
    slope = (tot[0] - tot[1]) / (2 * e)
    # rounding 1e-16 * |sum| / e and curvature e^2, both below 1e-7 here; the
    # gradient's own 1e-5 of its largest value, over its elements at random
    assert abs((f64(df) * d).sum() - slope) <= 1e-5 * np.abs(wdf).max() * \
        np.sqrt(d.size) * 10 + 1e-6


def test_refusals():
    say("[gpu] refusals of the recurrent model")
    for kw in (dict(channels=0), dict(channels=6, groups=4),
               dict(channels=4, taps=0)):
        with pytest.raises(ValueError):
            RecurrentHead(**kw)
    net = make_net(8)
    with pytest.raises(ValueError, match="channels"):
        RecurrentNet(net, RecurrentHead(9))
    with pytest.raises(ValueError, match="devices"):
        RecurrentNet(net, RecurrentHead(8, device="cpu"))
    head = RecurrentHead(8)
    with pytest.raises(ValueError, match="feats"):
        head.forward(torch.zeros(2, 1, 3, 3, 8, device="cuda"),
                     head.new_state(9))
    with pytest.raises(ValueError, match="window"):
        head.forward(torch.zeros(2, 1, 3, 3, 24, device="cuda"),
                     head.new_state(8))
    net.close()


def test_head_over_frames_equals_the_chunk():
    """The head's outputs for a chunk and for its frames, on maps whose norm
    is summed up in parts: the same bits, and the same memory."""
    say("[gpu] recurrent head, frames and chunk")
    t, n, hh, w, c = 6, 2, 64, 64, 512
    head = make_head(c, groups=32)
    g = torch.Generator().manual_seed(21)
    feats = torch.randn(t, n, hh, w, 3 * c, generator=g).cuda()
    a, b = head.new_state(n * hh * w), head.new_state(n * hh * w)
    y = head.forward(feats, a)
    for i in range(t):
        assert torch.equal(head.forward(feats[i:i + 1], b)[0], y[i])
    assert torch.equal(a.h, b.h) and torch.equal(a.window, b.window)


def test_refused_calls_leave_the_memory():
    """A call that is refused, by whichever of the head's operators, leaves
    the window and the state as they were; parameters that no call takes are
    refused when the head is made."""
    say("[gpu] recurrent head, refused calls")
    for kw in (dict(taps=9), dict(act=3), dict(act=-1), dict(eps=-1e-5),
               dict(eps=float("nan")), dict(eps=float("inf"))):
        with pytest.raises(ValueError):
            RecurrentHead(8, **kw)
    g = torch.Generator().manual_seed(22)
    feats = torch.randn(2, 1, 3, 3, 24, generator=g).cuda()
    spoil = [("gamma", torch.ones(7, device="cuda")),
             ("beta", torch.ones(8)),
             ("gamma", torch.ones(8, device="cuda", requires_grad=True))]
    for name, value in [("h", None)] + spoil:
        head = make_head(8)
        st = head.new_state(9)
        head.forward(feats, st)
        keep = [q.clone() for q in st]
        if name == "h":
            given = st._replace(h=st.h[:, :4])
        else:
            given = st
            setattr(head, name, value)
        with pytest.raises(ValueError):
            head.forward(feats, given)
        assert torch.equal(st.window, keep[0]) and torch.equal(st.h, keep[1])
