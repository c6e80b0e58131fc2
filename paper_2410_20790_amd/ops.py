"""Operators behind the encoder, on torch tensors: group norm with an
activation on channels-last maps, the causal depthwise convolution along time
and the gated linear recurrence, forward and backward (see
include/sparsetem.h for what each computes).

The functions check the tensors, allocate outputs and workspace from torch,
and pass addresses and the current stream of the tensors' device to the
library.  No computation happens here, and no autograd graph is recorded:
the backward calls are the gradients.  Where torch would record one -- a
tensor requires a gradient, outside torch.no_grad() and the methods of a
torch.autograd.Function -- a call is refused, not cut off in silence.

Maps are [n, ..., c] with one or two axes of sites, or views of such; sequences
are [t, b, c].  Channels are adjacent in memory, other strides are free.
Parameters, statistics and recurrent states are float32.
"""

import torch

from . import binding as B

_CODES = {torch.float32: B.ST_F32, torch.float16: B.ST_F16,
          torch.bfloat16: B.ST_BF16}


def _require(ok, msg):
    if not ok:
        raise ValueError(msg)


# The checks below run on every call, beside kernels of a few microseconds:
# their messages are only put together when one fails.

def _code(x, name):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    code = _CODES.get(x.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    return code


# what the library's 32-bit integers hold: ctypes would wrap the rest
_MOST = 0x7fffffff


def _too_large():
    return ValueError("sizes, groups and activations must lie below 2^31")


def _mismatch(name, shape, dtype, device, contiguous=False):
    return ValueError(
        f"{name} must be a {'contiguous ' if contiguous else ''}tensor "
        f"{tuple(shape)}{'' if dtype is None else ' of ' + str(dtype)} on "
        f"{device}")


def _no_graph(name):
    if torch.is_grad_enabled():
        raise ValueError(
            f"{name} requires a gradient, which the operators do not record: "
            "call them under torch.no_grad() or in a torch.autograd.Function "
            "with their backward calls, or detach it")


def _plain(x, shape, dtype, device, name):
    """Address of a contiguous tensor that may be absent."""
    if x is None:
        return None
    try:
        good = (x.shape == shape and x.dtype is dtype and x.device == device
                and x.is_contiguous())
    except AttributeError:
        good = False
    if not good:
        raise _mismatch(name, shape, dtype, device, True)
    if x.requires_grad:
        _no_graph(name)
    return x.data_ptr()


def _out_dtype(x, out, out_dtype):
    if out is not None:
        _require(out_dtype is None or out_dtype == out.dtype,
                 "out and out_dtype disagree")
        out_dtype = out.dtype
    if out_dtype is None or out_dtype == x.dtype:
        return x.dtype
    _require(x.dtype == torch.float32 and out_dtype in _CODES,
             "the output is of the input's type, or of any for float32")
    return out_dtype


def _workspace(x, nbytes):
    """A workspace beside x, and its address."""
    if not nbytes:
        return None, None
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    return ws, ws.data_ptr()


class _On:
    """Makes the tensors' device current for a call, where it is not, and
    gives its current stream."""
    __slots__ = ("index", "back")

    def __init__(self, device):
        self.index, self.back = device.index, None

    def __enter__(self):
        now = torch.cuda.current_device()
        if now != self.index:
            self.back = now
            torch.cuda.set_device(self.index)
        return _stream_of(self.index)

    def __exit__(self, *exc):
        if self.back is not None:
            torch.cuda.set_device(self.back)


def _stream_object(index):
    return torch.cuda.current_stream(index).cuda_stream


# the current stream's handle without a stream object around it (an eighth of
# a small call's time on the host), where torch offers it
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_object)


# -------------------------------------------------------------- group norm

def _map(x, shape, device, name, dtype=None):
    """Reference of a channels-last map of `shape` ([n, ..., c])."""
    try:
        good = (x.shape == shape and x.device == device
                and (dtype is None or x.dtype is dtype))
        st = x.stride()
    except AttributeError:
        good = False
    if not good:
        raise _mismatch(name, shape, dtype, device)
    if st[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{name}: channels must be adjacent")
    if x.requires_grad:
        _no_graph(name)
    if len(shape) == 4:
        return B.st_map_ref(x.data_ptr(), st[0], st[1], st[2])
    return B.st_map_ref(x.data_ptr(), st[0], st[1], st[1])


def _norm_desc(x, groups, act, eps, out_dtype):
    code = _code(x, "x")
    _require(x.dim() in (3, 4),
             "x must be [n, h, w, c] or [n, sites, c]")
    s = x.shape
    h, w = (s[1], s[2]) if len(s) == 4 else (s[1], 1)
    if not (s[0] <= _MOST and h <= _MOST and w <= _MOST and s[-1] <= _MOST
            and -_MOST <= groups <= _MOST and -_MOST <= act <= _MOST):
        raise _too_large()
    return B.st_norm_desc(code, _CODES[out_dtype], s[0], h, w, s[-1], groups,
                          act, eps)


def group_norm(x, groups, gamma=None, beta=None, act=0, eps=1e-5,
               out_dtype=None, out=None):
    """act(group norm of x): returns (y, mean, rstd), the statistics
    [n, groups] for group_norm_backward.  x: [n, h, w, c] or [n, sites, c];
    act: 0 none, 1 ReLU, 2 SiLU; out may be x."""
    dt = _out_dtype(x, out, out_dtype)
    d = _norm_desc(x, groups, act, eps, dt)
    dev, c = x.device, x.shape[-1]
    g = _plain(gamma, (c,), torch.float32, dev, "gamma")
    b = _plain(beta, (c,), torch.float32, dev, "beta")
    xr = _map(x, x.shape, dev, "x")
    y = x.new_empty(x.shape, dtype=dt) if out is None else out
    yr = _map(y, x.shape, dev, "out")
    n = B.st_group_norm_workspace(d, 0)
    stats = x.new_empty((2, d.n, groups), dtype=torch.float32)
    mean, rstd = stats.unbind(0)
    ws, wp = _workspace(x, n)
    with _On(dev) as stream:
        B.st_group_norm(d, xr, g, b, yr, mean.data_ptr(), rstd.data_ptr(),
                        wp, n, stream)
    return y, mean, rstd


def group_norm_backward(dy, x, groups, mean, rstd, gamma=None, beta=None,
                        act=0, out=None, need_params=True):
    """(dx, dgamma, dbeta) of group_norm from dy and the forward call's x,
    statistics and parameters (None, None for the last two unless
    need_params).  out, for dx, may be x, or dy where their types agree."""
    _code(dy, "dy")
    dt = _out_dtype(x, None, dy.dtype)
    d = _norm_desc(x, groups, act, 0.0, dt)
    dev, c = x.device, x.shape[-1]
    g = _plain(gamma, (c,), torch.float32, dev, "gamma")
    b = _plain(beta, (c,), torch.float32, dev, "beta")
    m = _plain(mean, (x.shape[0], groups), torch.float32, dev, "mean")
    r = _plain(rstd, (x.shape[0], groups), torch.float32, dev, "rstd")
    xr = _map(x, x.shape, dev, "x")
    dyr = _map(dy, x.shape, dev, "dy")
    dx = x.new_empty(x.shape, dtype=x.dtype) if out is None \
        else out
    dxr = _map(dx, x.shape, dev, "out", x.dtype)
    dgamma = dbeta = gp = bp = None
    if need_params:
        grads = x.new_empty((2, c), dtype=torch.float32)
        dgamma, dbeta = grads.unbind(0)
        gp, bp = dgamma.data_ptr(), dbeta.data_ptr()
    n = B.st_group_norm_workspace(d, 1)
    ws, wp = _workspace(x, n)
    with _On(dev) as stream:
        B.st_group_norm_backward(d, dyr, xr, m, r, g, b, dxr, gp, bp, wp, n,
                                 stream)
    return dx, dgamma, dbeta


# --------------------------------------------------------------- sequences

def _seq(x, shape, device, name, dtype=None):
    """Reference of a sequence tensor of `shape` ([t, b, c])."""
    try:
        good = (x.shape == shape and x.device == device
                and (dtype is None or x.dtype is dtype))
        st = x.stride()
    except AttributeError:
        good = False
    if not good:
        raise _mismatch(name, shape, dtype, device)
    if st[2] != 1 and shape[2] != 1:
        raise ValueError(f"{name}: channels must be adjacent")
    if x.requires_grad:
        _no_graph(name)
    return B.st_seq_ref(x.data_ptr(), st[0], st[1])


def _seq_desc(x, out_dtype, lengths, reset, reverse, act=0):
    code = _code(x, "the input")
    _require(x.dim() == 3, "sequences are [t, b, c]")
    t, b, c = x.shape
    if not (t <= _MOST and b <= _MOST and c <= _MOST
            and -_MOST <= act <= _MOST):
        raise _too_large()
    ln = _plain(lengths, (b,), torch.int32, x.device, "lengths")
    if reset is not None and reset.dtype == torch.bool:
        reset = reset.view(torch.uint8)
    rs = _plain(reset, (t, b), torch.uint8, x.device, "reset")
    return B.st_seq_desc(code, _CODES[out_dtype], t, b, c, bool(reverse), ln,
                         rs)


def time_conv(x, weight, bias=None, act=0, window=None, lengths=None,
              reset=None, reverse=False, out_dtype=None, out=None,
              window_out=None):
    """act(causal depthwise convolution of x along time): returns (y,
    window_out).  weight: [taps, c], the oldest input's tap first, at most 8
    taps; window: the taps - 1 inputs before the first step, oldest first,
    [taps - 1, b, c] of x's type (zeros if absent).  window_out, the window
    of the next call over the same rows, may be window itself."""
    dt = _out_dtype(x, out, out_dtype)
    d = _seq_desc(x, dt, lengths, reset, reverse, act)
    dev, (t, b, c) = x.device, x.shape
    _require(weight.dim() == 2 and
             1 <= weight.shape[0] <= B.TIME_CONV_MAX_TAPS,
             "weight must be [taps, c] with 1 to 8 taps")
    k = weight.shape[0]
    w = _plain(weight, (k, c), torch.float32, dev, "weight")
    bp = _plain(bias, (c,), torch.float32, dev, "bias")
    win = _plain(window, (k - 1, b, c), x.dtype, dev, "window")
    xr = _seq(x, x.shape, dev, "x")
    if out is None:
        y = x.new_empty((t, b, c), dtype=dt)
        yr = B.st_seq_ref(y.data_ptr(), b * c, c)
    else:
        y, yr = out, _seq(out, x.shape, dev, "out")
    if window_out is None:
        window_out = x.new_empty((k - 1, b, c))
        wo = window_out.data_ptr()
    else:
        wo = _plain(window_out, (k - 1, b, c), x.dtype, dev, "window_out")
    with _On(dev) as stream:
        B.st_time_conv(d, k, act, xr, w, bp, win, yr, wo, None, 0, stream)
    return y, window_out


def time_conv_backward(dy, x, weight, bias=None, act=0, window=None,
                       lengths=None, reset=None, reverse=False,
                       dwindow_out=None, out=None, need_params=True):
    """(dx, dweight, dbias, dwindow) of time_conv from dy and the forward
    call's inputs (None, None for dweight and dbias unless need_params);
    dwindow_out: the gradient with respect to window_out (zero if absent)."""
    _code(dy, "dy")
    dt = _out_dtype(x, None, dy.dtype)
    d = _seq_desc(x, dt, lengths, reset, reverse, act)
    dev, (t, b, c) = x.device, x.shape
    _require(weight.dim() == 2 and
             1 <= weight.shape[0] <= B.TIME_CONV_MAX_TAPS,
             "weight must be [taps, c] with 1 to 8 taps")
    k = weight.shape[0]
    w = _plain(weight, (k, c), torch.float32, dev, "weight")
    bp = _plain(bias, (c,), torch.float32, dev, "bias")
    win = _plain(window, (k - 1, b, c), x.dtype, dev, "window")
    dwo = _plain(dwindow_out, (k - 1, b, c), x.dtype, dev, "dwindow_out")
    xr = _seq(x, x.shape, dev, "x")
    dyr = _seq(dy, x.shape, dev, "dy")
    dx = x.new_empty(x.shape, dtype=x.dtype) if out is None \
        else out
    dxr = _seq(dx, x.shape, dev, "out", x.dtype)
    dwin = x.new_empty((k - 1, b, c))
    dw = db = dwp = dbp = None
    if need_params:
        grads = x.new_empty((k + 1, c), dtype=torch.float32)
        dw, db = grads[:k], grads[k]
        dwp, dbp = dw.data_ptr(), db.data_ptr()
    n = B.st_time_conv_workspace(d, k, 1)
    ws, wp = _workspace(x, n)
    with _On(dev) as stream:
        B.st_time_conv_backward(d, k, act, dyr, xr, w, bp, win, dwo, dxr, dwp,
                                dbp, dwin.data_ptr(), wp, n, stream)
    return dx, dw, db, dwin


def kept_states(t, b, c, device):
    """Room for the states that gated_scan keeps for its backward pass."""
    return torch.empty((-(-t // B.SCAN_STRIDE), b, c), dtype=torch.float32,
                       device=device)


def gated_scan(v, f, o=None, h=None, lengths=None, reset=None, reverse=False,
               out_dtype=None, out=None, h_out=None, save=False):
    """Gated linear recurrence h = sigmoid(f) h + sigmoid(-f) v along time,
    y = h sigmoid(o) (y = h without o): returns (y, h_out), and with save
    the states that gated_scan_backward needs.  h: the state before the
    first step, float32 [b, c] (zeros if absent); h_out, the state after each
    row's last step, may be h itself."""
    dt = _out_dtype(v, out, out_dtype)
    d = _seq_desc(v, dt, lengths, reset, reverse)
    dev, (t, b, c) = v.device, v.shape
    vr = _seq(v, v.shape, dev, "v")
    fr = _seq(f, v.shape, dev, "f", v.dtype)
    orf = None if o is None else _seq(o, v.shape, dev, "o", v.dtype)
    hp = _plain(h, (b, c), torch.float32, dev, "h")
    if out is None:
        y = v.new_empty((t, b, c), dtype=dt)
        yr = B.st_seq_ref(y.data_ptr(), b * c, c)
    else:
        y, yr = out, _seq(out, v.shape, dev, "out")
    if h_out is None:
        h_out = v.new_empty((b, c), dtype=torch.float32)
        ho = h_out.data_ptr()
    else:
        ho = _plain(h_out, (b, c), torch.float32, dev, "h_out")
    states = kept_states(t, b, c, dev) if save else None
    n = B.st_gated_scan_workspace(d, 0)
    ws, wp = _workspace(v, n)
    with _On(dev) as stream:
        B.st_gated_scan(d, vr, fr, orf, hp, yr, ho,
                        states.data_ptr() if save else None, wp, n, stream)
    return (y, h_out, states) if save else (y, h_out)


def gated_scan_backward(dy, v, f, o=None, *, states, dh=None, lengths=None,
                        reset=None, reverse=False, out=None):
    """(dv, df, do, dh) of gated_scan from dy, the forward call's inputs and
    the states it kept (do is None without o).  dh: the gradient with respect
    to h_out (zero if absent); the returned one is with respect to h.  out:
    a tuple (dv, df, do) to write into -- slices of one tensor, say, where v,
    f and o are slices of one."""
    _code(dy, "dy")
    dt = _out_dtype(v, None, dy.dtype)
    d = _seq_desc(v, dt, lengths, reset, reverse)
    dev, (t, b, c) = v.device, v.shape
    vr = _seq(v, v.shape, dev, "v")
    fr = _seq(f, v.shape, dev, "f", v.dtype)
    orf = None if o is None else _seq(o, v.shape, dev, "o", v.dtype)
    dyr = _seq(dy, v.shape, dev, "dy")
    sp = _plain(states, (-(-t // B.SCAN_STRIDE), b, c), torch.float32, dev,
                "states")
    dho = _plain(dh, (b, c), torch.float32, dev, "dh")
    if out is None:
        out = [v.new_empty(v.shape, dtype=v.dtype)
               for _ in range(2 if o is None else 3)]
    _require(len(out) in (2, 3), "out must hold dv, df and do")
    dv, df = out[0], out[1]
    do = out[2] if o is not None and len(out) == 3 else None
    _require(o is None or do is not None, "out must hold dv, df and do")
    dvr = _seq(dv, v.shape, dev, "dv", v.dtype)
    dfr = _seq(df, v.shape, dev, "df", v.dtype)
    dor = None if o is None else _seq(do, v.shape, dev, "do", v.dtype)
    dhi = v.new_empty((b, c), dtype=torch.float32)
    n = B.st_gated_scan_workspace(d, 1)
    ws, wp = _workspace(v, n)
    with _On(dev) as stream:
        B.st_gated_scan_backward(d, dyr, vr, fr, orf, sp, dho, dvr, dfr, dor,
                                 dhi.data_ptr(), wp, n, stream)
    return dv, df, do, dhi
