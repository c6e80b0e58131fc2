"""A recurrent video model: the diff encoder followed by a recurrent head, as
the paper's CRNN is a CNN encoder followed by a recurrent part.

The head works on the encoder's maps in place, every site a row of its own:
the net's last layer emits 3 c channels, [v | f | o]; v passes a causal
convolution along time with SiLU, f and o are the forget and output gates of
the gated recurrence, and a group norm per frame with an activation ends it.
Frames taken one by one, in chunks, or both in turn give the same outputs: the
window and the state are kept from call to call.
"""

from typing import NamedTuple, Optional

import torch

from . import binding as B
from . import ops
from .net import SparseTemNet


class HeadState(NamedTuple):
    """The head's memory of the frames so far: the last taps - 1 inputs of the
    convolution, [taps - 1, rows, c], and the recurrent state, [rows, c]."""
    window: torch.Tensor
    h: torch.Tensor


class Saved(NamedTuple):
    """What RecurrentHead.backward needs of a forward call."""
    feats: torch.Tensor
    reset: Optional[torch.Tensor]
    window: torch.Tensor
    u: torch.Tensor
    z: torch.Tensor
    states: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor


class RecurrentHead:
    """Parameters and calls of the head for maps of 3 * channels channels:
    weight [taps, channels] and bias [channels] of the convolution, gamma and
    beta [channels] of the norm, all float32 on `device`.  act: the activation
    behind the norm (0 none, 1 ReLU, 2 SiLU)."""

    def __init__(self, channels: int, taps: int = 4, groups: int = 1,
                 act: int = 2, eps: float = 1e-5, device="cuda"):
        if channels < 1 or taps < 1 or groups < 1 or channels % groups:
            raise ValueError("channels and taps must be positive, and groups "
                             "must divide the channels")
        if taps > B.TIME_CONV_MAX_TAPS:
            raise ValueError(f"taps must not exceed {B.TIME_CONV_MAX_TAPS}")
        if act not in (0, 1, 2):
            raise ValueError("act must be 0 (none), 1 (ReLU) or 2 (SiLU)")
        if not 0 <= eps < float("inf"):
            raise ValueError("eps must be finite and not negative")
        self.channels, self.taps, self.groups = channels, taps, groups
        self.act, self.eps = act, eps
        dev = torch.device(device)
        # the newest frame alone at first
        self.weight = torch.zeros(taps, channels, device=dev)
        self.weight[-1] = 1.0
        self.bias = torch.zeros(channels, device=dev)
        self.gamma = torch.ones(channels, device=dev)
        self.beta = torch.zeros(channels, device=dev)

    def new_state(self, rows: int, dtype=torch.float32) -> HeadState:
        """The memory before any frame, for maps of `rows` sites (images
        times height times width) of `dtype`."""
        dev = self.weight.device
        return HeadState(
            torch.zeros(self.taps - 1, rows, self.channels, dtype=dtype,
                        device=dev),
            torch.zeros(rows, self.channels, device=dev))

    def _split(self, feats):
        c = self.channels
        if feats.dim() != 5 or feats.shape[-1] != 3 * c:
            raise ValueError(f"feats must be [t, n, h, w, {3 * c}]")
        # one row for each site; views of the encoder's maps
        t, n, h, w, _ = feats.shape
        seq = feats.reshape(t, n * h * w, 3 * c)
        return seq[..., :c], seq[..., c:2 * c], seq[..., 2 * c:]

    def _check(self, feats, state):
        """What the operators would refuse once the first of them has moved
        the window on."""
        t, n, h, w, _ = feats.shape
        c, dev, f32 = self.channels, self.weight.device, torch.float32
        ops._plain(state.window, (self.taps - 1, n * h * w, c), feats.dtype,
                   dev, "window")
        ops._plain(state.h, (n * h * w, c), f32, dev, "h")
        ops._plain(self.gamma, (c,), f32, dev, "gamma")
        ops._plain(self.beta, (c,), f32, dev, "beta")

    def forward(self, feats, state: HeadState, reset=None, save=False):
        """y [t, n, h, w, c] of the maps feats [t, n, h, w, 3 c]; `state`
        moves on in place (a call that is refused leaves it as it was).
        reset: uint8 [t, rows], non-zero where a row forgets the frames before
        (a cut).  With save: (y, Saved)."""
        v, f, o = self._split(feats)
        t, n, h, w, _ = feats.shape
        self._check(feats, state)
        before = state.window.clone() if save else None
        u, _ = ops.time_conv(v, self.weight, self.bias, act=2,
                             window=state.window, window_out=state.window,
                             reset=reset)
        z, _, *kept = ops.gated_scan(u, f, o, h=state.h, h_out=state.h,
                                     reset=reset, save=save)
        z = z.view(t * n, h, w, self.channels)
        y, mean, rstd = ops.group_norm(z, self.groups, self.gamma, self.beta,
                                       act=self.act, eps=self.eps)
        y = y.view(t, n, h, w, self.channels)
        if not save:
            return y
        return y, Saved(feats, reset, before, u, z, kept[0], mean, rstd)

    def backward(self, dy, saved: Saved, dstate: Optional[HeadState] = None):
        """Gradients of a saved forward call: (dfeats, parameters, state), the
        parameters' as a dict by name, the state's with respect to the
        memory before the call; dstate: those with respect to the memory
        after it (zero if absent)."""
        t, n, h, w, _ = saved.feats.shape
        c = self.channels
        dz, dgamma, dbeta = ops.group_norm_backward(
            dy.reshape(t * n, h, w, c), saved.z, self.groups, saved.mean,
            saved.rstd, self.gamma, self.beta, act=self.act)
        v, f, o = self._split(saved.feats)
        dfeats = torch.empty_like(saved.feats,
                                  memory_format=torch.contiguous_format)
        gv, gf, go = self._split(dfeats)
        du = torch.empty_like(saved.u)
        _, _, _, dh = ops.gated_scan_backward(
            dz.view(t, n * h * w, c), saved.u, f, o, states=saved.states,
            dh=None if dstate is None else dstate.h, reset=saved.reset,
            out=(du, gf, go))
        _, dweight, dbias, dwindow = ops.time_conv_backward(
            du, v, self.weight, self.bias, act=2, window=saved.window,
            dwindow_out=None if dstate is None else dstate.window,
            reset=saved.reset, out=gv)
        return dfeats, dict(weight=dweight, bias=dbias, gamma=dgamma,
                            beta=dbeta), HeadState(dwindow, dh)


class RecurrentNet:
    """A SparseTemNet whose last layer emits 3 * head.channels channels, and a
    RecurrentHead: the encoder's calls, with the head's output [n, h, w, c]
    per frame in place of the maps.  The head's memory runs on from chunk to
    chunk (reset() clears it); the encoder restarts at every reference
    frame."""

    def __init__(self, net: SparseTemNet, head: RecurrentHead):
        if net.out_shape[3] != 3 * head.channels:
            raise ValueError(f"the net emits {net.out_shape[3]} channels, the "
                             f"head takes {3 * head.channels}")
        if head.weight.device != net.device:
            raise ValueError("net and head are on different devices")
        self.net, self.head = net, head
        n, h, w, _ = net.out_shape
        self.state = head.new_state(n * h * w)

    def reset(self):
        """Forget all frames."""
        self.state.window.zero_()
        self.state.h.zero_()

    def encode_reference(self, frame):
        return self.head.forward(self.net.encode_reference(frame)[None],
                                 self.state)[0]

    def encode_diff(self, frame, thr):
        return self.head.forward(self.net.encode_diff(frame, thr)[None],
                                 self.state)[0]

    def encode_chunk(self, frames, thr):
        """frames [t, n, H, W, C]; thr as SparseTemNet.encode_chunk."""
        return self.head.forward(self.net.encode_chunk(frames, thr),
                                 self.state)

    def close(self):
        self.net.close()
