"""What the operators behind the encoder refuse, and their workspaces, on the
host: every call here returns before anything is launched."""

import ctypes

import pytest
import torch

from paper_2410_20790_amd import binding as B
from paper_2410_20790_amd import ops

A = 1 << 20            # addresses nothing is read from
BAD, SMALL = B.ST_ERR_INVALID_ARG, B.ST_ERR_WORKSPACE


def refused(status, word, fn, *a, **k):
    with pytest.raises(B.StError) as e:
        fn(*a, **k)
    assert e.value.status == status
    assert word in str(e.value), str(e.value)


def norm_desc(**kw):
    d = dict(dtype=0, out_dtype=0, n=2, h=4, w=4, c=8, groups=2, act=0,
             eps=1e-5)
    d.update(kw)
    return B.st_norm_desc(**d)


def mref(addr, n=128, h=32, w=8):
    return B.st_map_ref(addr, n, h, w)


def norm(d=None, x=None, y=None, gamma=None, mean=None, rstd=None,
         ws=16 * A, n=1 << 20):
    B.st_group_norm(d or norm_desc(), x or mref(A), gamma, None,
                    y or mref(2 * A), mean, rstd, ws, n)


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=3), "types"), (dict(out_dtype=-1), "types"),
    (dict(dtype=1, out_dtype=0), "types"),
    (dict(dtype=1, out_dtype=2), "types"), (dict(n=-1), "sizes"),
    (dict(h=0), "sizes"), (dict(w=-2), "sizes"), (dict(c=0), "sizes"),
    (dict(n=1 << 20, c=1 << 11), "2^31"), (dict(groups=0), "groups"), (dict(groups=3), "groups"),
    (dict(act=3), "activation"), (dict(act=-1), "activation"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps")])
def test_norm_descriptors(kw, word):
    refused(BAD, word, norm, norm_desc(**kw))
    refused(BAD, word, B.st_group_norm_workspace, norm_desc(**kw), 0)


def test_norm_maps_and_memory():
    refused(BAD, "x is NULL", norm, x=mref(None))
    refused(BAD, "negative", norm, x=mref(A, -128))
    refused(BAD, "y: an output's elements overlap", norm,
            y=mref(2 * A, 128, 32, 7))
    refused(BAD, "elements overlap", norm, y=mref(2 * A, 0))
    refused(BAD, "elements overlap", norm, y=mref(2 * A, 120))
    refused(BAD, "both or neither", norm, mean=3 * A)
    refused(BAD, "overlaps", norm, y=mref(A + 64))
    refused(BAD, "overlaps", norm, y=mref(A, 256, 64, 16))  # x, other strides
    refused(BAD, "overlaps", norm, mean=2 * A, rstd=3 * A)
    refused(BAD, "overlaps", norm, mean=3 * A, rstd=3 * A)
    refused(BAD, "overlaps", norm, gamma=2 * A)
    refused(BAD, "overlaps", norm, ws=2 * A)
    refused(BAD, "aligned", norm, ws=16 * A + 8)
    # a map of this size is summed up in parts
    large = dict(d=norm_desc(n=1, h=512, w=512), x=mref(A, 0, 4096, 8),
                 y=mref(32 * A, 0, 4096, 8), ws=64 * A)
    need = B.st_group_norm_workspace(large["d"], 0)
    assert need > 0
    refused(BAD, "workspace is NULL", norm, **dict(large, ws=None))
    refused(SMALL, "small", norm, **large, n=need - 1)
    refused(BAD, "overlaps", norm, **dict(large, ws=33 * A))
    assert B.st_group_norm_workspace(norm_desc(), 0) == 0
    # types differ: not in place
    refused(BAD, "overlaps", norm, norm_desc(out_dtype=2), y=mref(A))
    assert B.library().st_group_norm(None, None, None, None, None, None, None,
                                     None, 0, None) == BAD
    assert B.library().st_group_norm_workspace(
        ctypes.byref(norm_desc()), 0, None) == BAD
    # no image: nothing to do, nothing needed
    norm(norm_desc(n=0), ws=None, n=0)
    assert B.st_group_norm_workspace(norm_desc(n=0), 1) == 0


def test_norm_backward_memory():
    def back(dy=None, x=None, mean=3 * A, rstd=4 * A, dx=None, dg=5 * A,
             db=6 * A, ws=16 * A, n=1 << 20, d=None):
        B.st_group_norm_backward(d or norm_desc(), dy or mref(A),
                                 x or mref(2 * A), mean, rstd, None, None,
                                 dx or mref(7 * A), dg, db, ws, n)
    refused(BAD, "mean or rstd", back, mean=None)
    refused(BAD, "dx: an output", back, dx=mref(7 * A, 128, 32, 4))
    refused(BAD, "overlaps", back, dx=mref(A + 4))
    refused(BAD, "overlaps", back, dg=6 * A)
    refused(BAD, "overlaps", back, dg=3 * A)
    refused(BAD, "overlaps", back, ws=A)
    refused(BAD, "overlaps", back, d=norm_desc(out_dtype=1), dx=mref(A))
    refused(SMALL, "small", back, n=16)


def seq_desc(**kw):
    d = dict(dtype=0, out_dtype=0, t=5, b=3, c=8, reverse=0, lengths=None,
             reset=None)
    d.update(kw)
    return B.st_seq_desc(**d)


def sref(addr, t=24, b=8):
    return B.st_seq_ref(addr, t, b)


def conv(d=None, k=3, act=0, x=None, w=3 * A, window=None, y=None, wo=None):
    B.st_time_conv(d or seq_desc(), k, act, x or sref(A), w, None, window,
                   y or sref(2 * A), wo)


def scan(d=None, v=None, f=None, o=None, h=None, y=None, ho=None, st=None,
         ws=16 * A, n=1 << 24):
    B.st_gated_scan(d or seq_desc(), v or sref(A), f or sref(2 * A), o, h,
                    y or sref(3 * A), ho, st, ws, n)


@pytest.mark.parametrize("call", [conv, scan])
@pytest.mark.parametrize("kw,word", [
    (dict(dtype=5), "types"), (dict(dtype=2, out_dtype=1), "types"),
    (dict(t=-1), "negative"), (dict(b=-1), "negative"),
    (dict(c=0), "positive"), (dict(b=1 << 20, c=1 << 11), "2^31"),
    (dict(t=(1 << 30) + 1), "2^30"), (dict(lengths=A + 2), "misaligned")])
def test_sequence_descriptors(call, kw, word):
    refused(BAD, word, call, seq_desc(**kw))
    for fn in (lambda d: B.st_time_conv_workspace(d, 3, 1),
               lambda d: B.st_gated_scan_workspace(d, 1)):
        refused(BAD, word, fn, seq_desc(**kw))


def test_conv_refusals():
    refused(BAD, "taps", conv, k=0)
    refused(BAD, "taps", conv, k=9)
    refused(BAD, "activation", conv, act=7)
    refused(BAD, "weight", conv, w=None)
    refused(BAD, "x is NULL", conv, x=sref(None))
    refused(BAD, "negative", conv, x=sref(A, -24))
    refused(BAD, "elements overlap", conv, y=sref(2 * A, 20, 8))
    refused(BAD, "elements overlap", conv, y=sref(2 * A, 24, 4))
    refused(BAD, "overlaps", conv, y=sref(A))
    refused(BAD, "overlaps", conv, y=sref(3 * A))
    refused(BAD, "overlaps", conv, window=2 * A)
    refused(BAD, "overlaps", conv, wo=A)
    refused(BAD, "overlaps", conv, window=5 * A, wo=5 * A + 4)
    refused(BAD, "overlaps", conv, d=seq_desc(lengths=2 * A))
    refused(BAD, "overlaps", conv, d=seq_desc(reset=2 * A))
    conv(seq_desc(b=0))

    def back(dx=None, dw=5 * A, db=6 * A, dwin=None, dwo=None, ws=16 * A,
             n=1 << 20, k=3):
        B.st_time_conv_backward(seq_desc(), k, 0, sref(A), sref(2 * A), 3 * A,
                                None, None, dwo, dx, dw, db, dwin, ws, n)
    refused(BAD, "taps", back, k=12)
    refused(BAD, "overlaps", back, dx=sref(A))
    refused(BAD, "overlaps", back, dx=sref(5 * A))
    refused(BAD, "overlaps", back, db=5 * A)
    refused(BAD, "overlaps", back, dwin=7 * A, dwo=7 * A)
    refused(BAD, "overlaps", back, ws=2 * A)
    refused(SMALL, "small", back, n=0)
    refused(BAD, "workspace is NULL", back, ws=None)


def test_scan_refusals():
    refused(BAD, "f is NULL", scan, f=sref(None))
    refused(BAD, "o is NULL", scan, o=sref(None))
    refused(BAD, "elements overlap", scan, y=sref(3 * A, 8, 8))
    refused(BAD, "overlaps", scan, y=sref(2 * A))
    refused(BAD, "overlaps", scan, h=4 * A, ho=4 * A + 32)
    refused(BAD, "overlaps", scan, h=3 * A)
    refused(BAD, "overlaps", scan, st=A)
    refused(BAD, "overlaps", scan, st=4 * A, ho=4 * A)
    refused(BAD, "aligned", scan, ws=16 * A + 1)
    scan(seq_desc(b=0))

    def back(dv=None, df=None, do=None, o=None, st=6 * A, dh=None, dho=None,
             ws=16 * A, n=1 << 24):
        B.st_gated_scan_backward(seq_desc(), sref(A), sref(2 * A),
                                 sref(3 * A), o, st, dho, dv or sref(4 * A),
                                 df or sref(5 * A), do, dh, ws, n)
    refused(BAD, "both or neither", back, o=sref(8 * A))
    refused(BAD, "both or neither", back, do=sref(8 * A))
    refused(BAD, "states", back, st=None)
    refused(BAD, "overlaps", back, dv=sref(5 * A))
    refused(BAD, "overlaps", back, df=sref(2 * A))
    refused(BAD, "overlaps", back, dh=6 * A)
    refused(BAD, "overlaps", back, dh=7 * A, dho=7 * A + 4)
    # slices of one tensor must lie side by side
    refused(BAD, "overlaps", back, dv=sref(4 * A, 72, 24),
            df=sref(4 * A + 28, 72, 24))
    refused(BAD, "overlaps", back, dv=sref(4 * A, 72, 24),
            df=sref(4 * A + 68, 72, 24))
    refused(BAD, "overlaps", back, dv=sref(4 * A, 72, 24),
            df=sref(4 * A + 32, 144, 24))


def test_misaligned_addresses():
    """Addresses between two elements are refused, in every place."""
    refused(BAD, "x is misaligned", norm, x=mref(A + 2))
    refused(BAD, "y is misaligned", norm, norm_desc(out_dtype=1),
            y=mref(2 * A + 1))
    refused(BAD, "misaligned", norm, gamma=A + 1)
    refused(BAD, "misaligned", norm, mean=3 * A + 2, rstd=4 * A)
    refused(BAD, "x is misaligned", conv, x=sref(A + 1))
    refused(BAD, "misaligned", conv, w=3 * A + 1)
    refused(BAD, "window", conv, window=5 * A + 2)
    refused(BAD, "window", conv, wo=5 * A + 1)
    refused(BAD, "f is misaligned", scan, f=sref(2 * A + 3))
    refused(BAD, "y is misaligned", scan, seq_desc(out_dtype=2),
            y=sref(3 * A + 1))
    refused(BAD, "misaligned", scan, ho=4 * A + 2)
    refused(BAD, "misaligned", B.st_gated_scan_backward, seq_desc(), sref(A),
            sref(2 * A), sref(3 * A), None, 6 * A, None, sref(4 * A + 2),
            sref(5 * A), None)
    refused(BAD, "misaligned", B.st_group_norm_backward, norm_desc(),
            mref(A), mref(2 * A), 3 * A, 4 * A, None, None, mref(7 * A),
            5 * A + 2)
    refused(BAD, "misaligned", B.st_time_conv_backward, seq_desc(), 3, 0,
            sref(A), sref(2 * A), 3 * A, None, None, 5 * A + 2, None)


def test_exported_constants():
    txt = open(B.__file__.rsplit("/", 2)[0] + "/include/sparsetem.h").read()
    assert f"#define ST_SCAN_STRIDE {B.SCAN_STRIDE}\n" in txt
    assert f"#define ST_TIME_CONV_MAX_TAPS {B.TIME_CONV_MAX_TAPS}\n" in txt


def test_workspaces_grow_with_the_work():
    small = B.st_group_norm_workspace(norm_desc(), 1)
    large = B.st_group_norm_workspace(norm_desc(n=64, h=64, w=64), 1)
    assert 0 < small < large < 1 << 28
    assert B.st_time_conv_workspace(seq_desc(), 3, 0) == 0
    assert 0 < B.st_time_conv_workspace(seq_desc(), 3, 1) < 1 << 20


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(2, 4, 4, 8)
    for call in (lambda: ops.group_norm(x, 2),
                 lambda: ops.time_conv(x[0], torch.zeros(3, 8)),
                 lambda: ops.gated_scan(x[0], x[0])):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def test_scan_gradients_that_cross_in_the_next_step():
    """Slices whose steps are narrower than all their rows side by side: the
    last row of one lies where the next step's first row of the other does."""
    d = seq_desc(t=2, b=2, c=4)
    for axes in ((16, 12), (12, 16)):
        refused(BAD, "overlaps", B.st_gated_scan_backward, d, sref(A),
                sref(2 * A), sref(3 * A), None, 6 * A, None,
                sref(4 * A, *axes), sref(4 * A + 16, *axes), None)


def test_maps_larger_than_any_memory():
    """Sizes whose product passes 64 bits are refused, not computed with."""
    for h, w, c in ((1 << 30, 1 << 30, 8), (1 << 30, 1 << 30, 4),
                    ((1 << 31) - 1, (1 << 31) - 1, 1), (1 << 20, 1 << 10, 2048)):
        d = norm_desc(n=1, h=h, w=w, c=c, groups=1)
        for back in (0, 1):
            refused(BAD, "2^40", B.st_group_norm_workspace, d, back)


@pytest.mark.parametrize("far", [2 ** 31, 2 ** 32 + 5, 2 ** 33 + 2])
def test_sizes_beyond_32_bits(far, monkeypatch):
    """What the descriptors' integers would wrap is refused, not taken for a
    small size (tensors without memory in place of device tensors)."""
    monkeypatch.setattr(ops, "_code", lambda x, name: 0)

    def t(*shape):
        return torch.empty(shape, device="meta")
    for call in (lambda: ops.group_norm(t(1, far, 1), 1),
                 lambda: ops.group_norm(t(far, 2, 2, 4), 2),
                 lambda: ops.group_norm(t(1, 2, far, 4), 2),
                 lambda: ops.group_norm(t(1, 2, 2, 4), far),
                 lambda: ops.group_norm(t(1, 2, 2, 4), 2, act=far),
                 lambda: ops.group_norm_backward(
                     t(1, far, 1), t(1, far, 1), 1, t(1, 1), t(1, 1)),
                 lambda: ops.time_conv(t(far, 1, 1), t(3, 1)),
                 lambda: ops.time_conv(t(2, 1, 1), t(3, 1), act=far),
                 lambda: ops.time_conv_backward(t(2, far, 1), t(2, far, 1),
                                                t(3, 1)),
                 lambda: ops.gated_scan(t(far, 1, 1), t(far, 1, 1)),
                 lambda: ops.gated_scan_backward(
                     t(far, 1, 1), t(far, 1, 1), t(far, 1, 1),
                     states=t(1, 1, 1))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_padding_need_not_be_there(tmp_path):
    """The recurrence's loads, compiled for the host: nothing behind a row's
    length is read, at any step of rows that end before it."""
    import os
    import subprocess

    from paper_2410_20790_amd import build
    exe = str(tmp_path / "padding_reads")
    src = os.path.join(os.path.dirname(__file__), "padding_reads.hip")
    subprocess.run([build.HIPCC, "-x", "hip", f"--offload-arch={build.ARCH}",
                    "--offload-host-only", "-O1", "-std=c++17",
                    "-I", build.OPS, src, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), (
        r.returncode, r.stdout[-200:])


def _calls(grad, t):
    """(name, call) of every operator with one input that requires a
    gradient; t makes a tensor, grad one that requires it."""
    x4, p, st = t(1, 2, 2, 4), t(4), t(1, 2)
    x, w, h = t(3, 2, 4), t(3, 4), t(2, 4)
    kept = t(1, 2, 4)
    return [
        ("x", lambda: ops.group_norm(grad(x4), 2)),
        ("gamma", lambda: ops.group_norm(x4, 2, grad(p))),
        ("beta", lambda: ops.group_norm(x4, 2, p, grad(p))),
        ("dy", lambda: ops.group_norm_backward(grad(x4), x4, 2, st, st)),
        ("x", lambda: ops.time_conv(grad(x), w)),
        ("weight", lambda: ops.time_conv(x, grad(w))),
        ("window", lambda: ops.time_conv(x, w, window=grad(t(2, 2, 4)))),
        ("weight", lambda: ops.time_conv_backward(x, x, grad(w))),
        ("v", lambda: ops.gated_scan(grad(x), x)),
        ("f", lambda: ops.gated_scan(x, grad(x))),
        ("o", lambda: ops.gated_scan(x, x, grad(x))),
        ("h", lambda: ops.gated_scan(x, x, h=grad(h))),
        ("dh", lambda: ops.gated_scan_backward(x, x, x, states=kept,
                                               dh=grad(h)))]


def test_gradients_that_nothing_would_record(monkeypatch):
    """An input that requires a gradient is refused where torch records."""
    monkeypatch.setattr(ops, "_code", lambda x, name: 0)
    for name, call in _calls(lambda x: x.clone().requires_grad_(),
                             lambda *s: torch.empty(s, device="meta")):
        with pytest.raises(ValueError, match=f"^{name} requires a gradient"):
            call()
