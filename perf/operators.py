"""Timed cases of the operators behind the encoder: group norm with an
activation on channels-last feature maps, the causal depthwise convolution
along time, and the gated linear recurrence -- forward and backward, over a
chunk of frames, single frames, text lines and long recordings.

Every case is one pass through one operator.  A plain form of each, in
elementary torch operations, stands beside the framework's calls.

Running order: step s of row b is time s, or lengths[b] - 1 - s in reverse;
a row ends at its own length (outputs behind it are zero, the state stays),
and a reset hides everything before its step.
"""

import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ES = {"f32": 4, "f16": 2, "bf16": 2}
NONE, RELU, SILU = 0, 1, 2
STRIDE = 16   # steps between the kept states of a scan


# ------------------------------------------------------------------- cases

def _norm(name, n, h, w, c, groups, dtype, out, act, grad=False,
          crop=False):
    return dict(name=name, op="norm", n=n, h=h, w=w, c=c, groups=groups,
                dtype=dtype, out=out, act=act, grad=grad, crop=crop)


def _conv(name, t, b, c, k, dtype, out, act, grad=False, sliced=False,
          padded=False, resets=False, reverse=False, state=True):
    return dict(name=name, op="conv", t=t, b=b, c=c, k=k, dtype=dtype,
                out=out, act=act, grad=grad, sliced=sliced, padded=padded,
                resets=resets, reverse=reverse, state=state)


def _scan(name, t, b, c, dtype, out, gate=True, grad=False, sliced=False,
          padded=False, resets=False, reverse=False, state=True):
    return dict(name=name, op="scan", t=t, b=b, c=c, dtype=dtype, out=out,
                gate=gate, grad=grad, sliced=sliced, padded=padded,
                resets=resets, reverse=reverse, state=state)


def listed():
    return [
        # one live frame of a detector backbone (EfficientNet-B0 at 512x512,
        # stride 32): the smallest norm, ten channels to a group
        _norm("norm_frame", 1, 16, 16, 320, 32, "f32", "f16", SILU),
        # a chunk from an odd-sized camera (ResNet-50 stage 2 of 375x621)
        _norm("norm_ragged", 8, 47, 78, 512, 32, "f16", "f16", RELU),
        # a chunk of driving video (ResNet-50 stage 1 of 1024x2048): the
        # largest
        _norm("norm_chunk", 9, 256, 512, 256, 32, "bf16", "bf16", RELU),
        # training a head on the stage-2 maps of such a chunk: the gradients
        _norm("norm_grad", 9, 128, 256, 512, 32, "bf16", "bf16", SILU,
              grad=True),
        # one live frame of ResNet-50 at 1024x2048 (32x64 sites): the step
        # of a single frame with its kept window
        _conv("conv_step", 1, 2048, 512, 4, "f32", "bf16", SILU,
              sliced=True),
        # the same for a chunk of nine diff frames at once
        _conv("conv_chunk", 9, 2048, 512, 4, "f32", "f32", SILU,
              sliced=True),
        # gradients over recordings of different lengths, pooled to rows
        _conv("conv_grad", 601, 48, 512, 4, "f16", "f16", SILU, grad=True,
              padded=True),
        # one live frame of 32 cameras (EfficientNet-B0 at 256x256)
        _scan("scan_step", 1, 2048, 320, "f32", "f32", sliced=True),
        # a chunk of nine diff frames of ResNet-50 at 1024x2048
        _scan("scan_chunk", 9, 2048, 2048, "f32", "f32", sliced=True),
        # text lines read backwards (CRNN-VGG: 32 columns, two rows each),
        # each as wide as its text
        _scan("scan_line", 32, 32, 512, "f16", "f16", padded=True,
              reverse=True, state=False),
        # one long recording (20 minutes at 30 frames a second), few rows
        _scan("scan_long", 36001, 1, 512, "bf16", "bf16"),
        # gradients over long recordings with cuts
        _scan("scan_grad", 4099, 8, 512, "bf16", "bf16", grad=True,
              resets=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(
        rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "conv", "scan"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    out = rng.choice(["f32", "f16", "bf16"]) if dtype == "f32" else dtype
    grad = rng.random() < 0.4
    if op == "norm":
        groups = rng.choice([1, 2, 4, 8, 16, 32])
        per = _log(rng, 1, max(1, 2048 // groups))
        c = groups * per
        n = _log(rng, 1, 32)
        sites = _log(rng, 1, max(1, min(1 << 18, 75_000_000 // (n * c))))
        h = _log(rng, 1, sites)
        return _norm("", n, h, max(1, sites // h), c, groups, dtype, out,
                     rng.choice([NONE, SILU]) if grad
                     else rng.choice([NONE, RELU, SILU]), grad,
                     rng.random() < 0.25)
    t = 1 if rng.random() < 0.2 else _log(rng, 1, 20000)
    c = _log(rng, 8, 2048)
    b = _log(rng, 1, max(1, min(4096, 40_000_000 // (t * c))))
    opts = dict(grad=grad, sliced=rng.random() < 0.4,
                padded=rng.random() < 0.3, resets=rng.random() < 0.3,
                reverse=rng.random() < 0.3, state=rng.random() < 0.7)
    if op == "conv":
        return _conv("", t, b, c, rng.randint(1, 8), dtype, out,
                     rng.choice([NONE, SILU]) if grad
                     else rng.choice([NONE, RELU, SILU]), **opts)
    return _scan("", t, b, c, dtype, out, rng.random() < 0.7, **opts)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _rand(g, *shape):
    return torch.rand(*shape, device="cuda", generator=g)


def _prepare_norm(case, seed):
    g = _gen(seed)
    n, h, w, c = (case[k] for k in ("n", "h", "w", "c"))
    e = 2 if case["crop"] else 0
    # feature maps: every channel has its own offset and spread
    x = _randn(g, n, h + e, w + e, c)
    x.mul_(0.3 + _rand(g, c)).add_(_randn(g, c))
    x = x.to(DT[case["dtype"]])
    if e:
        x = x[:, 1:-1, 1:-1, :]
    st = dict(case=case, x=x, gamma=1.0 + 0.2 * _randn(g, c),
              beta=0.1 * _randn(g, c))
    if case["grad"]:
        st["dy"] = _randn(g, n, h, w, c).to(DT[case["out"]])
        mean, var = _moments(x.float(), case["groups"])
        st["mean"] = mean
        st["rstd"] = torch.rsqrt(var + 1e-5)
    return st


def _prepare_seq(case, seed):
    g = _gen(seed)
    t, b, c, dt = case["t"], case["b"], case["c"], DT[case["dtype"]]
    st = dict(case=case, lengths=None, reset=None)
    if case["padded"]:
        # padded batches: from nothing to the whole axis, most of them long
        st["lengths"] = (t * _rand(g, b).sqrt() * 1.02).long().clamp_(
            max=t).to(torch.int32)
    if case["resets"]:
        # a cut now and then
        st["reset"] = (_rand(g, t, b) < 1 / 48).to(torch.uint8)
    # the encoder's last layer emits all inputs side by side
    parts = 3 if case["sliced"] else 1
    x = _randn(g, t, b, parts * c)
    if case["op"] == "conv":
        x = x.to(dt)
        k = case["k"]
        st.update(x=x[..., :c], weight=_randn(g, k, c) / math.sqrt(k),
                  bias=0.1 * _randn(g, c), window=None)
        if case["state"]:
            st["window"] = _randn(g, k - 1, b, c).to(dt)
        if case["grad"]:
            st["dy"] = _randn(g, t, b, c).to(DT[case["out"]])
            st["dwindow"] = None
        return st
    # forget gates that hold from a few steps to thousands, by channel
    off = 1.0 + 6.0 * _rand(g, c)
    if case["sliced"]:
        x[..., c:2 * c].add_(off)
        x = x.to(dt)
        v, f, o = x[..., :c], x[..., c:2 * c], x[..., 2 * c:]
    else:
        v = x.to(dt)
        f = (_randn(g, t, b, c) + off).to(dt)
        o = _randn(g, t, b, c).to(dt)
    st.update(v=v, f=f, o=o if case["gate"] else None, h=None)
    if case["state"]:
        st["h"] = _randn(g, b, c)
    if case["grad"]:
        st["dy"] = _randn(g, t, b, c).to(DT[case["out"]])
        st["dh"] = _randn(g, b, c) if case["state"] else None
        # the states a training program kept from the forward pass
        h = _states(st)
        first = h.new_zeros(1, b, c) if st["h"] is None else st["h"][None]
        kept = torch.cat([first, h])[:t:STRIDE]
        st["states"] = kept.contiguous()
    return st


def prepare(case, seed):
    if case["op"] == "norm":
        return _prepare_norm(case, seed)
    return _prepare_seq(case, seed)


# -------------------------------------------------------------- plain form

def _act(z, act):
    if act == RELU:
        return z.clamp_min(0)
    return z * torch.sigmoid(z) if act == SILU else z


def _dact(z, act):
    if act == RELU:
        return (z > 0).to(z.dtype)
    if act == SILU:
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _moments(x, groups):
    """Mean and variance of every image's groups, [n][groups]."""
    n, c = x.shape[0], x.shape[-1]
    v = x.reshape(n, -1, groups, c // groups)
    m = v.shape[1] * v.shape[3]
    mean = (v.sum((1, 3), dtype=torch.float64) / m).float()
    d = v - mean[:, None, :, None]
    var = (d * d).sum((1, 3), dtype=torch.float64) / m
    return mean, var.float()


def _per_channel(stat, c):
    """[n][groups] -> [n][1][1][c]."""
    n, groups = stat.shape
    return stat[:, :, None].expand(n, groups, c // groups).reshape(
        n, 1, 1, c)


def _plain_norm(st):
    case = st["case"]
    c, groups = case["c"], case["groups"]
    x = st["x"].float()
    if not case["grad"]:
        mean, var = _moments(x, groups)
        rstd = torch.rsqrt(var + 1e-5)
        z = (x - _per_channel(mean, c)) * _per_channel(rstd, c)
        z = z * st["gamma"] + st["beta"]
        return dict(y=_act(z, case["act"]).to(DT[case["out"]]), mean=mean,
                    rstd=rstd)
    rstd = _per_channel(st["rstd"], c)
    xh = (x - _per_channel(st["mean"], c)) * rstd
    dz = st["dy"].float() * _dact(xh * st["gamma"] + st["beta"],
                                  case["act"])
    n = case["n"]
    m = case["h"] * case["w"] * (c // groups)

    def group_mean(q):
        q = q.reshape(n, -1, groups, c // groups)
        return _per_channel((q.sum((1, 3), dtype=torch.float64) / m).float(),
                            c)

    dg = dz * st["gamma"]
    dx = rstd * (dg - group_mean(dg) - xh * group_mean(dg * xh))
    return dict(dx=dx.to(DT[case["dtype"]]),
                dgamma=(dz * xh).sum((0, 1, 2), dtype=torch.float64).float(),
                dbeta=dz.sum((0, 1, 2), dtype=torch.float64).float())


def _order(st):
    """The time of every running step, [t][b], and whether the row has it."""
    case = st["case"]
    t, b = case["t"], case["b"]
    s = torch.arange(t, device="cuda")[:, None].expand(t, b)
    n = (torch.full((b,), t, device="cuda") if st["lengths"] is None
         else st["lengths"].long())
    valid = s < n
    time = torch.where(valid, n - 1 - s, s) if case["reverse"] else s
    return time, valid, n


def _take(x, time, valid):
    """Rows of [t][b][c] by running step, f32, zero behind the lengths.
    A row's order is its own inverse: the same call brings results back."""
    x = torch.gather(x.float(), 0, time[:, :, None].expand(x.shape))
    return torch.where(valid[:, :, None], x, 0.0)


def _resets(st, time, valid):
    if st["reset"] is None:
        return torch.zeros_like(valid)
    return (torch.gather(st["reset"], 0, time) != 0) & valid


def _prefix(a, u):
    """h_s = a_s h_{s-1} + u_s for all s, by doubling."""
    d = 1
    while d < a.shape[0]:
        u = torch.cat([u[:d], a[d:] * u[:-d] + u[d:]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return u


def _gates(st, time, valid):
    """Decay (0 at a reset, 1 behind a row) and input of every step."""
    f = _take(st["f"], time, valid)
    live = valid[:, :, None]
    cut = _resets(st, time, valid)[:, :, None]
    a = torch.where(live, torch.sigmoid(f), 1.0)
    a = torch.where(cut, 0.0, a)
    u = torch.sigmoid(-f) * _take(st["v"], time, valid)
    return f, a, u


def _states(st):
    time, valid, _ = _order(st)
    _, a, u = _gates(st, time, valid)
    if st["h"] is not None:
        u[0] += a[0] * st["h"]
    return _prefix(a, u)


def _plain_scan(st):
    case = st["case"]
    time, valid, _ = _order(st)
    o = None if st["o"] is None else torch.sigmoid(
        _take(st["o"], time, valid))
    h = _states(st)
    if not case["grad"]:
        y = h if o is None else h * o
        return dict(y=_take(y, time, valid).to(DT[case["out"]]), h=h[-1])
    f, a, _ = _gates(st, time, valid)
    dy = _take(st["dy"], time, valid)
    g = dy if o is None else dy * o
    if st["dh"] is not None:
        g = torch.cat([g[:-1], g[-1:] + st["dh"]])
    nxt = torch.cat([a[1:], torch.ones_like(a[:1])])
    dh = _prefix(nxt.flip(0), g.flip(0)).flip(0)
    first = torch.zeros_like(h[:1]) if st["h"] is None else st["h"][None]
    prev = torch.cat([first, h[:-1]])
    prev = torch.where(_resets(st, time, valid)[:, :, None], 0.0, prev)
    keep, write = torch.sigmoid(f), torch.sigmoid(-f)
    dv = dh * write
    df = dh * (prev - _take(st["v"], time, valid)) * keep * write
    dt = DT[case["dtype"]]
    out = dict(dv=_take(dv, time, valid).to(dt),
               df=_take(df, time, valid).to(dt))
    if o is not None:
        out["do"] = _take(dy * h * o * (1 - o), time, valid).to(dt)
    if st["h"] is not None:
        out["dh"] = a[0] * dh[0]
    return out


def _plain_conv(st):
    case = st["case"]
    t, b, c, k = (case[q] for q in ("t", "b", "c", "k"))
    time, valid, n = _order(st)
    x = _take(st["x"], time, valid)
    win = (x.new_zeros(k - 1, b, c) if st["window"] is None
           else st["window"].float())
    line = torch.cat([win, x])                       # [k - 1 + t][b][c]
    cuts = _resets(st, time, valid).long().cumsum(0)  # cuts up to a step
    cuts = torch.cat([cuts.new_zeros(k - 1, b), cuts])
    w = st["weight"]

    def seen(j):   # tap j's value and the step see no cut between them
        return (cuts[j:j + t] == cuts[k - 1:])[:, :, None]

    z = st["bias"].expand(t, b, c)
    for j in range(k):
        z = z + w[j] * torch.where(seen(j), line[j:j + t], 0.0)
    if not case["grad"]:
        y = _take(_act(z, case["act"]), time, valid).to(DT[case["out"]])
        i = torch.arange(k - 1, device="cuda")[:, None] + n     # [k-1][b]
        last = torch.gather(line, 0, i[:, :, None].expand(k - 1, b, c))
        end = cuts[-1]
        last = torch.where((torch.gather(cuts, 0, i) == end)[:, :, None],
                           last, 0.0)
        return dict(y=y, window=last.to(DT[case["dtype"]]))
    dz = _take(st["dy"], time, valid) * _dact(z, case["act"])
    dline = torch.zeros_like(line)
    dw = []
    for j in range(k):
        q = torch.where(seen(j), dz, 0.0)
        dline[j:j + t] += w[j] * q
        dw.append((q * line[j:j + t]).sum((0, 1), dtype=torch.float64))
    dt = DT[case["dtype"]]
    out = dict(dx=_take(dline[k - 1:], time, valid).to(dt),
               dweight=torch.stack(dw).float(),
               dbias=dz.sum((0, 1), dtype=torch.float64).float())
    if st["window"] is not None:
        out["dwindow"] = dline[:k - 1].to(dt)
    return out


# ------------------------------------------------------- the framework's calls

def _own_norm(st):
    from paper_2410_20790_amd import ops
    case = st["case"]
    if not case["grad"]:
        y, mean, rstd = ops.group_norm(
            st["x"], case["groups"], st["gamma"], st["beta"],
            act=case["act"], eps=1e-5, out_dtype=DT[case["out"]])
        return dict(y=y, mean=mean, rstd=rstd)
    dx, dgamma, dbeta = ops.group_norm_backward(
        st["dy"], st["x"], case["groups"], st["mean"], st["rstd"],
        st["gamma"], st["beta"], act=case["act"])
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


def _own_conv(st):
    from paper_2410_20790_amd import ops
    case = st["case"]
    seq = dict(lengths=st["lengths"], reset=st["reset"],
               reverse=case["reverse"])
    if not case["grad"]:
        y, window = ops.time_conv(
            st["x"], st["weight"], st["bias"], act=case["act"],
            window=st["window"], out_dtype=DT[case["out"]], **seq)
        return dict(y=y, window=window)
    dx, dw, db, dwin = ops.time_conv_backward(
        st["dy"], st["x"], st["weight"], st["bias"], act=case["act"],
        window=st["window"], **seq)
    out = dict(dx=dx, dweight=dw, dbias=db)
    if st["window"] is not None:
        out["dwindow"] = dwin
    return out


def _own_scan(st):
    from paper_2410_20790_amd import ops
    case = st["case"]
    seq = dict(lengths=st["lengths"], reset=st["reset"],
               reverse=case["reverse"])
    if not case["grad"]:
        y, h = ops.gated_scan(st["v"], st["f"], st["o"], h=st["h"],
                              out_dtype=DT[case["out"]], **seq)
        return dict(y=y, h=h)
    dv, df, do, dh = ops.gated_scan_backward(
        st["dy"], st["v"], st["f"], st["o"], states=st["states"],
        dh=st["dh"], **seq)
    out = dict(dv=dv, df=df)
    if do is not None:
        out["do"] = do
    if st["h"] is not None:
        out["dh"] = dh
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "conv": _own_conv,
                "scan": _own_scan}[op](state)
    return {"norm": _plain_norm, "conv": _plain_conv,
            "scan": _plain_scan}[op](state)


# -------------------------------------------------------------------- work

def work(case):
    es, eo = ES[case["dtype"]], ES[case["out"]]
    if case["op"] == "norm":
        e = case["n"] * case["h"] * case["w"] * case["c"]
        if case["grad"]:
            return {"bytes": e * (2 * es + eo), "flops": 22 * e}
        return {"bytes": e * (es + eo), "flops": 12 * e}
    row = case["b"] * case["c"]
    e = case["t"] * row
    # padded rows are read to two thirds of the axis, and written whole
    r = 2 * e // 3 if case["padded"] else e
    if case["op"] == "conv":
        k = case["k"]
        win = 2 * (k - 1) * row * es * case["state"]
        if case["grad"]:
            return {"bytes": r * (es + eo) + e * es + win,
                    "flops": (6 * k + 10) * r}
        return {"bytes": r * es + e * eo + win, "flops": (2 * k + 6) * r}
    n = 2 + case["gate"]
    if case["grad"]:
        kept = -(-case["t"] // STRIDE) * row * 4
        return {"bytes": r * (n * es + eo) + e * n * es + kept,
                "flops": 36 * r}
    return {"bytes": r * n * es + e * eo + 8 * row, "flops": 16 * r}


# ----------------------------------------------------- definition in 64 bits

def _exact_norm(st):
    case = st["case"]
    n, h, w, c, groups = (case[q] for q in ("n", "h", "w", "c", "groups"))
    per = c // groups
    gam, bet = st["gamma"].double(), st["beta"].double()
    res = {}
    if not case["grad"]:
        y = torch.empty(n, h, w, c, dtype=torch.float64, device="cuda")
        mean = torch.empty(n, groups, dtype=torch.float64, device="cuda")
        rstd = torch.empty_like(mean)
        for i in range(n):
            for k in range(groups):
                ch = slice(k * per, (k + 1) * per)
                q = st["x"][i, :, :, ch].double()
                mean[i, k] = q.mean()
                q = q - mean[i, k]
                rstd[i, k] = (q.square().mean() + 1e-5) ** -0.5
                z = q * rstd[i, k] * gam[ch] + bet[ch]
                if case["act"] == RELU:
                    z = torch.maximum(z, torch.zeros_like(z))
                elif case["act"] == SILU:
                    z = z / (1 + torch.exp(-z))
                y[i, :, :, ch] = z
        return dict(y=y, mean=mean, rstd=rstd)
    dx = torch.empty(n, h, w, c, dtype=torch.float64, device="cuda")
    dgamma = torch.zeros(c, dtype=torch.float64, device="cuda")
    dbeta = torch.zeros_like(dgamma)
    for i in range(n):
        for k in range(groups):
            ch = slice(k * per, (k + 1) * per)
            r = st["rstd"][i, k].double()
            xh = (st["x"][i, :, :, ch].double()
                  - st["mean"][i, k].double()) * r
            dz = st["dy"][i, :, :, ch].double()
            if case["act"] != NONE:
                z = xh * gam[ch] + bet[ch]
                if case["act"] == SILU:
                    e = torch.exp(-z)
                    dz = dz * (1 + e + z * e) / (1 + e).square()
                else:
                    dz = torch.where(z > 0, dz, 0.0)
            dbeta[ch] += dz.sum((0, 1))
            dgamma[ch] += (dz * xh).sum((0, 1))
            d = dz * gam[ch]
            dx[i, :, :, ch] = r * (d - d.mean() - xh * (d * xh).mean())
    res.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return res


def _walk(st):
    """(time index [b], live [b][1], cut [b][1]) of every running step."""
    case = st["case"]
    t, b = case["t"], case["b"]
    n = (torch.full((b,), t, device="cuda") if st["lengths"] is None
         else st["lengths"].long())
    for s in range(t):
        i = torch.full((b,), s, device="cuda")
        if case["reverse"]:
            i = torch.where(n > s, n - 1 - s, i)
        live = (n > s)[:, None]
        cut = torch.zeros_like(live)
        if st["reset"] is not None:
            cut = (st["reset"].gather(0, i[None])[0] != 0)[:, None] & live
        yield i, live, cut


def _exact_scan(st):
    case = st["case"]
    t, b, c = case["t"], case["b"], case["c"]
    rows = torch.arange(b, device="cuda")
    plain = st["lengths"] is None and st["reset"] is None

    def sig(q):
        return 1 / (1 + torch.exp(-q))

    h = (torch.zeros(b, c, dtype=torch.float64, device="cuda")
         if st["h"] is None else st["h"].double())
    y = torch.zeros(t, b, c, dtype=torch.float64, device="cuda")
    before = torch.empty_like(y) if case["grad"] else None
    if plain:
        # no row differs from another: whole rows by their time
        steps = [(s if not case["reverse"] else t - 1 - s, None, None)
                 for s in range(t)]
    else:
        steps = list(_walk(st))
    for i, live, cut in steps:
        at = i if plain else (i, rows)
        f, v = st["f"][at].double(), st["v"][at].double()
        was = h if plain else torch.where(cut, 0.0, h)
        new = sig(f) * was + sig(-f) * v
        out = new if st["o"] is None else new * sig(st["o"][at].double())
        if case["grad"]:
            before[at] = was
        if plain:
            h, y[at] = new, out
        else:
            h = torch.where(live, new, h)
            y[at] = torch.where(live, out, 0.0)
    if not case["grad"]:
        return dict(y=y, h=h)
    dv, df, do = (torch.zeros_like(y) for _ in range(3))
    dh = (torch.zeros_like(h) if st["dh"] is None else st["dh"].double())
    for i, live, cut in reversed(steps):
        at = i if plain else (i, rows)
        f, v = st["f"][at].double(), st["v"][at].double()
        dy = st["dy"][at].double()
        keep, write = sig(f), sig(-f)
        here = keep * before[at] + write * v
        if st["o"] is not None:
            o = st["o"][at].double()
            d_o = dy * here * sig(o) * sig(-o)
            dy = dy * sig(o)
        else:
            d_o = None
        d = dh + (dy if plain else torch.where(live, dy, 0.0))
        d_v, d_f = d * write, d * (before[at] - v) * keep * write
        if plain:
            dv[at], df[at], dh = d_v, d_f, d * keep
            if d_o is not None:
                do[at] = d_o
        else:
            dv[at] = torch.where(live, d_v, 0.0)
            df[at] = torch.where(live, d_f, 0.0)
            if d_o is not None:
                do[at] = torch.where(live, d_o, 0.0)
            dh = torch.where(live, torch.where(cut, 0.0, d * keep), d)
    out = dict(dv=dv, df=df)
    if st["o"] is not None:
        out["do"] = do
    if st["h"] is not None:
        out["dh"] = dh
    return out


def _exact_conv(st):
    case = st["case"]
    t, b, c, k = (case[q] for q in ("t", "b", "c", "k"))
    rows = torch.arange(b, device="cuda")
    w, bias = st["weight"].double(), st["bias"].double()
    zero = torch.zeros(b, c, dtype=torch.float64, device="cuda")
    # the k - 1 values before the step, oldest first, and where each is from
    win = [zero if st["window"] is None else st["window"][j].double()
           for j in range(k - 1)]
    y = torch.zeros(t, b, c, dtype=torch.float64, device="cuda")
    steps = list(_walk(st))
    if not case["grad"]:
        for i, live, cut in steps:
            taps = [torch.where(cut, 0.0, q) for q in win]
            taps.append(st["x"][i, rows].double())
            z = bias + sum(w[j] * taps[j] for j in range(k))
            if case["act"] == RELU:
                z = torch.maximum(z, torch.zeros_like(z))
            elif case["act"] == SILU:
                z = z / (1 + torch.exp(-z))
            y[i, rows] = torch.where(live, z, 0.0)
            win = [torch.where(live, taps[j + 1], win[j])
                   for j in range(k - 1)]
        return dict(y=y, window=torch.stack(win) if k > 1 else
                    zero.new_zeros(0, b, c))
    # the window's gradient is carried back beside the window itself
    hist = []
    for i, live, cut in steps:
        hist.append(win)
        x = st["x"][i, rows].double()
        taps = [torch.where(cut, 0.0, q) for q in win] + [x]
        win = [torch.where(live, taps[j + 1], win[j]) for j in range(k - 1)]
    dx = torch.zeros_like(y)
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    dwin = [zero for _ in range(k - 1)]
    for (i, live, cut), old in zip(reversed(steps), reversed(hist)):
        taps = [torch.where(cut, 0.0, q) for q in old]
        taps.append(st["x"][i, rows].double())
        dz = torch.where(live, st["dy"][i, rows].double(), 0.0)
        if case["act"] != NONE:
            z = bias + sum(w[j] * taps[j] for j in range(k))
            if case["act"] == SILU:
                e = torch.exp(-z)
                dz = dz * (1 + e + z * e) / (1 + e).square()
            else:
                dz = torch.where(z > 0, dz, 0.0)
        db += dz.sum(0)
        dtaps = [w[j] * dz for j in range(k)]
        for j in range(k):
            dw[j] += (dz * taps[j]).sum(0)
        # taps[1:] went on as the next window
        for j in range(k - 1):
            dtaps[j + 1] = dtaps[j + 1] + dwin[j]
        dx[i, rows] = torch.where(live, dtaps[k - 1], dx[i, rows])
        dwin = [torch.where(live, torch.where(cut, 0.0, dtaps[j]), dwin[j])
                for j in range(k - 1)]
    out = dict(dx=dx, dweight=dw, dbias=db)
    if st["window"] is not None:
        out["dwindow"] = (torch.stack(dwin) if k > 1 else
                          zero.new_zeros(0, b, c))
    return out


def exact(case, seed):
    # about 40 us a step and direction, by the row operations of a step
    if case["op"] == "conv" and case["t"] * (20 + 14 * case["k"]) * (
            3 if case["grad"] else 1) > 2_000_000:
        return None
    if case["op"] == "conv" and case["grad"] and (
            case["t"] * case["b"] * case["c"] * case["k"] * 8 > 3e10):
        return None
    with torch.no_grad():
        st = prepare(case, seed)
        return {"norm": _exact_norm, "conv": _exact_conv,
                "scan": _exact_scan}[case["op"]](st)
