"""Timed cases of single operators, through the public entry points: the short causal convolution, the selective
state space scan, and the distillation loss over a vocabulary.

One pass is one call as a program makes it: a prompt ("forward"), the next token of every row ("token"), a training
pass (forward, then backward with every gradient), a loss, or a loss with its gradient.  Inputs, weights, output buffers
and workspaces are made beforehand, as such a program keeps them from call to call.

With ``own`` false the same outputs are computed by elementary tensor operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

_TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2}


def _conv(name, do, dtype, batch, t, channels, width, layout="time", ragged=False, state=False, silu=True):
    return {"name": name, "op": "conv", "do": do, "dtype": dtype, "batch": batch, "t": t, "channels": channels, "width": width,
            "layout": layout, "ragged": ragged, "state": state, "silu": silu}


def _scan(name, do, dtype, batch, t, channels, states, groups=1, spacing=8, layout="time", ragged=False, state=False, gate=True):
    return {"name": name, "op": "scan", "do": do, "dtype": dtype, "batch": batch, "t": t, "channels": channels, "states": states,
            "groups": groups, "spacing": spacing, "layout": layout, "ragged": ragged, "state": state, "gate": gate}


def _distill(name, do, dtype, rows, vocabulary, entries, temperature, masked=False):
    return {"name": name, "op": "distill", "do": do, "dtype": dtype, "rows": rows, "vocabulary": vocabulary, "entries": entries,
            "temperature": temperature, "masked": masked}


def listed():
    return [
        # the next token of a few rows: all latency
        _conv("conv_token_bf16", "token", "bf16", 4, 1, 512, 4, state=True),
        # the headline workload's sequences through the convolution of one layer
        _conv("conv_forward_bf16", "forward", "bf16", 64, 1000, 1024, 4),
        # a training pass over a ragged batch, sizes as a dataset gives them, in float32
        _conv("conv_train_fp32_ragged", "train", "fp32", 13, 1000, 300, 3, ragged=True, state=True),
        # the next token of a full batch: the states are read and written once
        _scan("scan_token_bf16", "token", "bf16", 64, 1, 2048, 16, state=True),
        # one long prompt: few rows, many steps, u and z and B and C as slices of their projections
        _scan("scan_prompt_bf16", "forward", "bf16", 1, 4000, 2048, 16, layout="sliced"),
        # a training pass of the headline workload's size, states kept as often as is fastest
        _scan("scan_train_bf16", "train", "bf16", 64, 1000, 1024, 16, spacing=8),
        # a training pass over long sequences that keeps few states, in float32 and batch-major
        _scan("scan_train_fp32_lean", "train", "fp32", 4, 2000, 512, 16, spacing=32, layout="batch"),
        # a short ragged batch with nothing a multiple of eight, continued from kept states
        _scan("scan_train_bf16_ragged", "train", "bf16", 13, 161, 300, 10, groups=2, spacing=16, ragged=True, state=True),
        # a small vocabulary, exact float32, some rows masked: evaluation only
        _distill("distill_loss_fp32", "loss", "fp32", 832, 1024, 16, 1.0, masked=True),
        # a vocabulary of ordinary size, loss and gradient in one read
        _distill("distill_train_bf16", "train", "bf16", 4096, 32000, 64, 2.0),
        # an odd vocabulary: rows that start anywhere
        _distill("distill_train_bf16_odd", "train", "bf16", 1000, 50257, 100, 1.5, masked=True),
        # few rows of a very large vocabulary
        _distill("distill_train_fp32_wide", "train", "fp32", 24, 128256, 32, 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("conv", "scan", "scan", "distill"))
    dtype = rng.choice(("fp32", "bf16", "bf16"))
    if op == "distill":
        rows, vocabulary = _log(rng, 1, 8192), _log(rng, 100, 200000)
        rows = max(1, min(rows, 100_000_000 // vocabulary))
        c = _distill(None, rng.choice(("loss", "train", "train")), dtype, rows, vocabulary, min(vocabulary, _log(rng, 1, 256)),
                     rng.choice((1.0, 1.0, 2.0, rng.uniform(0.5, 4.0))), rng.random() < 0.4)
    else:
        do = rng.choice(("token", "forward", "train", "train"))
        channels = _log(rng, 16, 2048)
        if rng.random() < 0.6:
            channels = max(16, channels - channels % 16)
        batch, t = _log(rng, 1, 64), 1 if do == "token" else _log(rng, 2, 4000)
        more = dict(layout=rng.choice(("time", "time", "batch", "sliced")), ragged=rng.random() < 0.4,
                    state=do == "token" or rng.random() < 0.4)
        if op == "conv":
            while batch * t * channels > 65_000_000:
                t = t * 3 // 4
            c = _conv(None, do, dtype, batch, t, channels, rng.choice((2, 3, 4, 4, 4, 5, 7)), silu=rng.random() < 0.8, **more)
        else:
            states = rng.choice((16, 16, 16, 8, 32, 64, rng.randint(1, 64)))
            groups = rng.choice((1, 1, 1, 2, 4))
            channels = max(groups, channels - channels % groups)
            while batch * t * channels * states > 500_000_000:
                t = t * 3 // 4
            c = _scan(None, do, dtype, batch, max(1, t), channels, states, groups, rng.choice((8, 8, 16, 32)),
                      gate=rng.random() < 0.8, **more)
    del c["name"]
    return c


# ---- what a program has in hand before the call ----------------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _array(layout, t, batch, width, parts, dtype, dev):
    """`parts` arrays [t, batch, width] of one type as the layout has them in memory, zeros."""
    if layout == "sliced":
        whole = torch.zeros(t, batch, parts * width, dtype=dtype, device=dev)
        return [whole[:, :, i * width:(i + 1) * width] for i in range(parts)]
    if layout == "batch":
        return [torch.zeros(batch, t, width, dtype=dtype, device=dev).transpose(0, 1) for _ in range(parts)]
    return [torch.zeros(t, batch, width, dtype=dtype, device=dev) for _ in range(parts)]


def _strides(x):
    return x.stride(0), x.stride(1)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(int(seed))
    return {"conv": _prepare_conv, "scan": _prepare_scan, "distill": _prepare_distill}[case["op"]](case, dev, g)


def _normal(g, dev, *shape):
    return torch.randn(shape, generator=g, device=dev)


def _lengths(c, dev, g):
    if not c["ragged"]:
        return None
    n = torch.randint(0, c["t"] + 1, (c["batch"],), generator=g, device=dev, dtype=torch.int32)
    n[0] = c["t"]
    return n


def _prepare_conv(c, dev, g):
    t, N, D, W, op = c["t"], c["batch"], c["channels"], c["width"], _TYPE[c["dtype"]]
    s = {"case": c, "lengths": _lengths(c, dev, g)}
    # the convolution reads the first half of a projection's columns where arrays are slices
    s["x"], s["dx"] = (_array(c["layout"], t, N, D, 2, op, dev)[0] for _ in range(2))
    s["y"], s["dy"] = (torch.zeros_like(s["x"]) for _ in range(2))
    s["x"].copy_(_normal(g, dev, t, N, D))
    s["dy"].copy_(_normal(g, dev, t, N, D))
    s["w"] = (_normal(g, dev, D, W) * W ** -0.5).to(op)
    s["bias"] = 0.3 * _normal(g, dev, D)
    s["s_in"] = _normal(g, dev, N, W - 1, D).to(op) if c["state"] else None
    s["ds_out"] = _normal(g, dev, N, W - 1, D).to(op) if c["state"] else None
    for k in ("s_out", "ds_in"):
        s[k] = torch.zeros(N, W - 1, D, dtype=op, device=dev) if c["state"] else None
    s["dw"], s["dbias"] = torch.zeros(D, W, device=dev), torch.zeros(D, device=dev)
    return s


def _prepare_scan(c, dev, g):
    t, N, D, S, G, op = c["t"], c["batch"], c["channels"], c["states"], c["groups"], _TYPE[c["dtype"]]
    s = {"case": c, "lengths": _lengths(c, dev, g)}
    for d in ("", "d"):
        s[d + "u"], s[d + "z"] = _array(c["layout"], t, N, D, 2, op, dev)
        s[d + "B"], s[d + "C"] = _array(c["layout"], t, N, G * S, 2, op, dev)
        s[d + "delta"] = torch.zeros_like(s[d + "u"])
        s[d + "y"] = torch.zeros_like(s[d + "u"])
    s["u"].copy_(torch.nn.functional.silu(_normal(g, dev, t, N, D)))       # what the convolution leaves
    s["z"].copy_(_normal(g, dev, t, N, D))
    s["B"].copy_(_normal(g, dev, t, N, G * S))
    s["C"].copy_(_normal(g, dev, t, N, G * S))
    s["delta"].copy_(0.5 * _normal(g, dev, t, N, D))
    s["dy"].copy_(_normal(g, dev, t, N, D))
    # step sizes of 0.001 to 0.1 and decay rates around 1 .. S, as such layers are initialised
    rate = torch.exp(torch.empty(D, device=dev).uniform_(math.log(1e-3), math.log(1e-1), generator=g))
    s["delta_bias"] = rate + torch.log(-torch.expm1(-rate))
    s["A"] = -torch.arange(1, S + 1, device=dev) * torch.exp(0.2 * _normal(g, dev, D, S))
    s["D"] = 1 + 0.1 * _normal(g, dev, D)
    if not c["gate"]:
        s["z"] = s["dz"] = None
    s["s_in"] = 0.3 * _normal(g, dev, N, D, S) if c["state"] else None
    s["ds_out"] = _normal(g, dev, N, D, S) if c["state"] else None
    s["ds_in"] = torch.zeros(N, D, S, device=dev) if c["state"] else None
    s["s_out"] = torch.zeros(N, D, S, device=dev)
    s["dA"], s["dD"], s["ddelta_bias"] = torch.zeros(D, S, device=dev), torch.zeros(D, device=dev), torch.zeros(D, device=dev)
    return s


def _prepare_distill(c, dev, g):
    R, V, K, op = c["rows"], c["vocabulary"], c["entries"], _TYPE[c["dtype"]]
    # logits of a trained readout: a few entries stand far out of the rest; the teacher's agree with them in part
    logits = 2 * _normal(g, dev, R, V)
    value, index = torch.topk(logits + _normal(g, dev, R, V), K, dim=1)
    s = {"case": c, "logits": logits.to(op), "indices": index.to(torch.int32), "values": (1.5 * value).contiguous()}
    s["weights"] = None
    if c["masked"]:
        s["weights"] = (torch.rand(R, generator=g, device=dev) < 0.8).float()       # prompt tokens and padding count nothing
        short = torch.randint(1, K + 1, (R, 1), generator=g, device=dev)            # fewer entries than there is room for
        s["indices"][torch.arange(K, device=dev)[None] >= short] = -1
    s["dloss"] = torch.ones(1, device=dev)
    s["loss"], s["row_loss"], s["row_stats"] = (torch.zeros(n, device=dev) for n in (1, R, 2 * R))
    s["dlogits"] = torch.zeros_like(s["logits"]) if c["do"] == "train" else None
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return {"conv": _own_conv, "scan": _own_scan, "distill": _own_distill}[state["case"]["op"]](state)
    return {"conv": _plain_conv, "scan": _plain_scan, "distill": _plain_distill}[state["case"]["op"]](state)


def _outputs(c, s):
    """The buffers that a pass fills."""
    names = {"conv": ("y", "s_out"), "scan": ("y", "s_out"), "distill": ("loss", "row_loss")}[c["op"]]
    if c["do"] == "train":
        names += {"conv": ("dx", "dw", "dbias", "ds_in"), "distill": ("dlogits",),
                  "scan": ("du", "ddelta", "dA", "dB", "dC", "dD", "dz", "ddelta_bias", "ds_in")}[c["op"]]
    return {n: s[n] for n in names if s[n] is not None}


def _own_conv(s):
    from paper_1606_03401_b200 import binding as B
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if "desc" not in s:
        s["desc"] = B.make_conv_desc(c["batch"], c["channels"], c["width"], c["t"], c["dtype"], silu=c["silu"],
                                     x_strides=_strides(s["x"]), y_strides=_strides(s["y"]))
        if c["do"] == "train":
            s["workspace"] = torch.empty(B.mebptt_conv_workspace_bytes(s["desc"]), dtype=torch.uint8, device=s["x"].device)
    B.mebptt_conv_forward(s["desc"], s["x"], s["w"], s["bias"], s["s_in"], s["lengths"], stream, s["y"], s["s_out"])
    if c["do"] == "train":
        B.mebptt_conv_backward(s["desc"], s["x"], s["w"], s["bias"], s["s_in"], s["lengths"], s["dy"], s["ds_out"], s["workspace"],
                               stream, s["dx"], s["dw"], s["dbias"], s["ds_in"])
    return _outputs(c, s)


def _own_scan(s):
    from paper_1606_03401_b200 import binding as B
    c, stream, train = s["case"], torch.cuda.current_stream().cuda_stream, s["case"]["do"] == "train"
    if "desc" not in s:
        at = {k + "_strides": _strides(s[k]) for k in ("u", "delta", "z", "B", "C", "y") if s[k] is not None}
        s["desc"] = d = B.make_scan_desc(c["batch"], c["channels"], c["states"], c["groups"], c["t"], c["dtype"], softplus=True,
                                         spacing=c["spacing"], **at)
        s["workspace"] = torch.empty(B.mebptt_scan_workspace_bytes(d, train), dtype=torch.uint8, device=s["u"].device)
        s["kept"] = torch.empty(B.mebptt_scan_kept_bytes(d), dtype=torch.uint8, device=s["u"].device) if train else None
    B.mebptt_scan_forward(s["desc"], s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["delta_bias"], s["s_in"],
                          s["lengths"], s["workspace"], stream, s["y"], s["s_out"], s["kept"])
    if train:
        B.mebptt_scan_backward(s["desc"], s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["delta_bias"],
                               s["lengths"], s["kept"], s["dy"], s["ds_out"], s["workspace"], stream, s["du"], s["ddelta"],
                               s["dA"], s["dB"], s["dC"], s["dD"], s["dz"], s["ddelta_bias"], s["ds_in"])
    return _outputs(c, s)


def _own_distill(s):
    from paper_1606_03401_b200 import binding as B
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if "desc" not in s:
        s["desc"] = B.make_distill_desc(c["rows"], c["vocabulary"], c["entries"], c["dtype"], temperature=c["temperature"],
                                        scale=1.0 / c["rows"])
    if c["do"] == "train":
        B.mebptt_distill_loss_grad(s["desc"], s["logits"], s["indices"], s["values"], s["weights"], s["dloss"], stream, s["loss"],
                                   s["row_loss"], s["dlogits"])
    else:
        B.mebptt_distill_loss(s["desc"], s["logits"], s["indices"], s["values"], s["weights"], stream, s["loss"], s["row_loss"],
                              s["row_stats"])
    return _outputs(c, s)


# ---- the same by elementary operations -------------------------------------------------------------------------------

def _within(s, t):
    """[t, batch, 1]: the steps that a row has; None: all of them."""
    return None if s["lengths"] is None else (torch.arange(t, device=s["lengths"].device)[:, None] < s["lengths"][None])[:, :, None]


def _only(x, within):
    return x if within is None else torch.where(within, x, torch.zeros_like(x))


def _dsilu(p):
    q = torch.sigmoid(p)
    return q * (1 + p * (1 - q))


def _plain_conv(s):
    c = s["case"]
    t, N, D, W, op = c["t"], c["batch"], c["channels"], c["width"], _TYPE[c["dtype"]]
    within, w = _within(s, t), s["w"].float()
    before = s["s_in"].float().transpose(0, 1) if c["state"] else torch.zeros(W - 1, N, D, device=w.device)
    x = torch.cat([before, _only(s["x"].float(), within)])
    p = (x.unfold(0, W, 1) * w).sum(-1) + s["bias"]
    out = {"y": _only(p * torch.sigmoid(p) if c["silu"] else p, within).to(op)}
    if c["state"]:
        n = s["lengths"].long() if c["ragged"] else torch.full((N,), t, device=w.device)
        last = n[:, None] + torch.arange(W - 1, device=w.device)               # places in x of the last W - 1 inputs
        out["s_out"] = x[last, torch.arange(N, device=w.device)[:, None]].to(op)
    if c["do"] != "train":
        return out
    dp = s["dy"].float() * _dsilu(p) if c["silu"] else s["dy"].float()
    dp = _only(dp, within)
    none = torch.zeros(W - 1, N, D, device=w.device)
    dx = (torch.cat([none, dp, none]).unfold(0, W, 1) * w.flip(1)).sum(-1)
    if c["state"]:
        dx[last, torch.arange(N, device=w.device)[:, None]] += s["ds_out"].float()
        out["ds_in"] = dx[:W - 1].transpose(0, 1).to(op)
    out["dx"] = _only(dx[W - 1:], within).to(op)
    out["dw"] = (x.unfold(0, W, 1) * dp[..., None]).sum((0, 1))
    out["dbias"] = dp.sum((0, 1))
    return out


def _recurrence(a, b):
    """s_k = a_k s_{k-1} + b_k from s_{-1} = 0, over dimension 0, in log2 of its length rounds."""
    reach = 1
    while reach < len(b):
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _by_channel(x, D, S):
    """[t, batch, groups * S] -> [t, batch, D, S]: every channel its group's."""
    t, N, GS = x.shape
    return x.float().view(t, N, GS // S, 1, S).expand(t, N, GS // S, D * S // GS, S).reshape(t, N, D, S)


def _plain_scan(s):
    c = s["case"]
    t, N, D, S, G, op = c["t"], c["batch"], c["channels"], c["states"], c["groups"], _TYPE[c["dtype"]]
    within = _within(s, t)
    u, pre = s["u"].float(), s["delta"].float() + s["delta_bias"]
    dt = _only(torch.where(pre > 20, pre, torch.log1p(torch.exp(pre))), within)
    a = torch.exp(dt[..., None] * s["A"])
    B, C = _by_channel(s["B"].contiguous(), D, S), _by_channel(s["C"].contiguous(), D, S)
    b = (dt * u)[..., None] * B
    if c["state"]:
        b[0] += a[0] * s["s_in"]
    h = _recurrence(a, b)
    del b
    v = (C * h).sum(-1) + s["D"] * u
    z = s["z"].float() if c["gate"] else None
    out = {"y": _only(v * z * torch.sigmoid(z) if c["gate"] else v, within).to(op), "s_out": h[-1]}
    if c["do"] != "train":
        return {"y": out["y"], "s_out": out["s_out"].clone()}
    dy = _only(s["dy"].float(), within)
    dv = dy * z * torch.sigmoid(z) if c["gate"] else dy
    if c["gate"]:
        out["dz"] = _only(dy * v * _dsilu(z), within).to(op)
    out["dC"] = (dv[..., None] * h).view(t, N, G, D // G, S).sum(3).view(t, N, G * S).to(op)
    before = torch.cat([(s["s_in"] if c["state"] else torch.zeros_like(h[0]))[None], h[:-1]])
    out["s_out"] = out["s_out"].clone()
    del h
    g = dv[..., None] * C
    del C
    if c["state"]:
        g[-1] += s["ds_out"]
    g = _recurrence(torch.cat([a[1:], torch.ones_like(a[:1])]).flip(0), g.flip(0)).flip(0)
    out["dB"] = (g * (dt * u)[..., None]).view(t, N, G, D // G, S).sum(3).view(t, N, G * S).to(op)
    gB = (g * B).sum(-1)
    out["du"] = _only(s["D"] * dv + dt * gB, within).to(op)
    if c["state"]:
        out["ds_in"] = a[0] * g[0]
    g = g.mul_(a).mul_(before)
    ddelta = _only((u * gB + (g * s["A"]).sum(-1)) * torch.sigmoid(pre), within)
    out["ddelta"] = ddelta.to(op)
    out["dA"] = (g * dt[..., None]).sum((0, 1))
    out["dD"] = (dv * u).sum((0, 1))
    out["ddelta_bias"] = ddelta.sum((0, 1))
    return out


def _plain_distill(s):
    c = s["case"]
    T, scale = c["temperature"], 1.0 / c["rows"]
    x = s["logits"].float() / T
    there = s["indices"] >= 0
    index = s["indices"].clamp(min=0).long()
    value = torch.where(there, s["values"] / T, torch.full_like(s["values"], -math.inf))
    e = torch.exp(value - value.amax(1, keepdim=True))
    q = e / e.sum(1, keepdim=True)
    top = x.amax(1, keepdim=True)
    x = x - top
    p = torch.exp(x)
    total = p.sum(1, keepdim=True)
    away = torch.log(total) - x.gather(1, index)                            # -log p of the listed entries
    weight = s["weights"] if c["masked"] else torch.ones(c["rows"], device=x.device)
    row = weight * T * T * torch.where(there, q * (torch.log(q) + away), torch.zeros_like(q)).sum(1)
    out = {"loss": scale * row.sum().view(1), "row_loss": row}
    if c["do"] == "train":
        d = (p / total).scatter_add_(1, index, torch.where(there, -q, torch.zeros_like(q)))
        out["dlogits"] = (d * (s["dloss"] * scale * T * weight)[:, None]).to(_TYPE[c["dtype"]])
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    e = _SIZE[c["dtype"]]
    if c["op"] == "distill":
        n = c["rows"] * c["vocabulary"]
        train = c["do"] == "train"
        return {"bytes": n * e * (2 if train else 1) + c["rows"] * (8 * c["entries"] + 12), "flops": n * (6 if train else 4)}
    n, D, N = c["batch"] * c["t"] * c["channels"], c["channels"], c["batch"]
    if c["op"] == "conv":
        W = c["width"]
        state = 2 * N * (W - 1) * D * e if c["state"] else 0
        bytes_, flops = 2 * n * e + state + D * (W * e + 4), n * (2 * W + 4)
        if c["do"] == "train":
            bytes_, flops = bytes_ + 3 * n * e + 2 * state + D * (W * (e + 4) + 8), flops + n * (6 * W + 8)
        return {"bytes": bytes_, "flops": flops}
    S, arrays, gs = c["states"], 4 if c["gate"] else 3, c["batch"] * c["t"] * 2 * c["groups"] * c["states"]
    state = 4 * N * D * S
    bytes_ = n * e * arrays + gs * e + D * (S + 2) * 4 + state * (2 if c["state"] else 1)
    flops = n * (6 * S + 10)
    if c["do"] == "train":
        bytes_ += n * e * (7 if c["gate"] else 5) + 2 * gs * e + 2 * D * (S + 2) * 4 + state * (2 if c["state"] else 0)
        flops += n * (20 * S + 20)
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits, a step or a row at a time -----------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "distill": _exact_distill}[case["op"]](case, s)


def _exact_conv(c, s):
    t, N, D, W = c["t"], c["batch"], c["channels"], c["width"]
    dev = s["w"].device
    n = s["lengths"].tolist() if c["ragged"] else [t] * N
    w = s["w"].double().requires_grad_(True)
    bias = s["bias"].double().requires_grad_(True)
    before = s["s_in"].double() if c["state"] else torch.zeros(N, W - 1, D, dtype=torch.float64, device=dev)
    out = {k: [] for k in ("y", "s_out", "dx", "ds_in")}
    dw, dbias = torch.zeros_like(w), torch.zeros_like(bias)
    for b in range(N):
        x = torch.cat([before[b], s["x"][:n[b], b].double()]).requires_grad_(True)
        p = sum(x[j:j + n[b]] * w[:, j] for j in range(W)) + bias
        y = p * torch.sigmoid(p) if c["silu"] else p
        rest = torch.zeros(t - n[b], D, dtype=torch.float64, device=dev)
        out["y"].append(torch.cat([y.detach(), rest]))
        out["s_out"].append(x.detach()[n[b]:])
        if c["do"] == "train":
            total = (y * s["dy"][:n[b], b].double()).sum()
            if c["state"]:
                total = total + (x[n[b]:] * s["ds_out"][b].double()).sum()
            gx, gw, gb = torch.autograd.grad(total, (x, w, bias), allow_unused=True)
            gx = torch.zeros_like(x) if gx is None else gx
            out["dx"].append(torch.cat([gx[W - 1:], rest]))
            out["ds_in"].append(gx[:W - 1])
            dw, dbias = dw if gw is None else dw + gw, dbias if gb is None else dbias + gb
    got = {"y": torch.stack(out["y"], 1)}
    if c["state"]:
        got["s_out"] = torch.stack(out["s_out"])
    if c["do"] == "train":
        got.update(dx=torch.stack(out["dx"], 1), dw=dw.detach(), dbias=dbias.detach())
        if c["state"]:
            got["ds_in"] = torch.stack(out["ds_in"])
    return got


def _exact_scan(c, s):
    t, N, D, S, G = c["t"], c["batch"], c["channels"], c["states"], c["groups"]
    if t * N * D * S > 1_100_000_000:       # the states of every step are held
        return None
    dev, of = s["A"].device, torch.float64
    n = s["lengths"] if c["ragged"] else torch.full((N,), t, device=dev)
    A, skip, bias = s["A"].double(), s["D"].double(), s["delta_bias"].double()
    h = [s["s_in"].double() if c["state"] else torch.zeros(N, D, S, dtype=of, device=dev)]
    out = {k: torch.zeros(t, N, D, dtype=of, device=dev) for k in ("y",)}
    group = torch.arange(D, device=dev) // (D // G)

    def step(k):
        live = (k < n)[:, None]
        u = torch.where(live, s["u"][k].double(), 0.0)
        pre = torch.where(live, s["delta"][k].double(), 0.0) + bias
        dt = torch.where(live, torch.nn.functional.softplus(pre, threshold=60.0), 0.0)
        B, C = (s[m][k].double().view(N, G, S)[:, group] for m in ("B", "C"))
        z = torch.where(live, s["z"][k].double(), 0.0) if c["gate"] else None
        return live, u, pre, dt, B, C, z

    def values(k, state, u, C):
        return torch.einsum("bds,bds->bd", C, state) + skip * u

    for k in range(t):
        live, u, pre, dt, B, C, z = step(k)
        h.append(h[-1] * torch.exp(dt[..., None] * A) + (dt * u)[..., None] * B)
        v = values(k, h[-1], u, C)
        out["y"][k] = torch.where(live, v * torch.nn.functional.silu(z) if c["gate"] else v, 0.0)
    out["s_out"] = h[-1].clone()
    if c["do"] != "train":
        return out
    for m in ("du", "ddelta") + (("dz",) if c["gate"] else ()):
        out[m] = torch.zeros(t, N, D, dtype=of, device=dev)
    out["dB"], out["dC"] = (torch.zeros(t, N, G * S, dtype=of, device=dev) for _ in range(2))
    dA, dD, dbias = torch.zeros(D, S, dtype=of, device=dev), torch.zeros(D, dtype=of, device=dev), torch.zeros(D, dtype=of, device=dev)
    carry = s["ds_out"].double() if c["state"] else torch.zeros(N, D, S, dtype=of, device=dev)
    for k in reversed(range(t)):
        live, u, pre, dt, B, C, z = step(k)
        dy = torch.where(live, s["dy"][k].double(), 0.0)
        dv = dy
        if c["gate"]:
            sig = torch.sigmoid(z)
            out["dz"][k] = dy * values(k, h[k + 1], u, C) * (sig + z * sig * (1 - sig))
            dv = dy * z * sig
        g = carry + dv[..., None] * C
        out["dC"][k] = (dv[..., None] * h[k + 1]).view(N, G, D // G, S).sum(2).view(N, G * S)
        out["dB"][k] = (g * (dt * u)[..., None]).view(N, G, D // G, S).sum(2).view(N, G * S)
        dtu = torch.einsum("bds,bds->bd", g, B)
        carry = g * torch.exp(dt[..., None] * A)
        da = carry * h[k]
        ddt = (torch.einsum("bds,ds->bd", da, A) + u * dtu) * torch.sigmoid(pre)
        ddt = torch.where(live, ddt, 0.0)
        out["du"][k] = torch.where(live, skip * dv + dt * dtu, 0.0)
        out["ddelta"][k] = ddt
        dA += (da * dt[..., None]).sum(0)
        dD += (dv * u).sum(0)
        dbias += ddt.sum(0)
    out.update(dA=dA, dD=dD, ddelta_bias=dbias)
    if c["state"]:
        out["ds_in"] = carry
    return out


def _exact_distill(c, s):
    T, R = c["temperature"], c["rows"]
    out = {"row_loss": torch.zeros(R, dtype=torch.float64, device=s["logits"].device)}
    if c["do"] == "train":
        out["dlogits"] = torch.zeros(R, c["vocabulary"], dtype=torch.float64, device=s["logits"].device)
    for r in range(0, R, 64):                                                # some rows at a time
        at = slice(r, min(R, r + 64))
        logp = torch.log_softmax(s["logits"][at].double() / T, 1)
        absent = s["indices"][at] < 0
        q = torch.softmax((s["values"][at].double() / T).masked_fill(absent, -math.inf), 1)
        index = s["indices"][at].long().masked_fill(absent, 0)
        logq = torch.log(q).masked_fill(absent, 0.0)
        weight = s["weights"][at].double() if c["masked"] else torch.ones(len(q), dtype=torch.float64, device=q.device)
        out["row_loss"][at] = weight * T * T * (q * (logq - logp.gather(1, index))).sum(1)
        if c["do"] == "train":
            target = torch.zeros_like(logp).scatter_add_(1, index, q)
            out["dlogits"][at] = (weight * T / R)[:, None] * (torch.exp(logp) - target)
    out["loss"] = out["row_loss"].sum().view(1) / R
    return out
