"""Slow float64 oracle of the operators over sequences: the short causal convolution, the selective scan and the
distillation loss, forward and backward, a step (or a row) at a time.

Everything is computed in ``Bounded`` numbers, which carry along what a float32 computation of the same formula may be off:
``bound`` holds that for every output, in units of 2**-24 (absolute).  Arrays over time are [t, batch, width]; ``lengths``
holds a row's steps (None: all).
"""
from __future__ import annotations

import numpy as np

from .bounded import Bounded, exp, lift, log, sigmoid, softplus

LEVELS = 160    # additions that a term of a sum over steps, rows or channels goes through, at the tests' sizes


def _put(out, bound, name, where, x):
    out[name][where], bound[name][where] = x.v, x.e


def _live(lengths, t, batch):
    n = np.full(batch, t) if lengths is None else np.clip(lengths, 0, t)
    return n.astype(int)


def conv(x, w, bias, s_in=None, lengths=None, silu=True, dy=None, ds_out=None):
    """y, s_out and, with dy, dx, dw, dbias, ds_in.  x [t,B,D], w [D,W], states [B,W-1,D]."""
    t, N, D = x.shape
    W = w.shape[1]
    n = _live(lengths, t, N)
    bias = np.zeros(D) if bias is None else bias
    shapes = {"y": (t, N, D), "s_out": (N, W - 1, D)}
    if dy is not None:
        shapes.update(dx=(t, N, D), dw=(D, W), dbias=(D,), ds_in=(N, W - 1, D))
    out, bound = ({k: np.zeros(v) for k, v in shapes.items()} for _ in range(2))
    dw, dbias = [], []
    for b in range(N):
        ext = np.concatenate([np.zeros((W - 1, D)) if s_in is None else s_in[b], x[:n[b], b]])
        out["s_out"][b] = ext[len(ext) - (W - 1):]
        dext = [Bounded(np.zeros(D)) for _ in ext]
        if dy is not None and ds_out is not None:
            dext[n[b]:] = [Bounded(v) for v in ds_out[b]]
        for k in range(n[b]):
            p = lift(bias)
            for j in range(W):
                p = p + lift(w[:, j]) * ext[k + j]
            sig = sigmoid(p)
            _put(out, bound, "y", (k, b), p * sig if silu else p)
            if dy is None:
                continue
            dp = dy[k, b] * (sig * (1 + p * (1 - sig))) if silu else lift(dy[k, b])
            for j in range(W):
                dext[k + j] = dext[k + j] + lift(w[:, j]) * dp
            dw.append([dp * ext[k + j] for j in range(W)])
            dbias.append(dp)
        if dy is not None:
            for i, d in enumerate(dext):
                if i < W - 1:
                    _put(out, bound, "ds_in", (b, i), d)
                else:
                    _put(out, bound, "dx", (i - W + 1, b), d)
    for j in range(W if dw else 0):
        _put(out, bound, "dw", (slice(None), j), _stack([d[j] for d in dw]).sum(0, LEVELS))
    if dbias:
        _put(out, bound, "dbias", slice(None), _stack(dbias).sum(0, LEVELS))
    out["bound"] = bound
    return out


def _stack(xs):
    return Bounded(np.stack([x.v for x in xs]), np.stack([x.e for x in xs]))


def scan(u, delta, A, Bm, Cm, skip=None, z=None, bias=None, s_in=None, lengths=None, soft=True, dy=None, ds_out=None, groups=1):
    """y, s_out and, with dy, every gradient.  u [t,B,D], Bm [t,B,G*N], A [D,N], states [B,D,N]."""
    t, N, D = u.shape
    S = A.shape[1]
    n = _live(lengths, t, N)
    skip = np.zeros(D) if skip is None else skip
    bias = np.zeros(D) if bias is None else bias
    group = np.arange(D) // (D // groups)
    shapes = {"y": (t, N, D), "s_out": (N, D, S)}
    if dy is not None:
        shapes.update(du=(t, N, D), ddelta=(t, N, D), dz=(t, N, D), dA=(D, S), dB=(t, N, groups * S), dC=(t, N, groups * S),
                      dskip=(D,), ddelta_bias=(D,), ds_in=(N, D, S))
    out, bound = ({k: np.zeros(v) for k, v in shapes.items()} for _ in range(2))
    over_time = {"dA": [], "dskip": [], "ddelta_bias": []}

    def by_group(v):                                            # [D, S] -> [G * S]: sums over a group's channels
        return v.reshape(groups, D // groups, S).sum(1, LEVELS).reshape(groups * S)

    def step(k, b):
        B, C = Bm[k, b].reshape(groups, S)[group], Cm[k, b].reshape(groups, S)[group]
        pre = lift(delta[k, b]) + bias
        dt, dsoft = (softplus(pre), sigmoid(pre)) if soft else (pre, lift(np.ones(D)))
        return B, C, dt, dsoft, exp(dt[:, None] * A)

    def value(C, s, k, b):
        return (C * s).sum(1) + skip * lift(u[k, b])

    for b in range(N):
        states = [lift(np.zeros((D, S)) if s_in is None else s_in[b])]
        for k in range(n[b]):
            B, C, dt, _, a = step(k, b)
            states.append(a * states[-1] + (dt * u[k, b])[:, None] * B)
            v = value(C, states[-1], k, b)
            _put(out, bound, "y", (k, b), v if z is None else v * (z[k, b] * sigmoid(z[k, b])))
        _put(out, bound, "s_out", b, states[-1])
        if dy is None:
            continue
        carry = lift(np.zeros((D, S)) if ds_out is None else ds_out[b])
        for k in reversed(range(n[b])):
            B, C, dt, dsoft, a = step(k, b)
            s = states[k + 1]
            dv = lift(dy[k, b])
            if z is not None:
                sig = sigmoid(z[k, b])
                _put(out, bound, "dz", (k, b), dy[k, b] * value(C, s, k, b) * (sig * (1 + z[k, b] * (1 - sig))))
                dv = dy[k, b] * z[k, b] * sig
            g = dv[:, None] * C + carry
            _put(out, bound, "dC", (k, b), by_group(dv[:, None] * s))
            _put(out, bound, "dB", (k, b), by_group(g * (dt * u[k, b])[:, None]))
            gB = (g * B).sum(1)
            _put(out, bound, "du", (k, b), skip * dv + dt * gB)
            da = g * (a * states[k])
            ddt = ((A * da).sum(1) + u[k, b] * gB) * dsoft
            _put(out, bound, "ddelta", (k, b), ddt)
            for name, x in (("dA", dt[:, None] * da), ("dskip", dv * u[k, b]), ("ddelta_bias", ddt)):
                over_time[name].append(x)
            carry = a * g
        _put(out, bound, "ds_in", b, carry)
    for name, xs in over_time.items():
        if xs:
            _put(out, bound, name, slice(None), _stack(xs).sum(0, LEVELS))
    out["bound"] = bound
    return out


def distill(logits, indices, values, weights=None, T=1.0, scale=1.0, dloss=1.0):
    """loss, row_loss, dlogits.  logits [R,V], indices and values [R,K]."""
    R, V = logits.shape
    out, bound = ({"row_loss": np.zeros(R), "dlogits": np.zeros((R, V))} for _ in range(2))
    over = 1 / T
    for r in range(R):
        w = 1.0 if weights is None else weights[r]
        there = (indices[r] >= 0) & (indices[r] < V) & (values[r] > -np.inf)
        if w == 0 or not there.any():
            continue
        i, v = indices[r][there], values[r][there]
        x, low = np.where(np.isneginf(logits[r]), -1e30, logits[r]), np.isneginf(logits[r])
        v, x = (lift(v) - v.max()) * over, (lift(x) - x[~low].max()) * over
        e, p = exp(v), exp(x)
        Q, S = e.sum(0, LEVELS), p.sum(0, LEVELS)
        q = e * Bounded(1 / Q.v, Q.e / Q.v ** 2 + 1 / Q.v)
        p = p * Bounded(1 / S.v, S.e / S.v ** 2 + 1 / S.v)
        term = q * ((v - log(Q)) - (x[i] - log(S)))
        term = Bounded(np.where(q.v > 0, term.v, 0), np.where(q.v > 0, term.e, 0))
        row = w * T * T * term.sum(0, LEVELS)
        _put(out, bound, "row_loss", r, row)
        d = p * 1.0
        for j, at in enumerate(i):
            d.v[at] -= q.v[j]
            d.e[at] += q.e[j] + np.abs(d.v[at]) + q.v[j]
        _put(out, bound, "dlogits", r, d * (lift(dloss) * scale * w * T))
    total = Bounded(out["row_loss"], bound["row_loss"]).sum(0, 2) * scale
    out["loss"], bound["loss"] = total.v, total.e
    out["bound"] = bound
    return out
