"""GPU: convolution, scan and distillation loss against the float64 oracle, element by element within the bounds it derives."""
import numpy as np
import pytest
import torch

from oracle import sequence_ops as O
from paper_1606_03401_b200 import binding as B
from tests.seq_util import Laid, assert_within, device, numpy, rounded

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _lengths(r, n, t, ragged):
    if not ragged:
        return None
    v = r.integers(0, t + 1, n)
    v[0] = t
    if n > 1:
        v[1] = 0
    if n > 2:
        v[2] = 1
    return v


def _hide(a, lengths):
    """NaN and infinities where a row has no steps."""
    if lengths is not None:
        for b, n in enumerate(lengths):
            a[n:, b] = np.nan
            a[n::2, b] = np.inf
    return a


class Conv:
    def __init__(self, dtype, N, t, D, W, layout="time", silu=True, state=True, ragged=True, bias=True, seed=0):
        r = np.random.default_rng(seed)
        self.dtype, self.silu = dtype, silu
        self.lengths = _lengths(r, N, t, ragged)
        self.x, self.dy = (_hide(rounded(r.standard_normal((t, N, D)), dtype), self.lengths) for _ in range(2))
        self.w, self.bias = rounded(r.standard_normal((D, W)), dtype), rounded(r.standard_normal(D), "fp32") if bias else None
        self.s_in, self.ds_out = (rounded(r.standard_normal((N, W - 1, D)), dtype) if state else None for _ in range(2))
        self.X, self.DY = Laid(self.x.shape, dtype, layout, self.x), Laid(self.x.shape, dtype, layout, self.dy)
        self.Y, self.DX = Laid(self.x.shape, dtype, layout), Laid(self.x.shape, dtype, layout)
        self.desc = B.make_conv_desc(N, D, W, t, dtype, silu, self.X.strides, self.Y.strides)
        self.dev = dict(w=device(self.w, dtype), bias=device(self.bias), s_in=device(self.s_in, dtype), ds_out=device(self.ds_out, dtype),
                        lengths=None if self.lengths is None else torch.tensor(self.lengths, dtype=torch.int32, device="cuda"))
        st = lambda: torch.full((N, W - 1, D), 7.0, device="cuda").to(self.X.x.dtype) if state else None  # noqa: E731
        self.s_out, self.ds_in = st(), st()
        self.dw, self.dbias = torch.full((D, W), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda") if bias else None
        self.workspace = torch.full((B.mebptt_conv_workspace_bytes(self.desc),), 255, dtype=torch.uint8, device="cuda")

    def forward(self):
        d = self.dev
        B.mebptt_conv_forward(self.desc, self.X.x, d["w"], d["bias"], d["s_in"], d["lengths"], _stream(), self.Y.x, self.s_out)

    def backward(self):
        d = self.dev
        B.mebptt_conv_backward(self.desc, self.X.x, d["w"], d["bias"], d["s_in"], d["lengths"], self.DY.x, d["ds_out"], self.workspace,
                               _stream(), self.DX.x, self.dw, self.dbias, self.ds_in)

    def outputs(self):
        return [v for v in (self.Y.x, self.s_out, self.DX.x, self.dw, self.dbias, self.ds_in) if v is not None]

    def check(self):
        z = lambda a: np.nan_to_num(a, nan=0.0, posinf=0.0) if self.lengths is not None else a  # noqa: E731  (not read)
        ref = O.conv(z(self.x), self.w, self.bias, self.s_in, self.lengths, self.silu, z(self.dy), self.ds_out)
        got = {"y": (self.Y.numpy(), self.dtype), "dx": (self.DX.numpy(), self.dtype), "dw": (numpy(self.dw), "fp32")}
        if self.bias is not None:
            got["dbias"] = (numpy(self.dbias), "fp32")
        if self.s_in is not None:
            got.update(s_out=(numpy(self.s_out), self.dtype), ds_in=(numpy(self.ds_in), self.dtype))
        for k, (v, dtype) in got.items():
            assert_within(k, v, ref[k], ref["bound"][k], dtype)
        assert all(a.untouched() for a in (self.X, self.Y, self.DX, self.DY))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,t,D,W,layout,kw", [
    (1, 1, 1, 4, "time", {}),
    (1, 2, 8, 8, "time", {}),                                   # fewer steps than the window
    (4, 9, 40, 4, "time", {}),
    (3, 33, 300, 3, "batch", {}),
    (3, 20, 37, 5, "odd", {}),
    (2, 50, 64, 4, "sliced", dict(silu=False)),
    (5, 17, 24, 2, "sliced", dict(state=False)),
    (3, 12, 520, 6, "time", dict(ragged=False, bias=False)),
    (2, 31, 16, 7, "batch", dict(ragged=False, state=False)),
    (9, 5, 264, 1, "time", {}),
])
def test_conv_matches_the_oracle(dtype, N, t, D, W, layout, kw):
    p = Conv(dtype, N, t, D, W, layout, **kw)
    p.forward()
    p.backward()
    p.check()


class Scan:
    def __init__(self, dtype, N, t, D, S, G=1, spacing=8, layout="time", gate=True, state=True, ragged=True, soft=True, extras=True, seed=0):
        r = np.random.default_rng(seed)
        self.dtype, self.soft, self.G = dtype, soft, G
        self.lengths = L = _lengths(r, N, t, ragged)
        draw = lambda *s: _hide(rounded(r.standard_normal(s), dtype), L)  # noqa: E731
        self.in_ = {"u": draw(t, N, D), "delta": draw(t, N, D) - 0.0, "Bm": draw(t, N, G * S), "Cm": draw(t, N, G * S),
                    "z": draw(t, N, D) if gate else None, "dy": draw(t, N, D)}
        if not soft:
            self.in_["delta"] = rounded(np.abs(self.in_["delta"]) * 0.25, dtype)
        self.A = rounded(-np.exp(r.standard_normal((D, S))), "fp32")
        self.skip, self.bias = (rounded(r.standard_normal(D), "fp32") if extras else None for _ in range(2))
        if extras:
            self.bias = rounded(np.abs(self.bias) - (2 if soft else 0), "fp32")
        self.s_in, self.ds_out = (rounded(r.standard_normal((N, D, S)), "fp32") if state else None for _ in range(2))
        lay = lambda a: None if a is None else Laid(a.shape, dtype, layout, a)  # noqa: E731
        self.L = {k: lay(v) for k, v in self.in_.items()}
        out = lambda k: None if self.in_[k] is None else Laid(self.in_[k].shape, dtype, layout)  # noqa: E731
        self.Lo = {"y": out("u"), "du": out("u"), "ddelta": out("delta"), "dz": out("z"), "dB": out("Bm"), "dC": out("Cm")}
        at = {n + "_strides": self.L[k].strides for n, k in (("u", "u"), ("delta", "delta"), ("z", "z"), ("B", "Bm"), ("C", "Cm"), ("y", "dy")) if self.L[k]}
        self.desc = B.make_scan_desc(N, D, S, G, t, dtype, soft, spacing, **at)
        self.dev = dict(A=device(self.A), skip=device(self.skip), bias=device(self.bias), s_in=device(self.s_in), ds_out=device(self.ds_out),
                        lengths=None if L is None else torch.tensor(L, dtype=torch.int32, device="cuda"))
        new = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
        self.s_out, self.ds_in, self.dA = new(N, D, S), new(N, D, S) if state else None, new(D, S)
        self.dskip, self.dbias = (new(D) if extras else None for _ in range(2))
        self.workspace = torch.full((B.mebptt_scan_workspace_bytes(self.desc, True),), 255, dtype=torch.uint8, device="cuda")
        self.kept = torch.full((B.mebptt_scan_kept_bytes(self.desc),), 255, dtype=torch.uint8, device="cuda")

    def _x(self, *names):
        return [None if self.L[k] is None else self.L[k].x for k in names]

    def forward(self, keep=True):
        d = self.dev
        u, delta, Bm, Cm, z = self._x("u", "delta", "Bm", "Cm", "z")
        B.mebptt_scan_forward(self.desc, u, delta, d["A"], Bm, Cm, d["skip"], z, d["bias"], d["s_in"], d["lengths"], self.workspace, _stream(),
                              self.Lo["y"].x, self.s_out, self.kept if keep else None)

    def backward(self):
        d = self.dev
        u, delta, Bm, Cm, z, dy = self._x("u", "delta", "Bm", "Cm", "z", "dy")
        o = {k: None if v is None else v.x for k, v in self.Lo.items()}
        B.mebptt_scan_backward(self.desc, u, delta, d["A"], Bm, Cm, d["skip"], z, d["bias"], d["lengths"], self.kept, dy, d["ds_out"],
                               self.workspace, _stream(), o["du"], o["ddelta"], self.dA, o["dB"], o["dC"], self.dskip, o["dz"], self.dbias,
                               self.ds_in)

    def outputs(self):
        return [v.x for v in self.Lo.values() if v is not None] + [v for v in (self.s_out, self.ds_in, self.dA, self.dskip, self.dbias) if v is not None]

    def check(self):
        z = {k: None if v is None else np.nan_to_num(v, nan=0.0, posinf=0.0) for k, v in self.in_.items()}
        ref = O.scan(z["u"], z["delta"], self.A, z["Bm"], z["Cm"], self.skip, z["z"], self.bias, self.s_in, self.lengths, self.soft,
                     z["dy"], self.ds_out, self.G)
        for k, v in self.Lo.items():
            if v is not None:
                assert_within(k, v.numpy(), ref[k], ref["bound"][k], self.dtype)
                assert v.untouched(), k
        for k, v in (("s_out", self.s_out), ("ds_in", self.ds_in), ("dA", self.dA), ("dskip", self.dskip), ("ddelta_bias", self.dbias)):
            if v is not None:
                assert_within(k, numpy(v), ref[k], ref["bound"][k], "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,t,D,S,kw", [
    (1, 1, 1, 1, dict(ragged=False)),
    (3, 1, 40, 16, {}),
    (3, 2, 5, 3, {}),
    (2, 33, 64, 16, dict(spacing=16)),
    (3, 32, 72, 16, dict(layout="batch")),
    (3, 70, 37, 10, dict(layout="odd", spacing=32)),
    (2, 41, 24, 16, dict(layout="sliced", G=3)),
    (2, 40, 300, 4, dict(state=False)),
    (2, 37, 150, 7, dict(spacing=32, gate=False)),
    (2, 50, 48, 20, dict(soft=False)),
    (2, 35, 20, 64, dict(G=2)),
    (2, 34, 17, 33, dict(extras=False, spacing=16)),
    (1, 300, 16, 16, dict(ragged=False)),                       # segments
    (2, 260, 24, 8, dict(spacing=32, layout="batch")),
    (3, 200, 12, 32, dict(spacing=16, G=2)),
    (3, 200, 9, 4, dict(state=False, gate=False)),
    (2, 43, 256, 16, dict(G=2)),                                # groups of whole blocks, columns that load as one
    (2, 90, 96, 12, dict(G=3, spacing=32, layout="sliced")),
])
def test_scan_matches_the_oracle(dtype, N, t, D, S, kw):
    p = Scan(dtype, N, t, D, S, **kw)
    p.forward()
    p.backward()
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("t,spacing", [(33, 8), (48, 8), (49, 16), (65, 8), (97, 32), (113, 16), (129, 32), (1024, 8)])
def test_scan_in_every_number_of_segments(dtype, t, spacing):
    """Three to sixty-four segments, whole batches of ends and rests of them, the last one of a single step; rows that end in the
    first ones or before them."""
    p = Scan(dtype, 5, t, 24, 16, spacing=spacing, ragged=True, seed=t)
    p.forward()
    p.backward()
    p.check()


def test_scan_without_kept_states_and_with_a_state_in_place():
    p = Scan("bf16", 3, 300, 24, 16, ragged=True)
    p.forward()
    y, s = p.Lo["y"].x.clone(), p.s_out.clone()
    p.Lo["y"].x.zero_()
    p.s_out = p.dev["s_in"]                                     # over the state it begins with, in segments
    p.forward(keep=False)
    assert torch.equal(p.Lo["y"].x, y) and torch.equal(p.s_out, s)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_token_by_token_is_the_prompt(dtype):
    """A prompt in one call, and the same steps one at a time with the states in place."""
    t, N, D, S, W = 12, 3, 40, 16, 4
    c, s = Conv(dtype, N, t, D, W, ragged=False), Scan(dtype, N, t, D, S, ragged=False)
    c.forward()
    s.forward()
    cd, sd = B.make_conv_desc(N, D, W, 1, dtype), B.make_scan_desc(N, D, S, 1, 1, dtype)
    cs, ss = c.dev["s_in"].clone(), s.dev["s_in"].clone()
    for k in range(t):
        y, v = torch.empty(N, D, dtype=c.X.x.dtype, device="cuda"), torch.empty(N, D, dtype=c.X.x.dtype, device="cuda")
        B.mebptt_conv_forward(cd, c.X.x[k], c.dev["w"], c.dev["bias"], cs, None, _stream(), y, cs)
        assert torch.equal(y, c.Y.x[k])
        u, delta, Bm, Cm, z = (x[k] for x in s._x("u", "delta", "Bm", "Cm", "z"))
        B.mebptt_scan_forward(sd, u, delta, s.dev["A"], Bm, Cm, s.dev["skip"], z, s.dev["bias"], ss, None, None, _stream(), v, ss)
        # the same operations in the same order but for the sum over states
        assert torch.allclose(v.float(), s.Lo["y"].x[k].float(), rtol=2 ** -7 if dtype == "bf16" else 1e-5, atol=1e-5)
    assert torch.equal(cs, c.s_out) and torch.allclose(ss, s.s_out, rtol=1e-6, atol=1e-7)


class Distill:
    def __init__(self, dtype, R, V, K, T=1.0, weights=True, pad=0, phase=0, seed=0, scale=None):
        r = np.random.default_rng(seed)
        self.dtype, self.T, self.scale = dtype, T, float(np.float32(1.0 / R if scale is None else scale))
        self.x = rounded(3 * r.standard_normal((R, V)), dtype)
        self.i = np.stack([r.permutation(V)[:K] if K <= V else r.integers(0, V, K) for _ in range(R)])
        self.v = rounded(2 * r.standard_normal((R, K)), "fp32")
        self.w = rounded(r.random(R) + 0.1, "fp32") if weights else None
        self.row = V + pad
        self.memory = torch.full((phase + R * self.row,), 977.0, device="cuda").to(device(self.x[:1], dtype).dtype)
        self.X = self.memory.as_strided((R, V), (self.row, 1), phase)
        self.dmemory = self.memory.clone()
        self.DX = self.dmemory.as_strided((R, V), (self.row, 1), phase)
        self.desc = B.make_distill_desc(R, V, K, dtype, T, self.scale, self.row, self.row)
        self.loss, self.row_loss, self.stats = (torch.full((n,), 7.0, device="cuda") for n in (1, R, 2 * R))
        self.dloss = torch.full((1,), 0.5, device="cuda")

    def upload(self):
        self.X.copy_(torch.from_numpy(self.x))
        self.dev = (torch.tensor(self.i, dtype=torch.int32, device="cuda"), device(self.v), device(self.w))
        return self

    def both(self):
        B.mebptt_distill_loss_grad(self.desc, self.X, *self.dev, self.dloss, _stream(), self.loss, self.row_loss, self.DX)

    def apart(self):
        B.mebptt_distill_loss(self.desc, self.X, *self.dev, _stream(), self.loss, self.row_loss, self.stats)
        B.mebptt_distill_grad(self.desc, self.X, *self.dev, self.stats, self.dloss, _stream(), self.DX)

    def check(self):
        ref = O.distill(self.x, self.i, self.v, self.w, float(np.float32(self.T)), self.scale, 0.5)
        assert_within("loss", numpy(self.loss)[0], ref["loss"], ref["bound"]["loss"], "fp32")
        assert_within("row_loss", numpy(self.row_loss), ref["row_loss"], ref["bound"]["row_loss"], "fp32")
        assert_within("dlogits", numpy(self.DX), ref["dlogits"], ref["bound"]["dlogits"], self.dtype)
        R, V = self.x.shape
        if self.row > V:
            assert bool((self.dmemory.as_strided((R - 1, self.row - V), (self.row, 1), self.DX.storage_offset() + V) == 977.0).all()) if R > 1 else True


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,V,K,kw", [
    (1, 1, 1, {}),
    (3, 7, 7, dict(T=0.5)),
    (5, 33, 4, dict(pad=3)),
    (40, 1024, 16, dict(T=2.0)),
    (3, 1000, 100, dict(phase=1)),
    (4, 5003, 33, dict(weights=False, phase=3, pad=1)),
    (2, 40000, 64, dict(T=1.5)),
    (400, 2048, 8, dict(T=4.0)),
    (2, 140001, 20, {}),                                        # longer than the registers of a cluster
    (2, 300000, 20, dict(T=3.0)),
])
def test_distill_matches_the_oracle(dtype, R, V, K, kw):
    p = Distill(dtype, R, V, K, **kw).upload()
    p.both()
    p.check()
    p.DX.fill_(7.0)
    p.apart()
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,K", [(50, 12), (20000, 700)])
def test_distill_entries_that_repeat_or_are_not_there(dtype, V, K):
    p = Distill(dtype, 8, V, K)
    p.i[0] = 5                                                  # one token, K times
    p.i[1] = np.random.default_rng(1).integers(0, 4, K)         # four tokens
    p.i[2, 3:] = -1
    p.i[3] = -1                                                 # no entry
    p.i[4, ::2] = V                                             # past the vocabulary
    p.v[5, 1:] = -np.inf
    p.v[6] = -np.inf                                            # no entry either
    p.w[7] = 0
    lowest = float(torch.finfo(p.X.dtype).min)
    p.upload()
    p.both()
    p.check()
    p.DX.fill_(7.0)
    p.apart()
    p.check()
    # masked tokens: logits of -inf and of the type's lowest value; rows that count nothing may hold anything
    p.x[:, 20:40] = -np.inf
    p.x[:, 40:45] = lowest
    for r in range(8):
        p.i[r][(p.i[r] >= 20) & (p.i[r] < 45)] = -1
    p.upload()
    p.X[3], p.X[6], p.X[7] = float("nan"), float("inf"), float("nan")
    p.both()
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distill_row_of_lowest_values_is_uniform_and_in_place(dtype):
    p = Distill(dtype, 3, 3000, 5)
    p.x[1] = float(torch.finfo(p.X.dtype).min)
    p.upload()
    p.DX, p.dmemory = p.X, p.memory                             # the gradient over the logits
    p.both()
    p.check()
    p.upload()
    B.mebptt_distill_loss(p.desc, p.X, *p.dev, _stream(), p.loss, p.row_loss, p.stats)
    B.mebptt_distill_grad(p.desc, p.X, *p.dev, p.stats, p.dloss, _stream(), p.X)
    p.check()


@pytest.mark.parametrize("make", [lambda: Conv("bf16", 4, 60, 72, 4), lambda: Scan("bf16", 2, 300, 40, 16), lambda: Scan("fp32", 2, 70, 40, 16, spacing=32),
                                  lambda: Distill("bf16", 9, 5001, 12).upload()], ids=["conv", "scan", "scan_lean", "distill"])
def test_captured_replayed_on_another_stream_and_bit_identical(make):
    p = make()

    def call():
        if isinstance(p, Distill):
            p.both()
        else:
            p.forward()
            p.backward()

    def outputs():
        return [p.loss, p.row_loss, p.DX] if isinstance(p, Distill) else p.outputs()

    call()
    torch.cuda.synchronize()
    want = [v.clone() for v in outputs()]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(outputs(), want))
    with torch.cuda.graph(graph):
        call()
    for v in outputs():
        v.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs(), want))


def test_float32_storage_has_two_names():
    a, b = Scan("fp32", 2, 40, 24, 16), Scan("fp32", 2, 40, 24, 16)
    b.desc.dtype = B.MEBPTT_TF32
    for p in (a, b):
        p.forward()
        p.backward()
    assert all(torch.equal(x, y) for x, y in zip(a.outputs(), b.outputs()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [60, 3000, 70001])
def test_distill_gradient_at_another_alignment_than_the_logits(dtype, V):
    p = Distill(dtype, 6, V, 9, pad=5, phase=1).upload()
    p.row = V + 2
    p.dmemory = torch.full((3 + 6 * p.row,), 977.0, device="cuda").to(p.X.dtype)
    p.DX = p.dmemory.as_strided((6, V), (p.row, 1), 3)
    p.desc.dlogits_row = p.row
    p.both()
    p.check()
    p.DX.fill_(7.0)
    p.apart()
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distill_many_rows_of_every_kernel(dtype):
    """More rows than there are warps, blocks or clusters at once, some of them without weight: rings go round, and clusters run
    through rows in which they do not meet."""
    for R, V in ((9000, 40), (1500, 3001), (330, 70000)):
        p = Distill(dtype, R, V, 6, T=1.3, seed=R)
        p.w[np.random.default_rng(0).random(R) < 0.4] = 0
        p.w[R // 3:R // 3 + 40] = 0
        p.upload()
        p.both()
        x = p.X.double() / float(np.float32(1.3))
        logp = torch.log_softmax(x, 1)
        q = torch.softmax(p.dev[1].double() / float(np.float32(1.3)), 1)
        idx = p.dev[0].long()
        w = p.dev[2].double()
        row = w * 1.3 ** 2 * (q * (torch.log(q) - logp.gather(1, idx))).sum(1)
        grad = (torch.exp(logp).scatter_add_(1, idx, -q) * (0.5 * p.scale * 1.3 * w)[:, None])
        # sums of thousands of exponentials in 32 bits, each with some six roundings: 3e-6 of a row's largest term is plenty
        assert torch.allclose(p.row_loss.double(), row, rtol=1e-5, atol=1e-5)
        tol = 2 ** -8 if dtype == "bf16" else 1e-5
        assert bool(((p.DX.double() - grad).abs() <= tol * grad.abs() + 3e-6 * grad.abs().amax(1, keepdim=True)).all())
        assert torch.allclose(p.loss.double(), p.scale * row.sum(), rtol=1e-5)
        first = [v.clone() for v in (p.loss, p.row_loss, p.DX)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.both()
        p.DX.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (p.loss, p.row_loss, p.DX)))


def test_longer_sequences_and_more_rows_agree_with_shorter_calls():
    """Two calls that hand a state on give what one call gives, in segments and without, with rows of every length."""
    for N, t, D, S in ((1, 2100, 40, 16), (40, 90, 264, 16), (2, 700, 20, 30)):
        p = Scan("fp32", N, t, D, S, ragged=N > 1, seed=t)
        p.forward()
        cut = t // 2 + 3
        parts, s = [], p.dev["s_in"].clone()
        for a, b in ((0, cut), (cut, t)):
            L = None if p.lengths is None else torch.tensor(np.clip(p.lengths - a, 0, b - a), dtype=torch.int32, device="cuda")
            u, delta, Bm, Cm, z = (x[a:b] for x in p._x("u", "delta", "Bm", "Cm", "z"))
            d = B.make_scan_desc(N, D, S, 1, b - a, "fp32")
            ws = torch.empty(B.mebptt_scan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
            y = torch.empty(b - a, N, D, device="cuda")
            B.mebptt_scan_forward(d, u, delta, p.dev["A"], Bm, Cm, p.dev["skip"], z, p.dev["bias"], s, L, ws, _stream(), y, s)
            parts.append(y)
        y = torch.cat(parts)
        # decays of up to t steps multiplied in another order: (4 + |x|) 2^-24 a step of what has not faded
        scale = p.Lo["y"].x.abs().amax()
        assert float((y - p.Lo["y"].x).abs().amax() / scale) < 2e-5 and torch.allclose(s, p.s_out, rtol=1e-4, atol=2e-5 * float(p.s_out.abs().max()))


def test_offsets_past_32_bits():
    """Steps, rows and logits' rows that lie 2^31 elements apart, against the same data close together."""
    far, t, N, D, S, W = 1 << 31, 3, 2, 24, 16, 4
    c, p = Conv("bf16", N, t, D, W, ragged=False), Scan("bf16", N, t, D, S, ragged=False)
    c.forward()
    c.backward()
    p.forward()
    p.backward()
    memory = torch.zeros((t - 1) * far + 4096, dtype=torch.bfloat16, device="cuda")
    used = 0

    def place(like=None, width=D):
        nonlocal used
        x = memory.as_strided((t, N, width), (far, 512, 1), used)
        used += width
        if like is not None:
            x.copy_(like)
        return x

    at = (far, 512)
    x, dy, y, dx = place(c.X.x), place(c.DY.x), place(), place()
    desc = B.make_conv_desc(N, D, W, t, "bf16", True, at, at)
    d, s_out, ds_in = c.dev, torch.empty_like(c.s_out), torch.empty_like(c.ds_in)
    B.mebptt_conv_forward(desc, x, d["w"], d["bias"], d["s_in"], None, _stream(), y, s_out)
    dw, db = torch.empty_like(c.dw), torch.empty_like(c.dbias)
    B.mebptt_conv_backward(desc, x, d["w"], d["bias"], d["s_in"], None, dy, d["ds_out"], c.workspace, _stream(), dx, dw, db, ds_in)
    for a, b in ((y, c.Y.x), (dx, c.DX.x), (s_out, c.s_out), (ds_in, c.ds_in), (dw, c.dw), (db, c.dbias)):
        assert torch.equal(a, b)
    memory.zero_()
    used, d = 0, p.dev
    u, delta, z, dy = (place(p.L[k].x) for k in ("u", "delta", "z", "dy"))
    Bm, Cm = (place(p.L[k].x, S) for k in ("Bm", "Cm"))
    y, du, dd, dz = (place() for _ in range(4))
    dB, dC = place(width=S), place(width=S)
    desc = B.make_scan_desc(N, D, S, 1, t, "bf16", True, 8, at, at, at, at, at, at)
    s_out, dA, dk, db, ds_in = (torch.empty_like(v) for v in (p.s_out, p.dA, p.dskip, p.dbias, p.ds_in))
    B.mebptt_scan_forward(desc, u, delta, d["A"], Bm, Cm, d["skip"], z, d["bias"], d["s_in"], None, p.workspace, _stream(), y, s_out, p.kept)
    B.mebptt_scan_backward(desc, u, delta, d["A"], Bm, Cm, d["skip"], z, d["bias"], None, p.kept, dy, d["ds_out"], p.workspace, _stream(), du, dd, dA,
                           dB, dC, dk, dz, db, ds_in)
    for a, b in ((y, p.Lo["y"].x), (du, p.Lo["du"].x), (dd, p.Lo["ddelta"].x), (dz, p.Lo["dz"].x), (dB, p.Lo["dB"].x), (dC, p.Lo["dC"].x),
                 (s_out, p.s_out), (dA, p.dA), (dk, p.dskip), (db, p.dbias), (ds_in, p.ds_in)):
        assert torch.equal(a, b)
    for V in (500, 3001):
        q = Distill("bf16", 3, V, 7).upload()
        q.both()
        x = memory.as_strided((3, V), (far, 1), 1)
        x.copy_(q.X)
        desc = B.make_distill_desc(3, V, 7, "bf16", 1.0, q.scale, far, far)
        row = torch.empty_like(q.row_loss)
        B.mebptt_distill_loss_grad(desc, x, *q.dev, q.dloss, _stream(), None, row, x)
        # (rows that begin elsewhere within 16 bytes sum in another order)
        assert torch.allclose(row, q.row_loss, rtol=1e-5) and torch.allclose(x.float(), q.DX.float(), rtol=2 ** -7, atol=1e-7)


def test_two_calls_at_once():
    """Different problems on two streams, each with workspaces of its own, again and again."""
    one = [Scan("bf16", 2, 500, 40, 16), Distill("bf16", 40, 70000, 9).upload(), Conv("bf16", 4, 60, 72, 4)]
    two = [Scan("fp32", 3, 300, 24, 8, spacing=32, seed=5), Distill("fp32", 60, 9000, 30, seed=5).upload(), Conv("fp32", 3, 90, 40, 3, seed=5)]

    def call(p):
        if isinstance(p, Distill):
            p.both()
        else:
            p.forward()
            p.backward()

    def outputs(p):
        return [p.loss, p.row_loss, p.DX] if isinstance(p, Distill) else p.outputs()

    for p in one + two:
        call(p)
    torch.cuda.synchronize()
    want = [[v.clone() for v in outputs(p)] for p in one + two]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(10):
        for a, b in zip(one, two):
            for p, st in ((a, streams[0]), (b, streams[1])):
                with torch.cuda.stream(st):
                    call(p)
    torch.cuda.synchronize()
    for p, w in zip(one + two, want):
        assert all(torch.equal(a, b) for a, b in zip(outputs(p), w))


@pytest.mark.parametrize("t", [1, 500, 3000])
def test_a_state_that_does_not_fade_stays_as_it_is(t):
    """A = 0: every decay is 1 exactly, however many steps, with and without segments; likewise steps of size 0."""
    N, D, S = 2, 24, 16
    r = np.random.default_rng(t)
    s_in = device(r.standard_normal((N, D, S)))
    zero = lambda *n: torch.zeros(*n, device="cuda")  # noqa: E731
    delta, one = torch.rand(t, N, D, device="cuda"), torch.rand(t, N, S, device="cuda")
    d = B.make_scan_desc(N, D, S, 1, t, "fp32", softplus=False)
    ws = torch.empty(B.mebptt_scan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    for step, A in ((delta, zero(D, S)), (zero(t, N, D), device(-np.exp(r.standard_normal((D, S)))))):
        out = zero(N, D, S)
        B.mebptt_scan_forward(d, zero(t, N, D), step, A, one, one, None, None, None, s_in, None, ws, _stream(), zero(t, N, D), out)
        assert torch.equal(out, s_in)


def test_lengths_outside_their_range_are_the_nearest_inside():
    a, b = Scan("fp32", 4, 40, 24, 16, seed=3), Scan("fp32", 4, 40, 24, 16, seed=3)
    c, e = Conv("fp32", 4, 40, 24, 4, seed=3), Conv("fp32", 4, 40, 24, 4, seed=3)
    wild = torch.tensor([1 << 30, -5, 1, int(a.lengths[3])], dtype=torch.int32, device="cuda")
    for p, q in ((a, b), (c, e)):
        assert p.lengths[0] == 40 and p.lengths[1] == 0
        q.dev["lengths"] = wild.clone()
        q.dev["lengths"][2:] = p.dev["lengths"][2:]
        for x in (p, q):
            x.forward()
            x.backward()
        assert all(torch.equal(x, y) for x, y in zip(p.outputs(), q.outputs()))


@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_distill_entries_that_are_not_there_may_hold_anything(V):
    p = Distill("fp32", 5, V, 8)
    p.i[:, 5:] = -1
    p.upload()
    p.both()
    want = [v.clone() for v in (p.loss, p.row_loss, p.DX)]
    p.dev[1][:, 5] = float("nan")
    p.dev[1][:, 6] = float("inf")
    p.dev[0][:, 7] = 1 << 30
    p.both()
    assert all(torch.equal(a, b) for a, b in zip(want, (p.loss, p.row_loss, p.DX)))
