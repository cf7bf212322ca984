"""GPU: the operators as a recurrent language model has them -- projection, convolution, scan, readout, distillation loss, and all of it
backwards -- against the same model in float64, and the same model token by token."""
import numpy as np
import pytest
import torch

from paper_1606_03401_b200 import binding as B
from paper_1606_03401_b200 import synth
from paper_1606_03401_b200.harness import rel_l2
from tests.seq_util import device, numpy

pytestmark = pytest.mark.gpu

# Everything is stored in float32 but what enters the tensor-core contractions, bfloat16: x and the weights exactly (they are drawn
# so), y, dlogits and the gradient of the projection with an error of 2^-9 of a value on average.  Some ten such errors add up in a
# gradient: less than 0.7 %, with room for terms that cancel, is the tolerance of bfloat16 training steps.
TOL = 2e-2


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Model:
    """logits = W_out y;  y = scan(silu(conv(W x)_1), W x_2 .. 5):  one contraction gives the convolution's input, the gate, the step
    sizes and B and C, as column slices of its result."""

    def __init__(self, t=40, N=3, I=64, D=48, S=16, W=4, V=200, K=8, seed=0):
        r = np.random.default_rng(seed)
        bf = lambda *s: synth.round_to_bf16(r.standard_normal(s))  # noqa: E731
        f = lambda *s: synth.round_to_fp32(r.standard_normal(s))  # noqa: E731
        self.t, self.N, self.I, self.D, self.S, self.W, self.V, self.K = t, N, I, D, S, W, V, K
        self.cols = 3 * D + 2 * S
        self.p = {"x": bf(t, N, I), "W_in": synth.round_to_bf16(r.standard_normal((self.cols, I)) * I ** -0.5),
                  "W_out": synth.round_to_bf16(r.standard_normal((V, D)) * D ** -0.5), "w": f(D, W) * 0.5, "bias": 0.1 * f(D), "A": -np.exp(f(D, S)),
                  "skip": f(D), "dbias": f(D) - 2, "values": f(t * N, K)}
        self.p = {k: v if k in ("x", "W_in", "W_out") else synth.round_to_fp32(v) for k, v in self.p.items()}
        self.idx = np.stack([r.permutation(V)[:K] for _ in range(t * N)])
        self.dev = {k: device(v, "bf16" if k in ("x", "W_in", "W_out") else "fp32") for k, v in self.p.items()}
        self.dev["idx"] = torch.tensor(self.idx, dtype=torch.int32, device="cuda")

    def slices(self, proj):
        """(convolution's input, z, delta, B, C) of a projection [t, batch, columns]."""
        D, S = self.D, self.S
        return tuple(proj[..., a:b] for a, b in ((0, D), (D, 2 * D), (2 * D, 3 * D), (3 * D, 3 * D + S), (3 * D + S, 3 * D + 2 * S)))

    def descs(self, t, train):
        N, D, S = self.N, self.D, self.S
        at = (N * self.cols, self.cols)
        conv = B.make_conv_desc(N, D, self.W, t, "fp32", x_strides=at)
        scan = B.make_scan_desc(N, D, S, 1, t, "fp32", spacing=16, delta_strides=at, z_strides=at, B_strides=at, C_strides=at)
        return conv, scan

    def gemm(self, A, a_mn, Bm, b_mn, M, N, K):
        out = torch.empty(M, N, device="cuda")
        B.mebptt_gemm_bf16(A, A.stride(0), int(a_mn), Bm, Bm.stride(0), int(b_mn), out, N, False, None, M, N, K, None, _stream())
        return out

    def forward(self, x, conv_state=None, scan_state=None, kept=None):
        """One call for t steps: logits, and what the backward pass needs.  States are updated in place."""
        d, t, N, D = self.dev, x.shape[0], self.N, self.D
        cd, sd = self.descs(t, kept is not None)
        proj = self.gemm(x.reshape(t * N, self.I), False, d["W_in"], False, t * N, self.cols, self.I).view(t, N, self.cols)
        xi, z, delta, Bm, Cm = self.slices(proj)
        u, y = torch.empty(t, N, D, device="cuda"), torch.empty(t, N, D, device="cuda")
        B.mebptt_conv_forward(cd, xi, d["w"], d["bias"], conv_state, None, _stream(), u, conv_state)
        ws = torch.empty(B.mebptt_scan_workspace_bytes(sd, True), dtype=torch.uint8, device="cuda")
        keep = torch.empty(B.mebptt_scan_kept_bytes(sd), dtype=torch.uint8, device="cuda") if kept is not None else None
        B.mebptt_scan_forward(sd, u, delta, d["A"], Bm, Cm, d["skip"], z, d["dbias"], scan_state, None, ws, _stream(), y, scan_state, keep)
        yb = y.view(t * N, D).to(torch.bfloat16)
        logits = self.gemm(yb, False, d["W_out"], False, t * N, self.V, D)
        return logits, dict(proj=proj, u=u, yb=yb, ws=ws, keep=keep, cd=cd, sd=sd)

    def backward(self, logits, s):
        d, t, N, D = self.dev, self.t, self.N, self.D
        R = t * N
        out = {"loss": torch.empty(1, device="cuda")}
        dd = B.make_distill_desc(R, self.V, self.K, "fp32", temperature=2.0, scale=1.0 / R)
        dlogits = torch.empty_like(logits)
        B.mebptt_distill_loss_grad(dd, logits, d["idx"], d["values"], None, None, _stream(), out["loss"], torch.empty(R, device="cuda"), dlogits)
        dlb = dlogits.to(torch.bfloat16)
        out["W_out"] = self.gemm(dlb, True, s["yb"], True, self.V, D, R)
        dy = self.gemm(dlb, False, d["W_out"], True, R, D, self.V).view(t, N, D)
        dproj = torch.empty_like(s["proj"])
        xi, z, delta, Bm, Cm = self.slices(s["proj"])
        dxi, dz, ddelta, dB, dC = self.slices(dproj)
        du = torch.empty(t, N, D, device="cuda")
        new = lambda *n: torch.empty(*n, device="cuda")  # noqa: E731
        out.update(A=new(D, self.S), skip=new(D), dbias=new(D), w=new(D, self.W), bias=new(D))
        B.mebptt_scan_backward(s["sd"], s["u"], delta, d["A"], Bm, Cm, d["skip"], z, d["dbias"], None, s["keep"], dy, None, s["ws"], _stream(),
                               du, ddelta, out["A"], dB, dC, out["skip"], dz, out["dbias"], None)
        ws = torch.empty(B.mebptt_conv_workspace_bytes(s["cd"]), dtype=torch.uint8, device="cuda")
        B.mebptt_conv_backward(s["cd"], xi, d["w"], d["bias"], None, None, du, None, ws, _stream(), dxi, out["w"], out["bias"], None)
        db = dproj.view(R, self.cols).to(torch.bfloat16)
        out["W_in"] = self.gemm(db, True, d["x"].view(R, self.I), True, self.cols, self.I, R)
        out["x"] = self.gemm(db, False, d["W_in"], True, R, self.I, self.cols)
        return out

    def reference(self):
        """The same in float64, with torch's own derivatives."""
        q = {k: torch.tensor(v, dtype=torch.float64, requires_grad=k != "values") for k, v in self.p.items()}
        t, N, D, S, W = self.t, self.N, self.D, self.S, self.W
        xi, z, delta, Bm, Cm = self.slices(q["x"] @ q["W_in"].T)
        ext = torch.cat([torch.zeros(W - 1, N, D, dtype=torch.float64), xi])
        u = torch.nn.functional.silu(sum(ext[j:j + t] * q["w"][:, j] for j in range(W)) + q["bias"])
        dt = torch.nn.functional.softplus(delta + q["dbias"])
        s, ys = torch.zeros(N, D, S, dtype=torch.float64), []
        for k in range(t):
            s = s * torch.exp(dt[k][..., None] * q["A"]) + (dt[k] * u[k])[..., None] * Bm[k][:, None]
            ys.append((s * Cm[k][:, None]).sum(-1) + q["skip"] * u[k])
        y = torch.stack(ys) * torch.nn.functional.silu(z)
        logits = y.reshape(t * N, D) @ q["W_out"].T
        logp = torch.log_softmax(logits / 2, 1)
        teacher = torch.softmax(q["values"] / 2, 1)
        idx = torch.tensor(self.idx)
        loss = 4 * (teacher * (torch.log(teacher) - logp.gather(1, idx))).sum(1).mean()
        loss.backward()
        return logits, loss, {k: v.grad for k, v in q.items() if v.grad is not None}


def test_a_training_step_of_a_recurrent_language_model():
    m = Model()
    logits, saved = m.forward(m.dev["x"], kept=True)
    got = m.backward(logits.clone(), saved)
    want_logits, loss, grads = m.reference()
    assert rel_l2(numpy(logits), want_logits.detach().numpy()) < TOL
    assert abs(float(got["loss"]) - loss.item()) < TOL * loss.item()
    errs = {k: rel_l2(numpy(got[k]), g.numpy()) for k, g in grads.items()}
    assert set(errs) == {"x", "W_in", "W_out", "w", "bias", "A", "skip", "dbias"} and max(errs.values()) < TOL, errs


def test_generation_continues_a_prompt():
    m = Model(t=20)
    whole, _ = m.forward(m.dev["x"])
    conv_state = torch.zeros(m.N, m.W - 1, m.D, device="cuda")
    scan_state = torch.zeros(m.N, m.D, m.S, device="cuda")
    rows = [m.forward(m.dev["x"][:13], conv_state, scan_state)[0]]
    for k in range(13, 20):
        rows.append(m.forward(m.dev["x"][k:k + 1], conv_state, scan_state)[0])
    # float32 sums over states in another order (1e-6), then y rounded to bfloat16: at most a step of it, 2^-8, in a few elements
    assert rel_l2(numpy(torch.cat(rows)), numpy(whole)) < 2 ** -9
