"""GPU: the operators over sequences where calls meet: several host threads, rows and states at the edge of what counts, waits that run out."""
import threading

import numpy as np
import pytest
import torch

from paper_1606_03401_b200 import binding as B
from tests.test_gpu_sequence_ops import Conv, Distill, Scan, _stream

pytestmark = pytest.mark.gpu


def _together(calls):
    """Each call by a host thread of its own, on a stream of its own; what a thread raises is raised here."""
    raised = []
    start = threading.Barrier(len(calls))

    def run(call):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                call()
                torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001  (handed on)
            raised.append(e)

    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if raised:
        raise raised[0]


@pytest.mark.parametrize("dtype,sizes", [("bf16", (32000, 20000, 5000)), ("fp32", (16000, 9000, 70000)), ("bf16", (2040, 1800, 1600))])
def test_distill_calls_of_host_threads_whose_rows_differ_in_length(dtype, sizes):
    """Kernels that take all these lengths with shared memory of another size for each: a call of one thread must not find the limit
    that another thread's call has just set for shorter rows."""
    problems = [Distill(dtype, 2, V, 9, seed=V).upload() for V in sizes]

    def outputs(p):
        return p.loss, p.row_loss, p.DX

    for p in problems:
        p.both()
    torch.cuda.synchronize()
    want = [[v.clone() for v in outputs(p)] for p in problems]

    def repeat(p):
        # (the C interface: what happens between its calls should be as little as possible)
        stream = torch.cuda.current_stream().cuda_stream
        a = [x.data_ptr() for x in (p.X, *p.dev, p.dloss)]
        o = [x.data_ptr() for x in outputs(p)]
        for _ in range(3000):
            st = B.lib.mebptt_distill_loss_grad(B.C.addressof(p.desc), *a, stream, *o)
            assert st == B.MEBPTT_OK, st

    _together([lambda p=p: repeat(p) for p in problems])
    for p, w in zip(problems, want):
        assert all(torch.equal(x, y) for x, y in zip(outputs(p), w))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("W", [2, 4, 8])
def test_conv_state_of_a_row_without_steps_is_handed_on_and_nothing_else(dtype, silu, W):
    """Rows that a batch has no use for: their states may hold anything, the gradients of the taps know nothing of them."""
    N, t, D = 5, 20, 40
    a, b = (Conv(dtype, N, t, D, W, silu=silu, seed=W) for _ in range(2))
    empty = [r for r in range(N) if a.lengths[r] == 0]
    assert empty
    for p, v in ((a, 0.0), (b, float("nan"))):
        p.dev["s_in"][empty] = v
        p.forward()
        p.backward()
    b.dev["s_in"][empty[0], :, ::2] = float("inf")
    b.backward()
    assert torch.equal(a.dw, b.dw) and torch.equal(a.dbias, b.dbias) and torch.equal(a.DX.x, b.DX.x) and torch.equal(a.ds_in, b.ds_in)
    assert torch.equal(a.Y.x, b.Y.x) and bool(b.s_out[empty].isnan().all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_conv_last_input_reaches_only_the_taps_that_saw_it(dtype):
    """The input of a row's last step was multiplied by the last tap alone, so that its value shows in that tap's gradient alone, where
    the array goes on and where it ends."""
    N, t, D, W = 3, 21, 24, 4
    a, b = (Conv(dtype, N, t, D, W, silu=False, seed=9) for _ in range(2))
    n = torch.tensor(a.lengths, device="cuda")
    for p, v in ((a, 0.0), (b, float("inf"))):
        for r in range(N):
            if n[r] > 0:
                p.X.x[int(n[r]) - 1, r] = v
        p.backward()
    assert torch.equal(a.dw[:, :W - 1], b.dw[:, :W - 1]) and not bool(b.dw[:, W - 1].isfinite().any())


@pytest.mark.parametrize("first,rate", [(1e-30, 7.0), (1e30, -9.0), (-3e-20, 6.25), (2e-3, -8.0)])
@pytest.mark.parametrize("t", [128, 700])
def test_scan_states_that_grow_or_fade_by_more_than_the_range_of_the_type_within_a_segment(t, first, rate):
    """Sixteen steps that multiply a state by e^100 and more, or by e^-128 and less, from a state small or large enough to stay a number
    throughout.  All other steps leave the state as it is, and nothing is added to it.

    Tolerance: the product e^(16 rate) is taken in one or two exponentials of the sum or in sixteen of the parts; sixteen parts are the
    most, each (2 |rate| + 4) + 1 half steps of float32 (argument, function, product).  The last pair ends at 5e-59, below the type's
    smallest normal number 2^-126, where results may be flushed to zero: off by less than that number."""
    N, D, S = 2, 8, 16
    zero = lambda *n: torch.zeros(*n, device="cuda")  # noqa: E731
    delta = zero(t, N, D)
    delta[64:80] = rate                                          # (whole segments: they begin at multiples of 16)
    A, one = torch.ones(D, S, device="cuda"), torch.ones(t, N, S, device="cuda")
    d = B.make_scan_desc(N, D, S, 1, t, "fp32", softplus=False)
    ws = torch.empty(B.mebptt_scan_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    kept = torch.empty(B.mebptt_scan_kept_bytes(d), dtype=torch.uint8, device="cuda")
    state, out, y, u = torch.full((N, D, S), first, device="cuda"), zero(N, D, S), zero(t, N, D), zero(t, N, D)
    want = float(np.float32(first)) * np.exp(16 * rate)
    tol = 16 * (2 * abs(rate) + 5) * 2.0 ** -24 * abs(want) + 2.0 ** -126
    B.mebptt_scan_forward(d, u, delta, A, one, one, None, None, None, state, None, ws, _stream(), y, out, kept)
    assert float((out.double() - want).abs().max()) <= tol
    assert bool(y.isfinite().all()) and float((y[-1].double() - S * want).abs().max()) <= S * (tol + 4 * 2.0 ** -24 * abs(want))
    # the same for what is handed back in time (from states of zeros, so that no other gradient is large)
    B.mebptt_scan_forward(d, u, delta, A, one, one, None, None, None, None, None, ws, _stream(), y, out, kept)
    du, dd, dA, dB, dC, back = zero(t, N, D), zero(t, N, D), zero(D, S), zero(t, N, S), zero(t, N, S), zero(N, D, S)
    B.mebptt_scan_backward(d, u, delta, A, one, one, None, None, None, None, kept, zero(t, N, D), state, ws, _stream(), du, dd, dA, dB, dC, None, None,
                           None, back)
    assert float((back.double() - want).abs().max()) <= tol
    assert not dA.any() and not dB.any() and not dC.any()


@pytest.fixture()
def fault():
    yield B.mebptt_test_wait_fault
    B.mebptt_test_wait_fault(0)


LOAD, SUMS, LOSS = 32, 64, 128
KERNELS = [("bf16", 15000, 40, 1), ("fp32", 9000, 1500, 1), ("bf16", 4000, 5001, 1), ("fp32", 700, 28001, 1), ("fp32", 700, 29001, 2), ("bf16", 700, 50257, 1),
           ("bf16", 500, 70000, 2), ("fp32", 300, 128256, 8)]     # type, rows, vocabulary, blocks of a row


def _wide(dtype, R, V, seed=0):
    """A problem made on the device (the oracle is not asked), every fifth row without weight, the middle one with."""
    p = Distill(dtype, 1, 8, 8)
    g = torch.Generator(device="cuda").manual_seed(seed)
    p.memory = p.X = torch.randn(R, V, device="cuda", generator=g).mul_(3).to(p.X.dtype)
    p.dmemory = p.DX = torch.empty_like(p.X)
    idx = torch.randint(0, V, (R, 8), device="cuda", generator=g).int()
    weights = torch.rand(R, device="cuda", generator=g) + 0.1
    weights[1::5] = 0
    weights[R // 2] = 0.5
    p.dev = (idx, torch.randn(R, 8, device="cuda", generator=g), weights)
    p.desc = B.make_distill_desc(R, V, 8, dtype, 1.5, 1 / R)
    p.row_loss, p.stats = (torch.empty(n * R, device="cuda") for n in (1, 2))
    return p


def _same(a, b):
    return torch.equal(a.nan_to_num(nan=-1.0), b.nan_to_num(nan=-1.0)) and torch.equal(a.isnan(), b.isnan())


@pytest.mark.parametrize("dtype,R,V,blocks,bit", [(*k, bit) for k in KERNELS for bit in (LOAD, SUMS, LOSS) if bit == LOAD or k[3] > 1])
def test_distill_waits_that_run_out_show_in_every_output(fault, dtype, R, V, blocks, bit):
    """The wait for the middle row's logits, the sums of its blocks or their parts of its loss expects more than ever comes and gives up.
    From that row on the block writes no numbers; rows of others, those before and those without weight are what they are."""
    p, row = _wide(dtype, R, V), R // 2
    live = p.dev[2] != 0
    p.both()
    clean = [v.clone() for v in (p.loss, p.row_loss, p.DX)]
    assert not any(bool(v.isnan().any()) for v in clean)

    def check(lost, grad):
        """`lost`: the rows that show it; grad: the gradient, of which at least the block's own part is lost in each of them."""
        rows = lost.nonzero().flatten()
        assert rows.numel() >= 2 and int(rows[0]) == row and bool(live[rows].all()) and rows.numel() < R // 4
        assert torch.equal(grad[~lost], clean[2][~lost])
        some = grad[rows].isnan()
        assert bool(some[1:].any(1).all()) and (blocks > 1 or bool(some.all()))
        return some[0]

    fault(bit)
    p.both()
    torch.cuda.synchronize()                                        # returns: the waits give up, the kernel ends
    fault(0)
    lost = p.row_loss.isnan()
    middle = check(lost, p.DX)
    assert bool(p.loss.isnan()) and torch.equal(p.row_loss[~lost], clean[1][~lost])
    if bit == LOAD:
        assert bool(middle.all())
    else:                                                           # (the others' parts of the middle row are right)
        assert bool(middle.any()) == (bit == SUMS) and not bool(middle.all())
        assert torch.equal(p.DX[row][~middle], clean[2][row][~middle])
    p.both()
    assert all(torch.equal(a, b) for a, b in zip((p.loss, p.row_loss, p.DX), clean))

    # the loss by itself: losses and statistics; the gradient by itself
    B.mebptt_distill_loss(p.desc, p.X, *p.dev, _stream(), p.loss, p.row_loss, p.stats)
    stats = p.stats.clone()
    fault(bit)
    B.mebptt_distill_loss(p.desc, p.X, *p.dev, _stream(), p.loss, p.row_loss, p.stats)
    torch.cuda.synchronize()
    lost, unknown = p.row_loss.isnan(), p.stats.view(R, 2).isnan()
    assert torch.equal(lost.nonzero().flatten()[:1], torch.tensor([row], device="cuda")) and bool(p.loss.isnan())
    assert torch.equal(p.stats.view(R, 2)[~lost], stats.view(R, 2)[~lost]) and torch.equal(p.row_loss[~lost], clean[1][~lost])
    after = lost.nonzero().flatten()[1:]
    assert after.numel() >= 1 and bool(unknown[after].all())
    assert bool(unknown[row].any()) if bit == LOAD else torch.equal(p.stats.view(R, 2)[row], stats.view(R, 2)[row])
    if bit == LOAD:
        p.DX.fill_(7.0)
        B.mebptt_distill_grad(p.desc, p.X, *p.dev, stats, p.dloss, _stream(), p.DX)
        torch.cuda.synchronize()
        middle = check(p.DX.isnan().any(1), p.DX)
        assert bool(middle.all()) == (blocks == 1)
    fault(0)
    p.DX.fill_(7.0)
    p.apart()
    again = [v.clone() for v in (p.loss, p.row_loss, p.DX)]
    p.apart()
    assert all(_same(a, b) for a, b in zip(again, (p.loss, p.row_loss, p.DX))) and not bool(p.DX.isnan().any())


def _fused_and_apart(p):
    p.upload()
    p.both()
    p.check()
    p.DX.fill_(7.0)
    p.apart()
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,K", [(1, 129), (300, 1024), (1000, 200), (2040, 130), (2049, 1024)])
def test_distill_more_entries_than_a_warp_takes_of_short_rows(dtype, V, K):
    """Blocks of as few as one warp that computes, with many times as many entries: tokens of their own, a few of them again and again, none."""
    p = Distill(dtype, 7, V, K, T=1.7, pad=3, phase=1)
    r = np.random.default_rng(K)
    p.i[1] = r.integers(0, V, K)
    p.i[2] = r.integers(0, min(V, 5), K)
    p.i[3, K // 3:] = -1
    p.i[4] = -1
    p.v[5, ::2] = -np.inf
    p.w[6] = 0
    _fused_and_apart(p)


@pytest.mark.parametrize("dtype,V,other", [("bf16", 140001, True), ("fp32", 140001, True), ("bf16", 300000, True), ("bf16", 600001, False), ("fp32", 260000, False)])
def test_distill_rows_that_no_ring_takes_and_no_registers_hold(dtype, V, other):
    """Rows that are read a second time for the gradient: too long for a cluster's shared memory, or for its registers where the gradient
    lies otherwise within 16 bytes than the logits."""
    p = Distill(dtype, 3, V, 20, T=0.8, pad=5, phase=1)
    if other:
        row = V + 2
        p.dmemory = torch.full((3 + 3 * row,), 977.0, device="cuda").to(p.X.dtype)
        p.DX = p.dmemory.as_strided((3, V), (row, 1), 3)
        p.row, p.desc.dlogits_row = row, row
    p.i[1, 4:9] = p.i[1, 3]
    p.w[2] = 0
    _fused_and_apart(p)


@pytest.mark.parametrize("low,high", [(1e-8, 1e-7), (1e-7, 1e-6), (1e-6, 1e-5), (1e-5, 1e-4), (1e-4, 1e-3), (1e-3, 1e-2), (1e-2, 0.1), (0.1, 0.5), (0.5, 2.0)])
def test_scan_decays_have_no_bias_where_states_last_for_thousands_of_steps(low, high):
    """A state that nothing is added to shows its decay; over 2^20 arguments the mean error is below a half step of float32, 2^-24 of the
    value, which single roundings stay within.  (A bias is what n steps raise to the n-th power; rounding errors average out.)"""
    D, S = 1 << 16, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (low + (high - low) * torch.rand(1, D, S, device="cuda", generator=g, dtype=torch.float64)).float()
    d = B.make_scan_desc(1, D, S, 1, 1, "fp32", softplus=False)
    one, u, out = torch.ones(1, 1, D, device="cuda"), torch.zeros(1, 1, D, device="cuda"), torch.empty(1, D, S, device="cuda")
    BC = torch.ones(1, 1, S, device="cuda")
    B.mebptt_scan_forward(d, u, one, -x[0].contiguous(), BC, BC, None, None, None, torch.ones(1, D, S, device="cuda"), None, None, _stream(), u.clone(), out)
    want = torch.exp(-x.double())
    error = (out.double() - want) / want
    assert abs(float(error.mean())) < 2.0 ** -24
    # argument (its two roundings), function and the product with the state, as the oracle counts them
    assert float((error.abs() - (2 * x.double() + 5) * 2.0 ** -24).max()) <= 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [40, 3001, 50257, 140000, 600001])
def test_distill_gradient_over_the_logits_in_every_kernel(dtype, V):
    p = Distill(dtype, 4, V, 12, T=1.2, pad=7, phase=1)
    p.DX, p.dmemory = p.X, p.memory
    p.w[2] = 0
    p.upload()
    p.both()
    p.check()
    p.upload()
    B.mebptt_distill_loss(p.desc, p.X, *p.dev, _stream(), p.loss, p.row_loss, p.stats)
    B.mebptt_distill_grad(p.desc, p.X, *p.dev, p.stats, p.dloss, _stream(), p.X)
    p.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("t,spacing", [(1, 8), (50, 8), (50, 32), (300, 16)])
def test_scan_state_of_a_row_without_steps_is_handed_on_and_nothing_else(dtype, t, spacing):
    a, b = (Scan(dtype, 5, t, 24, 16, spacing=spacing, seed=4) for _ in range(2))
    empty = [r for r in range(5) if a.lengths[r] == 0]
    assert empty
    for p, v in ((a, 0.0), (b, float("nan"))):
        p.dev["s_in"][empty] = v
        p.forward()
        p.backward()
    assert bool(b.s_out[empty].isnan().all()) and torch.equal(b.ds_in[empty], b.dev["ds_out"][empty])
    b.s_out[empty] = a.s_out[empty]
    assert all(torch.equal(x, y) for x, y in zip(a.outputs(), b.outputs()))
