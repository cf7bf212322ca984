"""Refusals and sizes of the operators over sequences: nothing here reaches a device."""
import ctypes as C

import pytest

from paper_1606_03401_b200 import binding as B

P = 0x10000          # an address that is aligned to anything; never followed: every call below is refused first


def _conv(back=False, desc=None, ws=P, nbytes=1 << 40, **kw):
    d = desc or B.make_conv_desc(2, 24, 4, 10, "bf16")
    for k, v in kw.items():
        if hasattr(d, k):
            setattr(d, k, v)
    p = {k: kw.get(k, P) for k in ("x", "w", "bias", "s_in", "lengths", "y", "s_out", "dy", "ds_out", "dx", "dw", "dbias", "ds_in")}
    if not back:
        return B.lib.mebptt_conv_forward(C.addressof(d), p["x"], p["w"], p["bias"], p["s_in"], p["lengths"], None, p["y"], p["s_out"])
    return B.lib.mebptt_conv_backward(C.addressof(d), p["x"], p["w"], p["bias"], p["s_in"], p["lengths"], p["dy"], p["ds_out"], ws, nbytes, None,
                                      p["dx"], p["dw"], p["dbias"], p["ds_in"])


def _scan(back=False, ws=P, nbytes=1 << 50, **kw):
    d = B.make_scan_desc(2, 24, 16, 1, 10, "bf16")
    for k, v in kw.items():
        if k in dict(d._fields_):
            setattr(d, k, v)
    names = ("u", "delta", "A", "Bm", "Cm", "skip", "z", "bias", "s_in", "lengths", "y", "s_out", "kept", "dy", "ds_out", "du", "ddelta",
             "dA", "dB", "dC", "dskip", "dz", "dbias", "ds_in")
    p = {k: kw.get("p_" + k, P) for k in names}
    if not back:
        return B.lib.mebptt_scan_forward(C.addressof(d), *(p[k] for k in names[:10]), ws, nbytes, None, p["y"], p["s_out"], p["kept"])
    return B.lib.mebptt_scan_backward(C.addressof(d), *(p[k] for k in names[:8]), p["lengths"], p["kept"], p["dy"], p["ds_out"], ws, nbytes, None,
                                      *(p[k] for k in names[15:]))


def _distill(which="both", **kw):
    d = B.make_distill_desc(4, 100, 8, "bf16")
    for k, v in kw.items():
        if k in dict(d._fields_):
            setattr(d, k, v)
    p = {k: kw.get("p_" + k, P) for k in ("logits", "indices", "values", "weights", "dloss", "loss", "row_loss", "stats", "dlogits")}
    a = (C.addressof(d), p["logits"], p["indices"], p["values"], p["weights"])
    if which == "loss":
        return B.lib.mebptt_distill_loss(*a, None, p["loss"], p["row_loss"], p["stats"])
    if which == "grad":
        return B.lib.mebptt_distill_grad(*a, p["stats"], p["dloss"], None, p["dlogits"])
    return B.lib.mebptt_distill_loss_grad(*a, p["dloss"], None, p["loss"], p["row_loss"], p["dlogits"])


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(channels=0), dict(width=0), dict(width=9), dict(t=0), dict(t=(1 << 30) + 1), dict(dtype=3), dict(flags=2), dict(reserved=1),
    dict(x=None), dict(w=None), dict(y=None), dict(x=P + 1), dict(w=P + 1), dict(s_in=P + 1), dict(bias=P + 2), dict(lengths=P + 2),
    dict(x_step=-48, x_row=24), dict(x_step=23, x_row=24), dict(x_step=48, x_row=0), dict(y_step=0, y_row=24),
    dict(x_step=24, x_row=100),                 # rows that begin inside one another
    dict(y_step=47, y_row=24), dict(x_step=1 << 41, x_row=24),
])
def test_conv_forward_refuses(kw):
    assert _conv(**kw) == B.MEBPTT_ERR_ARG


def test_conv_backward_refuses():
    for kw in (dict(dy=None), dict(dx=None), dict(dw=None), dict(dy=P + 1), dict(dw=P + 2), dict(dbias=P + 2), dict(ds_in=P + 1), dict(width=9)):
        assert _conv(True, **kw) == B.MEBPTT_ERR_ARG, kw
    need = B.mebptt_conv_workspace_bytes(B.make_conv_desc(2, 24, 4, 10, "bf16"))
    assert need > 0
    for ws, nbytes in ((None, need), (P + 128, need), (P, need - 1)):
        assert _conv(True, ws=ws, nbytes=nbytes) == B.MEBPTT_ERR_WORKSPACE
    assert B.mebptt_conv_workspace_bytes(B.make_conv_desc(2, 24, 9, 10, "bf16")) == 0


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(channels=0), dict(states=0), dict(states=65), dict(groups=0), dict(groups=5), dict(t=0), dict(dtype=-1), dict(flags=2),
    dict(spacing=0), dict(spacing=12), dict(spacing=64), dict(reserved=1),
    dict(u_step=10, u_row=24), dict(delta_step=24, delta_row=24), dict(z_step=-1, z_row=24), dict(b_step=31, b_row=16), dict(c_step=16, c_row=16),
    dict(y_step=1, y_row=1), dict(p_u=None), dict(p_delta=None), dict(p_A=None), dict(p_Bm=None), dict(p_Cm=None), dict(p_u=P + 1), dict(p_A=P + 2),
    dict(p_lengths=P + 1), dict(p_kept=P + 8),
])
@pytest.mark.parametrize("back", [False, True])
def test_scan_refuses(back, kw):
    assert _scan(back, **kw) == B.MEBPTT_ERR_ARG


def test_scan_refuses_more():
    assert _scan(p_y=None) == B.MEBPTT_ERR_ARG
    for k in ("kept", "dy", "du", "ddelta", "dA", "dB", "dC", "dz", "z"):
        assert _scan(True, **{"p_" + k: None}) == B.MEBPTT_ERR_ARG, k
    for k in ("dB", "dA", "dskip", "dbias", "ds_out"):
        assert _scan(True, **{"p_" + k: P + 1}) == B.MEBPTT_ERR_ARG, k
    assert _scan(batch=70000) == B.MEBPTT_ERR_UNSUPPORTED
    d = B.make_scan_desc(2, 24, 16, 1, 10, "bf16")
    assert B.mebptt_scan_workspace_bytes(d) == 0                      # nothing to hold: one segment
    need = B.mebptt_scan_workspace_bytes(d, True)
    for ws, nbytes in ((None, need), (P + 64, need), (P, need - 1)):
        assert _scan(True, ws=ws, nbytes=nbytes) == B.MEBPTT_ERR_WORKSPACE
    d.t = 4000
    assert B.mebptt_scan_workspace_bytes(d) > 0 and _scan(t=4000, ws=None) == B.MEBPTT_ERR_WORKSPACE


def test_states_that_are_kept_take_what_the_spacing_says():
    for spacing in (8, 16, 32):
        d = B.make_scan_desc(3, 40, 10, 2, 100, "fp32", spacing=spacing)
        assert B.mebptt_scan_kept_bytes(d) == -(-100 // spacing) * 3 * 40 * 16 * 4
    d.spacing = 9
    assert B.mebptt_scan_kept_bytes(d) == 0


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(vocabulary=0), dict(entries=0), dict(entries=1025), dict(dtype=7), dict(reserved=1), dict(temperature=0.0),
    dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(scale=float("inf")), dict(scale=float("nan")),
    dict(logits_row=99), dict(dlogits_row=99), dict(logits_row=-1), dict(p_logits=None), dict(p_indices=None), dict(p_values=None),
    dict(p_logits=P + 1), dict(p_indices=P + 2), dict(p_values=P + 2), dict(p_weights=P + 2),
])
@pytest.mark.parametrize("which", ["loss", "grad", "both"])
def test_distill_refuses(which, kw):
    assert _distill(which, **kw) == B.MEBPTT_ERR_ARG


def test_distill_refuses_more():
    assert _distill("loss", p_row_loss=None) == _distill("loss", p_stats=None) == _distill("loss", p_loss=P + 2) == B.MEBPTT_ERR_ARG
    assert _distill("grad", p_stats=None) == _distill("grad", p_dlogits=None) == _distill("grad", p_dlogits=P + 1) == B.MEBPTT_ERR_ARG
    assert _distill("both", p_row_loss=None) == _distill("both", p_dlogits=None) == _distill("both", p_dloss=P + 1) == B.MEBPTT_ERR_ARG
    assert _distill("both", rows=1 << 31) == B.MEBPTT_ERR_UNSUPPORTED


def test_null_descriptors_are_refused():
    assert B.lib.mebptt_conv_forward(*[None] * 9) == B.MEBPTT_ERR_ARG
    assert B.lib.mebptt_conv_workspace_bytes(None) == B.lib.mebptt_scan_kept_bytes(None) == B.lib.mebptt_scan_workspace_bytes(None, 1) == 0
    assert B.lib.mebptt_scan_forward(*[None] * 12, 0, *[None] * 4) == B.MEBPTT_ERR_ARG
    assert B.lib.mebptt_distill_loss(*[None] * 9) == B.MEBPTT_ERR_ARG


def test_tensors_of_another_type_or_place_are_refused():
    import torch
    d = B.make_conv_desc(1, 8, 2, 1, "bf16")
    x = torch.zeros(1, 1, 8, dtype=torch.bfloat16)
    with pytest.raises(B.MebpttError) as e:
        B.mebptt_conv_forward(d, x, x, None, None, None, None, x, None)
    assert e.value.status == B.MEBPTT_ERR_ARG


def test_scan_refuses_rows_of_sums_that_pass_32_bits():
    wide = dict(batch=1, t=1, channels=1 << 24, groups=1 << 24)
    for states in (33, 64):                                         # in memory 64 states a group, dB and dC: 2^31 values
        assert _scan(True, states=states, **wide) == B.MEBPTT_ERR_UNSUPPORTED
    assert _scan(True, states=64, nbytes=0, batch=1, t=1, channels=1 << 23, groups=1 << 23) == B.MEBPTT_ERR_WORKSPACE      # half as many: taken


@pytest.mark.parametrize("which", ["loss", "grad", "both"])
def test_distill_refuses_temperatures_whose_square_is_not_a_normal_number(which):
    for T in (1e-45, 1e-40, 1e-30, 1.0e-19, 1.9e19, 1e30, 3e38):
        assert _distill(which, temperature=T) == B.MEBPTT_ERR_ARG, T
    for T in (1.1e-19, 1e-3, 1e4, 1.8e19):
        assert _distill(which, temperature=T, rows=1 << 31) == B.MEBPTT_ERR_UNSUPPORTED, T        # taken, but for the rows


def _tensors(op, e="bf16", t=5, batch=3, D=8, W=4, S=16, G=2, rows=6, V=40, K=4):
    """The tensors of each call."""
    import torch
    o = torch.bfloat16 if e == "bf16" else torch.float32
    z = lambda *n, dtype=o: torch.zeros(*n, dtype=dtype)  # noqa: E731
    f = lambda *n: z(*n, dtype=torch.float32)  # noqa: E731
    i = lambda *n: z(*n, dtype=torch.int32)  # noqa: E731
    if op.startswith("conv"):
        d = B.make_conv_desc(batch, D, W, t, e)
        a = dict(x=z(t, batch, D), w=z(D, W), bias=f(D), s_in=z(batch, W - 1, D), lengths=i(batch))
        if op == "conv_forward":
            return d, dict(**a, stream=None, y=z(t, batch, D), s_out=z(batch, W - 1, D))
        return d, dict(**a, dy=z(t, batch, D), ds_out=z(batch, W - 1, D), workspace=None, stream=None, dx=z(t, batch, D), dw=f(D, W), dbias=f(D),
                       ds_in=z(batch, W - 1, D))
    if op.startswith("scan"):
        d = B.make_scan_desc(batch, D, S, G, t, e)
        a = dict(u=z(t, batch, D), delta=z(t, batch, D), A=f(D, S), Bm=z(t, batch, G * S), Cm=z(t, batch, G * S), skip=f(D), z=z(t, batch, D), delta_bias=f(D))
        if op == "scan_forward":
            return d, dict(**a, s_in=f(batch, D, S), lengths=i(batch), workspace=None, stream=None, y=z(t, batch, D), s_out=f(batch, D, S), kept=None)
        return d, dict(**a, lengths=i(batch), kept=None, dy=z(t, batch, D), ds_out=f(batch, D, S), workspace=None, stream=None, du=z(t, batch, D),
                       ddelta=z(t, batch, D), dA=f(D, S), dB=z(t, batch, G * S), dC=z(t, batch, G * S), dskip=f(D), dz=z(t, batch, D), ddelta_bias=f(D),
                       ds_in=f(batch, D, S))
    d = B.make_distill_desc(rows, V, K, e)
    a = dict(logits=z(rows, V), indices=i(rows, K), values=f(rows, K), weights=f(rows))
    if op == "distill_loss":
        return d, dict(**a, stream=None, loss=f(1), row_loss=f(rows), row_stats=f(rows, 2))
    if op == "distill_grad":
        return d, dict(**a, row_stats=f(rows, 2), dloss=f(1), stream=None, dlogits=z(rows, V))
    return d, dict(**a, dloss=f(1), stream=None, loss=f(1), row_loss=f(rows), dlogits=z(rows, V))


OK = "taken"


def _says(op, desc, kw):
    """What the call is refused with, or OK."""
    try:
        getattr(B, "mebptt_" + op)(desc, **kw)
    except B.MebpttError as e:
        assert e.status == B.MEBPTT_ERR_ARG
        return str(e)
    return OK


@pytest.fixture()
def hosted(monkeypatch):
    """The binding as it is where the host is the current device, with a library whose calls do nothing."""
    class Library:
        def __getattr__(self, name):
            return real[name] if name.endswith("_bytes") or name == "mebptt_strerror" else lambda *a: B.MEBPTT_OK

    real = {n: getattr(B.lib, n) for n in B._SIGS}
    monkeypatch.setattr(B, "_DEVICE", -1)                                  # get_device() of a host tensor
    monkeypatch.setattr(B, "lib", Library())


CALLS = ["conv_forward", "conv_backward", "scan_forward", "scan_backward", "distill_loss", "distill_grad", "distill_loss_grad"]


@pytest.mark.parametrize("e", ["bf16", "fp32"])
@pytest.mark.parametrize("op", CALLS)
def test_tensors_that_lie_otherwise_or_end_too_early_are_refused(hosted, op, e):
    import torch
    desc, right = _tensors(op, e)
    assert _says(op, desc, right) == OK
    for name, x in right.items():
        if x is None:
            continue
        other = torch.float32 if x.dtype is not torch.float32 else torch.float64
        assert f"a {other} tensor" in _says(op, desc, {**right, name: x.to(other)}), name
        wide = torch.zeros(*x.shape[:-1], 2 * x.shape[-1], dtype=x.dtype)
        if x.numel() > 1:
            assert "strides" in _says(op, desc, {**right, name: wide[..., ::2]}), name              # every second column
            assert "strides" in _says(op, desc, {**right, name: wide[:1, ..., :1].expand(x.shape) if x.dim() > 1 else wide[:1].expand(x.shape)}), name
        if x.dim() > 1:
            assert "strides" in _says(op, desc, {**right, name: x.transpose(-1, -2).contiguous().transpose(-1, -2)}), name
            assert "strides" in _says(op, desc, {**right, name: wide[..., :x.shape[-1]]}), name      # a slice, where the descriptor has a dense array
        assert "belong" in _says(op, desc, {**right, name: x.flatten()[:-1]}) or "ends" in _says(op, desc, {**right, name: x.flatten()[:-1]}), name
        assert _says(op, desc, {**right, name: x.flatten()}) == OK, name                              # as many, in one dimension
        assert _says(op, desc, {**right, name: torch.cat([x.flatten()] * 2)}) == OK, name


def test_arrays_over_time_with_gaps_are_taken_as_the_descriptor_says(hosted):
    import torch
    t, N, D = 5, 3, 8
    _, right = _tensors("conv_forward")
    memory = torch.zeros(N, t, 2 * D, dtype=torch.bfloat16)
    x = memory[:, :, :D].transpose(0, 1)                            # [t, N, D], batch-major, half of the columns
    desc = B.make_conv_desc(N, D, 4, t, "bf16", x_strides=(x.stride(0), x.stride(1)))
    assert _says("conv_forward", desc, {**right, "x": x}) == OK
    assert _says("conv_forward", desc, {**right, "x": memory[:, :, :D]}) == OK      # the same places under other names
    assert _says("conv_forward", desc, {**right, "x": memory}) == OK                # a buffer that holds them
    assert "strides" in _says("conv_forward", desc, right)                          # a dense array is not what this descriptor says
    assert "ends" in _says("conv_forward", desc, {**right, "x": memory.flatten()[:-D - 1]})
    assert _says("conv_forward", desc, {**right, "x": memory.flatten()[:-D]}) == OK  # (nothing is read behind the last column)
    assert "ends" in _says("conv_forward", desc, {**right, "x": x[:-1]})
    assert "columns" in _says("conv_forward", desc, {**right, "x": memory.transpose(1, 2)})
    # rows in one dimension, a longer array; gaps that the descriptor does not have, or has otherwise
    wide = torch.zeros(t + 2, N, 2 * D, dtype=torch.bfloat16)
    gaps = B.make_conv_desc(N, D, 4, t, "bf16", x_strides=(wide.stride(0), wide.stride(1)))
    for v in (wide[:t, :, :D], wide[:, :, :D], wide.view(-1, 2 * D)[:t * N, :D], wide):
        assert _says("conv_forward", gaps, {**right, "x": v}) == OK
    dense = B.make_conv_desc(N, D, 4, t, "bf16")
    for v in (wide.view(-1, 2 * D)[:, :D], wide[:, :, :D], wide[:, 0, :D]):
        assert "strides" in _says("conv_forward", dense, {**right, "x": v})
    assert "strides" in _says("conv_forward", gaps, {**right, "x": torch.zeros(t * N, 3 * D, dtype=torch.bfloat16)[:, :D]})
    assert _says("conv_forward", gaps, {**right, "x": memory[:, :, :D]}) == OK      # (the same rows: which is which the descriptor says)
    # one step: rows of a wider array, with and without the dimension of time
    one = B.make_conv_desc(N, D, 4, 1, "bf16", x_strides=(99, t * 2 * D), y_strides=(0, 0))
    right["y"] = right["y"][:1]
    for v in (x[:1], x[0], memory[:, 0], memory[:, 0, :D]):
        assert _says("conv_forward", one, {**right, "x": v}) == OK
    assert "ends" in _says("conv_forward", one, {**right, "x": x[0, :-1]})
    # logits: rows with gaps
    _, right = _tensors("distill_loss")
    desc = B.make_distill_desc(6, 40, 4, "bf16", logits_row=48)
    rows = torch.zeros(6, 48, dtype=torch.bfloat16)
    for v in (rows, rows[:, :40], rows.view(2, 3, 48)[..., :40]):
        assert _says("distill_loss", desc, {**right, "logits": v}) == OK
    assert "strides" in _says("distill_loss", desc, right) and "ends" in _says("distill_loss", desc, {**right, "logits": rows[:5]})
    # an optional tensor may be missing, and a width of one has no state
    desc, right = _tensors("conv_forward", W=1)
    assert _says("conv_forward", desc, {**right, "bias": None, "lengths": None, "s_in": None, "s_out": None}) == OK


def test_tensors_of_another_device_than_the_current_one_are_refused(hosted, monkeypatch):
    import torch

    class On:
        """A tensor as if it were on a CUDA device."""
        def __init__(self, x, device):
            self.x, self.device_at = x, device

        def __getattr__(self, k):
            return getattr(self.x, k)

        is_cuda = True

        def get_device(self):
            return self.device_at

    for op in CALLS:
        desc, right = _tensors(op)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(B, "_DEVICE", -2)
        assert "current CUDA device" in _says(op, desc, right)              # host tensors
        here = {k: v if v is None else On(v, 0) for k, v in right.items()}
        assert _says(op, desc, here) == OK
        for name, x in right.items():
            if x is not None:
                assert "current CUDA device" in _says(op, desc, {**here, name: On(x, 1)}), name
                assert "current CUDA device" in _says(op, desc, {**here, name: x}), name


def test_rooms_are_contiguous_and_on_the_current_device(hosted):
    import torch
    desc, right = _tensors("scan_backward")
    room = torch.zeros(2, B.mebptt_scan_kept_bytes(desc), dtype=torch.uint8)
    for name in ("kept", "workspace"):
        assert _says("scan_backward", desc, {**right, name: room[0]}) == OK
        assert "contiguous" in _says("scan_backward", desc, {**right, name: room.t()}), name
    with pytest.raises(B.MebpttError) as e:
        B.mebptt_scan_backward(desc, **{**right, "kept": room[0, :-1]})
    assert e.value.status == B.MEBPTT_ERR_WORKSPACE
