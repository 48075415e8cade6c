"""Row layouts at the binding of the operators around the recurrence: what is passed on has
one distance between the rows, and every other layout is refused before the library is
called (CPU only: tensors that say they are on a device, calls that end before the library)."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from paper_2509_25223_gb300 import _abi, layer_ops


class OnDevice(torch.Tensor):
    """A host tensor that calls itself device 0's."""

    def get_device(self):
        return 0


class Torch:
    """torch, its allocations on the host."""

    def __getattr__(self, name):
        return getattr(torch, name)

    @staticmethod
    def empty(*shape, dtype=None, device=None):
        return torch.empty(*shape, dtype=dtype).as_subclass(OnDevice)


STRUCTS = {"rdn_conv_fwd": _abi.ConvArgs, "rdn_conv_bwd": _abi.ConvArgs, "rdn_conv_step": _abi.ConvStepArgs,
           "rdn_scan_fwd": _abi.ScanArgs, "rdn_scan_bwd": _abi.ScanArgs, "rdn_scan_step": _abi.ScanStepArgs,
           "rdn_norm_fwd": _abi.NormArgs, "rdn_norm_bwd": _abi.NormArgs}


@pytest.fixture
def calls(monkeypatch):
    """The argument structs that would have reached the library."""
    seen = []
    monkeypatch.setattr(layer_ops, "torch", Torch())
    monkeypatch.setattr(layer_ops, "_size", lambda name, args: 64)
    monkeypatch.setattr(layer_ops, "_call", lambda name, args, dev: seen.append(STRUCTS[name].from_buffer_copy(args)))
    return seen


def t(*shape):
    return torch.zeros(*shape).as_subclass(OnDevice)


B, T, C, S, G, H, N = 3, 5, 8, 4, 2, 2, 6


def conv(fn, **kw):
    back = dict(dy=t(B, T, C)) if fn is rdn.causal_conv_bwd else {}
    args = {**dict(x=t(B, T, C), weight=t(C, 4)), **back, **kw}
    return fn(**args)


def conv_bwd_out(**kw):
    return conv(rdn.causal_conv_bwd, out=kw)


def conv_step(**kw):
    return rdn.causal_conv_step(**{**dict(x=t(N, C), weight=t(C, 4), state=t(N, 3, C)), **kw})


def scan(fn, **kw):
    back = dict(dout=t(B, T, C)) if fn is rdn.selective_scan_bwd else {}
    args = {**dict(x=t(B, T, C), dt=t(B, T, C), A=t(C, S), B=t(B, T, G, S), C=t(B, T, G, S), z=t(B, T, C)), **back,
            **kw}
    return fn(**args)


def scan_bwd_out(**kw):
    return scan(rdn.selective_scan_bwd, out=kw)


def scan_step(**kw):
    return rdn.selective_scan_step(**{**dict(x=t(N, C), dt=t(N, C), A=t(C, S), B=t(N, G, S), C=t(N, G, S),
                                             h=t(N, C, S), z=t(N, C)), **kw})


def norm(fn, lead, **kw):
    shape = (*lead, C)
    heads = len(lead) == 3
    back = dict(dr=t(*shape)) if fn is rdn.block_norm_bwd else {}
    args = {**dict(f=t(*shape), weight=t(H, C) if heads else t(C), z=t(*shape), x=None if heads else t(*shape)),
            **back, **kw}
    return fn(**args)


def bind(f, *a):
    return lambda **kw: f(*a, **kw)


SEQ, BC, STEP, STEP_BC = ((B, T), (C,)), ((B, T), (G, S)), ((N,), (C,)), ((N,), (G, S))
# (what, call, operand, (leading axes, axes of a row), its row stride's field)
OPERANDS = [
    ("conv_fwd", bind(conv, rdn.causal_conv_fwd), "x", SEQ, "x_ld"),
    ("conv_fwd", bind(conv, rdn.causal_conv_fwd), "out", SEQ, "y_ld"),
    ("conv_bwd", bind(conv, rdn.causal_conv_bwd), "x", SEQ, "x_ld"),
    ("conv_bwd", bind(conv, rdn.causal_conv_bwd), "dy", SEQ, "dy_ld"),
    ("conv_bwd out", conv_bwd_out, "dx", SEQ, "dx_ld"),
    ("conv_step", conv_step, "x", STEP, "x_ld"), ("conv_step", conv_step, "out", STEP, "y_ld"),
]
for _fn in (rdn.selective_scan_fwd, rdn.selective_scan_bwd):
    _name = _fn.__name__
    OPERANDS += [(_name, bind(scan, _fn), "x", SEQ, "x_ld"), (_name, bind(scan, _fn), "dt", SEQ, "dt_ld"),
                 (_name, bind(scan, _fn), "z", SEQ, "z_ld"), (_name, bind(scan, _fn), "B", BC, "b_ld"),
                 (_name, bind(scan, _fn), "C", BC, "c_ld")]
OPERANDS += [("scan_fwd", bind(scan, rdn.selective_scan_fwd), "out", SEQ, "out_ld"),
             ("scan_bwd", bind(scan, rdn.selective_scan_bwd), "dout", SEQ, "dout_ld"),
             ("scan_bwd out", scan_bwd_out, "dx", SEQ, "dx_ld"), ("scan_bwd out", scan_bwd_out, "ddt", SEQ, "ddt_ld"),
             ("scan_bwd out", scan_bwd_out, "dz", SEQ, "dz_ld"),
             ("scan_step", scan_step, "x", STEP, "x_ld"), ("scan_step", scan_step, "dt", STEP, "dt_ld"),
             ("scan_step", scan_step, "z", STEP, "z_ld"), ("scan_step", scan_step, "B", STEP_BC, "b_ld"),
             ("scan_step", scan_step, "C", STEP_BC, "c_ld"), ("scan_step", scan_step, "out", STEP, "out_ld")]
for _fn in (rdn.block_norm_fwd, rdn.block_norm_bwd):
    for _lead in ((N,), (B, T), (B, T, H)):
        for _k in ("f", "z") + (("x",) if len(_lead) < 3 else ()):
            OPERANDS.append((f"{_fn.__name__} {_lead}", bind(norm, _fn, _lead), _k, (_lead, (C,)), _k + "_ld"))
IDS = [f"{o[0]}-{o[2]}" for o in OPERANDS]


def uneven(lead, row):
    """{name: tensor} of shape lead + row whose rows are not one non-zero distance apart."""
    shape = (*lead, *row)
    out = {}
    for a in range(len(lead)):
        one = list(shape)
        one[a] = 1
        out[f"axis {a} expanded"] = t(*one).expand(shape)
    out["expanded"] = t(*[1] * len(lead), *row).expand(shape)
    for a in range(1, len(lead)):
        wide = list(shape)
        wide[a] += 3
        out[f"the first of axis {a}"] = t(*wide).narrow(a, 0, shape[a])
        out[f"the last of axis {a}"] = t(*wide).narrow(a, 3, shape[a])
    if len(lead) > 1:
        out["every other batch row"] = t(2 * lead[0], *shape[1:])[::2]
        out["batch rows in turn"] = t(lead[1], lead[0], *shape[2:]).transpose(0, 1)
    if len(lead) > 2:
        out["every other token"] = t(lead[0], 2 * lead[1], *shape[2:])[:, ::2]
    out["every other element"] = t(*shape[:-1], 2 * shape[-1])[..., ::2]
    out["elements first"] = t(*shape[:-2], shape[-1], shape[-2]).transpose(-1, -2)
    if len(row) > 1:
        out["part of every group"] = t(*shape[:-1], 2 * shape[-1])[..., :shape[-1]]
        out["every other group"] = t(*lead, 2 * row[0], *row[1:])[(slice(None),) * len(lead) + (slice(None, None, 2),)]
    return out


@pytest.mark.parametrize("what,call,name,axes,field", OPERANDS, ids=IDS)
def test_uneven_rows_are_refused(calls, what, call, name, axes, field):
    call()
    assert len(calls) == 1
    for layout, bad in uneven(*axes).items():
        assert bad.shape == (*axes[0], *axes[1])
        with pytest.raises(ValueError, match=rf"\b{name}\b"):
            call(**{name: bad})
        assert len(calls) == 1, (layout, bad.stride(), getattr(calls[-1], field))


@pytest.mark.parametrize("what,call,name,axes,field", OPERANDS, ids=IDS)
def test_even_rows_are_passed_on(calls, what, call, name, axes, field):
    """Slices of a wider row's last axis, and every other row where there is one leading axis."""
    lead, row = axes
    width = row[0] * (row[1] if len(row) > 1 else 1)
    good = {}
    part = t(*lead, width + 12)[..., 4:4 + width]
    if len(lead) < 3:
        good[width + 12] = part.unflatten(-1, row) if len(row) > 1 else part
    if len(lead) == 1:
        good[2 * width] = t(2 * lead[0], *row)[::2]
    good[0] = t(*lead, *row)
    for ld, tensor in good.items():
        call(**{name: tensor})
        assert getattr(calls[-1], field) == ld


def test_single_rows():
    """Axes of one element have no distance: one batch row's tokens, one token of each row."""
    ld = lambda x, lead=2: layer_ops._rows("x", x, x.shape, x.dtype, 0, lead)[1]  # noqa: E731
    assert ld(t(2, 9, C)[:1, 2:7]) == 0
    assert ld(t(B, 9, C)[:, 3:4]) == 9 * C and ld(t(B, 9, C + 4)[:, 3:4, :C]) == 9 * (C + 4)
    assert ld(t(B, 9, C)[:, -1], 1) == 9 * C
    assert ld(t(1, 7, C).expand(1, 7, C)) == 0
    assert ld(t(B, T, H, 3 * C)[..., C:2 * C], 3) == 3 * C
    assert ld(t(B, T, 0, C).flatten(2)) == 0 and ld(t(B, 0, C)) == 0
