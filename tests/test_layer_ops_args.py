"""The operators around the recurrence: argument checks of the C entry points
and of the binding, struct layouts, workspace sizes, and the 64-bit oracle's own
pins (CPU only; nothing reaches a GPU)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2509_25223_gb300 as rdn
from paper_2509_25223_gb300 import _abi, layer_ops
from tests import layer_oracle as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # aligned, never dereferenced: validation fails first
INVALID, UNSUPPORTED, WORKSPACE, MISALIGNED = 1, 2, 5, 6

_STRUCTS = {"rdn_conv_args": "ConvArgs", "rdn_conv_step_args": "ConvStepArgs", "rdn_scan_args": "ScanArgs",
            "rdn_scan_step_args": "ScanStepArgs", "rdn_norm_args": "NormArgs"}


def test_struct_layouts_match_the_header(tmp_path):
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "rdn.h"', "int main(void) {"]
    for cname, pyname in _STRUCTS.items():
        src.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        for f, _ in getattr(_abi, pyname)._fields_:
            src.append(f'  printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));')
    src += ['  printf("chunk chunk %d\\n", RDN_SCAN_CHUNK);', "  return 0;", "}"]
    c = tmp_path / "layout.c"
    c.write_text("\n".join(src))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in out.splitlines()}
    assert got.pop(("chunk", "chunk")) == _abi.SCAN_CHUNK
    for cname, pyname in _STRUCTS.items():
        st = getattr(_abi, pyname)
        assert got[(cname, "size")] == ctypes.sizeof(st), cname
        for f, _ in st._fields_:
            assert got[(cname, f)] == getattr(st, f).offset, (cname, f)


def _fill(cls, **kw):
    a = cls()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _conv(**kw):
    base = dict(B=2, T=64, C=128, W=4, dtype=_abi.RDN_BF16, silu=1, x=FAKE, w=FAKE, y=FAKE + 4096, dy=FAKE,
                dx=FAKE + 8192, dw=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
    return _fill(_abi.ConvArgs, **{**base, **kw})


def _scan(**kw):
    base = dict(B=2, T=64, D=128, S=16, G=1, dtype=_abi.RDN_BF16, dt_softplus=1, x=FAKE, dt=FAKE, Bm=FAKE, Cm=FAKE,
                A=FAKE, out=FAKE, dout=FAKE, dx=FAKE, ddt=FAKE, dB=FAKE, dC=FAKE, dA=FAKE, workspace=FAKE,
                workspace_bytes=1 << 40)
    return _fill(_abi.ScanArgs, **{**base, **kw})


def _norm(**kw):
    base = dict(rows=6, D=64, heads=1, dtype=_abi.RDN_BF16, x_dtype=_abi.RDN_F32, eps=1e-6, scale_const=1.0, f=FAKE,
                x=FAKE, w=FAKE, w_next=FAKE, r_out=FAKE, h=FAKE, dr=FAKE, dh=FAKE, df=FAKE, dx=FAKE, dw=FAKE,
                dw_next=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
    return _fill(_abi.NormArgs, **{**base, **kw})


def _refused(fn, a, status, says):
    lib = _abi.load()
    # a call that got past its checks would launch: the injected failure stops it before
    os.environ["RDN_FAULT_INJECT"] = "launch"
    try:
        st = lib[fn](ctypes.byref(a) if a is not None else None, None)
    finally:
        del os.environ["RDN_FAULT_INJECT"]
    msg = lib.rdn_last_error().decode()
    assert st == status and says in msg, (fn, st, msg)


SEQ = [(dict(B=0), INVALID, "B >= 1"), (dict(T=-1), INVALID, "T >= 0"), (dict(T=1 << 30), UNSUPPORTED, "too large"),
       (dict(cu_seqlens=FAKE, num_seqs=2), INVALID, "B = 1"),
       (dict(B=1, cu_seqlens=FAKE, num_seqs=0), INVALID, "num_seqs"),
       (dict(B=1, cu_seqlens=FAKE + 2, num_seqs=2), MISALIGNED, "cu_seqlens"),
       (dict(dtype=5), UNSUPPORTED, "dtype")]


@pytest.mark.parametrize("kw,status,says", SEQ + [
    (dict(C=0), INVALID, "C"), (dict(W=1), UNSUPPORTED, "W in"), (dict(W=5), UNSUPPORTED, "W in"),
    (dict(silu=2), INVALID, "silu"), (dict(x_ld=127), INVALID, "x_ld"), (dict(x_ld=-1), INVALID, "x_ld"),
    (dict(x=0), INVALID, "x is NULL"), (dict(w=0), INVALID, "w is NULL"), (dict(x=FAKE + 1), MISALIGNED, "x is"),
    (dict(w=FAKE + 2), MISALIGNED, "w is"), (dict(state0=FAKE + 1), MISALIGNED, "state0"),
    (dict(), 3, "injected")])
def test_conv_refusals(kw, status, says):
    for fn in ("rdn_conv_fwd", "rdn_conv_bwd"):
        _refused(fn, _conv(**kw), status, says)


def test_conv_refusals_of_one_direction():
    _refused("rdn_conv_fwd", None, INVALID, "args is NULL")
    _refused("rdn_conv_fwd", _conv(y=0), INVALID, "y is NULL")
    _refused("rdn_conv_fwd", _conv(y=FAKE), INVALID, "aliases")
    _refused("rdn_conv_bwd", _conv(dy=0), INVALID, "dy is NULL")
    _refused("rdn_conv_bwd", _conv(dx=FAKE), INVALID, "aliases")
    _refused("rdn_conv_bwd", _conv(dw=0), INVALID, "dw is NULL")
    _refused("rdn_conv_bwd", _conv(workspace=0), WORKSPACE, "workspace")
    _refused("rdn_conv_bwd", _conv(workspace_bytes=16), WORKSPACE, "workspace")
    _refused("rdn_conv_bwd", _conv(workspace=FAKE + 8), WORKSPACE, "aligned")


@pytest.mark.parametrize("kw,status,says", SEQ + [
    (dict(D=0), INVALID, "D"), (dict(G=3), INVALID, "G dividing"), (dict(S=0), INVALID, "S >= 1"),
    (dict(S=65), UNSUPPORTED, "64 states"), (dict(dt_softplus=3), INVALID, "dt_softplus"),
    (dict(b_ld=15), INVALID, "b_ld"), (dict(dt=0), INVALID, "dt is NULL"), (dict(Bm=0), INVALID, "Bm is NULL"),
    (dict(A=0), INVALID, "A is NULL"), (dict(A=FAKE + 4), MISALIGNED, "A is"), (dict(h0=FAKE + 4), MISALIGNED, "h0"),
    (dict(z=FAKE + 1), MISALIGNED, "z is"), (dict(), 3, "injected")])
def test_scan_refusals(kw, status, says):
    for fn in ("rdn_scan_fwd", "rdn_scan_bwd"):
        _refused(fn, _scan(**kw), status, says)


def test_scan_refusals_of_one_direction():
    _refused("rdn_scan_fwd", _scan(out=0), INVALID, "out is NULL")
    _refused("rdn_scan_fwd", _scan(T=4096, workspace=0), WORKSPACE, "workspace")
    _refused("rdn_scan_bwd", _scan(dout=0), INVALID, "dout is NULL")
    _refused("rdn_scan_bwd", _scan(z=FAKE), INVALID, "dz is NULL")
    _refused("rdn_scan_bwd", _scan(dA=0), INVALID, "dA is NULL")
    _refused("rdn_scan_bwd", _scan(workspace_bytes=64), WORKSPACE, "workspace")


@pytest.mark.parametrize("kw,status,says", [
    (dict(rows=0), INVALID, "rows"), (dict(D=0), INVALID, "D >= 2"), (dict(D=1), UNSUPPORTED, "2 to 16384"),
    (dict(D=16385), UNSUPPORTED, "16384"),
    (dict(heads=4), INVALID, "heads"), (dict(heads=3), INVALID, "neither"), (dict(dtype=3), UNSUPPORTED, "dtype"),
    (dict(x_dtype=3), UNSUPPORTED, "x_dtype"), (dict(gate=2), INVALID, "gate"), (dict(eps=-1.0), INVALID, "eps"),
    (dict(eps=float("nan")), INVALID, "eps"), (dict(scale_const=float("nan")), INVALID, "scale_const"),
    (dict(f=0, w_next=0), INVALID, "without f"), (dict(f=0, x=0), INVALID, "without f"),
    (dict(f_ld=63), INVALID, "f_ld"), (dict(w=0), INVALID, "w is NULL"), (dict(x=FAKE + 2), MISALIGNED, "x is"),
    (dict(), 3, "injected")])
def test_norm_refusals(kw, status, says):
    for fn in ("rdn_norm_fwd", "rdn_norm_bwd"):
        _refused(fn, _norm(**kw), status, says)


def test_norm_refusals_of_one_direction():
    _refused("rdn_norm_fwd", _norm(h=0), INVALID, "h is NULL")
    _refused("rdn_norm_fwd", _norm(w_next=0, r_out=0), INVALID, "r_out is NULL")
    _refused("rdn_norm_bwd", _norm(dh=0), INVALID, "dh is NULL")
    _refused("rdn_norm_bwd", _norm(w_next=0, dr=0), INVALID, "dr is NULL")
    _refused("rdn_norm_bwd", _norm(z=FAKE), INVALID, "dz is NULL")
    _refused("rdn_norm_bwd", _norm(scale=FAKE), INVALID, "dscale is NULL")
    _refused("rdn_norm_bwd", _norm(workspace_bytes=0), WORKSPACE, "workspace")


def test_step_refusals():
    c = dict(N=2, C=64, W=4, dtype=1, silu=1, num_slots=2, x=FAKE, w=FAKE, state=FAKE, y=FAKE)
    for kw, st, says in ((dict(N=0), INVALID, "N >= 1"), (dict(num_slots=1), INVALID, "num_slots"),
                         (dict(W=6), UNSUPPORTED, "W in"), (dict(state=0), INVALID, "state is NULL"),
                         (dict(slots=FAKE + 1), MISALIGNED, "slots"), (dict(dtype=9), UNSUPPORTED, "dtype"),
                         (dict(), 3, "injected")):
        _refused("rdn_conv_step", _fill(_abi.ConvStepArgs, **{**c, **kw}), st, says)
    s = dict(N=2, D=64, S=16, G=1, dtype=1, dt_softplus=1, num_slots=2, x=FAKE, dt=FAKE, Bm=FAKE, Cm=FAKE, A=FAKE,
             h=FAKE, out=FAKE)
    for kw, st, says in ((dict(N=0), INVALID, "N >= 1"), (dict(num_slots=0), INVALID, "num_slots"),
                         (dict(S=70), UNSUPPORTED, "64 states"), (dict(G=5), INVALID, "G dividing"),
                         (dict(h=FAKE + 8), MISALIGNED, "h is"), (dict(c_ld=3), INVALID, "c_ld"),
                         (dict(), 3, "injected")):
        _refused("rdn_scan_step", _fill(_abi.ScanStepArgs, **{**s, **kw}), st, says)


def test_size_queries():
    lib = _abi.load()
    n, slots = ctypes.c_size_t(0), ctypes.c_longlong(0)
    for fn, a in (("rdn_conv_bwd_workspace_size", _conv(x=0, w=0)), ("rdn_scan_bwd_workspace_size", _scan(x=0)),
                  ("rdn_norm_bwd_workspace_size", _norm(f=FAKE))):
        assert lib[fn](ctypes.byref(a), ctypes.byref(n)) == 0 and n.value > 0, fn
        assert lib[fn](ctypes.byref(a), None) == INVALID
        assert lib[fn](None, ctypes.byref(n)) == INVALID
    # given states leave out their place in the workspace
    with_, without = ctypes.c_size_t(0), ctypes.c_size_t(0)
    lib.rdn_scan_bwd_workspace_size(ctypes.byref(_scan(h_chunks=FAKE)), ctypes.byref(with_))
    lib.rdn_scan_bwd_workspace_size(ctypes.byref(_scan()), ctypes.byref(without))
    assert without.value - with_.value == 2 * 4 * 128 * 16 * 4
    assert lib.rdn_scan_chunk_slots(ctypes.byref(_scan(T=33)), ctypes.byref(slots)) == 0 and slots.value == 2 * 3
    a = _scan(B=1, T=33, cu_seqlens=FAKE, num_seqs=5)
    assert lib.rdn_scan_chunk_slots(ctypes.byref(a), ctypes.byref(slots)) == 0 and slots.value == 5 + 3


def test_row_strides():
    rows = lambda t: layer_ops._rows("t", t, t.shape, t.dtype, t.get_device())[1]  # noqa: E731
    t = torch.zeros(3, 5, 40)
    assert rows(t) == 0
    assert rows(t[..., 8:24]) == 40 and rows(t[:, :1, 8:24]) == 200 and rows(t[1:2, :, :4]) == 40
    assert rows(t[..., 4:20].unflatten(-1, (2, 8))) == 40
    assert rows(t[:1, :1, :4]) == 0  # a single row is contiguous
    for bad in (t.transpose(1, 2), t[:, :3, :16], t[..., ::2]):
        with pytest.raises(ValueError):
            rows(bad)


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(1, 4, 8)
    bc = torch.zeros(1, 4, 1, 2)
    with pytest.raises(ValueError, match="CUDA"):
        rdn.causal_conv_fwd(x, torch.zeros(8, 4))
    with pytest.raises(ValueError, match="CUDA"):
        rdn.selective_scan_fwd(x, x, torch.zeros(8, 2), bc, bc)
    with pytest.raises(ValueError, match="CUDA"):
        rdn.block_norm_fwd(x, torch.zeros(8))
    with pytest.raises(ValueError, match="f or x"):
        rdn.block_norm_fwd()
    with pytest.raises(ValueError, match="activation"):
        layer_ops._silu("relu")


def test_oracle_against_closed_forms():
    """One token, and constant decays: the oracle's loops against sums written out."""
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, st = r(1, 5, 3), r(3, 4), r(3), r(1, 3, 3)
    y, last = ref.conv(x, w, b, st, False)
    full = torch.cat([st, x], 1)[0]
    want = torch.nn.functional.conv1d(full.T[None], w[:, None], b, groups=3)[0].T
    assert torch.allclose(y[0], want, atol=1e-13) and torch.equal(last[0], x[0, -3:])
    A, B, C, dt = -torch.rand(3, 2, generator=g, dtype=torch.float64), r(1, 5, 1, 2), r(1, 5, 1, 2), r(1, 5, 3).abs()
    out, hT, kept = ref.scan(x, dt, A, B, C, None, None, None, None, False)
    t = 4
    h = sum(torch.exp(dt[0, i + 1:t + 1].sum(0)[:, None] * A) * (dt[0, i] * x[0, i])[:, None] * B[0, i, 0]
            for i in range(t + 1))
    assert torch.allclose(hT[0], h, atol=1e-13) and torch.allclose(out[0, t], (h * C[0, t, 0]).sum(-1), atol=1e-13)
    assert not kept.any()
    f = r(4, 6)
    n, _ = ref.norm(f, torch.ones(6, dtype=torch.float64), None, "silu", None, None, None, 0.0)
    assert torch.allclose(n.pow(2).mean(-1), torch.ones(4, dtype=torch.float64), atol=1e-13)


def test_oracle_gradients_by_differences():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_()  # noqa: E731
    assert torch.autograd.gradcheck(lambda *a: ref.conv(*a, True, [2, 0, 4]), (r(1, 6, 2), r(2, 3), r(2), r(3, 2, 2)))
    args = (r(1, 5, 4), r(1, 5, 4), r(4, 3), r(1, 5, 2, 3), r(1, 5, 2, 3), r(4), r(1, 5, 4), r(4), r(2, 4, 3))
    assert torch.autograd.gradcheck(lambda *a: ref.scan(*a, True, [2, 3])[:2], args)
    assert torch.autograd.gradcheck(lambda f, w, z, x, s, n: ref.norm(f, w, z, "silu", x, s, n, 1e-3),
                                    (r(3, 5), r(5), r(3, 5), r(3, 5), r(5), r(5)))
