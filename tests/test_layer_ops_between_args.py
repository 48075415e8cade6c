"""Gated recurrence, 8-bit norm and matrix products: argument checks of the C entry points and
of the binding, struct layouts and workspace sizes (CPU only; nothing reaches a GPU)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2509_25223_gb300 as rdn
from paper_2509_25223_gb300 import _abi, layer_ops
from tests.test_layer_ops_args import FAKE, INVALID, MISALIGNED, ROOT, UNSUPPORTED, WORKSPACE, _fill, _refused

_STRUCTS = {"rdn_gscan_args": "GscanArgs", "rdn_gscan_step_args": "GscanStepArgs", "rdn_norm_q8_args": "NormQ8Args",
            "rdn_linear_args": "LinearArgs"}
AT = 1 << 32  # (clear of the other fake operands)


def test_struct_layouts_match_the_header(tmp_path):
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "rdn.h"', "int main(void) {"]
    for cname, pyname in _STRUCTS.items():
        src.append(f'  printf("{cname} size %zu\\n", sizeof({cname}));')
        for f, _ in getattr(_abi, pyname)._fields_:
            src.append(f'  printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));')
    src += ['  printf("chunk chunk %d\\n", RDN_GSCAN_CHUNK);', '  printf("type type %d\\n", RDN_E4M3);', "  return 0;", "}"]
    c, exe = tmp_path / "layout.c", tmp_path / "layout"
    c.write_text("\n".join(src))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in out.splitlines()}
    assert got.pop(("chunk", "chunk")) == _abi.GSCAN_CHUNK and got.pop(("type", "type")) == _abi.RDN_E4M3
    for cname, pyname in _STRUCTS.items():
        st = getattr(_abi, pyname)
        assert got[(cname, "size")] == ctypes.sizeof(st), cname
        for f, _ in st._fields_:
            assert got[(cname, f)] == getattr(st, f).offset, (cname, f)


def _gscan(**kw):
    base = dict(B=2, T=200, D=128, dtype=_abi.RDN_BF16, c=8.0, x=FAKE, r=FAKE, i=FAKE, lam=FAKE, y=FAKE + 4096, dy=FAKE,
                dx=FAKE + 4096, dr=FAKE + 8192, di=FAKE + 12288, dlam=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
    return _fill(_abi.GscanArgs, **{**base, **kw})


def _gstep(**kw):
    base = dict(N=4, D=128, dtype=_abi.RDN_BF16, c=8.0, num_slots=4, x=FAKE, r=FAKE, i=FAKE, lam=FAKE, h=FAKE, y=FAKE)
    return _fill(_abi.GscanStepArgs, **{**base, **kw})


def _q8(**kw):
    base = dict(rows=6, D=64, x_dtype=_abi.RDN_BF16, f_dtype=_abi.RDN_BF16, eps=1e-6, x=FAKE, f=FAKE + 4096, w=FAKE,
                r_out=FAKE + 8192, q=FAKE + 12288, scale=FAKE)
    return _fill(_abi.NormQ8Args, **{**base, **kw})


def _linear(**kw):
    base = dict(M=6, N=64, K=32, dtype=_abi.RDN_BF16, y_dtype=_abi.RDN_BF16, x=FAKE, w=FAKE + 4096, y=FAKE + 8192,
                dw_dtype=_abi.RDN_BF16, dy=FAKE + 16384, dx=FAKE + 20480, dw=FAKE + 24576, workspace=FAKE,
                workspace_bytes=1 << 40)
    return _fill(_abi.LinearArgs, **{**base, **kw})


def _q8_linear(**kw):
    return _linear(**{**dict(dtype=_abi.RDN_E4M3, x_scale=FAKE, w_scale=FAKE), **kw})


LAUNCH = 3  # a call that passes its checks ends in the injected failure
CASES = [
    ("rdn_gscan_fwd", None, INVALID, "args is NULL"),
    ("rdn_gscan_fwd", _gscan(), LAUNCH, "injected"),
    ("rdn_gscan_fwd", _gscan(B=0), INVALID, "B >= 1"),
    ("rdn_gscan_fwd", _gscan(T=-1), INVALID, "T >= 0"),
    ("rdn_gscan_fwd", _gscan(D=0), INVALID, "D"),
    ("rdn_gscan_fwd", _gscan(D=(1 << 19) + 1), INVALID, "D"),
    ("rdn_gscan_fwd", _gscan(B=1 << 24, T=1, D=1 << 19), UNSUPPORTED, "too many"),
    ("rdn_gscan_fwd", _gscan(dtype=_abi.RDN_E4M3), UNSUPPORTED, "dtype"),
    ("rdn_gscan_fwd", _gscan(c=0.0), INVALID, "c must be"),
    ("rdn_gscan_fwd", _gscan(c=float("nan")), INVALID, "c must be"),
    ("rdn_gscan_fwd", _gscan(c=float("inf")), INVALID, "c must be"),
    ("rdn_gscan_fwd", _gscan(r_ld=127), INVALID, "r_ld"),
    ("rdn_gscan_fwd", _gscan(i_ld=1 << 24), UNSUPPORTED, "2^24"),
    ("rdn_gscan_bwd", _gscan(di_ld=1 << 24), UNSUPPORTED, "2^24"),
    ("rdn_gscan_fwd", _gscan(i_ld=(1 << 24) - 1), LAUNCH, "injected"),
    ("rdn_gscan_fwd", _gscan(x=0), INVALID, "x is NULL"),
    ("rdn_gscan_fwd", _gscan(T=0, x=0, r=0, i=0, y=0), LAUNCH, "injected"),
    ("rdn_gscan_fwd", _gscan(i=FAKE + 1), MISALIGNED, "i is not"),
    ("rdn_gscan_fwd", _gscan(h0=FAKE + 2), MISALIGNED, "h0"),
    ("rdn_gscan_fwd", _gscan(lam=0), INVALID, "lam"),
    ("rdn_gscan_fwd", _gscan(y=FAKE), INVALID, "aliases"),
    ("rdn_gscan_fwd", _gscan(cu_seqlens=FAKE, num_seqs=2), INVALID, "B = 1"),
    ("rdn_gscan_fwd", _gscan(B=1, cu_seqlens=FAKE, num_seqs=0), INVALID, "num_seqs"),
    ("rdn_gscan_fwd", _gscan(h0=AT, hT=AT + 2 * 128 * 4 - 4), INVALID, "overlaps"),
    ("rdn_gscan_fwd", _gscan(h0=AT, hT=AT + 2 * 128 * 4), LAUNCH, "injected"),
    ("rdn_gscan_fwd", _gscan(h0=AT, h_chunks=AT - 2 * 4 * 128 * 4 + 4), INVALID, "overlaps"),
    ("rdn_gscan_fwd", _gscan(hT=AT, h_chunks=AT), INVALID, "overlaps"),
    ("rdn_gscan_bwd", _gscan(), LAUNCH, "injected"),
    ("rdn_gscan_bwd", _gscan(dy=0), INVALID, "dy"),
    ("rdn_gscan_bwd", _gscan(dr=0), INVALID, "dr"),
    ("rdn_gscan_bwd", _gscan(di=FAKE), INVALID, "aliases"),
    ("rdn_gscan_bwd", _gscan(dlam=0), INVALID, "dlam"),
    ("rdn_gscan_bwd", _gscan(dh0=AT, dhT=AT), INVALID, "overlaps"),
    ("rdn_gscan_bwd", _gscan(dh0=AT, h0=AT), INVALID, "overlaps"),
    ("rdn_gscan_bwd", _gscan(workspace=0), WORKSPACE, "workspace"),
    ("rdn_gscan_bwd", _gscan(workspace_bytes=64), WORKSPACE, "workspace"),
    ("rdn_gscan_bwd", _gscan(workspace=FAKE + 4), WORKSPACE, "aligned"),
    ("rdn_gscan_step", _gstep(), LAUNCH, "injected"),
    ("rdn_gscan_step", _gstep(N=0), INVALID, "N >= 1"),
    ("rdn_gscan_step", _gstep(num_slots=3), INVALID, "num_slots"),
    ("rdn_gscan_step", _gstep(D=0), INVALID, "D"),
    ("rdn_gscan_step", _gstep(c=-1.0), INVALID, "c must be"),
    ("rdn_gscan_step", _gstep(h=0), INVALID, "h is NULL"),
    ("rdn_gscan_step", _gstep(y_ld=3), INVALID, "y_ld"),
    ("rdn_norm_q8", _q8(), LAUNCH, "injected"),
    ("rdn_norm_q8", _q8(rows=0, x=0, f=0, q=0, scale=0), LAUNCH, "injected"),
    ("rdn_norm_q8", _q8(rows=-1), INVALID, "rows"),
    ("rdn_norm_q8", _q8(D=0), INVALID, "D"),
    ("rdn_norm_q8", _q8(D=16385), UNSUPPORTED, "16384"),
    ("rdn_norm_q8", _q8(x_dtype=2), UNSUPPORTED, "dtype"),
    ("rdn_norm_q8", _q8(f_dtype=7), UNSUPPORTED, "dtype"),
    ("rdn_norm_q8", _q8(f=0, f_dtype=7), LAUNCH, "injected"),
    ("rdn_norm_q8", _q8(eps=-1.0), INVALID, "eps"),
    ("rdn_norm_q8", _q8(x=0), INVALID, "x is NULL"),
    ("rdn_norm_q8", _q8(x=FAKE + 1), MISALIGNED, "x is not"),
    ("rdn_norm_q8", _q8(scale=0), INVALID, "scale"),
    ("rdn_norm_q8", _q8(x_ld=63), INVALID, "x_ld"),
    ("rdn_norm_q8", _q8(r_out=FAKE + 4096), INVALID, "r_out"),
    ("rdn_norm_q8", _q8(r_out=FAKE), LAUNCH, "injected"),
    ("rdn_norm_q8", _q8(r_out=FAKE, x_ld=72), INVALID, "r_out"),
    ("rdn_norm_q8", _q8(q=FAKE), INVALID, "q aliases"),
    ("rdn_linear_fwd", _linear(), LAUNCH, "injected"),
    ("rdn_linear_fwd", _linear(M=0, x=0, y=0), LAUNCH, "injected"),
    ("rdn_linear_fwd", _linear(M=-1), INVALID, "M >= 0"),
    ("rdn_linear_fwd", _linear(N=0), INVALID, "N"),
    ("rdn_linear_fwd", _linear(N=68), UNSUPPORTED, "multiple"),
    ("rdn_linear_fwd", _linear(K=36), UNSUPPORTED, "multiple of 8"),
    ("rdn_linear_fwd", _q8_linear(K=40), UNSUPPORTED, "multiple of 16"),
    ("rdn_linear_fwd", _linear(M=1 << 31), UNSUPPORTED, "too large"),
    ("rdn_linear_fwd", _linear(M=1 << 30, K=2048), UNSUPPORTED, "too large"),
    ("rdn_linear_fwd", _linear(dtype=_abi.RDN_F32), UNSUPPORTED, "dtype"),
    ("rdn_linear_fwd", _linear(y_dtype=2), UNSUPPORTED, "y_dtype"),
    ("rdn_linear_fwd", _linear(act=4), INVALID, "act"),
    ("rdn_linear_fwd", _linear(x=FAKE + 8), MISALIGNED, "x is not"),
    ("rdn_linear_fwd", _linear(x_ld=36), MISALIGNED, "rows of x"),
    ("rdn_linear_fwd", _q8_linear(x_ld=40), MISALIGNED, "rows of x"),
    ("rdn_linear_fwd", _linear(x_ld=1 << 39), UNSUPPORTED, "too far apart"),
    ("rdn_linear_fwd", _linear(w_ld=28), INVALID, "w_ld"),
    ("rdn_linear_fwd", _linear(w=0), INVALID, "w is NULL"),
    ("rdn_linear_fwd", _linear(x_scale=FAKE), INVALID, "scales"),
    ("rdn_linear_fwd", _q8_linear(), LAUNCH, "injected"),
    ("rdn_linear_fwd", _q8_linear(x_scale=0), INVALID, "x_scale"),
    ("rdn_linear_fwd", _q8_linear(w_scale=0), INVALID, "w_scale"),
    ("rdn_linear_fwd", _linear(y=FAKE), INVALID, "aliases"),
    ("rdn_linear_fwd", _linear(pre=FAKE + 8192), INVALID, "aliases"),
    ("rdn_linear_fwd", _linear(pre=AT + 8), MISALIGNED, "pre"),
    ("rdn_linear_fwd", _linear(res=FAKE + 8192), LAUNCH, "injected"),
    ("rdn_linear_fwd", _linear(res=FAKE + 8192, res_ld=72), INVALID, "same rows"),
    ("rdn_linear_bwd", _linear(), LAUNCH, "injected"),
    ("rdn_linear_bwd", _q8_linear(), UNSUPPORTED, "dtype"),
    ("rdn_linear_bwd", _linear(act=1), INVALID, "pre"),
    ("rdn_linear_bwd", _linear(act=1, pre=AT), LAUNCH, "injected"),
    ("rdn_linear_bwd", _linear(dy_ld=68), MISALIGNED, "rows of dy"),
    ("rdn_linear_bwd", _linear(dy=0), INVALID, "dy"),
    ("rdn_linear_bwd", _linear(dx=FAKE + 16384), INVALID, "aliases"),
    ("rdn_linear_bwd", _linear(dw=FAKE + 4096), INVALID, "aliases"),
    ("rdn_linear_bwd", _linear(dw_dtype=5), UNSUPPORTED, "dw_dtype"),
    ("rdn_linear_bwd", _linear(workspace=0, act=1, pre=FAKE), WORKSPACE, "workspace"),
    ("rdn_linear_bwd", _linear(workspace=0, M=1000, dbias=FAKE), WORKSPACE, "workspace"),
]


@pytest.mark.parametrize("fn,args,status,says", CASES, ids=[f"{c[0]}-{n}" for n, c in enumerate(CASES)])
def test_entry_points(fn, args, status, says):
    _refused(fn, args, status, says)


def test_workspace_sizes():
    lib, n = _abi.load(), ctypes.c_size_t(0)
    # the sums of the batch's rows, if several, and the kept states (4 a row) where they are not given
    for B, kept, want in ((2, 0, 2 * 128 * 4 * (1 + 4)), (2, FAKE, 2 * 128 * 4), (1, 0, 128 * 4 * 4), (1, FAKE, 0)):
        assert lib.rdn_gscan_bwd_workspace_size(ctypes.byref(_gscan(B=B, h_chunks=kept)), ctypes.byref(n)) == 0
        assert n.value == want
    assert lib.rdn_gscan_bwd_workspace_size(ctypes.byref(_gscan()), None) == INVALID
    assert lib.rdn_linear_bwd_workspace_size(ctypes.byref(_linear(M=100)), ctypes.byref(n)) == 0
    none = n.value
    assert lib.rdn_linear_bwd_workspace_size(ctypes.byref(_linear(M=100, act=1)), ctypes.byref(n)) == 0
    assert n.value - none == 100 * 64 * 2
    assert lib.rdn_linear_bwd_workspace_size(ctypes.byref(_linear(N=4)), ctypes.byref(n)) == UNSUPPORTED


def test_binding_refusals():
    x, lam = torch.zeros(2, 3, 8), torch.zeros(8)
    for call in (lambda: rdn.gated_scan_fwd(x, x, x, lam), lambda: rdn.gated_scan_bwd(x, x, x, lam, x),
                 lambda: rdn.gated_scan_step(x[0], x[0], x[0], lam, torch.zeros(3, 8)), lambda: rdn.add_norm_q8(x),
                 lambda: rdn.linear_fwd(x, torch.zeros(8, 8)), lambda: rdn.linear_bwd(x, torch.zeros(8, 8), x)):
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    with pytest.raises(ValueError, match="act must be"):
        layer_ops._act("relu")


@pytest.mark.gpu
def test_binding_refusals_on_the_device():
    dev, bf = "cuda", torch.bfloat16
    x, lam = torch.zeros(2, 4, 16, device=dev, dtype=bf), torch.zeros(16, device=dev)
    w = torch.zeros(8, 16, device=dev, dtype=bf)
    f8 = torch.float8_e4m3fn
    bad = [
        lambda: rdn.gated_scan_fwd(x, x[:, :2], x, lam),
        lambda: rdn.gated_scan_fwd(x, x.float(), x, lam),
        lambda: rdn.gated_scan_fwd(x[:, :2], x[:, :2], x[:, :2], lam),  # rows of two distances
        lambda: rdn.gated_scan_fwd(x, x, x, lam.double()),
        lambda: rdn.gated_scan_fwd(x, x, x, lam, h0=torch.zeros(3, 16, device=dev)),
        lambda: rdn.gated_scan_bwd(x, x, x, lam, x, h_chunks=torch.zeros(2, 2, 16, device=dev)),
        lambda: rdn.gated_scan_step(x[0], x[0], x[0], lam, torch.zeros(4, 16, device=dev, dtype=bf)),
        lambda: rdn.add_norm_q8(x, x[..., :8]),
        lambda: rdn.add_norm_q8(x, weight=lam[:8]),
        lambda: rdn.add_norm_q8(x.half()),
        lambda: rdn.linear_fwd(x, w[:, :8]),
        lambda: rdn.linear_fwd(x.float(), w.float()),
        lambda: rdn.linear_fwd(x, w, act="relu"),
        lambda: rdn.linear_fwd(x, w, x_scale=torch.zeros(2, 4, device=dev)),
        lambda: rdn.linear_fwd(x.to(f8), w.to(f8)),
        lambda: rdn.linear_fwd(x, w, residual=x),
        lambda: rdn.linear_fwd(x.expand(3, 2, 4, 16), w),
        lambda: rdn.linear_bwd(x, w, torch.zeros(2, 4, 8, device=dev, dtype=bf), act="silu"),
        lambda: rdn.linear_bwd(x, w, x),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {n} was taken")
    for call in (lambda: rdn.linear_fwd(x, w[:4]), lambda: rdn.linear_fwd(x[..., 1:9], w[:, :8].contiguous()),
                 lambda: rdn.gated_scan_fwd(x, x, x, lam, c=0.0)):
        with pytest.raises(rdn.RdnError):
            call()
