"""The operators around the recurrence (include/rdn.h, "Operators around the
recurrence"): the short causal convolution, the selective state space scan, the
gated linear recurrence, the norms before and after a block with its gate and
scaled residual, the norm with an output in 8 bits, and the matrix product with
bias, activation and residual; for prompts and training, and for single tokens.

As in the rest of the package these functions only check and marshal
arguments, allocate results and the workspace the library asks for, and raise
on a non-OK status; every step runs in the library's CUDA kernels on the
current stream of the operands' device.

Token rows may be strided: a [B, T, C] operand can be a slice of the last axis
of a wider, otherwise contiguous tensor (`proj[..., a:b]`), without a copy.  All
its rows have to be one distance apart: a slice of the tokens of several batch
rows (`x[:, a:b]`) and expanded tensors are refused (make them contiguous).
Parameters (weights, biases, A, D, scales) and the scans' states are fp32;
results and convolution states have the inputs' type (bf16 or fp32).  The matrix
product's operands are bf16, or 8-bit with scales.
"""
from __future__ import annotations

import ctypes

import torch

from . import _abi

__all__ = ["causal_conv_fwd", "causal_conv_bwd", "causal_conv_step", "selective_scan_fwd",
           "selective_scan_bwd", "selective_scan_step", "block_norm_fwd", "block_norm_bwd", "gated_scan_fwd",
           "gated_scan_bwd", "gated_scan_step", "add_norm_q8", "linear_fwd", "linear_bwd"]

_DTYPES = {torch.bfloat16: _abi.RDN_BF16, torch.float32: _abi.RDN_F32}
_GATES = {"silu": 0, "sigmoid": 1}
_F32 = torch.float32


def _code(dtype):
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"rdn: unsupported dtype {dtype}")
    return code


# A step of one token is a few microseconds of device time, so the checks below
# are kept to a few attribute reads per operand (device indexes instead of device
# objects, dtypes by identity) and the argument structs are packed in one call.

def _bad(name, t, shape, dtype, dev):
    raise ValueError(f"rdn: {name} must be {tuple(shape)} {dtype} on CUDA device {dev} "
                     f"(got {tuple(t.shape)} {t.dtype} on {t.device})")


def _rows(name, t, shape, dtype, dev, lead=2):
    """(address, row stride) of t's rows: one for each index of the first `lead` axes, of the
    elements of the others.  Stride 0: contiguous."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        _bad(name, t, shape, dtype, dev)
    return t.data_ptr(), 0 if t.is_contiguous() else _stride(name, t, lead)


def _stride(name, t, lead):
    """The one distance between consecutive rows that the library takes: the elements of a row
    lie side by side, and every leading axis of more than one element continues the one below
    it (an expanded axis, of stride 0, does not, nor does a slice of the tokens of several
    batch rows)."""
    shape, strides = t.shape, t.stride()
    if lead == 2 and len(shape) == 3:  # (the common case: a slice of a projection's rows)
        n0, n1, width = shape
        s0, ld, one = strides
        if one == 1 and ld >= width and n1 > 1 and (n0 == 1 or s0 == ld * n1):
            return ld
    width = 1
    for a in range(len(shape) - 1, lead - 1, -1):
        if shape[a] != 1 and strides[a] != width:
            axes = "axis" if len(shape) - lead == 1 else f"{len(shape) - lead} axes"
            raise ValueError(f"rdn: the last {axes} of {name} must be contiguous")
        width *= shape[a]
    ld = span = 0  # distance of the rows; of the next axis's indexes, if the rows go on evenly
    for a in range(lead - 1, -1, -1):
        if shape[a] == 1:
            continue
        if strides[a] < width if ld == 0 else strides[a] != span:
            raise ValueError(f"rdn: the rows of {name} must be evenly spaced, without overlap (got strides "
                             f"{tuple(strides)} of {tuple(shape)}); pass {name}.contiguous()")
        ld = ld or strides[a]
        span = strides[a] * shape[a]
    return ld


def _whole(name, t, shape, dtype, dev):
    """The address of an optional contiguous tensor (0 = None)."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        _bad(name, t, shape, dtype, dev)
    if not t.is_contiguous():
        raise ValueError(f"rdn: {name} must be contiguous")
    return t.data_ptr()


def _cuda(name, t, dims):
    """(device index, shape)"""
    dev, shape = t.get_device(), t.shape
    if dev < 0:
        raise ValueError("rdn: tensors must be on a CUDA device")
    if len(shape) != dims:
        raise ValueError(f"rdn: {name} must have {dims} axes (got {tuple(shape)})")
    return dev, shape


def _table(cu, B, dev):
    """(address, sequences of the table or 0, sequences of the call)"""
    if cu is None:
        return 0, 0, B
    if cu.dtype != torch.int32 or cu.dim() != 1 or cu.numel() < 2 or cu.get_device() != dev:
        raise ValueError("cu_seqlens must be a 1-D int32 device tensor of num_seqs + 1 offsets")
    if not cu.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous")
    return cu.data_ptr(), cu.numel() - 1, cu.numel() - 1


def _error(name, st):
    from . import RdnError
    raise RdnError(name, st, _abi.load().rdn_last_error().decode())


_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(name, args, dev):
    # the library launches on the current device: make it the operands'
    if dev == _current_device():
        st = _abi.packed(name)(args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            st = _abi.packed(name)(args, _raw_stream(dev))
    if st:
        _error(name, st)


def _size(name, args):
    n = ctypes.c_longlong(0)
    st = _abi.packed(name)(args, ctypes.addressof(n))
    if st:
        _error(name, st)
    return n.value


def _workspace(workspace, nbytes, dev):
    if workspace is not None and workspace.numel() * workspace.element_size() >= nbytes:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("rdn: workspace must be contiguous and on the operands' device")
        return workspace
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=dev)


def _with_workspace(query, args, workspace, dev):
    """args, whose last two fields are the workspace and its bytes, with a workspace of the size that `query`
    asks for."""
    nbytes = _size(query, args)
    if not nbytes and workspace is None:
        return None, args
    ws = _workspace(workspace, nbytes, dev)
    return ws, args[:-16] + _abi.WORKSPACE_PACK(ws.data_ptr(), ws.numel() * ws.element_size())


def _silu(activation):
    if activation not in ("silu", None):
        raise ValueError('rdn: activation must be "silu" or None')
    return 1 if activation == "silu" else 0


def causal_conv_fwd(x, weight, bias=None, state=None, activation="silu", cu_seqlens=None,
                    return_state=False, out=None):
    """Depthwise causal convolution over tokens with W = 2..4 taps, then SiLU
    (activation=None: none): y_t = act(bias + sum_j weight[:, j] x_{t-W+1+j}).

    x [B,T,C]; weight [C,W], bias [C] fp32.  state [B,W-1,C] (packed:
    [num_seqs,W-1,C]): the inputs before each sequence's start, oldest first
    (None: zeros).  Returns y [B,T,C], or (y, last state) with return_state.
    cu_seqlens: packed sequences, as for rdn_fwd (B = 1)."""
    dev, shape = _cuda("x", x, 3)
    B, T, C = shape
    W = weight.shape[-1]
    cu, ns, n = _table(cu_seqlens, B, dev)
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
    last = torch.empty(n, W - 1, C, dtype=x.dtype, device=dev) if return_state else None
    px, x_ld = _rows("x", x, (B, T, C), x.dtype, dev)
    py, y_ld = _rows("out", y, (B, T, C), x.dtype, dev)
    args = _abi.CONV_PACK(
        B, T, C, W, _code(x.dtype), _silu(activation), x_ld, y_ld, 0, 0, px,
        _whole("weight", weight, (C, W), _F32, dev), _whole("bias", bias, (C,), _F32, dev),
        _whole("state", state, (n, W - 1, C), x.dtype, dev), py,
        0 if last is None else last.data_ptr(), cu, ns, 0, 0, 0, 0, 0, 0, 0, 0)
    _call("rdn_conv_fwd", args, dev)
    return (y, last) if return_state else y


def causal_conv_bwd(x, weight, dy, bias=None, state=None, d_state=None, activation="silu",
                    cu_seqlens=None, workspace=None, out=None):
    """Backward of causal_conv_fwd (recomputes the sums before the activation).
    dy: gradient of y; d_state: of the returned last state, or None.  Returns a
    dict with dx, dweight [C,W], dbias [C] (fp32; with bias) and dstate (with
    state).  out: tensors to write into, by those names."""
    dev, shape = _cuda("x", x, 3)
    B, T, C = shape
    W = weight.shape[-1]
    cu, ns, n = _table(cu_seqlens, B, dev)
    e = lambda *s, dtype=x.dtype: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
    res = dict(out) if out else {}
    if res.get("dx") is None:
        res["dx"] = e(B, T, C)
    if res.get("dweight") is None:
        res["dweight"] = e(C, W, dtype=_F32)
    if bias is not None and res.get("dbias") is None:
        res["dbias"] = e(C, dtype=_F32)
    if state is not None and res.get("dstate") is None:
        res["dstate"] = e(n, W - 1, C)
    px, x_ld = _rows("x", x, (B, T, C), x.dtype, dev)
    pdy, dy_ld = _rows("dy", dy, (B, T, C), x.dtype, dev)
    pdx, dx_ld = _rows("dx", res["dx"], (B, T, C), x.dtype, dev)

    def pack(ws, nbytes):
        return _abi.CONV_PACK(
            B, T, C, W, _code(x.dtype), _silu(activation), x_ld, 0, dy_ld, dx_ld, px,
            _whole("weight", weight, (C, W), _F32, dev), _whole("bias", bias, (C,), _F32, dev),
            _whole("state", state, (n, W - 1, C), x.dtype, dev), 0, 0, cu, ns, pdy,
            _whole("d_state", d_state, (n, W - 1, C), x.dtype, dev), pdx,
            _whole("dweight", res["dweight"], (C, W), _F32, dev),
            _whole("dbias", res.get("dbias"), (C,), _F32, dev),
            _whole("dstate", res.get("dstate"), (n, W - 1, C), x.dtype, dev), ws, nbytes)

    ws = _workspace(workspace, _size("rdn_conv_bwd_workspace_size", pack(0, 0)), dev)
    _call("rdn_conv_bwd", pack(ws.data_ptr(), ws.numel() * ws.element_size()), dev)
    return res


def causal_conv_step(x, weight, state, bias=None, activation="silu", slots=None, out=None):
    """One token of causal_conv_fwd for N requests: x [N,C]; state
    [num_slots,W-1,C] is updated in place.  slots [N] int32: each request's row
    of state (distinct); a negative one is an idle row (y = 0).  None: row n."""
    dev, shape = _cuda("x", x, 2)
    N, C = shape
    W = weight.shape[-1]
    ty = x.dtype
    px, x_ld = (x.data_ptr(), 0) if x.is_contiguous() else _rows("x", x, shape, ty, dev, 1)
    if out is None:
        y = torch.empty(shape, dtype=ty, device=dev)
        py, y_ld = y.data_ptr(), 0
    else:
        y = out
        py, y_ld = _rows("out", y, shape, ty, dev, 1)
    num = state.shape[0]
    args = _abi.CONV_STEP_PACK(
        N, C, W, _code(ty), _silu(activation), num, x_ld, y_ld, px,
        _whole("weight", weight, (C, W), _F32, dev), _whole("bias", bias, (C,), _F32, dev),
        _whole("state", state, (num, W - 1, C), ty, dev),
        _whole("slots", slots, (N,), torch.int32, dev), py)
    _call("rdn_conv_step", args, dev)
    return y


class _Scan:
    """The operands of a scan, checked, as the leading values of SCAN_PACK."""

    def __init__(self, x, dt, A, B, C, D, z, dt_bias, h0, dt_softplus, cu_seqlens):
        self.dev, shape = _cuda("x", x, 3)
        dev = self.dev
        b, t, d = shape
        if B.dim() != 4:
            raise ValueError(f"rdn: B must be [B, T, G, S] (got {tuple(B.shape)})")
        g, s = B.shape[2:]
        self.shape, self.bc, self.dtype = (b, t, d), (b, t, g, s), x.dtype
        self.cu, self.ns, self.n = _table(cu_seqlens, b, dev)
        self.states = (self.n, d, s)
        rows = [_rows("x", x, self.shape, x.dtype, dev), _rows("dt", dt, self.shape, x.dtype, dev),
                (0, 0) if z is None else _rows("z", z, self.shape, x.dtype, dev),
                _rows("B", B, self.bc, x.dtype, dev), _rows("C", C, self.bc, x.dtype, dev)]
        self.head = (b, t, d, s, g, _code(x.dtype), 1 if dt_softplus else 0)
        self.lds, self.ptrs = [r[1] for r in rows], [r[0] for r in rows]
        self.params = (_whole("A", A, (d, s), _F32, dev), _whole("D", D, (d,), _F32, dev),
                       _whole("dt_bias", dt_bias, (d,), _F32, dev),
                       _whole("h0", h0, self.states, _F32, dev))

    def slots(self):
        """Blocks of the kept states (rdn_scan_chunk_slots)."""
        b, t = self.shape[:2]
        nc = (t + _abi.SCAN_CHUNK - 1) // _abi.SCAN_CHUNK
        return self.ns + nc if self.ns else b * nc

    def pack(self, out=(0, 0), hT=0, chunks=0, grads=(0,) * 15, ws=0, nbytes=0):
        return _abi.SCAN_PACK(*self.head, *self.lds, out[1], *self.ptrs, *self.params, out[0], hT,
                              chunks, self.cu, self.ns, *grads, ws, nbytes)


def selective_scan_fwd(x, dt, A, B, C, D=None, z=None, dt_bias=None, h0=None, dt_softplus=True,
                       cu_seqlens=None, return_final_state=True, return_chunk_states=False,
                       out=None, workspace=None):
    """Selective state space scan over d channels of s states each:
        dl_t = softplus(dt_t + dt_bias)   (dt_softplus=False: dt_t + dt_bias)
        h_t = exp(dl_t A) h_{t-1} + dl_t x_t B_t,   y_t = C_t . h_t + D x_t
        out_t = y_t silu(z_t)             (z=None: y_t)

    x, dt, z [B,T,d]; A [d,s] fp32; B, C [B,T,G,s] (group g for channels
    g d/G ..); D, dt_bias [d] fp32; h0 [B or num_seqs, d, s] fp32; s <= 64.
    Returns (out, hT); with return_chunk_states also the states at every 16
    tokens [slots,d,s], which selective_scan_bwd can read instead of computing
    them again; only out with both off.  cu_seqlens: packed sequences."""
    a = _Scan(x, dt, A, B, C, D, z, dt_bias, h0, dt_softplus, cu_seqlens)
    dev = a.dev
    y = torch.empty(a.shape, dtype=a.dtype, device=dev) if out is None else out
    hT = torch.empty(a.states, dtype=_F32, device=dev) if return_final_state else None
    hc = None
    if return_chunk_states:
        hc = torch.empty((a.slots(),) + a.states[1:], dtype=_F32, device=dev)
    o = _rows("out", y, a.shape, a.dtype, dev)
    hTp = 0 if hT is None else hT.data_ptr()
    hcp = 0 if hc is None else hc.data_ptr()
    nbytes = _size("rdn_scan_fwd_workspace_size", a.pack())
    ws = _workspace(workspace, nbytes, dev) if nbytes else None
    args = a.pack(o, hTp, hcp, ws=0 if ws is None else ws.data_ptr(),
                  nbytes=0 if ws is None else ws.numel() * ws.element_size())
    _call("rdn_scan_fwd", args, dev)
    res = (y,) + ((hT,) if return_final_state else ()) + ((hc,) if return_chunk_states else ())
    return res if len(res) > 1 else y


def selective_scan_bwd(x, dt, A, B, C, dout, D=None, z=None, dt_bias=None, h0=None, dhT=None,
                       h_chunks=None, dt_softplus=True, cu_seqlens=None, workspace=None, out=None):
    """Backward of selective_scan_fwd.  dout: gradient of out; dhT: of hT or
    None; h_chunks: the forward's states (return_chunk_states) or None.
    Returns a dict with dx, ddt, dB, dC (and dz) in the inputs' type and dA (and
    dD, ddt_bias, dh0, each with its operand) in fp32.  out: tensors to write
    into, by those names."""
    a = _Scan(x, dt, A, B, C, D, z, dt_bias, h0, dt_softplus, cu_seqlens)
    dev = a.dev
    d, s = a.states[1:]
    res = dict(out) if out else {}
    for name, shape, dtype, given in (
            ("dx", a.shape, a.dtype, x), ("ddt", a.shape, a.dtype, dt), ("dz", a.shape, a.dtype, z),
            ("dB", a.bc, a.dtype, B), ("dC", a.bc, a.dtype, C), ("dA", (d, s), _F32, A),
            ("dD", (d,), _F32, D), ("ddt_bias", (d,), _F32, dt_bias), ("dh0", a.states, _F32, h0)):
        if given is not None and res.get(name) is None:
            res[name] = torch.empty(shape, dtype=dtype, device=dev)
    rows = [_rows("dout", dout, a.shape, a.dtype, dev)]
    rows += [(0, 0) if res.get(k) is None else _rows(k, res[k], a.shape, a.dtype, dev)
             for k in ("dx", "ddt", "dz")]
    grads = [r[1] for r in rows] + [rows[0][0], _whole("dhT", dhT, a.states, _F32, dev)]
    grads += [r[0] for r in rows[1:]]
    grads += [_whole("dB", res["dB"], a.bc, a.dtype, dev), _whole("dC", res["dC"], a.bc, a.dtype, dev),
              _whole("dA", res["dA"], (d, s), _F32, dev), _whole("dD", res.get("dD"), (d,), _F32, dev),
              _whole("ddt_bias", res.get("ddt_bias"), (d,), _F32, dev),
              _whole("dh0", res.get("dh0"), a.states, _F32, dev)]
    hc = _whole("h_chunks", h_chunks, (a.slots(), d, s), _F32, dev)
    nbytes = _size("rdn_scan_bwd_workspace_size", a.pack(chunks=hc))
    ws = _workspace(workspace, nbytes, dev)
    _call("rdn_scan_bwd", a.pack(chunks=hc, grads=grads, ws=ws.data_ptr(),
                                 nbytes=ws.numel() * ws.element_size()), dev)
    return res


def selective_scan_step(x, dt, A, B, C, h, D=None, z=None, dt_bias=None, dt_softplus=True,
                        slots=None, out=None):
    """One token of selective_scan_fwd for N requests: x, dt, z [N,d]; B, C
    [N,G,s]; h [num_slots,d,s] fp32 is updated in place; slots as in
    causal_conv_step.  Returns out [N,d]."""
    dev, shape = _cuda("x", x, 2)
    n, d = shape
    bshape = B.shape
    if len(bshape) != 3 or bshape[0] != n:
        raise ValueError(f"rdn: B must be [N, G, S] (got {tuple(bshape)})")
    g, s = bshape[1], bshape[2]
    ty = x.dtype
    px, x_ld = (x.data_ptr(), 0) if x.is_contiguous() else _rows("x", x, shape, ty, dev, 1)
    pdt, dt_ld = _rows("dt", dt, shape, ty, dev, 1)
    pz, z_ld = (0, 0) if z is None else _rows("z", z, shape, ty, dev, 1)
    pB, b_ld = _rows("B", B, bshape, ty, dev, 1)
    pC, c_ld = _rows("C", C, bshape, ty, dev, 1)
    if out is None:
        y = torch.empty(shape, dtype=ty, device=dev)
        py, y_ld = y.data_ptr(), 0
    else:
        y = out
        py, y_ld = _rows("out", y, shape, ty, dev, 1)
    num = h.shape[0]
    args = _abi.SCAN_STEP_PACK(
        n, d, s, g, _code(ty), 1 if dt_softplus else 0, num, x_ld, dt_ld, z_ld, b_ld, c_ld, y_ld, px,
        pdt, pz, pB, pC, _whole("A", A, (d, s), _F32, dev), _whole("D", D, (d,), _F32, dev),
        _whole("dt_bias", dt_bias, (d,), _F32, dev), _whole("h", h, (num, d, s), _F32, dev),
        _whole("slots", slots, (n,), torch.int32, dev), py)
    _call("rdn_scan_step", args, dev)
    return y


class _Norm:
    """The operands of a block norm, checked, as the leading values of NORM_PACK."""

    def __init__(self, f, weight, z, gate, x, scale, weight_next, eps, h_dtype=None):
        first = f if f is not None else x
        if first is None:
            raise ValueError("rdn: f or x is required")
        self.dev = dev = first.get_device()
        if dev < 0:
            raise ValueError("rdn: tensors must be on a CUDA device")
        self.shape = shape = first.shape
        D, lead = shape[-1], len(shape) - 1
        self.heads, self.wshape = 1, (D,)
        if f is not None:
            if weight is None:
                raise ValueError("rdn: f needs its weight")
            self.wshape = weight.shape
            if len(self.wshape) == 2:
                self.heads = self.wshape[0]
            elif len(self.wshape) != 1:
                raise ValueError("rdn: weight must be [D] or [heads, D]")
            if self.wshape[-1] != D:
                raise ValueError(f"rdn: weight must have {D} columns (got {tuple(self.wshape)})")
            if self.heads > 1 and lead > 1 and shape[-2] != self.heads:
                raise ValueError(f"rdn: weight of {self.heads} heads needs f [..., {self.heads}, {D}], or the rows of "
                                 f"one [rows, {D}] (got {tuple(shape)})")
        if gate not in _GATES:
            raise ValueError('rdn: gate must be "silu" or "sigmoid"')
        self.dtype = h_dtype if f is None and h_dtype is not None else first.dtype
        self.xdtype = x.dtype if x is not None else self.dtype
        self.vec = scale if isinstance(scale, torch.Tensor) else None
        const = 1.0 if scale is None or self.vec is not None else float(scale)
        pf, f_ld = (0, 0) if f is None else _rows("f", f, shape, self.dtype, dev, lead)
        pz, z_ld = (0, 0) if z is None else _rows("z", z, shape, self.dtype, dev, lead)
        px, x_ld = (0, 0) if x is None else _rows("x", x, shape, self.xdtype, dev, lead)
        n = first.numel() // D if D else 0
        self.head = (n, D, self.heads, _DTYPES.get(self.dtype, -1), _DTYPES.get(self.xdtype, -1),
                     _GATES[gate], float(eps), const, f_ld, z_ld, x_ld, pf, pz, px,
                     0 if f is None else _whole("weight", weight, self.wshape, _F32, dev),
                     _whole("scale", self.vec, (D,), _F32, dev),
                     _whole("weight_next", weight_next, (D,), _F32, dev))


def block_norm_fwd(f=None, weight=None, z=None, gate="silu", x=None, scale=None, weight_next=None,
                   eps=1e-6, h_dtype=None, out=None):
    """The norms after and before a block, per row of the last axis:
        u = f / rms(f) * weight * act(z)     act: gate = "silu" or "sigmoid"
        r = x + scale * u                    (x=None: r = u)
        h = r / rms(r) * weight_next
    with rms(t) = sqrt(mean(t^2) + eps).  Returns (r, h); h is None without
    weight_next.  f=None: only the norm before a block, r is x itself.

    f, z [..., D] (z=None: no gate); x [..., D] in f's type or fp32; weight [D],
    or [heads, D] for f [..., heads, D], or its rows flattened to [rows, D] with the
    heads in turn (without x and weight_next); scale: a [D] fp32 tensor or a number; weight_next [D] fp32.  r has x's type, h f's
    (f=None: h_dtype, or x's).  out: (r, h) to write into."""
    a = _Norm(f, weight, z, gate, x, scale, weight_next, eps, h_dtype)
    r, h = out if out is not None else (None, None)
    pr = ph = 0
    if f is None:
        r = x
    elif r is None:
        r = torch.empty(a.shape, dtype=a.xdtype, device=a.dev)
        pr = r.data_ptr()
    else:
        pr = _whole("r", r, a.shape, a.xdtype, a.dev)
    if weight_next is None:
        h = None
    elif h is None:
        h = torch.empty(a.shape, dtype=a.dtype, device=a.dev)
        ph = h.data_ptr()
    else:
        ph = _whole("h", h, a.shape, a.dtype, a.dev)
    _call("rdn_norm_fwd", _abi.NORM_PACK(*a.head, pr, ph, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), a.dev)
    return r, h


def block_norm_bwd(f=None, weight=None, z=None, gate="silu", x=None, scale=None, weight_next=None,
                   eps=1e-6, dr=None, dh=None, workspace=None, out=None):
    """Backward of block_norm_fwd.  dr: gradient of r (or None with weight_next:
    zero), dh: of h.  Returns a dict with df, dz, dx and (fp32) dweight, dscale
    (with a scale tensor), dweight_next, each with its operand.  out: tensors to
    write into, by those names."""
    a = _Norm(f, weight, z, gate, x, scale, weight_next, eps, None if dh is None else dh.dtype)
    res = dict(out) if out else {}
    D = a.shape[-1:]
    for name, shape, dtype, given in (
            ("df", a.shape, a.dtype, f), ("dz", a.shape, a.dtype, z if f is not None else None),
            ("dx", a.shape, a.xdtype, x), ("dweight", a.wshape, _F32, f),
            ("dscale", D, _F32, a.vec if f is not None and x is not None else None),
            ("dweight_next", D, _F32, weight_next)):
        if given is not None and res.get(name) is None:
            res[name] = torch.empty(shape, dtype=dtype, device=a.dev)
    p = lambda k, shape, ty: _whole(k, res.get(k), shape, ty, a.dev)  # noqa: E731
    tail = (0, 0, _whole("dr", dr, a.shape, a.xdtype, a.dev), _whole("dh", dh, a.shape, a.dtype, a.dev),
            p("df", a.shape, a.dtype), p("dz", a.shape, a.dtype), p("dx", a.shape, a.xdtype),
            p("dweight", a.wshape, _F32), p("dscale", D, _F32), p("dweight_next", D, _F32))
    nbytes = _size("rdn_norm_bwd_workspace_size", _abi.NORM_PACK(*a.head, *(0,) * 12))
    ws = _workspace(workspace, nbytes, a.dev)
    _call("rdn_norm_bwd", _abi.NORM_PACK(*a.head, *tail, ws.data_ptr(),
                                         ws.numel() * ws.element_size()), a.dev)
    return res


class _Gated:
    """The operands of a gated recurrence, checked, as the leading values of GSCAN_PACK."""

    def __init__(self, x, r, i, lam, c, h0, cu_seqlens):
        self.dev, self.shape = dev, shape = _cuda("x", x, 3)
        self.dtype = ty = x.dtype
        b, t, d = shape
        self.cu, self.ns, self.n = _table(cu_seqlens, b, dev)
        self.states = (self.n, d)
        px, x_ld = _rows("x", x, shape, ty, dev)
        pr, r_ld = _rows("r", r, shape, ty, dev)
        pi, i_ld = _rows("i", i, shape, ty, dev)
        self.head = (b, t, d, _code(ty), float(c))
        self.lds, self.ptrs = (x_ld, r_ld, i_ld), (px, pr, pi)
        self.params = (_whole("lam", lam, (d,), _F32, dev), _whole("h0", h0, self.states, _F32, dev))

    def chunks(self):
        """Shape of the kept states."""
        b, t, d = self.shape
        return (b, (t + _abi.GSCAN_CHUNK - 1) // _abi.GSCAN_CHUNK, d)

    def pack(self, y=(0, 0), hT=0, chunks=0, grads=(0,) * 11, ws=0, nbytes=0):
        return _abi.GSCAN_PACK(*self.head, *self.lds, y[1], *self.ptrs, *self.params, y[0], hT, chunks,
                               self.cu, self.ns, *grads, ws, nbytes)


def gated_scan_fwd(x, r, i, lam, c=8.0, h0=None, cu_seqlens=None, return_final_state=True,
                   return_chunk_states=False, out=None):
    """Gated linear recurrence over d channels of one state each:
        a_t = exp(-c softplus(lam) sigmoid(r_t))
        h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t,   y_t = h_t

    x, r, i [B,T,d]; lam [d] fp32; h0 [B or num_seqs, d] fp32.  Returns (y, hT);
    with return_chunk_states also the states before every 64 tokens
    [B, ceil(T/64), d], which gated_scan_bwd can read instead of computing them
    again; only y with both off.  cu_seqlens: packed sequences."""
    a = _Gated(x, r, i, lam, c, h0, cu_seqlens)
    dev, shape = a.dev, a.shape
    hT = hc = None
    phT = phc = 0
    if out is None:
        y = torch.empty(shape, dtype=a.dtype, device=dev)
        py = (y.data_ptr(), 0)
    else:
        y = out
        py = _rows("out", y, shape, a.dtype, dev)
    if return_final_state:
        hT = torch.empty(a.states, dtype=_F32, device=dev)
        phT = hT.data_ptr()
    if return_chunk_states:
        hc = torch.empty(a.chunks(), dtype=_F32, device=dev)
        phc = hc.data_ptr()
    _call("rdn_gscan_fwd", a.pack(py, phT, phc), dev)
    if return_final_state:
        return (y, hT, hc) if return_chunk_states else (y, hT)
    return (y, hc) if return_chunk_states else y


def gated_scan_bwd(x, r, i, lam, dy, c=8.0, h0=None, dhT=None, cu_seqlens=None, h_chunks=None,
                   workspace=None, out=None):
    """Backward of gated_scan_fwd.  dy: gradient of y; dhT: of the final states, or
    None; h_chunks: the forward's return_chunk_states (None: computed again).
    Returns a dict with dx, dr, di, dlam (fp32) and, with h0, dh0.  out: tensors
    to write into, by those names."""
    a = _Gated(x, r, i, lam, c, h0, cu_seqlens)
    dev, shape, ty = a.dev, a.shape, a.dtype
    d = shape[2]
    pdy, dy_ld = _rows("dy", dy, shape, ty, dev)
    dx_ld = dr_ld = di_ld = pdh = 0
    if out is None:
        dx, dr = torch.empty(shape, dtype=ty, device=dev), torch.empty(shape, dtype=ty, device=dev)
        di, dlam = torch.empty(shape, dtype=ty, device=dev), torch.empty(d, dtype=_F32, device=dev)
        pdx, pdr, pdi, pdl = dx.data_ptr(), dr.data_ptr(), di.data_ptr(), dlam.data_ptr()
        res = dict(dx=dx, dr=dr, di=di, dlam=dlam)
        if h0 is not None:
            res["dh0"] = dh = torch.empty(a.states, dtype=_F32, device=dev)
            pdh = dh.data_ptr()
    else:
        res = dict(out)
        for name in ("dx", "dr", "di"):
            if res.get(name) is None:
                res[name] = torch.empty(shape, dtype=ty, device=dev)
        if res.get("dlam") is None:
            res["dlam"] = torch.empty(d, dtype=_F32, device=dev)
        if h0 is not None and res.get("dh0") is None:
            res["dh0"] = torch.empty(a.states, dtype=_F32, device=dev)
        pdx, dx_ld = _rows("dx", res["dx"], shape, ty, dev)
        pdr, dr_ld = _rows("dr", res["dr"], shape, ty, dev)
        pdi, di_ld = _rows("di", res["di"], shape, ty, dev)
        pdl = _whole("dlam", res["dlam"], (d,), _F32, dev)
        pdh = _whole("dh0", res.get("dh0"), a.states, _F32, dev)
    grads = (dy_ld, dx_ld, dr_ld, di_ld, pdy, _whole("dhT", dhT, a.states, _F32, dev), pdx, pdr, pdi, pdl, pdh)
    args = a.pack(chunks=_whole("h_chunks", h_chunks, a.chunks(), _F32, dev), grads=grads)
    ws, args = _with_workspace("rdn_gscan_bwd_workspace_size", args, workspace, dev)
    _call("rdn_gscan_bwd", args, dev)
    return res


def gated_scan_step(x, r, i, lam, h, c=8.0, slots=None, out=None):
    """One token of gated_scan_fwd for N requests: x, r, i [N,d]; h [num_slots,d]
    fp32 is updated in place.  slots [N] int32: each request's row of h (distinct);
    a negative one is an idle row (y = 0).  None: row n."""
    dev, shape = _cuda("x", x, 2)
    n, d = shape
    ty = x.dtype
    px, x_ld = _rows("x", x, shape, ty, dev, 1)
    pr, r_ld = _rows("r", r, shape, ty, dev, 1)
    pi, i_ld = _rows("i", i, shape, ty, dev, 1)
    if out is None:
        y = torch.empty(shape, dtype=ty, device=dev)
        py, y_ld = y.data_ptr(), 0
    else:
        y = out
        py, y_ld = _rows("out", y, shape, ty, dev, 1)
    num = h.shape[0]
    args = _abi.GSCAN_STEP_PACK(
        n, d, _code(ty), float(c), num, x_ld, r_ld, i_ld, y_ld, px, pr, pi, _whole("lam", lam, (d,), _F32, dev),
        _whole("h", h, (num, d), _F32, dev), _whole("slots", slots, (n,), torch.int32, dev), py)
    _call("rdn_gscan_step", args, dev)
    return y


_E4M3 = torch.float8_e4m3fn


def add_norm_q8(x, f=None, weight=None, eps=1e-6, out=None):
    """The residual's addition and the norm before a block, per row of the last
    axis, with an output in 8 bits and a scale per row:
        r = x + f                       (f=None: r is x itself)
        h = r / rms(r) * weight         (weight=None: h = r)
        scale = max|h| / 448,  q = h / scale rounded to float8_e4m3fn
    x, f [..., D] (bf16 or fp32, each its own); weight [D] fp32.  Returns
    (r, q, scale): r in x's type, scale [...] fp32; q and scale are the first
    operand of linear_fwd.  out: (r, q, scale) to write into, each a tensor or None; r may be x.
    Backward (straight through the rounding): block_norm_bwd(x=r,
    weight_next=weight, dr=dr, dh=dh)["dx"] is the gradient of x and of f."""
    dev, shape, ty = x.get_device(), x.shape, x.dtype
    if dev < 0 or not shape:
        raise ValueError("rdn: tensors must be on a CUDA device, with at least one axis")
    d, lead, over = shape[-1], len(shape) - 1, shape[:-1]
    px, x_ld = _rows("x", x, shape, ty, dev, lead)
    pf = f_ld = pr = fc = 0
    if f is not None:
        pf, f_ld = _rows("f", f, shape, f.dtype, dev, lead)
        fc = _code(f.dtype)
    if out is None:
        if f is None:
            r = x
        else:
            r = torch.empty(shape, dtype=ty, device=dev)
            pr = r.data_ptr()
        q = torch.empty(shape, dtype=_E4M3, device=dev)
        s = torch.empty(over, dtype=_F32, device=dev)
        pq, ps = q.data_ptr(), s.data_ptr()
    else:
        r, q, s = out
        if f is None and (r is None or r is x):
            r = x
        else:
            r = torch.empty(shape, dtype=ty, device=dev) if r is None else r
            pr = _whole("r", r, shape, ty, dev)
        q = torch.empty(shape, dtype=_E4M3, device=dev) if q is None else q
        s = torch.empty(over, dtype=_F32, device=dev) if s is None else s
        pq, ps = _whole("q", q, shape, _E4M3, dev), _whole("scale", s, over, _F32, dev)
    args = _abi.NORM_Q8_PACK(over.numel(), d, _code(ty), fc, float(eps), x_ld, f_ld, px, pf,
                             _whole("weight", weight, (d,), _F32, dev), pr, pq, ps)
    _call("rdn_norm_q8", args, dev)
    return r, q, s


_ACTS = {None: 0, "silu": 1, "sigmoid": 2, "gelu": 3}


def _act(act):
    if act not in _ACTS:
        raise ValueError(f'rdn: act must be None, "silu", "sigmoid" or "gelu" (got {act!r})')
    return _ACTS[act]


def _linear_operands(x, w):
    """(device, rows' shape, M, N, K, x's and w's (address, row stride))"""
    dev, shape, ty = x.get_device(), x.shape, x.dtype
    if dev < 0 or not shape:
        raise ValueError("rdn: tensors must be on a CUDA device, with at least one axis")
    ws, lead = w.shape, shape[:-1]
    if len(ws) != 2 or ws[1] != shape[-1]:
        raise ValueError(f"rdn: w must be [N, {shape[-1]}] (got {tuple(ws)})")
    n, k = ws
    return (dev, lead, lead.numel(), n, k, _rows("x", x, shape, ty, dev, len(lead)), _rows("w", w, ws, ty, dev, 1))


def linear_fwd(x, w, bias=None, act=None, residual=None, x_scale=None, w_scale=None, out_dtype=None,
               return_pre=False, out=None):
    """Matrix product with bias, activation and residual:
        p = x w^T (x_scale w_scale) + bias,   y = act(p) + residual
    act: None, "silu", "sigmoid" or "gelu".

    x [..., K], w [N, K] bf16, or float8_e4m3fn with x_scale [...] and w_scale [N]
    fp32 (add_norm_q8 makes both); bias [N] bf16 or fp32; residual [..., N] in y's
    type.  y [..., N]: out_dtype, or the residual's type, or bf16.  K a multiple
    of 8 (8-bit: 16), N of 8; rows of x and w start on 16 bytes.  Returns y, or
    (y, p in bf16) with return_pre, which linear_bwd reads.  out: y to write into;
    it may be the residual."""
    dev, lead, m, n, k, (px, x_ld), (pw, w_ld) = _linear_operands(x, w)
    q8 = x.dtype is _E4M3
    if not q8 and x.dtype is not torch.bfloat16:
        raise ValueError(f"rdn: unsupported dtype {x.dtype}")
    pxs = pws = pb = bt = pr = r_ld = pp = 0
    if q8:
        if x_scale is None or w_scale is None:
            raise ValueError("rdn: 8-bit operands need x_scale and w_scale")
        pxs, pws = _whole("x_scale", x_scale, lead, _F32, dev), _whole("w_scale", w_scale, (n,), _F32, dev)
    elif x_scale is not None or w_scale is not None:
        raise ValueError("rdn: x_scale and w_scale go with 8-bit operands")
    shape = (*lead, n)
    if out_dtype is not None:
        ty = out_dtype
    else:
        ty = out.dtype if out is not None else torch.bfloat16 if residual is None else residual.dtype
    if residual is not None:
        pr, r_ld = _rows("residual", residual, shape, ty, dev, len(lead))
    if bias is not None:
        bt, pb = _code(bias.dtype), _whole("bias", bias, (n,), bias.dtype, dev)
    if out is None:
        y = torch.empty(shape, dtype=ty, device=dev)
        py, y_ld = y.data_ptr(), 0
    else:
        y = out
        py, y_ld = _rows("out", y, shape, ty, dev, len(lead))
    if return_pre:
        pre = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        pp = pre.data_ptr()
    args = _abi.LINEAR_PACK(m, n, k, _abi.RDN_E4M3 if q8 else _abi.RDN_BF16, _code(ty), bt, _act(act), x_ld, w_ld,
                            r_ld, y_ld, px, pw, pxs, pws, pb, pr, py, pp, 0, 0, 0, 0, 0, 0, 0, 0)
    _call("rdn_linear_fwd", args, dev)
    return (y, pre) if return_pre else y


def linear_bwd(x, w, dy, pre=None, act=None, bias=None, need_dx=True, need_dw=True, dw_dtype=None,
               workspace=None, out=None):
    """Backward of linear_fwd in bf16: dp = dy act'(pre), dx = dp w, dw = dp^T x,
    dbias = the sum of dp's rows; the residual's gradient is dy itself.

    dy [..., N] bf16; pre: linear_fwd's return_pre, needed with an activation;
    bias: the forward's bias, or None.  Returns a dict with dx (bf16), dw (dw_dtype,
    or w's type) and, with a bias, dbias in its type.  out: tensors to write into,
    by those names."""
    dev, lead, m, n, k, (px, x_ld), (pw, w_ld) = _linear_operands(x, w)
    bf = torch.bfloat16
    if x.dtype is not bf:
        raise ValueError(f"rdn: unsupported dtype {x.dtype}")
    if act is not None and pre is None:
        raise ValueError("rdn: the backward of an activation needs pre")
    pdy, dy_ld = _rows("dy", dy, (*lead, n), bf, dev, len(lead))
    res = dict(out) if out else {}
    pdx = pdw = pdb = bt = pp = 0
    wt = dw_dtype or (res["dw"].dtype if res.get("dw") is not None else w.dtype)
    if need_dx:
        if res.get("dx") is None:
            res["dx"] = torch.empty(x.shape, dtype=bf, device=dev)
        pdx = _whole("dx", res["dx"], x.shape, bf, dev)
    else:
        res.pop("dx", None)
    if need_dw:
        if res.get("dw") is None:
            res["dw"] = torch.empty(w.shape, dtype=wt, device=dev)
        pdw = _whole("dw", res["dw"], w.shape, wt, dev)
    else:
        res.pop("dw", None)
    if bias is not None:
        bt = _code(bias.dtype)
        if bias.shape != (n,) or bias.get_device() != dev:
            _bad("bias", bias, (n,), bias.dtype, dev)
        if res.get("dbias") is None:
            res["dbias"] = torch.empty(n, dtype=bias.dtype, device=dev)
        pdb = _whole("dbias", res["dbias"], (n,), bias.dtype, dev)
    else:
        res.pop("dbias", None)
    if act is not None:
        pp = _whole("pre", pre, (*lead, n), bf, dev)
    args = _abi.LINEAR_PACK(m, n, k, _abi.RDN_BF16, 0, bt, _act(act), x_ld, w_ld, 0, 0, px, pw, 0, 0, 0, 0, 0, pp,
                            _code(wt), dy_ld, pdy, pdx, pdw, pdb, 0, 0)
    if act is not None or bias is not None:
        ws, args = _with_workspace("rdn_linear_bwd_workspace_size", args, workspace, dev)
    _call("rdn_linear_bwd", args, dev)
    return res
