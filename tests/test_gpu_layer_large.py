"""The operators around the recurrence on tensors of more than 2^31 elements: what lies past a
32-bit offset equals a call on that part alone."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rand(*shape, dtype=BF16):
    return torch.randn(*shape, device="cuda", dtype=dtype)


def test_conv():
    C, T, tail = 4096, 530000, 300
    x, w, b = rand(1, T, C), rand(C, 4, dtype=F32), rand(C, dtype=F32)
    assert x.numel() > 2 ** 31
    y, last = rdn.causal_conv_fwd(x, w, b, return_state=True)
    part, plast = rdn.causal_conv_fwd(x[:, -tail:], w, b, state=x[:, -tail - 3:-tail].contiguous(),
                                      return_state=True)
    assert torch.equal(y[:, -tail:], part) and torch.equal(last, plast)
    dx = rdn.causal_conv_bwd(x, w, y, b)["dx"]
    dpart = rdn.causal_conv_bwd(x[:, -tail:], w, part, b, state=x[:, -tail - 3:-tail].contiguous())["dx"]
    assert torch.equal(dx[:, -tail:], dpart)


def test_scan():
    D, S, T, tail = 4096, 16, 524800, 320
    x, dt, B, C = rand(1, T, D), rand(1, T, D), rand(1, T, 1, S), rand(1, T, 1, S)
    A = -torch.exp(rand(D, S, dtype=F32))
    assert x.numel() > 2 ** 31
    out, hT, hc = rdn.selective_scan_fwd(x, dt, A, B, C, return_chunk_states=True)
    assert hc.numel() > 2 ** 31
    cut = lambda t: t[:, -tail:]  # noqa: E731
    h0 = hc[(T - tail) // 16][None].clone()
    part, phT = rdn.selective_scan_fwd(cut(x), cut(dt), A, cut(B), cut(C), h0=h0)
    # (cut into other units, the states may differ by rounding: 2^-24 a step over the tail)
    assert (phT - hT).norm() <= 2e-5 * hT.norm()
    assert (cut(out).float() - part.float()).abs().max() <= 2.0 ** -7 * part.float().abs().max()


def test_steps():
    D, S, slots = 4096, 16, 33000
    h = torch.zeros(slots, D, S, device="cuda")
    assert h.numel() > 2 ** 31
    x, dt, B = rand(2, D), rand(2, D), rand(2, 1, S)
    A = -torch.exp(rand(D, S, dtype=F32))
    h[-1] = 1.5
    at = torch.tensor([slots - 1, 3], dtype=torch.int32, device="cuda")
    small = torch.zeros(2, D, S, device="cuda")
    small[0] = 1.5
    o = rdn.selective_scan_step(x, dt, A, B, B, h, slots=at)
    o2 = rdn.selective_scan_step(x, dt, A, B, B, small)
    assert torch.equal(o, o2) and torch.equal(h[-1], small[0]) and torch.equal(h[3], small[1])
    assert not h[-2].any() and not h[4].any()
    del h
    C, slots = 8192, 90000
    state = torch.zeros(slots, 3, C, device="cuda", dtype=BF16)
    assert state.numel() > 2 ** 31
    xc, w = rand(1, C), rand(C, 4, dtype=F32)
    state[-1] = 0.5
    y = rdn.causal_conv_step(xc, w, state, slots=torch.tensor([slots - 1], dtype=torch.int32, device="cuda"))
    small = torch.full((1, 3, C), 0.5, device="cuda", dtype=BF16)
    assert torch.equal(y, rdn.causal_conv_step(xc, w, small)) and torch.equal(state[-1], small[0])


def test_norm():
    D, rows, tail = 2048, 1100000, 700
    f, x, w = rand(rows, D), rand(rows, D), rand(D, dtype=F32)
    assert f.numel() > 2 ** 31
    r, h = rdn.block_norm_fwd(f, w, x=x, weight_next=w)
    pr, ph = rdn.block_norm_fwd(f[-tail:], w, x=x[-tail:], weight_next=w)
    assert torch.equal(r[-tail:], pr) and torch.equal(h[-tail:], ph)
    d = rdn.block_norm_bwd(f, w, x=x, weight_next=w, dr=r, dh=h)
    p = rdn.block_norm_bwd(f[-tail:], w, x=x[-tail:], weight_next=w, dr=pr, dh=ph)
    assert torch.equal(d["df"][-tail:], p["df"]) and torch.equal(d["dx"][-tail:], p["dx"])
