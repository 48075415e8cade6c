"""Gated recurrence, 8-bit norm and matrix products past 2^31 elements: the last rows are those of a call of
their own."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn

pytestmark = pytest.mark.gpu

T, D = (1 << 20) + 200, 2056  # 2.16e9 elements


def big(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, D, generator=g, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("off", [0, 1])
def test_gated_scan(off):
    """off = 1: rows that do not start on 16 bytes."""
    x, r, i, dy = (big(k)[None][..., off:] for k in range(4))
    d = D - off
    lam = torch.full((d,), -4.0, device="cuda")
    y, hT, hc = rdn.gated_scan_fwd(x, r, i, lam, return_chunk_states=True)
    at = T - T % 64 - 640  # the tail, from a kept state
    tail = [t[:, at:] for t in (x, r, i, dy)]
    # (the same tiles, in clusters of another number of CTAs: other roundings of 2^-24, 2^-8 where bf16 falls the
    # other way)
    y1, h1 = rdn.gated_scan_fwd(*tail[:3], lam, h0=hc[0, at // 64][None].contiguous())
    assert ((y[:, at:] - y1).float().abs() <= 2.0 ** -7 * y1.float().abs() + 1e-5).all()
    assert (hT - h1).abs().max() <= 1e-5
    g = rdn.gated_scan_bwd(x, r, i, lam, dy, h_chunks=hc)
    g1 = rdn.gated_scan_bwd(*tail[:3], lam, tail[3], h0=hc[0, at // 64][None].contiguous())
    for k in ("dx", "dr", "di"):
        a, b = g[k][:, at:].float(), g1[k].float()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 1e-4 * b.pow(2).mean().sqrt()).all(), k


def test_norm_q8():
    x, f = big(0), big(1)
    w = torch.ones(D, device="cuda")
    r, q, s = rdn.add_norm_q8(x, f, w)
    r1, q1, s1 = rdn.add_norm_q8(x[-70:], f[-70:], w)
    assert torch.equal(r[-70:], r1)
    # (few rows are shared out over more lanes: sums in another order, codes a step apart at most)
    assert ((s[-70:] - s1).abs() <= 2.0 ** -20 * s1).all()
    a, b = q[-70:].float(), q1.float()
    assert ((a - b).abs() <= 0.126 * b.abs() + 2.0 ** -9).all() and (a != b).float().mean() < 1e-3


def test_linear():
    """y, dx and dw of more than 2^31 elements of x, y and dy."""
    x, dy = big(0), big(1)
    w = torch.randn(D, D, device="cuda").to(torch.bfloat16)
    y, pre = rdn.linear_fwd(x, w, act="silu", residual=dy, return_pre=True)
    n = 4096  # (tiles of the same kernel: the same bits)
    y1, p1 = rdn.linear_fwd(x[-n:], w, act="silu", residual=dy[-n:], return_pre=True)
    assert torch.equal(y[-n:], y1) and torch.equal(pre[-n:], p1)
    d = rdn.linear_bwd(x, w, dy, pre, "silu")
    d1 = rdn.linear_bwd(x[-n:], w, dy[-n:], pre[-n:], "silu")
    assert torch.equal(d["dx"][-n:], d1["dx"])
    # dw of all rows: halves add up.  The tensor core cuts its sum to 24 bits at every 16 products: 65549 steps of
    # less than 2^-23 of the sum so far, half as many in each half; rounded to bf16
    h = T // 2 // 8 * 8
    parts = [rdn.linear_bwd(x[a:b], w, dy[a:b], pre[a:b], "silu", need_dx=False, dw_dtype=torch.float32)["dw"]
             for a, b in ((0, h), (h, T))]
    want = parts[0] + parts[1]
    cut = 1.5 * 65549 * 2.0 ** -23
    size = want.abs() + want.pow(2).mean().sqrt()
    assert ((d["dw"].float() - want).abs() <= 2.0 ** -8 * want.abs() + cut * size).all()


def test_long_sums():
    """The error of a product's sums, against 64 bits: toward zero and below what its steps cut off."""
    for rows in (4096, 65536):
        g = torch.Generator(device="cuda").manual_seed(rows)
        x, dy = (torch.randn(rows, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        got = rdn.linear_bwd(x, x[:128], dy, need_dx=False, dw_dtype=torch.float32)["dw"].double()
        want = dy.double().T @ x.double()
        size = want.abs() + want.pow(2).mean().sqrt()
        assert ((got - want).abs() <= rows / 16 * 2.0 ** -23 * size).all()
