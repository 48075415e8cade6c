"""GELU below zero, where it is small: each value and derivative to its own digits, in both of the product's kernels."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def points(m):
    """bf16 numbers over [-8, 8]"""
    return torch.linspace(-8, 8, m, device="cuda").to(BF)


def cdf(p):
    return 0.5 * torch.erfc(p.double() * -(0.5 ** 0.5))


@pytest.mark.parametrize("M,N,kernel", [(300, 8, "linear_split"), (300, 2600, "linear_tiles")])
@pytest.mark.parametrize("out", [F32, BF])
def test_values(M, N, kernel, out):
    """p = x itself: one weight of 1 and zeros.  The roundings of p^2 / 2 times log2 e, 2^-23 in all, move the
    exponential by p^2 / 2 times that of itself, and a 2-unit exponential, a 1-unit reciprocal, the polynomial's 1.7e-7
    (1.4 units of 2^-23) and some products add less than 8."""
    p = points(M)
    x, w = torch.zeros(M, 8, device="cuda", dtype=BF), torch.zeros(N, 8, device="cuda", dtype=BF)
    x[:, 3], w[:, 3] = p, 1.0
    with rdn.LaunchTimer(4) as lt:
        y = rdn.linear_fwd(x, w, act="gelu", out_dtype=out)
    assert [k for k, _ in lt.records] == [kernel]
    want = (p.double() * cdf(p))[:, None]
    rel = (p.double().pow(2) + p.double().abs() + 8)[:, None] * 2.0 ** -23 + (2.0 ** -8 if out is BF else 0)
    assert ((y.double() - want).abs() <= rel * want.abs()).all()


def test_derivative():
    """dx of a single weight of 1 is dp, in bf16: half a step, and what the two terms of the derivative are off: the
    distribution function's as above, the density's by its exponent of p^2 / 2 and its 2-unit exponential."""
    M = 3000
    p, N = points(M), 16
    x, w = torch.zeros(M, 8, device="cuda", dtype=BF), torch.zeros(N, 8, device="cuda", dtype=BF)
    w[5, 3] = 1.0
    d = rdn.linear_bwd(x, w, torch.ones(M, N, device="cuda", dtype=BF), p[:, None].expand(M, N).contiguous(), "gelu",
                       need_dw=False)["dx"]
    v = p.double()
    dens = v * torch.exp(-0.5 * v * v) / (2 * torch.pi) ** 0.5
    want = cdf(p) + dens
    bound = 2.0 ** -8 * want.abs() + (2 * v * v + 16) * 2.0 ** -23 * (cdf(p) + dens.abs())
    assert ((d[:, 3].double() - want).abs() <= bound).all()
    assert not d[:, [0, 1, 2, 4, 5, 6, 7]].any()


def test_zero_and_far_out():
    x = torch.tensor([0.0, -0.0, 40.0, -40.0, 1e4, -1e4, float("inf"), float("nan")], device="cuda").to(BF)
    eye = torch.eye(8, device="cuda", dtype=BF)
    y = rdn.linear_fwd(x.nan_to_num(0, 3e38).diag(), eye, act="gelu", out_dtype=F32).diag()
    assert not y[[0, 1, 3, 5, 7]].any() and y[2] == 40 and y[4] == x[4].float() and y[6] > 1e38
