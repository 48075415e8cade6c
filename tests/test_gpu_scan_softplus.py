"""The step sizes alone: one token from a zero state with x = B = C = 1 returns
dl = softplus(dt), and its gradient the sigmoid.

Bound, relative.  The exponent |v| log2 e is a 32-bit product with a 32-bit constant: off by at most
|v| (2^-24 + 1.34e-8) in e^-|v|, 7.3e-8 |v|; the rest -- an exponential of 2^-22, a reciprocal of
one unit (2^-23), five roundings (2^-24 each) and the polynomial (8e-9) -- stays below 7e-7.
Above 0 the exponential is a small part of the result."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn

pytestmark = pytest.mark.gpu


def bound(v):
    return 7.3e-8 * (-v).clamp(min=0) + 7e-7


@pytest.mark.parametrize("D", [1 << 16, (1 << 16) - 1])  # (16-byte rows, single elements)
@pytest.mark.parametrize("lo,hi", [(-80, 20), (-10, -1), (-1, 1)])
def test_step_sizes(D, lo, hi):
    g = torch.Generator(device="cuda").manual_seed(D)
    dt = torch.rand(1, 1, D, generator=g, device="cuda") * (hi - lo) + lo
    x, A, B = torch.ones_like(dt), -torch.ones(D, 1, device="cuda"), torch.ones(1, 1, 1, 1, device="cuda")
    v = dt.double()
    want, slope = v.clamp(min=0) + torch.log1p(torch.exp(-v.abs())), torch.sigmoid(v)
    out = rdn.selective_scan_fwd(x, dt, A, B, B, return_final_state=False)
    step = rdn.selective_scan_step(x[0], dt[0], A, B[0], B[0], torch.zeros(1, D, 1, device="cuda"))
    ddt = rdn.selective_scan_bwd(x, dt, A, B, B, torch.ones_like(dt))["ddt"]
    for name, got, ref in (("fwd", out, want), ("step", step[None], want), ("ddt", ddt, slope)):
        err = ((got.double() - ref).abs() / ref / bound(v)).max().item()
        assert err <= 1, (name, err)
