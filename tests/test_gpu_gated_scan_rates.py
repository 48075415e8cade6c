"""The gated linear recurrence at the ends of its rate c: channels that never decay and ones that decay at once."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref
from tests.test_gpu_gated_scan import DT, T32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,D", [(2, 64), (36, 64), (2, 33)])
@pytest.mark.parametrize("c", [3.4028234663852886e38, 2.5e38, 1e-30])
def test_the_largest_and_smallest_rates(c, B, D, dtype):
    """lam = -200: softplus is 0 in 32 bits, and c softplus(lam) below 1e-48 for the largest c: the state stays.
    lam = 2 with a large c: nothing of the state is left; with a small one everything is."""
    x = make(B, 70, D, dtype)
    x["lam"][:] = 2.0
    x["lam"][::2] = -200.0
    y, hT = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], c, x["h0"])
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], c, x["h0"])
    for t in (y, hT, *d.values()):
        assert torch.isfinite(t).all()
    assert torch.equal(hT[:, ::2], x["h0"][:, ::2])
    if c < 1:
        assert (hT - x["h0"]).abs().max() <= 1e-12  # (inputs come in with sqrt(2 c) of them)
    else:
        want = torch.sigmoid(x["i"].double()) * x["x"].double()
        ref.check("y", y[..., 1::2], want[..., 1::2].cpu(), T32)
    # a step gives the same
    h = x["h0"].clone()
    o = rdn.gated_scan_step(*(x[k][:, 0].contiguous() for k in ("x", "r", "i")), x["lam"], h, c)
    assert torch.isfinite(o).all() and o.dtype == DT[dtype]
    ref.check("step", o, y[:, 0].double().cpu(), T32)
