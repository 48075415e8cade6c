"""The operators together, as examples/selective_block.py uses them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "selective_block.py")
spec = importlib.util.spec_from_file_location("selective_block", PATH)
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)


def test_training_lowers_the_loss():
    losses = ex.train()
    assert losses[-1] < 0.5 * losses[0], losses


def test_decoding_is_the_sequence():
    # bf16 activations: a few roundings of 2^-9 each between the two orders of the same products
    assert ex.serve() < 3e-2


def test_layer_gradient_by_differences():
    """The layer in fp32: the chained backwards against a difference quotient along the gradient."""
    layer = ex.SelectiveLayer(64, 96, 16, rank=8, dtype=torch.float32)
    x = torch.randn(2, 40, 64, device="cuda")
    dr, dh = torch.randn_like(x), torch.randn_like(x)

    def loss():
        r, hn, s = layer.forward(x, ex.norm_in(x, torch.float32))
        return (r.double() * dr).sum().item() + (hn.double() * dh).sum().item(), s

    g = layer.backward(loss()[1], dr, dh)[0]
    for k, p in layer.p.items():
        keep = p.clone()
        v = g[k] / g[k].norm()
        e = 2e-3 * max(1.0, p.norm().item())
        p.copy_(keep + e * v)
        up = loss()[0]
        p.copy_(keep - e * v)
        down = loss()[0]
        p.copy_(keep)
        slope, want = (up - down) / (2 * e), g[k].norm().item()
        assert abs(slope - want) <= 3e-2 * want, (k, slope, want)
