"""The operators between the recurrences together, as examples/gated_block.py uses them."""
import importlib.util
import math
import os

import pytest
import torch

from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
spec = importlib.util.spec_from_file_location("gated_block", PATH)
ex = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ex)


def test_training_runs():
    losses = ex.train(3)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)


@pytest.mark.parametrize("q8", [False, True])
def test_decoding_is_the_sequence(q8):
    """A token's rows come from other kernels than the sequence's.  In bf16 the two differ by roundings of
    2^-9 of some intermediate rows, each of which moves the output by at most that of its own magnitude (a few
    times the RMS).  In 8 bits a value may fall on the code next to it, 2^-3 of itself; one of an inner row's
    512 moves the output by 2^-3 * 4 / sqrt(512), and few do."""
    assert ex.serve(q8) < (0.1 if q8 else 3e-2)


def formulas(layer, x, v):
    """The layer in 64 bits."""
    def rms(t):
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)

    n, T = layer.inner, x.shape[1]
    u = rms(x) * v["norm"] @ v["w_in"].T + v["b_in"]
    c = ref.conv(u[..., :n], v["conv_w"], v["conv_b"], None, True)[0]
    la = -8.0 * torch.nn.functional.softplus(v["lam"]) * torch.sigmoid(u[..., n:2 * n])
    a, b = torch.exp(la), torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(u[..., 2 * n:]) * c
    h, y = torch.zeros_like(a[:, 0]), []
    for t in range(T):
        h = a[:, t] * h + b[:, t]
        y.append(h)
    return x + torch.stack(y, 1) @ v["w_out"].T


def test_layer_against_the_formulas():
    """Forward and gradients against differentiation of the layer in 64 bits.  Between the operators h, u, c,
    y and their gradients are held in bf16, each rounding 2^-9 / sqrt(3) of its value on average: some ten of
    them in a chain, unrelated, give 0.7 % of the RMS, and 6 times that is not passed in some 10^5 values."""
    layer = ex.GatedLayer(64, 96)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 70, 64, generator=gen, device="cuda").to(torch.bfloat16)
    dout = torch.randn(2, 70, 64, generator=gen, device="cuda").to(torch.bfloat16)
    out, s = layer.forward(x)
    g, dx = layer.backward(s, dout)
    v = {k: ref.double(t, True) for k, t in dict(layer.p, x=x).items()}
    want = formulas(layer, v["x"], v)
    ref.check("out", out, want, 4e-2)
    d = ref.grads([(want, ref.double(dout))], v)
    ref.check("dx", dx, d["x"], 4e-2)
    for k in layer.p:
        ref.check(k, g[k], d[k], 4e-2)


def test_block_in_graphs():
    """Two captured passes that live at the same time, replayed in turn on new inputs, and an eager one between."""
    layer = ex.GatedLayer(128, 128)
    xs = [torch.randn(2, 150, 128, device="cuda").to(torch.bfloat16) for _ in range(2)]

    def once(x):
        out, s = layer.forward(x)
        g, dx = layer.backward(s, x)
        return [out, dx, *g.values()]

    graphs, held = [], []
    for x in xs:
        once(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(once(x))
        graphs.append(g)
    for x in xs:
        x.copy_(torch.randn_like(x))
    want = [once(x) for x in xs]
    for g in graphs + graphs[::-1]:
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(held, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
