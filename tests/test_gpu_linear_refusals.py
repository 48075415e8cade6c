"""Refusals of the matrix product's backward by the binding."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn

pytestmark = pytest.mark.gpu


def test_a_bias_that_is_not_the_forwards():
    """Its values are not read, but its gradient is of its shape."""
    bf = torch.bfloat16
    x, w, dy = (torch.ones(s, device="cuda", dtype=bf) for s in ((4, 16), (8, 16), (4, 8)))
    for bias in (torch.zeros(16, device="cuda", dtype=bf), torch.zeros(1, 8, device="cuda", dtype=bf),
                 torch.zeros(8, dtype=bf)):
        with pytest.raises(ValueError, match="bias"):
            rdn.linear_bwd(x, w, dy, bias=bias)
    with pytest.raises(ValueError, match="dtype"):
        rdn.linear_bwd(x, w, dy, bias=torch.zeros(8, device="cuda", dtype=torch.float16))
    d = rdn.linear_bwd(x, w, dy, bias=torch.zeros(8, device="cuda", dtype=bf))
    assert (d["dbias"] == 4).all()


def test_gradients_over_operands():
    """out= with an operand in a gradient's place."""
    bf = torch.bfloat16
    x, w, dy = (torch.ones(64, 64, device="cuda", dtype=bf) for _ in range(3))
    other = torch.empty_like(x)
    for out in (dict(dx=w), dict(dw=x), dict(dw=dy), dict(dx=dy), dict(dw=w), dict(dx=other, dw=other)):
        with pytest.raises(rdn.RdnError, match="aliases"):
            rdn.linear_bwd(x, w, dy, out=out)
    for t in (x, w, dy):
        assert (t == 1).all()
