"""Outputs given to add_norm_q8 without a block's output to add."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests.test_gpu_norm_q8 import rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [512, 33, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
def test_the_sum_is_written_where_it_is_asked_for(D, dtype, norm):
    x, w = rows(9, D, dtype=dtype, pad=8), 1 + 0.1 * rows(D, dtype="f32") if norm else None
    _, q, s = rdn.add_norm_q8(x, weight=w)
    given = torch.full((9, D), 7.0, device="cuda", dtype=x.dtype)
    r, q1, s1 = rdn.add_norm_q8(x, weight=w, out=(given, None, None))
    assert r is given and torch.equal(r, x)
    assert torch.equal(q.view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s, s1)


def test_the_sum_that_is_x_itself():
    x = rows(9, 64)
    want = x.clone()
    for out in ((None, None, None), (x, None, None)):
        r, _, _ = rdn.add_norm_q8(x, out=out)
        assert r is x and torch.equal(x, want)
    view = x.view(9, 64)
    assert rdn.add_norm_q8(x, out=(view, None, None))[0] is view and torch.equal(x, want)


def test_refusals():
    x = rows(9, 64)
    for r in (rows(9, 63), rows(9, 64, dtype="f32"), rows(9, 64, pad=8), torch.zeros(9, 64, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            rdn.add_norm_q8(x, out=(r, None, None))
