"""weight [heads, D] of the block norms belongs to rows [..., heads, D], or to rows flattened from
them: a head axis of another size is refused (CPU only; calls that end before the library)."""
import pytest

import paper_2509_25223_gb300 as rdn
from tests.test_layer_ops_rows import calls, t  # noqa: F401

D = 8


@pytest.mark.parametrize("fn", [rdn.block_norm_fwd, rdn.block_norm_bwd])
@pytest.mark.parametrize("shape,heads", [((2, 8, D), 4), ((2, 8, D), 2), ((4, 3, D), 6), ((2, 4, 3, D), 4),
                                         ((2, 4, 1, D), 4), ((5, 3, D), 15)])
def test_other_head_axes_are_refused(calls, fn, shape, heads):  # noqa: F811
    with pytest.raises(ValueError, match="heads"):
        fn(t(*shape), t(heads, D), **dict(dr=t(*shape)) if fn is rdn.block_norm_bwd else {})
    assert not calls


@pytest.mark.parametrize("fn", [rdn.block_norm_fwd, rdn.block_norm_bwd])
@pytest.mark.parametrize("shape,heads", [((2, 8, D), 8), ((2, 4, 3, D), 3), ((8, D), 4), ((8, D), 8), ((2, 8, D), 1),
                                         ((8, D), 1), ((2, 5, 1, D), 1)])
def test_head_axes_and_flattened_rows(calls, fn, shape, heads):  # noqa: F811
    fn(t(*shape), t(heads, D), **dict(dr=t(*shape)) if fn is rdn.block_norm_bwd else {})
    a, = calls
    assert a.heads == heads and a.D == D and a.rows * D == t(*shape).numel()
