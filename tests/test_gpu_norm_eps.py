"""The norms without eps: slots of rows past the last one, which are worked on as zeros, leave
the sums over the rows alone (bounds: those of the other norm tests)."""
import pytest

from tests import test_gpu_norm as tn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def no_eps(monkeypatch):
    monkeypatch.setattr(tn, "EPS", 0.0)


@pytest.mark.parametrize("rows", [1, 7, 33, 301])
@pytest.mark.parametrize("D,dtype", [(63, "bf16"), (64, "bf16"), (64, "f32"), (128, "bf16"), (300, "f32"),
                                     (1000, "bf16"), (2055, "f32")])
def test_rows_that_fill_no_cta(D, dtype, rows):
    tn.compare(tn.make(rows, D, dtype, seed=rows))
    tn.compare(tn.make(rows, D, dtype, x=False, nxt=False, seed=rows), "sigmoid")


@pytest.mark.parametrize("D", [64, 512, 1000])
def test_norm_before_a_block(D):
    tn.compare(tn.make(37, D, "bf16", "f32", f=False))
    tn.compare(tn.make(37, D, "f32", z=False, x=False, nxt=True))


@pytest.mark.parametrize("heads", [2, 5, 16])
def test_heads(heads):
    tn.compare(tn.make((11, heads), 64, heads=heads, x=False, nxt=False))
    tn.compare(tn.make((11, heads), 128, heads=heads, z=False, x=False, nxt=False))


@pytest.mark.parametrize("rows,D", [(5, 8200), (5, 16384), (77, 6000)])
def test_long_rows(rows, D):
    tn.compare(tn.make(rows, D))
