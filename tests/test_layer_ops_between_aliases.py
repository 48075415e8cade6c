"""Results of the operators between the recurrences that would lie on what other CTAs of the call still read
or write are refused by the C entry points (CPU only; nothing reaches a GPU)."""
import random

import pytest

from paper_2509_25223_gb300 import _abi
from tests.test_layer_ops_args import FAKE, INVALID, _refused
from tests.test_layer_ops_between_args import AT, LAUNCH, _gscan, _linear, _q8

FAR = 1 << 40  # (clear of AT)


def _bwd(**kw):
    """M = N = K = 64: every operand could take another's place."""
    base = dict(M=64, N=64, K=64, act=1, bias_dtype=_abi.RDN_BF16, x=AT, w=AT + 0x10000, dy=AT + 0x20000,
                pre=AT + 0x30000, dx=AT + 0x40000, dw=AT + 0x50000, dbias=AT + 0x60000)
    return _linear(**{**base, **kw})


SIZE = 64 * 64 * 2


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("out,other", [("dx", "w"), ("dx", "x"), ("dx", "dy"), ("dw", "x"), ("dw", "dy"), ("dw", "w"),
                                       ("dx", "dw"), ("dbias", "dw"), ("dbias", "dx"), ("dbias", "x"), ("dbias", "w"),
                                       ("dbias", "dy")])
def test_gradients_over_operands(out, other, act):
    at = getattr(_bwd(), other)
    size = 128 if out == "dbias" else SIZE
    for place, refused in ((at, True), (at + 16, True), (at + SIZE - 16, True), (at + SIZE, False), (at - size, False),
                           (at - size + 16, True)):
        _refused("rdn_linear_bwd", _bwd(act=act, **{out: place}), INVALID if refused else LAUNCH,
                 "aliases" if refused else "injected")


def test_gradients_over_what_the_activation_reads():
    for out in ("dx", "dw", "dbias"):
        _refused("rdn_linear_bwd", _bwd(**{out: AT + 0x30000}), INVALID, f"{out} aliases pre")
        _refused("rdn_linear_bwd", _bwd(act=0, **{out: AT + 0x30000}), LAUNCH, "injected")


def test_gradients_that_are_not_asked_for():
    _refused("rdn_linear_bwd", _bwd(dx=0), LAUNCH, "injected")
    _refused("rdn_linear_bwd", _bwd(dw=0, dbias=0), LAUNCH, "injected")
    # without rows x and dy have no bytes; w has
    _refused("rdn_linear_bwd", _bwd(M=0, dw=AT), LAUNCH, "injected")
    _refused("rdn_linear_bwd", _bwd(M=0, dw=AT + 0x10000), INVALID, "dw aliases w")


@pytest.mark.parametrize("name,size", [("x", 6 * 64), ("w", 64 * 64), ("bias", 128), ("res", 6 * 128)])
def test_forward_results_over_operands(name, size):
    base = dict(bias_dtype=_abi.RDN_BF16, x=AT, w=AT + 0x10000, bias=AT + 0x20000, res=AT + 0x30000, y=FAR,
                pre=FAR + 0x10000)
    at = base[name]
    for out in ("y", "pre"):
        for place in (at + 16, at + size - 16, at - 6 * 128 + 16):
            says = "same rows" if (out, name) == ("y", "res") else f"{out} aliases {name}"
            _refused("rdn_linear_fwd", _linear(**{**base, out: place}), INVALID, says)
        for place in (at + size, at - 6 * 128):
            _refused("rdn_linear_fwd", _linear(**{**base, out: place}), LAUNCH, "injected")
    _refused("rdn_linear_fwd", _linear(**{**base, "pre": FAR + 16}), INVALID, "pre aliases y")
    _refused("rdn_linear_fwd", _linear(**{**base, "y": base["res"]}), LAUNCH, "injected")


def test_forward_results_over_scales():
    base = dict(dtype=_abi.RDN_E4M3, x=AT, w=AT + 0x10000, x_scale=AT + 0x20000, w_scale=AT + 0x30000, y=FAR)
    _refused("rdn_linear_fwd", _linear(**base), LAUNCH, "injected")
    for name, size in (("x_scale", 24), ("w_scale", 256)):
        _refused("rdn_linear_fwd", _linear(**{**base, "y": base[name] + size - 4}), INVALID, f"y aliases {name}")
        _refused("rdn_linear_fwd", _linear(**{**base, "y": base[name] + size}), LAUNCH, "injected")


def test_strided_rows_against_their_bytes():
    """Slices of one wider tensor's columns are taken; every placement against the bytes themselves."""
    rng, seen = random.Random(5), set()
    for _ in range(3000):
        M, N, K = rng.randint(1, 4), 8 * rng.randint(1, 3), 8 * rng.randint(1, 3)
        x_ld = rng.choice([K, 64])
        y_ld = rng.choice([N, 64])
        d = 2 * rng.randint(-4 * 64, 4 * 64)
        bytes_of = lambda p, ld, n: {p + 2 * (r * ld) + b for r in range(M) for b in range(2 * n)}  # noqa: E731
        shared = bool(bytes_of(AT, x_ld, K) & bytes_of(AT + d, y_ld, N))
        seen.add((shared, x_ld == 64, y_ld == 64))
        _refused("rdn_linear_fwd", _linear(M=M, N=N, K=K, x=AT, x_ld=x_ld, w=FAR, y=AT + d, y_ld=y_ld),
                 INVALID if shared else LAUNCH, "y aliases x" if shared else "injected")
    assert len(seen) == 8


def test_far_apart_rows_of_many():
    """Distances whose products pass 63 bits."""
    _refused("rdn_linear_fwd", _linear(M=1 << 30, N=8, K=8, x=AT, x_ld=(1 << 38) - 8, w=FAR, y=AT - 4096, y_ld=1 << 40),
             INVALID, "y aliases x")
    _refused("rdn_linear_fwd", _linear(M=1 << 30, N=8, K=8, x=AT, x_ld=1 << 30, w=AT + 128, y=AT + 256, y_ld=1 << 30),
             LAUNCH, "injected")


@pytest.mark.parametrize("a,b", [("dr", "dx"), ("di", "dx"), ("di", "dr")])
def test_gradients_of_the_recurrence_over_one_another(a, b):
    for cu in (dict(), dict(B=1, cu_seqlens=FAKE, num_seqs=3)):
        _refused("rdn_gscan_bwd", _gscan(**{a: AT, b: AT}, **cu), INVALID, f"{a} aliases {b}")
    _refused("rdn_gscan_bwd", _gscan(**{a: AT, b: AT}, T=0), LAUNCH, "injected")
    # slices of one tensor's columns
    _refused("rdn_gscan_bwd", _gscan(**{a: AT, b: AT + 256, a + "_ld": 384, b + "_ld": 384}), LAUNCH, "injected")


@pytest.mark.parametrize("name,size", [("x", 768), ("f", 768), ("w", 256)])
def test_results_of_the_norm_over_operands(name, size):
    base = dict(x=AT, f=AT + 0x10000, w=AT + 0x20000, r_out=FAR, q=FAR + 0x10000)
    at = base[name]
    for out, own in (("r_out", 768), ("q", 384)):
        if (out, name) == ("r_out", "w"):
            continue
        for place, refused in ((at + 16, 1), (at + size - 16, 1), (at - own + 16, 1), (at + size, 0), (at - own, 0)):
            _refused("rdn_norm_q8", _q8(**{**base, out: place}), INVALID if refused else LAUNCH,
                     "injected" if not refused else f"q aliases {name}" if out == "q" else "r_out may be")
    for place in (FAR, FAR + 16, FAR + 752, FAR - 368):
        _refused("rdn_norm_q8", _q8(**{**base, "q": place}), INVALID, "q aliases r_out")
    _refused("rdn_norm_q8", _q8(**{**base, "r_out": base["x"]}), LAUNCH, "injected")
    # r_out in the columns beside x's
    _refused("rdn_norm_q8", _q8(**{**base, "rows": 1, "r_out": AT + 128}), LAUNCH, "injected")
