"""States that a call reads may not share memory with those that it writes: other CTAs may
still read them.  Refused by the C entry points (CPU only; nothing reaches a GPU)."""
import pytest

from tests.test_layer_ops_args import FAKE, INVALID, _conv, _refused, _scan

AT = 1 << 32  # (clear of the other fake operands)
N_CONV = 2 * 3 * 128 * 2  # bytes of [2, W-1, C] bf16
N_SCAN = 2 * 128 * 16 * 4  # of [2, D, S] fp32
N_KEPT = 2 * 4 * 128 * 16 * 4  # of [2 * ceil(T/16), D, S]


def apart(fn, make, out, into, size, at, **kw):
    """`out` of `size` bytes from `at` on against `into` at AT: refused if they overlap."""
    a = make(**{into: AT, out: at}, **kw)
    if AT - size < at < AT + (N_SCAN if make is _scan else N_CONV):
        _refused(fn, a, INVALID, f"{out} overlaps {into}")
    else:
        _refused(fn, a, 3, "injected")


@pytest.mark.parametrize("fn,make,out,into,size", [
    ("rdn_conv_fwd", _conv, "stateT", "state0", N_CONV), ("rdn_conv_bwd", _conv, "dstate0", "dstateT", N_CONV),
    ("rdn_conv_bwd", _conv, "dstate0", "state0", N_CONV), ("rdn_scan_fwd", _scan, "hT", "h0", N_SCAN),
    ("rdn_scan_fwd", _scan, "h_chunks", "h0", N_KEPT), ("rdn_scan_bwd", _scan, "dh0", "dhT", N_SCAN)])
def test_states_in_place_are_refused(fn, make, out, into, size):
    n = N_SCAN if make is _scan else N_CONV
    for at in (AT, AT + 16, AT + n - 16, AT + n, AT - 16, AT - size + 16, AT - size):
        apart(fn, make, out, into, size, at)


def test_packed_states_in_place_are_refused():
    """(their number is the table's)"""
    kw = dict(B=1, T=64, cu_seqlens=FAKE, num_seqs=5)
    for at, st in ((AT + 5 * 3 * 128 * 2 - 2, INVALID), (AT + 5 * 3 * 128 * 2, 3)):
        _refused("rdn_conv_fwd", _conv(state0=AT, stateT=at, **kw), st, "overlaps" if st == INVALID else "injected")
    for at, st in ((AT + 5 * 128 * 16 * 4 - 16, INVALID), (AT + 5 * 128 * 16 * 4, 3)):
        _refused("rdn_scan_fwd", _scan(h0=AT, hT=at, **kw), st, "overlaps" if st == INVALID else "injected")


def test_absent_states():
    _refused("rdn_conv_fwd", _conv(stateT=AT), 3, "injected")
    _refused("rdn_scan_fwd", _scan(h0=AT), 3, "injected")
