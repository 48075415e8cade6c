"""Waits of the gated linear recurrence's kernels that run out: they end their rounds, and what is in flight is
waited for, so that the context stays usable."""
import time

import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests.test_gpu_gated_scan import make
from tests.test_gpu_gated_scan_tiles import WIDE, ran

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("T,d,tiles", [(40000, WIDE, True), (6400, 28032, True), (131072, 256, False)])
def test_a_wait_that_runs_out(T, d, tiles, back, packed, monkeypatch):
    """RDN_FAULT_INJECT=device_wait (device_wait_bwd): the copies of each strip's first CTA are made to seem short, or
    (rows addressed one by one) it sends nothing to its cluster.  The waits on that give up after 5 ms instead of a
    second; the CTAs go on without waiting, end when what they have in flight is there, and the next call is right.
    In clusters of up to six and eight CTAs, and without one (438 strips).  100 rounds and more: waits in each of
    them would take half a second; a CTA has at most five, and there are at most two CTAs one after the other."""
    x = make(1, T, d, "bf16", lens=[1000, 0, T - 1010, 10] if packed else None)
    ins = (x["x"], x["r"], x["i"], x["lam"])
    kw = dict(h0=x["h0"], cu_seqlens=x["cu"])

    def call(hc=None):
        if back:
            return rdn.gated_scan_bwd(*ins, x["dy"], h_chunks=hc, dhT=x["dhT"], **kw)
        return dict(zip("yhc", rdn.gated_scan_fwd(*ins, return_chunk_states=True, **kw)))

    hc = rdn.gated_scan_fwd(*ins, return_chunk_states=True, **kw)[2]
    want = call(hc)
    rdn.device_status()  # whatever an earlier test left
    monkeypatch.setenv("RDN_FAULT_INJECT", "device_wait_bwd" if back else "device_wait")
    began = time.monotonic()
    with ran(tiles, not back, back):
        call(hc)
    assert rdn.device_status() == 4  # RDN_ERR_TIMEOUT
    assert time.monotonic() - began < 0.25
    monkeypatch.delenv("RDN_FAULT_INJECT")
    got = call(hc)
    assert rdn.device_status() == 0
    for k in want:
        assert torch.equal(got[k], want[k]), k
