"""Waits of the matrix product's kernels that run out: the kernels drain and return, and the context stays usable."""
import time

import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests.test_gpu_linear import forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N,K,kernel", [(3, 2048, 4096, "linear_split"), (512, 2048, 2048, "linear_split"),
                                          (2100, 2048, 256, "linear_tiles"), (8200, 4104, 512, "linear_tiles")])
def test_a_wait_that_runs_out(M, N, K, kernel, kind, monkeypatch):
    """RDN_FAULT_INJECT=device_wait: the first tile's sums are not signalled, so that the waits on them give up after
    5 ms instead of a second; a CTA has at most ten waits one after the other."""
    x = make(M, N, K, kind)
    want = forward(x, "silu")
    rdn.device_status()  # whatever an earlier test left
    monkeypatch.setenv("RDN_FAULT_INJECT", "device_wait")
    began = time.monotonic()
    with rdn.LaunchTimer(4) as lt:
        forward(x, "silu")
    assert [k for k, _ in lt.records] == [kernel]
    assert rdn.device_status() == 4  # RDN_ERR_TIMEOUT
    assert time.monotonic() - began < 0.25
    monkeypatch.delenv("RDN_FAULT_INJECT")
    got = forward(x, "silu")
    assert rdn.device_status() == 0 and torch.equal(got, want)


@pytest.mark.parametrize("M,N,K", [(130, 264, 96), (4100, 2056, 2048)])
def test_a_wait_of_the_backward_that_runs_out(M, N, K, monkeypatch):
    x = make(M, N, K, residual=None)
    pre = forward(x, "silu", return_pre=True)[1]

    def call():
        return rdn.linear_bwd(x["x"], x["w"], x["dy"], pre, "silu", x["bias"])

    want = call()
    rdn.device_status()
    monkeypatch.setenv("RDN_FAULT_INJECT", "device_wait_bwd")
    began = time.monotonic()
    call()
    assert rdn.device_status() == 4
    assert time.monotonic() - began < 0.5  # (two products)
    monkeypatch.delenv("RDN_FAULT_INJECT")
    got = call()
    assert rdn.device_status() == 0
    for k in want:
        assert torch.equal(got[k], want[k]), k
