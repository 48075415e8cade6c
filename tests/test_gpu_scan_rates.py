"""States without memory: a rate A of -inf (A_log past the type's range), or one whose product
with log2 e is, leaves of a state what its token adds; also in the tokens past the end of a
sequence's last group, whose steps are zero."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref
from tests.test_gpu_scan import INS, T32, call, make

pytestmark = pytest.mark.gpu


def rates(x, value):
    A = x["A"].clone()
    A[::3, ::2] = value
    A[1] = value
    return A


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 4, 5, 16, 21, 70, 130, 200])
@pytest.mark.parametrize("value", [float("-inf"), -3e38])
def test_states_without_memory(value, T, dtype):
    """Against the 64-bit loop with rates of -1e30, whose decays are zero as well (and whose
    derivatives, rate times decay, are zero instead of undefined)."""
    x = make(2, T, 40, 16, dtype=dtype, seed=T)
    v = {k: ref.double(x[k] if k != "A" else rates(x, -1e30), True) for k in INS}
    o, hTr, kept = ref.scan(*(v[k] for k in INS), True, None)
    g = ref.grads([(o, ref.double(x["dout"])), (hTr, ref.double(x["dhT"]))], v)
    x["A"] = rates(x, value)
    out, hT, hc = call(rdn.selective_scan_fwd, x, return_chunk_states=True)
    ref.check("out", out, o, T32)
    ref.check("hT", hT, hTr, T32)
    ref.check("h_chunks", hc[:kept.shape[0]], kept, T32)
    for chunks in (hc, None):
        d = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"], h_chunks=chunks)
        for name, k in (("dx", "x"), ("ddt", "dt"), ("dz", "z"), ("dB", "B"), ("dC", "C"), ("dA", "A"),
                        ("dD", "D"), ("ddt_bias", "dt_bias"), ("dh0", "h0")):
            ref.check(name, d[name], g[k], T32)


def test_packed_and_steps():
    lens = [5, 0, 33, 1, 18]
    x = make(1, sum(lens), 40, 16, dtype="f32", lens=lens)
    v = {k: ref.double(x[k] if k != "A" else rates(x, -1e30)) for k in INS}
    o, hTr, _ = ref.scan(*(v[k] for k in INS), True, lens)
    x["A"] = rates(x, float("-inf"))
    out, hT = call(rdn.selective_scan_fwd, x)
    ref.check("out", out, o, T32)
    ref.check("hT", hT, hTr, T32)
    h = x["h0"][:1].clone()
    for t in range(lens[0]):
        y = rdn.selective_scan_step(x["x"][:, t], x["dt"][:, t], x["A"], x["B"][:, t], x["C"][:, t], h, x["D"],
                                    x["z"][:, t], x["dt_bias"])
        ref.check("step", y, o[:, t], T32)
    ref.check("h", h, hTr[:1], T32)


def test_undefined_rates_stay_undefined():
    x = make(1, 21, 40, 16, dtype="f32")
    x["A"][3, 2] = float("nan")
    out, hT = call(rdn.selective_scan_fwd, x)
    assert torch.isnan(out[..., 3]).all() and torch.isnan(hT[0, 3, 2])
    assert torch.isfinite(out[..., [0, 1, 2, 4, 39]]).all()
