"""The short causal convolution on the GPU against a plain 64-bit loop."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# 32-bit bounds.  y, dx: at most 6 products and sums (2^-24 each) of terms whose sum of
# magnitudes is a few RMS, and the activation's 2-ulp exponential and divide: below 4e-6.
# dw, dbias: sums of some 200 terms in chains of at most 64 + 8 + 16: below 2e-5.
T32, TSUM = 4e-6, 2e-5


def make(B, T, C, W, dtype, lens=None, state=True, bias=True, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=DT[dtype]: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    n = B if lens is None else len(lens)
    x = r(B, T, C + pad)[..., pad // 2:pad // 2 + C] if pad else r(B, T, C)
    f32 = torch.float32
    return dict(x=x, w=r(C, W, dt=f32) * 0.5, bias=r(C, dt=f32) * 0.1 if bias else None,
                state=r(n, W - 1, C) if state else None, dy=r(B, T, C),
                dlast=r(n, W - 1, C),
                cu=None if lens is None else torch.tensor([0] + [sum(lens[:i + 1]) for i in range(n)],
                                                         dtype=torch.int32, device="cuda"))


def compare(x, silu=True, lens=None, dlast=True, back=True):
    act = "silu" if silu else None
    y, last = rdn.causal_conv_fwd(x["x"], x["w"], x["bias"], x["state"], act, x["cu"], return_state=True)
    v = {k: ref.double(x[k], True) for k in ("x", "w", "bias", "state")}
    yr, lr = ref.conv(v["x"], v["w"], v["bias"], v["state"], silu, lens)
    ref.check("y", y, yr, T32)
    assert torch.equal(last.double().cpu(), lr.detach())
    if not back:
        return
    d = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"] if dlast else None, act,
                            x["cu"])
    outs = [(yr, ref.double(x["dy"]))] + ([(lr, ref.double(x["dlast"]))] if dlast else [])
    g = ref.grads(outs, v)
    ref.check("dx", d["dx"], g["x"], T32)
    ref.check("dweight", d["dweight"], g["w"], TSUM)
    if x["bias"] is not None:
        ref.check("dbias", d["dbias"], g["bias"], TSUM)
    if x["state"] is not None:
        ref.check("dstate", d["dstate"], g["state"], T32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 9, 65, 150])
def test_lengths(T, W, dtype):
    compare(make(2, T, 40, W, dtype, seed=T))


@pytest.mark.parametrize("C", [1, 3, 8, 100, 129, 512])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_channels(C, dtype):
    compare(make(3, 20, C, 4, dtype, seed=C))


@pytest.mark.parametrize("state,bias,silu,dlast", [(False, False, False, False), (False, True, True, True),
                                                   (True, False, True, False), (True, True, False, True)])
def test_options(state, bias, silu, dlast):
    compare(make(2, 33, 64, 4, "bf16", state=state, bias=bias), silu, dlast=dlast)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [2, 6, 64])
def test_strided_rows(pad, dtype):
    compare(make(2, 40, 96, 4, dtype, pad=pad))


@pytest.mark.parametrize("lens", [[5], [0, 1, 2, 3, 0, 40, 64, 0], [1] * 20, [0, 0], [130, 0, 7]])
@pytest.mark.parametrize("W", [2, 4])
def test_packed(lens, W):
    compare(make(1, sum(lens), 72, W, "f32", lens=lens), lens=lens)
    compare(make(1, sum(lens), 72, W, "bf16", lens=lens, state=False), lens=lens)


def test_no_tokens():
    x = make(2, 0, 16, 4, "bf16")
    y, last = rdn.causal_conv_fwd(x["x"], x["w"], x["bias"], x["state"], return_state=True)
    assert y.shape == (2, 0, 16) and torch.equal(last, x["state"])
    d = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"])
    assert torch.equal(d["dstate"], x["dlast"])
    assert not d["dweight"].any() and not d["dbias"].any()


def test_sequences_do_not_touch():
    """NaN and infinities in one packed sequence, its state and its gradient stay there."""
    lens = [20, 3, 41]
    x = make(1, 64, 48, 4, "bf16", lens=lens)
    clean = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"], cu_seqlens=x["cu"])
    yc = rdn.causal_conv_fwd(x["x"], x["w"], x["bias"], x["state"], cu_seqlens=x["cu"])
    x["x"][0, 20:23] = float("nan")
    x["state"][1] = float("inf")
    x["dy"][0, 20:23] = float("nan")
    y = rdn.causal_conv_fwd(x["x"], x["w"], x["bias"], x["state"], cu_seqlens=x["cu"])
    d = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"], cu_seqlens=x["cu"])
    for a, b in ((y, yc), (d["dx"], clean["dx"])):
        assert torch.equal(a[0, :20], b[0, :20]) and torch.equal(a[0, 23:], b[0, 23:])
        assert torch.isnan(a[0, 20:23]).all()
    assert torch.equal(d["dstate"][[0, 2]], clean["dstate"][[0, 2]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,W", [(64, 4), (100, 3), (7, 2)])
def test_steps_are_the_sequence(C, W, dtype):
    """Tokens one by one, in shuffled slots with an idle row, equal the sequence call."""
    x = make(3, 6, C, W, dtype, seed=5)
    y, last = rdn.causal_conv_fwd(x["x"], x["w"], x["bias"], x["state"], return_state=True)
    slots = torch.tensor([4, -1, 0, 2], dtype=torch.int32, device="cuda")
    state = torch.randn(5, W - 1, C, device="cuda").to(DT[dtype])
    rows = [0, 2, 3]
    state[slots[rows].long()] = x["state"]
    kept = state.clone()
    for t in range(6):
        xt = torch.full((4, C), float("nan"), device="cuda").to(DT[dtype])
        xt[rows] = x["x"][:, t]
        o = rdn.causal_conv_step(xt, x["w"], state, x["bias"], slots=slots)
        assert not o[1].any()
        ref.check("step", o[rows], y[:, t].double().cpu(), T32)
    assert torch.equal(state[slots[rows].long()], last)
    assert torch.equal(state[[1, 3]], kept[[1, 3]])


def test_step_without_slots_and_far_slots():
    x = make(2, 1, 64, 4, "bf16")
    a, b = x["state"].clone(), x["state"].clone()
    y = rdn.causal_conv_step(x["x"][:, 0], x["w"], a, x["bias"])
    far = torch.tensor([0, 2], dtype=torch.int32, device="cuda")  # 2: no such slot
    y2 = rdn.causal_conv_step(x["x"][:, 0], x["w"], b, x["bias"], slots=far)
    assert torch.equal(y[0], y2[0]) and not y2[1].any()
    assert torch.equal(a[0], b[0]) and torch.equal(b[1], x["state"][1])


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e through the fp32 forward.  e = 2^-6: the
    curvature's e^2 term and the outputs' rounding (2^-24 / e) are both below 1e-3 of the slope."""
    x = make(2, 30, 24, 4, "f32", seed=3)
    names = ("x", "w", "bias", "state")
    d = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"])
    got = dict(x=d["dx"], w=d["dweight"], bias=d["dbias"], state=d["dstate"])

    def loss(p):
        return (rdn.causal_conv_fwd(p["x"], p["w"], p["bias"], p["state"]).double() * x["dy"].double()).sum().item()

    for n in names:
        v = torch.sign(got[n])
        e = 2.0 ** -6
        up, down = ({**x, n: x[n] + s * e * v} for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * e)
        want = (got[n].double() * v.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * abs(want), (n, slope, want)


def test_same_bits_and_other_stream():
    x = make(2, 200, 256, 4, "bf16")
    a = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = rdn.causal_conv_bwd(x["x"], x["w"], x["dy"], x["bias"], x["state"], x["dlast"])
    torch.cuda.current_stream().wait_stream(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k
