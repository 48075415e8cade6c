"""The gated linear recurrence on the GPU against a plain 64-bit loop."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# 32-bit bounds, for rows of at most 400 tokens.  The sigmoids are within 1e-6 (the exponent's
# rounding at |r| < 6, a 2-ulp exponential, a 1-ulp reciprocal), the log decay and 1 - a within
# 1.6e-6, and the state follows 1 - a; rounding a itself adds at most 2^-25 of the state a
# token, 1.2e-5 over 400.  Gradients carry the states' and the reverse scan's errors: twice that.
# dlam: sums of some hundred terms, whose errors are each below that and unrelated.
T32, TGRAD, TSUM = 2e-5, 4e-5, 1e-4


def cu_of(lens):
    return torch.tensor([0] + [sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32, device="cuda")


def make(B, T, D, dtype, lens=None, state=True, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=DT[dtype]: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    n = B if lens is None else len(lens)
    f32 = torch.float32
    gates = r(B, T, 2 * D + pad)
    a = 0.9 + 0.099 * torch.rand(D, generator=g, device="cuda")
    return dict(x=r(B, T, D), r=gates[..., :D] if pad else gates[..., :D].contiguous(),
                i=gates[..., D:2 * D] if pad else gates[..., D:].contiguous(),
                lam=torch.log(torch.expm1(-torch.log(a) / 8)), h0=r(n, D, dt=f32) if state else None,
                dy=r(B, T, D), dhT=r(n, D, dt=f32), cu=None if lens is None else cu_of(lens))


def loop(v, c, lens):
    """(y, last states, states before every 64th token of a row)"""
    la = -c * torch.nn.functional.softplus(v["lam"], threshold=700.0) * torch.sigmoid(v["r"])
    a, b = torch.exp(la), torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(v["i"]) * v["x"]
    y, last, kept, D = [], [], [], v["x"].shape[2]
    for s, (row, lo, hi) in enumerate(ref.spans(v["x"], lens)):
        h = torch.zeros(D, dtype=torch.float64) if v["h0"] is None else v["h0"][s]
        for t in range(lo, hi):
            if t % 64 == 0 and t > lo:
                kept.append((row, t // 64, h.detach()))
            h = a[row, t] * h + b[row, t]
            y.append(h)
        last.append(h)
    y = torch.stack(y).view(v["x"].shape) if y else torch.zeros_like(v["x"])
    return y, torch.stack(last), kept


def compare(x, c=8.0, lens=None, dhT=True, keep=True, times=1):
    y, hT, hc = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], c, x["h0"], x["cu"], return_chunk_states=True)
    v = {k: ref.double(x[k], True) for k in ("x", "r", "i", "lam", "h0")}
    yr, hr, kept = loop(v, c, lens)
    ref.check("y", y, yr, times * T32)
    ref.check("hT", hT, hr, times * T32)
    for row, k, h in kept:
        ref.check("h_chunks", hc[row, k], h, times * T32)
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], c, x["h0"], x["dhT"] if dhT else None, x["cu"],
                           h_chunks=hc if keep else None)
    g = ref.grads([(yr, ref.double(x["dy"]))] + ([(hr, ref.double(x["dhT"]))] if dhT else []), v)
    for k, n in (("dx", "x"), ("dr", "r"), ("di", "i")):
        ref.check(k, d[k], g[n], times * TGRAD)
    ref.check("dlam", d["dlam"], g["lam"], times * TSUM)
    assert ("dh0" in d) == (x["h0"] is not None)
    if x["h0"] is not None:
        ref.check("dh0", d["dh0"], g["h0"], times * TGRAD)
    return y, hT, hc, d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 400])
def test_lengths(T, dtype):
    compare(make(2, T, 40, dtype, seed=T))


@pytest.mark.parametrize("D", [1, 2, 3, 8, 31, 33, 40, 64, 65, 72, 130, 512])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_channels(D, dtype):
    compare(make(2, 70, D, dtype, seed=D))


@pytest.mark.parametrize("state,dhT,keep", [(False, False, False), (False, True, True), (True, False, False),
                                            (True, True, False)])
def test_options(state, dhT, keep):
    compare(make(3, 150, 64, "bf16", state=state), dhT=dhT, keep=keep)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rounds(dtype):
    """Rows longer than the tokens that a cluster has at one time, kept states or not: the same bits."""
    x = make(1, 1300, 72, dtype, seed=4)
    a = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], return_chunk_states=True)
    v = {k: ref.double(x[k]) for k in ("x", "r", "i", "lam", "h0")}
    yr, hr, _ = loop(v, 8.0, None)
    # (the bound grows with the tokens: 2^-25 of the state each)
    ref.check("y", a[0], yr, 6e-5)
    ref.check("hT", a[1], hr, 6e-5)
    d = [rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], h_chunks=hc) for hc in (a[2], None)]
    for k in d[0]:
        assert torch.equal(d[0][k], d[1][k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [2, 5, 64])
def test_strided_rows(pad, dtype):
    compare(make(2, 40, 96, dtype, pad=pad))


@pytest.mark.parametrize("lens", [None, [30, 0, 100, 70]])
@pytest.mark.parametrize("off", [1, 2])
def test_odd_addresses(off, lens):
    """Rows that do not start on 16 bytes."""
    x = make(1, 200, 64, "bf16", lens=lens)
    wide = {k: torch.cat([x[k][..., :off], x[k]], -1)[..., off:] for k in ("x", "r", "i", "dy")}
    compare({**x, **wide}, lens=lens)


@pytest.mark.parametrize("lens", [[5], [0, 1, 2, 3, 0, 40, 64, 0], [1] * 20, [0, 0], [130, 0, 7], [64, 64, 1], [200, 199]])
@pytest.mark.parametrize("D", [72, 33])
def test_packed(lens, D):
    compare(make(1, sum(lens), D, "f32", lens=lens), lens=lens)
    compare(make(1, sum(lens), D, "bf16", lens=lens, state=False), lens=lens, keep=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_many_rounds(dtype):
    """(sequences of up to 700 tokens: 2^-25 of the state a token, twice the bounds above)"""
    lens = [600, 0, 3, 700, 64, 1]
    compare(make(1, sum(lens), 64, dtype, lens=lens, seed=9), lens=lens, times=2)


def test_no_tokens():
    x = make(2, 0, 16, "bf16")
    y, hT = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"])
    assert y.shape == (2, 0, 16) and torch.equal(hT, x["h0"])
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"])
    assert torch.equal(d["dh0"], x["dhT"]) and not d["dlam"].any()
    y, hT = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"])
    assert not hT.any()


def test_sequences_do_not_touch():
    """NaN and infinities in one packed sequence, its state and its gradient stay there."""
    lens = [20, 3, 41, 600]
    x = make(1, sum(lens), 48, "bf16", lens=lens)

    def both():
        y, hT = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], cu_seqlens=x["cu"])
        return y, hT, rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"],
                                         cu_seqlens=x["cu"])

    yc, hc, clean = both()
    for k in ("x", "dy"):
        x[k][0, 20:23] = float("nan")
    x["r"][0, 21] = float("nan")
    x["h0"][1] = float("inf")
    x["dhT"][1] = float("nan")
    y, hT, d = both()
    for a, b in ((y, yc), (d["dx"], clean["dx"]), (d["dr"], clean["dr"]), (d["di"], clean["di"])):
        assert torch.equal(a[0, :20], b[0, :20]) and torch.equal(a[0, 23:], b[0, 23:])
        assert torch.isnan(a[0, 20:23]).all()
    for a, b in ((hT, hc), (d["dh0"], clean["dh0"])):
        assert torch.equal(a[[0, 2, 3]], b[[0, 2, 3]])


def test_gates_at_their_ends():
    """Gates closed and open to the last digit, and decays of 1 and 0, stay finite; a closed
    decay gate keeps the state, an open one with a large lam forgets it."""
    x = make(1, 100, 64, "f32")
    x["r"][0, :, :16], x["r"][0, :, 16:32] = -200.0, 200.0
    x["i"][0, :, 32:40], x["i"][0, :, 40:48] = -200.0, 200.0
    x["lam"][48:52], x["lam"][52:56], x["lam"][16:20], x["lam"][56:60] = -120.0, -float("inf"), 60.0, float("inf")
    y, hT = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"])
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"])
    for t in (y, hT, *d.values()):
        assert torch.isfinite(t).all()
    assert torch.equal(hT[0, 48:56], x["h0"][0, 48:56])
    ref.check("closed", hT[:, :16], x["h0"][:, :16].double().cpu(), 1e-6)
    want = (torch.sigmoid(x["i"][0, -1, 16:20].double()) * x["x"][0, -1, 16:20].double()).cpu()
    ref.check("forgets", hT[0, 16:20], want, T32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 101])
def test_steps_are_the_sequence(D, dtype):
    """Tokens one by one, in shuffled slots with an idle row, equal the sequence call."""
    x = make(3, 6, D, dtype, seed=5)
    y, last = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"])
    slots = torch.tensor([4, -1, 0, 2], dtype=torch.int32, device="cuda")
    h, rows = torch.randn(5, D, device="cuda"), [0, 2, 3]
    h[slots[rows].long()] = x["h0"]
    kept = h.clone()
    for t in range(6):
        one = {k: torch.full((4, D), float("nan"), device="cuda").to(DT[dtype]) for k in "xri"}
        for k in one:
            one[k][rows] = x[k][:, t]
        o = rdn.gated_scan_step(one["x"], one["r"], one["i"], x["lam"], h, slots=slots)
        assert not o[1].any()
        ref.check("step", o[rows], y[:, t].double().cpu(), T32)
    ref.check("states", h[slots[rows].long()], last.double().cpu(), T32)
    assert torch.equal(h[[1, 3]], kept[[1, 3]])


def test_step_without_slots_and_far_slots():
    x = make(2, 1, 64, "bf16", pad=6)
    a, b = x["h0"].clone(), x["h0"].clone()
    ins = (x["x"][:, 0], x["r"][:, 0], x["i"][:, 0], x["lam"])
    y = rdn.gated_scan_step(*ins, a)
    y2 = rdn.gated_scan_step(*ins, b, slots=torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(y[0], y2[0]) and not y2[1].any()
    assert torch.equal(a[0], b[0]) and torch.equal(b[1], x["h0"][1])


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e through the fp32 forward.  e = 2^-6: the
    curvature's e^2 term and the outputs' rounding (2^-24 / e) are both below 1e-3 of the slope."""
    x = make(2, 90, 24, "f32", seed=3)
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"])
    got = dict(x=d["dx"], r=d["dr"], i=d["di"], lam=d["dlam"], h0=d["dh0"])

    def loss(p):
        y = rdn.gated_scan_fwd(p["x"], p["r"], p["i"], p["lam"], h0=p["h0"], return_final_state=False)
        return (y.double() * x["dy"].double()).sum().item()

    for n, gr in got.items():
        v, e = torch.sign(gr), 2.0 ** -6
        slope = (loss({**x, n: x[n] + e * v}) - loss({**x, n: x[n] - e * v})) / (2 * e)
        want = (gr.double() * v.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * abs(want), (n, slope, want)


@pytest.mark.parametrize("off", [8, 4])
def test_outputs_given_and_their_surroundings(off):
    """Results written into slices of wider tensors leave what is beside them.  (Rows that do not start on 16
    bytes take other kernels, which add up in another order: each within its bound of the exact
    values, so within twice that of one another.)"""
    x = make(2, 70, 40, "bf16")
    y, _, hc = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], return_chunk_states=True)
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], h_chunks=hc)
    wide = {k: torch.full((2, 70, 56), 7.0, device="cuda", dtype=torch.bfloat16) for k in ("y", "dx", "dr", "di")}
    rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], out=wide["y"][..., off:off + 40])
    rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], h_chunks=hc,
                       out={k: wide[k][..., off:off + 40] for k in ("dx", "dr", "di")})
    for k, t in dict(d, y=y).items():
        if k in wide:
            got = wide[k][..., off:off + 40]
            if off == 8:
                assert torch.equal(got, t), k
            else:
                g, r = got.double(), t.double()
                most = torch.maximum(g.abs(), r.abs())
                assert ((g - r).abs() <= 2 * (TGRAD * (most + r.pow(2).mean().sqrt()) + 2.0 ** -8 * most)).all(), k
            assert (wide[k][..., :off] == 7).all() and (wide[k][..., off + 40:] == 7).all()


def test_same_bits_other_stream_and_graph():
    x = make(2, 700, 256, "bf16")

    def both():
        y, hT, hc = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], return_chunk_states=True)
        return dict(rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"]), y=y,
                    hT=hT, hc=hc)

    a = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = both()
    torch.cuda.current_stream().wait_stream(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c = both()
    y = make(2, 700, 256, "bf16", seed=1)
    for k in ("x", "r", "i", "dy", "h0", "dhT"):
        x[k].copy_(y[k])
    want = both()
    g.replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(c[k], want[k]), k
