"""The selective state space scan on the GPU against a plain 64-bit loop."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# 32-bit bound: a state forgets over at most some 300 tokens here, two roundings (2^-24) each,
# if none of them cancelled: 4e-5 of its size; sums over states, channels and tokens average out.
T32 = 4e-5
INS = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h0")


def make(B, T, D, S, G=1, dtype="bf16", lens=None, state=True, gate=True, skip=True, bias=True, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=DT[dtype]: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    n = B if lens is None else len(lens)
    rows = lambda *s: r(*s) if not pad else r(*s[:-1], s[-1] + pad)[..., pad // 2:pad // 2 + s[-1]]  # noqa: E731
    f32 = torch.float32
    x = dict(x=rows(B, T, D), dt=rows(B, T, D) * 0.5 if not pad else rows(B, T, D),
             A=-torch.exp(torch.rand(D, S, generator=g, device="cuda") * 3 - 1),
             B=r(B, T, G, S), C=r(B, T, G, S), D=r(D, dt=f32) if skip else None,
             z=rows(B, T, D) if gate else None, dt_bias=r(D, dt=f32) - 2 if bias else None,
             h0=r(n, D, S, dt=f32) if state else None, dout=r(B, T, D), dhT=r(n, D, S, dt=f32))
    x["cu"] = None if lens is None else torch.tensor([0] + [sum(lens[:i + 1]) for i in range(n)],
                                                     dtype=torch.int32, device="cuda")
    return x


def call(fn, x, *more, **kw):
    return fn(*(x[k] for k in INS[:5]), *more, **{k: x[k] for k in INS[5:]}, cu_seqlens=x["cu"], **kw)


def compare(x, softplus=True, lens=None, dhT=True, back=True, chunks=True, t32=T32):
    out, hT, hc = call(rdn.selective_scan_fwd, x, dt_softplus=softplus, return_chunk_states=True)
    v = {k: ref.double(x[k], True) for k in INS}
    o, hTr, kept = ref.scan(*(v[k] for k in INS), softplus, lens)
    ref.check("out", out, o, t32)
    ref.check("hT", hT, hTr, t32)
    if kept is not None:
        ref.check("h_chunks", hc[:kept.shape[0]], kept, t32)
    if not back:
        return
    d = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"] if dhT else None,
             h_chunks=hc if chunks else None, dt_softplus=softplus)
    outs = [(o, ref.double(x["dout"]))] + ([(hTr, ref.double(x["dhT"]))] if dhT else [])
    g = ref.grads(outs, v)
    for name, k in (("dx", "x"), ("ddt", "dt"), ("dz", "z"), ("dB", "B"), ("dC", "C"), ("dA", "A"),
                    ("dD", "D"), ("ddt_bias", "dt_bias"), ("dh0", "h0")):
        if x[k] is not None:
            ref.check(name, d[name], g[k], t32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 4, 15, 16, 17, 63, 64, 65, 130, 200])
def test_lengths(T, dtype):
    """(beyond 64 tokens these few channels are cut into units)"""
    compare(make(2, T, 24, 16, dtype=dtype, seed=T))


@pytest.mark.parametrize("T", [3, 5, 8, 9, 12, 13, 25])
def test_lengths_within_a_tile(T):
    """(the backward keeps states at every fourth token of sixteen)"""
    compare(make(2, T, 24, 16, seed=T))


@pytest.mark.parametrize("S", [1, 3, 4, 5, 8, 9, 12, 16, 20, 32, 33, 48, 64])
def test_states(S):
    compare(make(1, 70, 16, S, dtype="f32", seed=S))
    compare(make(2, 20, 16, S, dtype="bf16", seed=S))


@pytest.mark.parametrize("D,G", [(1, 1), (2, 2), (7, 1), (64, 1), (65, 1), (130, 2), (200, 4), (96, 3), (256, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_channels_and_groups(D, G, dtype):
    compare(make(1, 21, D, 16, G, dtype, seed=D))
    compare(make(1, 18, D, 6, G, dtype, seed=D))


@pytest.mark.parametrize("S", [8, 16, 32, 64])
def test_wide(S):
    """More channels than a CTA's, whole and ragged, on 16-byte and on odd rows."""
    compare(make(1, 33, 280, S, dtype="bf16"))
    compare(make(1, 17, 139, S, dtype="bf16"))


@pytest.mark.parametrize("state,gate,skip,bias,softplus,dhT", [
    (False, False, False, False, True, False), (True, False, True, False, True, True),
    (False, True, False, True, True, True), (False, True, True, True, True, False)])
def test_options(state, gate, skip, bias, softplus, dhT):
    compare(make(2, 90, 40, 16, state=state, gate=gate, skip=skip, bias=bias), softplus, dhT=dhT)


def test_steps_given_directly():
    x = make(2, 40, 40, 16, dtype="f32", bias=False)
    x["dt"] = x["dt"].abs() * 0.2
    compare(x, softplus=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [2, 64])
def test_strided_rows(pad, dtype):
    compare(make(2, 40, 48, 16, dtype=dtype, pad=pad))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parameters_at_odd_addresses(dtype):
    x = make(1, 40, 64, 16, dtype=dtype, seed=3)
    for k in ("D", "dt_bias"):
        at = torch.empty(65, device="cuda")
        at[1:] = x[k]
        x[k] = at[1:]
        assert x[k].data_ptr() % 16
    compare(x)


def test_operands_of_one_projection():
    """x, z, dt, B and C as slices of one row."""
    x = make(2, 50, 64, 16)
    proj = torch.randn(2, 50, 64 * 3 + 32, device="cuda").bfloat16()
    x["x"], x["z"], x["dt"] = proj[..., :64], proj[..., 64:128], proj[..., 128:192]
    x["B"], x["C"] = proj[..., 192:208].unflatten(-1, (1, 16)), proj[..., 208:].unflatten(-1, (1, 16))
    compare(x)


@pytest.mark.parametrize("lens", [[5], [0, 1, 2, 0, 16, 40, 70, 0], [1] * 40, [0, 0], [150, 0, 17]])
def test_packed(lens):
    compare(make(1, sum(lens), 40, 16, dtype="f32", lens=lens), lens=lens)
    compare(make(1, sum(lens), 40, 16, dtype="bf16", lens=lens, state=False), lens=lens)


def test_states_computed_by_the_backward():
    for lens in (None, [30, 0, 100]):
        compare(make(1, 130, 40, 16, lens=lens), lens=lens, chunks=False)


def test_no_tokens():
    x = make(2, 0, 16, 16)
    out, hT = call(rdn.selective_scan_fwd, x)
    assert out.shape == (2, 0, 16) and torch.equal(hT, x["h0"])
    d = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"])
    assert torch.equal(d["dh0"], x["dhT"])
    for k in ("dA", "dD", "ddt_bias"):
        assert not d[k].any()


def test_long_memory():
    """Steps of 0.001 to 0.01 and A = -1: a state remembers up to 1,000 tokens.  Decays that come
    out 2e-8 low on average would put the state off by 2e-8 * 600 = 1.2e-5; rounding alone leaves
    6e-8 * sqrt(600 / 2) = 1e-6, allowed four times."""
    T, D = 1200, 32
    x = make(1, T, D, 16, dtype="f32", state=False, gate=False, bias=False)
    x["A"] = torch.full_like(x["A"], -1.0)
    x["dt"] = torch.rand(1, T, D, device="cuda") * 0.009 + 0.001
    x["x"], x["B"] = x["x"].abs(), x["B"].abs()
    out, hT = call(rdn.selective_scan_fwd, x, dt_softplus=False)
    v = {k: ref.double(x[k]) for k in INS}
    o, hTr, _ = ref.scan(*(v[k] for k in INS), False)
    rel = ((hT.double().cpu() - hTr).norm() / hTr.norm()).item()
    assert rel <= 4e-6, rel


def test_sequences_and_channels_do_not_touch():
    lens = [20, 3, 100]
    x = make(1, 123, 48, 16, lens=lens)
    o, hT, hc = call(rdn.selective_scan_fwd, x, return_chunk_states=True)
    d = call(rdn.selective_scan_bwd, x, x["dout"], h_chunks=hc)
    for k in ("x", "dt", "dout", "z"):
        x[k][0, 20:23] = float("nan")
    x["B"][0, 20:23] = float("inf")
    x["h0"][1] = float("nan")
    o2, hT2, hc2 = call(rdn.selective_scan_fwd, x, return_chunk_states=True)
    d2 = call(rdn.selective_scan_bwd, x, x["dout"], h_chunks=hc2)
    for a, b in ((o, o2), (d["dx"], d2["dx"]), (d["ddt"], d2["ddt"]), (d["dz"], d2["dz"]),
                 (d["dB"], d2["dB"]), (d["dC"], d2["dC"])):
        assert torch.equal(a[0, :20], b[0, :20]) and torch.equal(a[0, 23:], b[0, 23:])
        assert torch.isnan(b[0, 20:23]).all()
    assert torch.equal(hT[[0, 2]], hT2[[0, 2]]) and torch.equal(d["dh0"][[0, 2]], d2["dh0"][[0, 2]])
    # one channel's infinity stays out of the others' results
    x = make(1, 40, 48, 16, state=False)
    o = call(rdn.selective_scan_fwd, x)[0]
    x["x"][0, 7, 5] = float("inf")
    o2 = call(rdn.selective_scan_fwd, x)[0]
    keep = [c for c in range(48) if c != 5]
    assert torch.equal(o[..., keep], o2[..., keep])


def test_large_steps():
    """Decays that underflow (exp of -2000) and very negative steps (softplus underflows)."""
    x = make(1, 40, 32, 16, dtype="f32", state=True, bias=False)
    x["dt"][..., ::3] = 100.0
    x["dt"][..., 1::3] = -200.0
    compare(x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S,G", [(64, 16, 1), (30, 5, 2), (100, 64, 1), (128, 8, 4)])
def test_steps_are_the_sequence(D, S, G, dtype):
    x = make(3, 5, D, S, G, dtype, seed=9)
    out, hT = call(rdn.selective_scan_fwd, x)
    slots = torch.tensor([4, -1, 0, 2], dtype=torch.int32, device="cuda")
    rows, h = [0, 2, 3], torch.randn(5, D, S, device="cuda")
    h[slots[rows].long()] = x["h0"]
    kept = h.clone()
    for t in range(5):
        a = {}
        for k in ("x", "dt", "z", "B", "C"):
            a[k] = torch.full((4,) + x[k].shape[2:], float("nan"), device="cuda").to(DT[dtype])
            a[k][rows] = x[k][:, t]
        o = rdn.selective_scan_step(a["x"], a["dt"], x["A"], a["B"], a["C"], h, x["D"], a["z"], x["dt_bias"],
                                    slots=slots)
        assert not o[1].any()
        # (two roundings to bf16 may fall on different sides: a whole unit in the last place)
        err = (o[rows].double() - out[:, t].double()).abs()
        ulp = 2.0 ** -7 if dtype == "bf16" else 0.0
        assert (err <= (T32 + ulp) * (out[:, t].double().abs() + out.double().pow(2).mean().sqrt())).all()
    ref.check("h", h[slots[rows].long()], hT.double().cpu(), T32)
    assert torch.equal(h[[1, 3]], kept[[1, 3]])


def test_continuation():
    """A prompt in two calls equals one call."""
    x = make(2, 100, 64, 16, dtype="f32")
    out, hT = call(rdn.selective_scan_fwd, x)
    cut = lambda lo, hi: {**x, **{k: x[k][:, lo:hi] for k in ("x", "dt", "z", "B", "C")}}  # noqa: E731
    first = {k: (t.contiguous() if isinstance(t, torch.Tensor) else t) for k, t in cut(0, 37).items()}
    rest = {k: (t.contiguous() if isinstance(t, torch.Tensor) else t) for k, t in cut(37, 100).items()}
    o1, h1 = call(rdn.selective_scan_fwd, first)
    rest["h0"] = h1
    o2, h2 = call(rdn.selective_scan_fwd, rest)
    ref.check("out", torch.cat([o1, o2], 1), out.double().cpu(), T32)
    ref.check("hT", h2, hT.double().cpu(), T32)


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e through the fp32 forward; steps small
    enough for the curvature (e^2) and large enough for the outputs' rounding (2^-24 / e)."""
    x = make(1, 70, 16, 16, dtype="f32", seed=4)
    d = call(rdn.selective_scan_bwd, x, x["dout"])
    got = dict(x=d["dx"], dt=d["ddt"], A=d["dA"], B=d["dB"], C=d["dC"], D=d["dD"], z=d["dz"],
               dt_bias=d["ddt_bias"], h0=d["dh0"])

    def loss(p):
        return (call(rdn.selective_scan_fwd, p)[0].double() * x["dout"].double()).sum().item()

    for n, gr in got.items():
        v, e = torch.sign(gr), 2.0 ** -8
        up, down = ({**x, n: x[n] + s * e * v} for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * e)
        want = (gr.double() * v.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * abs(want), (n, slope, want)


def test_same_bits_and_other_stream():
    x = make(2, 200, 256, 16)
    a = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"])
    torch.cuda.current_stream().wait_stream(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_in_a_graph():
    """A captured forward and backward replay on new inputs."""
    x = make(2, 100, 64, 16)
    new = make(2, 100, 64, 16, seed=1)
    out, hT, hc = call(rdn.selective_scan_fwd, x, return_chunk_states=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, hT, hc = call(rdn.selective_scan_fwd, x, return_chunk_states=True)
        d = call(rdn.selective_scan_bwd, x, x["dout"], h_chunks=hc)
    for k in INS + ("dout",):
        x[k].copy_(new[k])
    g.replay()
    o2, _, hc2 = call(rdn.selective_scan_fwd, new, return_chunk_states=True)
    d2 = call(rdn.selective_scan_bwd, new, new["dout"], h_chunks=hc2)
    assert torch.equal(out, o2)
    for k in d:
        assert torch.equal(d[k], d2[k]), k


def test_steps_of_zero_keep_the_state():
    """dl = 0 is a decay of exactly one: the state passes through bit by bit, both ways."""
    x = make(2, 37, 40, 16, dtype="f32", bias=False)
    x["dt"].zero_()
    out, hT = call(rdn.selective_scan_fwd, x, dt_softplus=False)
    assert torch.equal(hT, x["h0"])
    x["C"].zero_()
    d = call(rdn.selective_scan_bwd, x, x["dout"], dhT=x["dhT"], dt_softplus=False)
    assert torch.equal(d["dh0"], x["dhT"])
