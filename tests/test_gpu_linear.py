"""The matrix product with bias, activation and residual, on the GPU against the formulas in
64 bits."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ACTS = {None: lambda p: p, "silu": lambda p: p * torch.sigmoid(p), "sigmoid": torch.sigmoid,
        "gelu": lambda p: 0.5 * p * (1 + torch.erf(p / 2 ** 0.5))}
# 32-bit bound: the products are exact and their fp32 sum has at most K / 16 = 256 roundings of a
# partial sum near the result's RMS, 2^-23 each: 3e-5.  The activations add a few 2^-22 and
# have slopes below 1.13.
T32 = 4e-5


def rnd(*shape, dtype=BF, std=1.0, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.randn(*shape[:-1], shape[-1] + pad, generator=g, device="cuda") * std).to(dtype)
    return t[..., pad:] if pad else t


def make(M, N, K, kind="bf16", bias=BF, residual=BF, seed=0):
    if kind == "bf16":
        x, w, xs, ws = rnd(M, K, seed=seed), rnd(N, K, std=K ** -0.5, seed=seed + 1), None, None
    else:
        _, x, xs = rdn.add_norm_q8(rnd(M, K, seed=seed))
        _, w, ws = rdn.add_norm_q8(rnd(N, K, std=K ** -0.5, seed=seed + 1))
    return dict(x=x, w=w, xs=xs, ws=ws, bias=None if bias is None else rnd(N, dtype=bias, std=0.3, seed=seed + 2),
                res=None if residual is None else rnd(M, N, dtype=residual, seed=seed + 3), dy=rnd(M, N, seed=seed + 4))


def exact(x, act):
    """(p, y) in 64 bits"""
    p = x["x"].double() @ x["w"].double().T
    if x["xs"] is not None:
        p = p * x["xs"].double()[..., None] * x["ws"].double()
    if x["bias"] is not None:
        p = p + x["bias"].double()
    y = ACTS[act](p)
    return p.cpu(), (y if x["res"] is None else y + x["res"].double()).cpu()


def forward(x, act, **kw):
    return rdn.linear_fwd(x["x"], x["w"], x["bias"], act, x["res"], x["xs"], x["ws"], **kw)


def compare(x, act=None, out_dtype=None, **kw):
    p, y = exact(x, act)
    got = forward(x, act, out_dtype=out_dtype, **kw)
    ref.check("y", got, y, T32)
    return got


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N,K", [
    (1, 8, 16), (1, 16, 64), (1, 128, 2048), (2, 136, 208), (7, 1000, 1040), (16, 128, 64), (17, 256, 128),
    (32, 264, 80), (33, 128, 4096), (64, 2048, 1024), (65, 520, 144), (127, 128, 128), (128, 128, 64),
    (129, 384, 192), (200, 1000, 2064), (256, 256, 64), (257, 8, 1024), (1000, 16, 256)])
def test_sizes(M, N, K, kind):
    compare(make(M, N, K, kind, seed=M + N), "silu")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(2048, 2048, 64), (1900, 2056, 80), (4100, 1000, 400), (777, 4096, 2048),
                                   (16400, 136, 128), (130, 16392, 64), (1, 65536, 64)])
def test_many_tiles(M, N, K, kind):
    compare(make(M, N, K, kind, seed=N), "gelu")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(1, 16392, 1040), (40, 12296, 208), (64, 40008, 64), (3, 2048, 2064),
                                   (128, 4096, 1024), (250, 1288, 2048), (512, 2048, 2048), (500, 4096, 4096),
                                   (2048, 136, 4096)])
def test_parts_of_the_sum(M, N, K, kind):
    """Few rows of wide results, and one to eight parts of the sum over k, on one and two CTAs an SM."""
    compare(make(M, N, K, kind, seed=K), "silu")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,N", [(5, 136), (2050, 2056)])
@pytest.mark.parametrize("act", [None, "silu", "sigmoid", "gelu"])
def test_options(M, N, act, kind):
    for bias, residual, out in ((None, None, None), (BF, None, F32), (F32, BF, None), (None, F32, None), (F32, F32, F32),
                                (BF, BF, BF)):
        got = compare(make(M, N, 96, kind, bias, residual), act, out)
        assert got.dtype == (out or residual or BF)


@pytest.mark.parametrize("M,N", [(5, 136), (70, 264), (2050, 2056)])
def test_pre(M, N):
    x = make(M, N, 96)
    y, pre = forward(x, "silu", return_pre=True)
    p, want = exact(x, "silu")
    ref.check("pre", pre, p, T32)
    ref.check("y", y, want, T32)


@pytest.mark.parametrize("M", [6, 2100])
@pytest.mark.parametrize("out", [BF, F32])
def test_strided_rows_and_axes(M, out):
    """Slices of wider tensors, more axes, odd rows of the residual and the result; what is beside
    the result is left as it was."""
    N, K = 2056, 128
    x = make(M, N, K, bias=F32, residual=None)
    x["x"], x["w"] = rnd(2, M // 2, K, pad=24), rnd(N, K, std=K ** -0.5, pad=8, seed=1)
    for pad in (3, 16):
        x["res"] = rnd(2, M // 2, N, dtype=out, pad=pad, seed=2)
        wide = torch.full((2, M // 2, N + 2 * pad), 7.0, dtype=out, device="cuda")
        got = compare(x, "silu", out=wide[..., pad:pad + N])
        assert got.shape == (2, M // 2, N)
        assert (wide[..., :pad] == 7).all() and (wide[..., pad + N:] == 7).all()


@pytest.mark.parametrize("M", [3, 2100])
def test_residual_in_place(M):
    x = make(M, 2056, 128)
    want = forward(x, "silu")
    got = forward(x, "silu", out=x["res"])
    assert got is x["res"] and torch.equal(got, want)


def test_no_rows():
    x = make(0, 64, 32)
    assert forward(x, "silu").shape == (0, 64)
    d = rdn.linear_bwd(x["x"], x["w"], x["dy"], pre=x["dy"], act="silu", bias=x["bias"])
    assert d["dx"].shape == (0, 32) and not d["dw"].any() and not d["dbias"].any()
    assert d["dw"].shape == (64, 32)


def test_a_row_that_is_not_finite_stays_alone():
    for M in (4, 2100):
        x = make(M, 2048, 64)
        want = forward(x, None)
        x["x"][1, 3], x["x"][2, 5] = float("nan"), float("inf")
        got = forward(x, None)
        keep = [0] + list(range(3, M))
        assert torch.equal(got[keep], want[keep]) and torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()


def rounded_dp(x, pre, act):
    """dy act'(pre), rounded to bf16 as the products take it, in 64 bits on the GPU."""
    if act is None:
        return x["dy"].double()
    p = pre.double().requires_grad_()
    d = torch.autograd.grad(ACTS[act](p).sum(), p)[0]
    return (x["dy"].double() * d).to(BF).double()


def backward(M, N, K, act, bias=BF, dw_dtype=None, seed=0):
    x = make(M, N, K, bias=bias, residual=None, seed=seed)
    pre = None if act is None else forward(x, act, return_pre=True)[1]
    d = rdn.linear_bwd(x["x"], x["w"], x["dy"], pre, act, x["bias"], dw_dtype=dw_dtype)
    dp = rounded_dp(x, pre, act)
    # a dp near a rounding tie may fall the other way: 2^-8 of it, of which a sum of n terms has
    # few; one is below 5 RMS of a term, 5 / sqrt(n) RMS of the sum
    flip = lambda n: T32 if act is None else T32 + 2.0 ** -8 * 5 / n ** 0.5  # noqa: E731
    ref.check("dx", d["dx"], (dp @ x["w"].double()).cpu(), flip(N))
    ref.check("dw", d["dw"], (dp.T @ x["x"].double()).cpu(), flip(M))
    assert d["dw"].dtype == (dw_dtype or BF)
    if bias is not None:
        exact_dp = x["dy"].double()
        if act is not None:
            p = pre.double().requires_grad_()
            exact_dp = exact_dp * torch.autograd.grad(ACTS[act](p).sum(), p)[0]
        # chains of at most M / 8 terms a warp, 8 and 16 + M / 64 joins, of 2^-24 each
        assert d["dbias"].dtype == bias
        ref.check("dbias", d["dbias"], exact_dp.sum(0).cpu(), 4e-5)
    return x, pre, d


@pytest.mark.parametrize("M,N,K", [(1, 16, 64), (5, 136, 208), (64, 1000, 64), (200, 128, 1000), (300, 16, 2048),
                                   (2500, 264, 128), (128, 4096, 2048), (4100, 2056, 136), (3000, 2048, 2048),
                                   (63, 136, 64), (512, 264, 64), (513, 264, 64)])
def test_backward_sizes(M, N, K):
    backward(M, N, K, "silu", seed=M)


@pytest.mark.parametrize("act", [None, "silu", "sigmoid", "gelu"])
@pytest.mark.parametrize("bias,dw", [(None, None), (F32, F32), (BF, F32)])
def test_backward_options(act, bias, dw):
    backward(130, 264, 96, act, bias, dw)


def test_backward_parts():
    x, pre, d = backward(130, 264, 96, "silu")
    ins = (x["x"], x["w"], x["dy"], pre, "silu")
    a = rdn.linear_bwd(*ins, need_dx=False)
    b = rdn.linear_bwd(*ins, need_dw=False)
    c = rdn.linear_bwd(*ins, bias=x["bias"], need_dw=False, need_dx=False)
    assert set(a) == {"dw"} and set(b) == {"dx"} and set(c) == {"dbias"}
    assert torch.equal(a["dw"], d["dw"]) and torch.equal(b["dx"], d["dx"]) and torch.equal(c["dbias"], d["dbias"])


def test_backward_strided_rows():
    x, pre, d = backward(130, 264, 96, None)
    wide = {k: torch.cat([x[k][:, :8], x[k]], 1)[:, 8:] for k in ("x", "w", "dy")}
    got = rdn.linear_bwd(wide["x"], wide["w"], wide["dy"], bias=x["bias"])
    for k in d:
        assert torch.equal(got[k], d[k]), k


@pytest.mark.parametrize("act", ["silu", "sigmoid", "gelu"])
def test_gradient_of_the_formula(act):
    """Against differentiation in 64 bits of the unrounded pass.  Rounding pre and dp to bf16 (2^-8
    each at most, 2^-8 / sqrt(3) RMS) moves a sum of unrelated terms by 0.33 % of its RMS, and
    5 times that is not passed by any of some 10^5 elements; the activations' second derivatives
    times p stay below their slopes' RMS."""
    x = make(150, 256, 192, residual=None, seed=2)
    y, pre = forward(x, act, return_pre=True)
    d = rdn.linear_bwd(x["x"], x["w"], x["dy"], pre, act, x["bias"])
    v = {k: ref.double(x[k], True) for k in ("x", "w", "bias")}
    out = ACTS[act](v["x"] @ v["w"].T + v["bias"])
    g = ref.grads([(out, ref.double(x["dy"]))], v)
    for k, n in (("dx", "x"), ("dw", "w"), ("dbias", "bias")):
        ref.check(k, d[k], g[n], 1.7e-2)


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e with L in 64 bits of an fp32 result.  The
    steps are whole powers of two on values below 4, kept in bf16: e = 2^-5 moves every one (their
    step is at most 2^-6); the curvature's e^2 term and the roundings of pre and dp are below 1 %."""
    x = make(64, 128, 96, residual=None, seed=5)
    for k in ("x", "w"):
        x[k] = ((x[k].float() * (1 if k == "x" else 8)).clamp(-3.9, 3.9) * 64).round().div(64).to(BF)
    pre = forward(x, "silu", return_pre=True)[1]
    d = rdn.linear_bwd(x["x"], x["w"], x["dy"], pre, "silu", x["bias"], dw_dtype=F32)

    def loss(p):
        return (rdn.linear_fwd(p["x"], p["w"], p["bias"], "silu", out_dtype=F32).double() * x["dy"].double()).sum().item()

    for n, gr in (("x", d["dx"]), ("w", d["dw"])):
        v = torch.sign(gr.float()) * (torch.arange(gr.numel(), device="cuda").view(gr.shape) % 7 == 0)
        e = 2.0 ** -5
        up, down = ({**x, n: (x[n].float() + s * e * v).to(BF)} for s in (1, -1))
        moved = (up[n].double() - down[n].double())
        want = (gr.double() * moved).sum().item()
        assert abs(loss(up) - loss(down) - want) <= 2e-2 * abs(want), (n, loss(up) - loss(down), want)


@pytest.mark.parametrize("M", [3, 300, 2500])
def test_same_bits_other_stream_and_graph(M):
    x = make(M, 2048, 256)

    def both():
        y, pre = forward(x, "silu", return_pre=True)
        return dict(rdn.linear_bwd(x["x"], x["w"], x["dy"], pre, "silu", x["bias"]), y=y)

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
    y = make(M, 2048, 256, seed=9)
    for k in ("x", "w", "bias", "res", "dy"):
        x[k].copy_(y[k])
    want = both()
    g.replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(c[k], want[k]), k
    assert rdn.device_status() == 0
